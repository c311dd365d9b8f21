"""What the orthogonalised updates, the embedding and the cross entropy launch
(CPU: launches are taken down, nothing runs; addresses are numbers)."""

import pytest

import launch_recorder


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    shim = launch_recorder.build(str(tmp_path_factory.mktemp("shim")))
    return lambda body: launch_recorder.run(shim, body)


ANY_SIZES = r"""
        import random
        rng = random.Random(7)
        B, MOST = 1 << 40, (1 << 63) - 1

        def size():
            return rng.choice([0, 1, 2, 3, 7, 64, 127, 128, 129, 4096, 8192, 8193, 1 << 14, (1 << 14) + 1, 1 << 20, (1 << 20) + 1, (1 << 31) - 1, 1 << 31,
                               1 << 40, 1 << 62, MOST, -1, rng.randrange(1, 1 << 17)])

        def orthogonalize():
            batch, r, k = rng.choice([0, 1, 3, 50, size()]), size(), size()
            if min(r, k) > 300 and batch > 3:
                batch = 3
            need = c.mtdao_orthogonalize_workspace_bytes(min(batch, 200), r, k)
            c.mtdao_orthogonalize(B, rng.choice([0, 1]), min(batch, 200), r, k, B << 8, rng.choice([0, 1]), rng.choice([1, 2, 3, 5, 7]), 1e-7, B << 16, need, None)

        def muon():
            n = rng.randrange(1, 40)
            cfg = c.MuonConfig(rng.choice([0, 1]), rng.choice([0, 1]), n, rng.choice([0, 1]), rng.choice([1, 5]), 0, 0.9, 1e-7)
            few = [rng.randrange(1, 3000) for _ in range(rng.choice([2, 30]))]
            rows = (c.MuonMatrix * n)(*(c.MuonMatrix(*(B + (i << 46) + (j << 43) for j in range(3)), rng.choice(few), rng.choice(few + [0]), 0.1, 1.0)
                                        for i in range(n)))
            need = c.mtdao_muon_workspace_bytes(cfg, rows)
            h = c.mtdao_muon_init(cfg, rows, B << 20, need, None)
            c.mtdao_muon_set_grads(h, [r.g for r in rows], None)
            c.mtdao_muon_step(h, 1e-3, None)
            c.mtdao_muon_destroy(h)

        def embedding():
            n, rows, d = size(), size(), size()
            ld = rng.choice([d, size()])
            if rng.random() < 0.5:
                c.mtdao_embedding(B, rng.choice([32, 64]), n, B << 14, rng.choice([0, 1]), rows, d, ld, 1.0, B << 16, rng.choice([0, 1]), d, None)
            else:
                need = c.mtdao_embedding_backward_workspace_bytes(n, rows, d)
                c.mtdao_embedding_backward(B << 14, rng.choice([0, 1]), ld, B, rng.choice([32, 64]), n, 1.0, B << 16, rows, d, d, rng.choice([0, 1]), B << 18,
                                           need, None)

        def loss():
            a = c.CrossEntropyArgs(size(), size(), 0, 0, rng.choice([0, 1]), rng.choice([32, 64]), rng.choice([0, 1, 2]), 0.0, 1.0, 0, B, B << 14, None)
            a.ld_logits = rng.choice([a.cols, size()])
            a.ld_d = rng.choice([a.cols, a.ld_logits])
            for name, at in (("losses", B << 16), ("loss", B << 17), ("d_logits", rng.choice([B << 18, B]))):
                if rng.random() < 0.6:
                    setattr(a, name, at)
            c.mtdao_cross_entropy(a, B << 20, c.mtdao_cross_entropy_workspace_bytes(a), None)

        taken = refused = 0
        for _ in range(6000):
            try:
                rng.choice([orthogonalize, muon, embedding, embedding, loss, loss])()
                taken += 1
            except abi.MtdaoError:
                refused += 1
        say([taken, refused])
"""


def test_any_sizes_are_refused_or_fit_their_launches(run):
    launches, said = run(ANY_SIZES)
    assert min(said[0]) > 1000, said
    for name, (x, y, z), threads, _ in launches:
        assert x >= 1 and y >= 1 and z == 1 and x * threads < 1 << 32 and y <= 65535, (name, x, y, threads)
    assert {"k_muon_product", "k_muon_split", "k_embedding", "k_embedding_sums", "k_cross_entropy"} <= {name for name, *_ in launches}


def test_matrices_of_a_step_share_their_launches(run):
    """Launches go by the products, not by the number of matrices."""
    counts = []
    for n in (1, 24):
        launches, _ = run(f"""
            B = 1 << 40
            cfg = c.MuonConfig(0, 0, 4 * {n}, 1, 5, 0, 0.9, 1e-7)
            shapes = [(768, 256), (256, 256), (1024, 256), (256, 1024)] * {n}
            rows = (c.MuonMatrix * len(shapes))(*(c.MuonMatrix(*(B + (i << 46) + (j << 43) for j in range(3)), *s, 0.1, 1.0) for i, s in enumerate(shapes)))
            h = c.mtdao_muon_init(cfg, rows, B << 20, c.mtdao_muon_workspace_bytes(cfg, rows), None)
            say("steps")
            c.mtdao_muon_step(h, 1e-3, None)
            c.mtdao_muon_destroy(h)
        """)
        counts.append(len([1 for name, *_ in launches if name != "k_muon_table"]))
    assert counts[1] <= counts[0] <= counts[1] + 5  # (few matrices' A, five times, is formed in parts and joined)

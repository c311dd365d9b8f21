"""MT-DAO optimizer hot path on MI355X (gfx950).

``mtdao`` is the ctypes binding of the C ABI declared in include/mtdao.h
(libmtdao.so, built by ``python -m paper_2510_05361_amd.build``);
``optimizer.MtdaoOptimizer`` holds torch-allocated state buffers for it.
``ops`` has operators of the models that it trains (AdamW, the boundary of a
Peri-LN block, 8-bit linear layers) on torch tensors, ``mtdao_ops`` the binding
of their C ABI, include/mtdao_ops.h.
Importing the package loads nothing; the library is loaded on first use and
its absence is an error.
"""

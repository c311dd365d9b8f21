"""What the library would launch, on a machine without a GPU.

A small C library answers the HIP calls of libmtdao.so: it takes kernels,
grids and the first bytes of the arguments down and runs nothing.  Loaded
with RTLD_GLOBAL before libmtdao.so, in a process of its own, its symbols
come before those of the HIP runtime, which is never called.  Device addresses
may be any number.
"""

from __future__ import annotations

import json
import os
import re
import subprocess
import sys
import textwrap

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#include <stddef.h>
#include <stdio.h>
typedef struct { unsigned x, y, z; } dim3_t;
static const void* fn[4096];
static const char* name[4096];
static int n;
static dim3_t grid, block;
static size_t shared;
static void* stream;
void** __hipRegisterFatBinary(const void* p) { (void)p; static void* h; return &h; }
void __hipUnregisterFatBinary(void** h) { (void)h; }
void __hipRegisterVar(void** h, void* v, char* a, char* b, int c, size_t d, int e, int f) {
  (void)h; (void)v; (void)a; (void)b; (void)c; (void)d; (void)e; (void)f;
}
void __hipRegisterFunction(void** h, const void* host, char* dev, const char* what, unsigned l, void* a, void* b, void* c, void* d, int* e) {
  (void)h; (void)dev; (void)l; (void)a; (void)b; (void)c; (void)d; (void)e;
  if (n < 4096) { fn[n] = host; name[n++] = what; }
}
int __hipPushCallConfiguration(dim3_t g, dim3_t b, size_t s, void* st) { grid = g; block = b; shared = s; stream = st; return 0; }
int __hipPopCallConfiguration(dim3_t* g, dim3_t* b, size_t* s, void** st) { *g = grid; *b = block; *s = shared; *st = stream; return 0; }
int hipLaunchKernel(const void* f, dim3_t g, dim3_t b, void** args, size_t s, void* st) {
  (void)args; (void)st;
  const char* what = "?";
  for (int i = 0; i < n; ++i)
    if (fn[i] == f) what = name[i];
  printf("launch %s %u %u %u %u %zu\n", what, g.x, g.y, g.z, b.x, s);
  fflush(stdout);
  return 0;
}
int hipGetLastError(void) { return 0; }
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipFuncSetAttribute(const void* f, int a, int v) { (void)f; (void)a; (void)v; return 0; }
const char* hipGetErrorString(int e) { (void)e; return "error"; }
"""


def build(folder) -> str:
    src, lib = os.path.join(folder, "shim.c"), os.path.join(folder, "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["gcc", "-std=c11", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", lib, src], check=True)
    return lib


def _lines(shim: str, body: str):
    """What the Python lines ``body`` (``c``: mtdao_ops, ``abi``: mtdao) print and launch over the shim."""
    head = f"""
        import ctypes, json, sys
        sys.path.insert(0, {ROOT!r})
        ctypes.CDLL({shim!r}, mode=ctypes.RTLD_GLOBAL)
        from paper_2510_05361_amd import mtdao as abi, mtdao_ops as c
        def say(value):
            print("say " + json.dumps(value), flush=True)
    """
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(head) + textwrap.dedent(body)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])
    return r.stdout.splitlines()


_KERNEL = re.compile(r"(?:12_GLOBAL__N_1|^_Z)\d+(k_[a-z0-9_]+?)(?:I|E)")


def run(shim: str, body: str):
    """Run the Python lines ``body`` (``c``: mtdao_ops, ``abi``: mtdao) over the
    shim.  Returns (launches, printed): launches as (kernel's name without
    template arguments, grid, threads of a workgroup, bytes of dynamic LDS), printed as the JSON
    values that ``say(value)`` was given, both in order."""
    launches, said = [], []
    for line in _lines(shim, body):
        if line.startswith("say "):
            said.append(json.loads(line[4:]))
        elif line.startswith("launch "):
            _, what, gx, gy, gz, threads, lds = line.split()
            launches.append((_KERNEL.search(what).group(1), (int(gx), int(gy), int(gz)), int(threads), int(lds)))
    return launches, said


def instances(shim: str, body: str):
    """The kernels that ``body`` launches, in order, with their template arguments: "k_name<128, 2, float>"
    (bf16 is its storage type)."""
    out = []
    for line in _lines(shim, body):
        if line.startswith("launch "):
            what = line.split()[1]
            name = _KERNEL.search(what).group(1)
            args = what[what.index(name) + len(name):]
            args = args[1:args.index("EEv")] + "E" if args.startswith("I") else ""
            args = [number or {"0": "false", "1": "true", "f": "float", "t": "bf16"}[truth or kind]
                    for number, truth, kind in re.findall(r"Li(\d+)E|Lb([01])E|([ft])", args)]
            out.append(name + ("<" + ", ".join(args) + ">" if args else ""))
    return out

"""The rules of csrc/linear_rules.hpp, built with the host compiler."""

import collections
import ctypes
import functools
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2511_11505_amd", "csrc")
CUS = 256   # of gfx950
Plan = collections.namedtuple("Plan", "height width slices per mid")
FORWARD, INPUT, WEIGHT = (True, True), (True, False), (False, False)   # how A and B lie


@functools.lru_cache(maxsize=None)
def _lib():
    with tempfile.TemporaryDirectory() as d:
        so = os.path.join(d, "rules.so")
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, "-o", so,
                        os.path.join(HERE, "linear_rules_shim.cpp")], check=True)
        lib = ctypes.CDLL(so)
    i, q = ctypes.c_int, ctypes.c_longlong
    lib.rule_product.argtypes = [i, i, i, i, q, q, q, i, ctypes.POINTER(i)]
    lib.rule_product_ws.argtypes = [i, i, i, q, q, q, i]
    lib.rule_product_ws.restype = q
    lib.rule_tile_operand.argtypes = [ctypes.c_ulonglong, q, q]
    return lib


def plan(kind, M, N, K, dtype="bf16", tiles_ok=True, cus=CUS):
    out = (ctypes.c_int * 5)()
    _lib().rule_product(int(dtype == "bf16"), int(tiles_ok), *map(int, kind), M, N, K, cus, out)
    return Plan(*out)


def workspace(kind, M, N, K, dtype="bf16", cus=CUS):
    return _lib().rule_product_ws(int(dtype == "bf16"), *map(int, kind), M, N, K, cus)


def tile_operand(base, ld, row):
    return bool(_lib().rule_tile_operand(base, ld, row))


def route(kind, M, N, K, dtype="bf16", tiles_ok=True):
    """Kernel of a product: "few" is not the plan's to choose."""
    p = plan(kind, M, N, K, dtype, tiles_ok)
    name = f"tile{p.height}" if p.height else f"mid{p.mid}" if p.mid else "any"
    return name + ("+slices" if p.slices > 1 else "")

"""MXFP4 products over the whole range of sizes that the header names: what is planned, on the CPU, and the ends of the range on the GPU.  Tolerances
as derived in test_mx.py (16 waves at most, K/32 + 16 + 128 roundings: whatever the pieces that K comes in, a wave's sums are one chain)."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import test_mx as tmx
from oracle import mx_oracle as mo

gpu = pytest.mark.gpu

LDS = 160 << 10   # of a compute unit
LONGEST = 1 << 17  # K


@pytest.fixture(scope="module")
def mx():
    from paper_2601_16536_amd import binding, build, mx
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    mx.lib()
    return mx


def _how(kind):
    import torch
    return dict(x_mx=True) if kind == "mx" else dict(dtype=getattr(torch, kind))


def _product(mx, kind, rng, M, N, K):
    """(Y, its check's reference and terms)."""
    import torch
    wc, ws = tmx._random_mx(rng, N, K)
    if kind == "mx":
        xc, xs = tmx._random_mx(rng, M, K)
        return (mx.gemm_mx(tmx._torch(xc), tmx._torch(xs), tmx._torch(wc), tmx._torch(ws)), *mo.gemm(mo.values(xc, xs), wc, ws))
    X = tmx._torch(rng.standard_normal((M, K)) * (2.0 ** -6 if kind == "float16" else 1.0)).to(getattr(torch, kind))
    return (mx.gemm(X, tmx._torch(wc), tmx._torch(ws)), *mo.gemm(tmx._exact(X), wc, ws))


@pytest.mark.parametrize("kind", ["float16", "bfloat16", "mx"])
def test_every_plan_fits_lds(mx, kind):
    lengths = [*range(32, 1025, 32), *range(1056, LONGEST, 2080), 31488, 31520, 32768, 42784, 64288, 65280, 65312, 65536, LONGEST - 32, LONGEST]
    how = _how(kind)
    for M in (*range(1, 18), 32, 33, 100, 3000):
        for N in (1, 17, 1000, 4096, 4097, 16384, 70000):
            for K in lengths:
                lds, chunks = mx.query_lds(M, N, K, **how)
                assert 0 < lds <= LDS and 1 <= chunks <= (K + 255) // 256, (M, N, K, lds, chunks)


# where scales of a row fill much of LDS: X in pieces shorter than the threads could hold, down to one tile of W
LONG = [("mx", 16, 20, LONGEST), ("mx", 16, 100, 32768), ("mx", 8, 40, 42784), ("mx", 13, 33, LONGEST - 32), ("bfloat16", 1, 33, 65536), ("bfloat16", 8, 17, 64288),
        ("bfloat16", 6, 20, LONGEST), ("float16", 1, 18, LONGEST), ("float16", 3, 50, LONGEST - 96), ("float16", 8, 40, 65312)]


def test_the_longest_rows_are_of_the_kernel_for_few_rows(mx):
    assert {mx.query_tile(M, N, K, **_how(kind)) for kind, M, N, K in LONG} == {(16, 16)}


@gpu
@pytest.mark.parametrize("kind,M,N,K", LONG)
def test_longest_rows_match_the_oracle(mx, kind, M, N, K):
    Y, ref, terms = _product(mx, kind, np.random.default_rng([M, N, K]), M, N, K)
    tmx.check(Y, ref, terms, K, "M=%d N=%d K=%d %s" % (M, N, K, kind))

"""Every form of the MXFP4 products and of the experts' kernels that the library chooses by size, ragged in each dimension, against the oracle.  Tolerances
as derived in test_mx.py and test_moe.py: neither depends on the form (at most eight shares of K and 128 terms inside an instruction)."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import test_moe as tmoe
import test_mx as tmx
from oracle import mx_oracle as mo

gpu = pytest.mark.gpu

# (M, N, K): sizes that are no multiple of a tile, K that ends inside a stage, a step or a share
SHAPES = [(1, 33, 2080), (16, 6205, 4128), (13, 45, 416), (9, 6300, 160), (20, 6211, 288), (50, 2107, 1056), (33, 6205, 544), (70, 6203, 160), (150, 6210, 672), (1000, 1037, 288),
          (1003, 2111, 416), (1001, 4205, 160), (1000, 6203, 160), (1999, 8100, 224)]
ALL = {(16, 16), (16, 32), (32, 32), (32, 64), (64, 64), (64, 128), (128, 128), (128, 256)}
TILES = {"float16": ALL - {(128, 256)}, "bfloat16": ALL, "mx": ALL - {(32, 64)}}


@pytest.fixture(scope="module")
def mx():
    from paper_2601_16536_amd import binding, build, mx
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    mx.lib()
    return mx


def _kinds():
    import torch
    return {"float16": dict(dtype=torch.float16), "bfloat16": dict(dtype=torch.bfloat16), "mx": dict(x_mx=True)}


def test_the_shapes_reach_every_form(mx):
    for kind, how in _kinds().items():
        assert {mx.query_tile(M, N, K, **how) for M, N, K in SHAPES} == TILES[kind], kind


def test_query_refuses_what_the_products_refuse(mx):
    from paper_2601_16536_amd.binding import W4A16Error
    for M, N, K in ((0, 8, 32), (1, 0, 32), (1, 8, 40), (1, 8, (1 << 17) + 32)):
        with pytest.raises(W4A16Error):
            mx.query_tile(M, N, K)
    assert mx.query_tile(5, 40, 96) == (16, 16)


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "mx"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_every_form_matches_the_oracle(mx, kind, M, N, K):
    import torch
    rng = np.random.default_rng([M, N, K, 7])
    wc, ws = tmx._random_mx(rng, N, K)
    if kind == "mx":
        xc, xs = tmx._random_mx(rng, M, K)
        ref, terms = mo.gemm(mo.values(xc, xs), wc, ws)
        Y = mx.gemm_mx(tmx._torch(xc), tmx._torch(xs), tmx._torch(wc), tmx._torch(ws))
    else:
        X = tmx._torch(rng.standard_normal((M, K)) * (2.0 ** -4 if kind == "float16" else 1.0)).to(getattr(torch, kind))
        ref, terms = mo.gemm(tmx._exact(X), wc, ws)
        Y = mx.gemm(X, tmx._torch(wc), tmx._torch(ws))
    tmx.check(Y, ref, terms, K, "M=%d N=%d K=%d %s" % (M, N, K, kind))


@gpu
@pytest.mark.parametrize("kind", ["bfloat16", "mx"])
@pytest.mark.parametrize("M,N,K", [(70, 6203, 160), (1003, 2111, 416), (1001, 4205, 160)])
def test_not_a_number_stays_put_in_wide_tiles(mx, kind, M, N, K):
    import torch
    rng = np.random.default_rng(M)
    wc, ws = tmx._random_mx(rng, N, K)
    ws[N - 1, K // 32 - 1] = 255  # the last block of the last row: beside blocks and rows that are not there
    xc, xs = tmx._random_mx(rng, M, K)
    if kind == "mx":
        xs[M - 1, K // 32 - 1] = 255
        Y = mx.gemm_mx(tmx._torch(xc), tmx._torch(xs), tmx._torch(wc), tmx._torch(ws))
    else:
        X = tmx._torch(rng.standard_normal((M + 1, K)) * 0.01).to(torch.bfloat16)
        X[M - 1, K - 1] = float("inf")
        X[M] = float("nan")  # what lies behind the matrix
        Y = mx.gemm(X[:M], tmx._torch(wc), tmx._torch(ws))
    y = tmx._exact(Y)
    bad = ~np.isfinite(y)
    want = np.zeros((M, N), bool)
    want[:, N - 1] = True
    if kind == "mx":
        want[M - 1] = True
    else:
        want[M - 1] = mo.values(wc, ws)[:, K - 1] != 0  # infinity times an element
        want[M - 1] |= mo.values(wc, ws)[:, K - 1] == 0  # or NaN
    assert np.array_equal(bad, want)


# T, E, top_k, H, I: many tokens to an expert; I or H large enough for the tiles, neither a multiple of them
TILE_LAYERS = [(64, 4, 2, 96, 4128), (64, 4, 2, 8224, 96), (64, 16, 2, 160, 1056), (64, 16, 2, 2080, 160), (150, 8, 2, 224, 736), (70, 5, 5, 1312, 1248)]


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("T,E,top_k,H,I", TILE_LAYERS)
def test_experts_with_many_tokens_match_the_oracle(kind, T, E, top_k, H, I):
    import torch
    from paper_2601_16536_amd import moe
    tmoe.check_layer(moe, np.random.default_rng([T, E, H]), T, E, top_k, H, I, getattr(torch, kind), ldx=8 * (T % 3))


@gpu
def test_experts_with_many_tokens_unevenly(mx):
    """All tokens to one expert of four, ids out of range, an expert twice for a token."""
    import torch
    from paper_2601_16536_amd import moe
    rng = np.random.default_rng(6)
    for H, I in ((96, 4128), (8224, 96)):
        ids = np.full((64, 3), 2)
        ids[:, 1] = rng.integers(-2, 6, 64)
        ids[5] = [3, 3, 0]
        tmoe.check_layer(moe, rng, 64, 4, 3, H, I, torch.bfloat16, ids=ids)


@gpu
@pytest.mark.parametrize("apart", [0, 6, 22, 23, 24, 60])
@pytest.mark.parametrize("M,N,K", [(16, 6205, 4128), (50, 2107, 1056), (33, 6205, 1056), (150, 6210, 672), (1003, 2111, 416), (1000, 1037, 288)])
def test_blocks_beside_much_larger_ones(mx, M, N, K, apart):
    """FP16: blocks of W whose scales are 2^apart times their neighbours', where X is zero: the small ones' values are all there is."""
    import torch
    rng = np.random.default_rng([M, N, apart])
    wc, ws = tmx._random_mx(rng, N, K)
    large = np.arange(K // 32) % 4 == rng.integers(0, 4)
    ws[:] = rng.integers(119, 122, (N, 1)) + apart * large
    ws[::7] = 120  # rows without large blocks among them
    x = rng.standard_normal((M, K)).reshape(M, K // 32, 32)
    x[:, large] = 0.0
    X = tmx._torch(x.reshape(M, K)).to(torch.float16)
    ref, terms = mo.gemm(tmx._exact(X), wc, ws)
    tmx.check(mx.gemm(X, tmx._torch(wc), tmx._torch(ws)), ref, terms, K, "M=%d N=%d K=%d apart=%d" % (M, N, K, apart))

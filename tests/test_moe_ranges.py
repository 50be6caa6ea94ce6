"""The experts' layer over the whole range of sizes that the header names: what is planned, on the CPU, and the ends of the range on the GPU, with the
tolerances derived in test_moe.py (they do not depend on how a layer runs)."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import test_moe as tmoe

gpu = pytest.mark.gpu

LDS = 160 << 10   # of a compute unit
LONGEST = 1 << 15  # H and I


@pytest.fixture(scope="module")
def moe():
    from paper_2601_16536_amd import binding, build, moe
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    moe.lib()
    return moe


def test_every_plan_has_rows_and_fits_lds(moe):
    lengths = [32, 64, 96, 1024, 4096, 6144, 14336, *range(15008, LONGEST, 1056), 29664, 29696, 29728, 30080, LONGEST - 32, LONGEST]
    layers = [(1, 1), (1, 8), (8, 2), (8, 8), (64, 8), (128, 32), (1024, 5)]
    for E, top_k in layers:
        for T in (1, 2, 5, 16, 24, 31, 64, 65, 300, 1 << 21):
            for H in lengths:
                for I in lengths:
                    p = moe.query_plan(T, E, top_k, H, I)
                    where = (T, E, top_k, H, I, p)
                    assert 0 < p["lds_up"] <= LDS and 0 < p["lds_down"] <= LDS, where
                    assert p["rows_up"] >= 1 and p["rows_down"] >= 1, where


def test_query_refuses_what_the_layer_refuses(moe):
    from paper_2601_16536_amd import binding as b
    for sizes, status in (((0, 4, 2, 64, 64), b.ERR_SHAPE), ((1, 0, 2, 64, 64), b.ERR_SHAPE), ((1, 4, 33, 64, 64), b.ERR_SHAPE), ((1, 4, 2, 40, 64), b.ERR_SHAPE),
                          ((1, 4, 2, LONGEST + 32, 64), b.ERR_UNSUPPORTED), ((1, 4, 2, 64, LONGEST + 32), b.ERR_UNSUPPORTED), (((1 << 21) + 1, 4, 2, 64, 64), b.ERR_UNSUPPORTED)):
        with pytest.raises(b.W4A16Error) as e:
            moe.query_plan(*sizes)
        assert e.value.status == status


# rows of the hidden values that no longer fit LDS, the longest that do, one at a time; rows of X likewise
LONG = [(1, 2, 2, 32, LONGEST), (10, 4, 2, 96, LONGEST), (3, 4, 2, 64, 29728), (3, 2, 2, 64, 29664), (1, 2, 2, LONGEST, 32), (20, 3, 2, LONGEST - 32, 32), (64, 4, 2, 32, LONGEST - 32)]


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("T,E,top_k,H,I", LONG)
def test_longest_rows_match_the_oracle(moe, kind, T, E, top_k, H, I):
    import torch
    tmoe.check_layer(moe, np.random.default_rng([T, E, H]), T, E, top_k, H, I, getattr(torch, kind), ldx=8 * (T % 3))


@gpu
def test_more_tokens_than_one_grid_has_threads_for(moe):
    """Four tokens to 256 threads: 2^26 tokens are 2^32 threads.  Two experts, the larger logit's one wanted."""
    import torch
    T = 2 ** 26 + 5
    logits = torch.zeros(T, 2, dtype=torch.bfloat16, device="cuda")
    logits[::3, 1] = 1
    ids = torch.full((T, 1), 7, dtype=torch.int32, device="cuda")
    w = torch.full((T, 1), 7.0, device="cuda")
    moe.route(logits, 1, factor=0.5, out=(ids, w))
    assert torch.equal(ids[:, 0], logits[:, 1].int()) and bool((w == 0.5).all())

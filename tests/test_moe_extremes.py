"""The experts' layer where the hidden values leave the range of BF16 or of FP32."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import test_moe as tmoe
from oracle import mx_oracle as mo

gpu = pytest.mark.gpu

# one token and few rows to an expert (weights streamed), many rows (tiles)
TOKENS = [1, 5, 40]


@pytest.fixture(scope="module")
def moe():
    from paper_2601_16536_amd import binding, build, moe
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    moe.lib()
    return moe


def _layer(rng, E, H, I):
    """Weights that are 0 but for what a test sets: codes and scales of W13 [E, 2 I, H], and of W2 [E, H, I] with elements of both signs, none of them 0."""
    c13 = np.zeros((E, 2 * I, H // 2), np.uint8)
    s13 = np.full((E, 2 * I, H // 32), 127, np.uint8)
    q = rng.integers(1, 8, (E, H, I)) + 8 * rng.integers(0, 2, (E, H, I))
    c2 = (q[..., 0::2] | (q[..., 1::2] << 4)).astype(np.uint8)
    s2 = rng.integers(96, 99, (E, H, I // 32)).astype(np.uint8)
    return c13, s13, c2, s2


def _run(moe, x, ids, w, c13, s13, c2, s2):
    t = tmoe._torch
    return tmoe._exact(moe.experts(x, t(ids.astype(np.int32)), t(w), t(c13), t(s13), t(c2), t(s2)))


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("sign", [1, -1])
def test_hidden_values_beyond_bf16(moe, kind, T, sign):
    """h = +-(2^128 - 2^112), an FP32 number above BF16's largest, in hidden value 7; the others are 0.  g = 2^64, which SiLU leaves as it is; u = (1 - 2^-8)(2^64 + 2^56);
    both, h and h's two terms are exact, so an output is off by its rounding alone, half a unit in the last place (the FP32 sum has one term in two parts: 2^-23)."""
    import torch
    rng = np.random.default_rng(T)
    E, H, I, at = 2, 96, 64, 7
    c13, s13, c2, s2 = _layer(rng, E, H, I)
    one = 2 if sign > 0 else 10                     # the code of 1 or -1
    c13[:, at, 0] = 2 << 4                          # gate: x[1] = 1, times 2^64
    s13[:, at, 0] = 127 + 64
    c13[:, I + at, 0] = one                         # up: x[0] times 2^64 and x[32] times 2^56
    c13[:, I + at, 16] = one
    s13[:, I + at, :2] = 127 + 64, 127 + 56
    if kind == "float16":
        s2 -= 24                                    # FP16's range
    x = np.zeros((T, H))
    x[:, 1] = 1.0
    x[:, [0, 32]] = 1.0 - 2.0 ** -8
    X = tmoe._torch(x).to(getattr(torch, kind))
    ids = rng.integers(0, E, (T, 1))
    w = np.full((T, 1), 2.0 ** -97 if kind == "bfloat16" else 2.0 ** -73, np.float32)  # results of about 1
    Y = _run(moe, X, ids, w, c13, s13, c2, s2)
    h = sign * (2.0 ** 128 - 2.0 ** 112)
    want = float(w[0, 0]) * h * mo.values(c2, s2)[ids[:, 0], :, at]
    assert np.all(np.abs(want) < 60000) and np.all(np.abs(want) > 2.0 ** -10)
    half = 2.0 ** -11 if kind == "float16" else 2.0 ** -8
    assert np.all(np.abs(Y - want) <= (half + 2.0 ** -22) * np.abs(want))


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("sign", [1, -1])
def test_hidden_values_beyond_fp32(moe, kind, T, sign):
    """Finite x and weights whose hidden value 7 is about 2^160: infinite in FP32, and with it every output of a weight that is not 0, by its sign; a token of another expert,
    whose weights are 0, has zeros."""
    import torch
    rng = np.random.default_rng(T)
    E, H, I, at = 2, 96, 64, 7
    c13, s13, c2, s2 = _layer(rng, E, H, I)
    c13[0, at, 0], s13[0, at, 0] = 2, 127 + 80
    c13[0, I + at, 0], s13[0, I + at, 0] = 2 if sign > 0 else 10, 127 + 80
    x = np.zeros((T, H))
    x[:, 0] = 1.0
    ids = np.zeros((T, 1), np.int64)
    ids[1::2] = 1
    Y = _run(moe, tmoe._torch(x).to(getattr(torch, kind)), ids, np.ones((T, 1), np.float32), c13, s13, c2, s2)
    want = np.zeros((T, H))
    want[::2] = sign * np.sign(mo.values(c2, s2)[0, :, at]) * np.inf
    assert np.array_equal(Y, want)


@gpu
@pytest.mark.parametrize("T", TOKENS)
def test_infinite_x(moe, T):
    """x[5] infinite, every weight that it meets positive: g, u and h are infinite, an output the sum of infinities of W2's signs: one sign to a row here."""
    import torch
    rng = np.random.default_rng(T)
    E, H, I = 2, 96, 64
    c13, s13, c2, s2 = _layer(rng, E, H, I)
    c13[:] = 0x22
    c2 = (c2 & 0x77) | (rng.integers(0, 2, (E, H, 1)) * 0x88).astype(np.uint8)
    x = rng.standard_normal((T, H))
    x[:, 5] = np.inf
    ids = rng.integers(0, E, (T, 1))
    Y = _run(moe, tmoe._torch(x).to(torch.bfloat16), ids, np.ones((T, 1), np.float32), c13, s13, c2, s2)
    assert np.array_equal(Y, np.sign(mo.values(c2, s2)[ids[:, 0], :, 0]) * np.inf)


# ---- routing: sigmoids below FP32's range ----

def test_oracle_divides_sigmoids_that_vanish():
    for l in (0.0, -50.0, -89.0, -800.0, -1e30):
        _, w = mo.route([[l] * 8], 4, sigmoid=True)
        assert np.allclose(w, 0.25, rtol=1e-12)
    _, w = mo.route([[-800.0, -801.0, -802.0]], 2, sigmoid=True)
    assert np.allclose(w, [[1 / (1 + np.exp(-1.0)), 1 / (1 + np.exp(1.0))]], rtol=1e-12)
    rng = np.random.default_rng(1)
    l = rng.standard_normal((5, 9)) * 3
    ids, w = mo.route(l, 3, sigmoid=True)
    s = np.take_along_axis(1 / (1 + np.exp(-l)), ids, 1)
    assert np.allclose(w, s / s.sum(1, keepdims=True), rtol=1e-12)


@gpu
@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("E", [8, 130, 700])
def test_renormalized_sigmoids_of_very_negative_logits(moe, kind, E):
    """The tolerance of test_moe.py: at most 32 terms of 2 roundings each in a sum, and l - top rounded: |l - top| <= 104 where the result is an FP32 number, 52 of 2^-23;
    below (32 / 2 + 8 + 52) 2^-23."""
    import torch
    rng = np.random.default_rng(E)
    rows = np.stack([np.full(E, l) for l in (-1.0, -50.0, -88.0, -89.0, -90.0, -100.0, -104.0, -300.0, -6e4)])
    near = -rng.uniform(80, 200, (40, 1)) - rng.uniform(0, 20, (40, E))       # some beside each other, all beyond the range
    wide = -np.exp(rng.uniform(0, 10, (40, E)))                               # of every size
    both = rng.standard_normal((40, E)) * 60                                  # a positive one among them
    holes = near.copy()
    holes[rng.random((40, E)) < 0.9] = -np.inf
    logits = tmoe._torch(np.concatenate([rows, near, wide, both, holes])).to(getattr(torch, kind))
    for renormalize in (True, False):
        ids, w = moe.route(logits, 8, scoring="sigmoid", renormalize=renormalize, factor=2.5)
        want, ww = mo.route(tmoe._exact(logits), 8, True, renormalize, 2.5)
        assert np.array_equal(ids.cpu().numpy(), want)
        got = tmoe._exact(w)
        assert np.all(np.abs(got - ww) <= (32 / 2 + 8 + 52) * 2.0 ** -23 * ww + 2.5 * 2.0 ** -126)
        if renormalize:
            assert np.allclose(got[(want >= 0).any(1)].sum(1), 2.5, rtol=1e-5)


# ---- a workspace that is none ----

@gpu
def test_workspace_on_the_host_or_with_gaps_is_refused(moe):
    import torch
    from paper_2601_16536_amd import mx
    (c13, s13), (c2, s2) = mx.quantize(torch.zeros(4, 64, 64, device="cuda")), mx.quantize(torch.zeros(4, 64, 32, device="cuda"))
    x = torch.zeros(2, 64, dtype=torch.float16, device="cuda")
    ids, w = moe.route(torch.zeros(2, 4, device="cuda"), 2)
    need = moe.workspace_bytes(2, 2, 64, 32)
    for workspace in (torch.empty(need, dtype=torch.uint8), torch.empty(need, dtype=torch.uint8, pin_memory=True), torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(TypeError):
            moe.experts(x, ids, w, c13, s13, c2, s2, workspace=workspace)
    flat = torch.empty(need // 4, device="cuda")  # of any type
    assert not bool(moe.experts(x, ids, w, c13, s13, c2, s2, workspace=flat).any())

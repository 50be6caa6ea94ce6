"""The mixture-of-experts layer: pins of the CPU oracle, refusals, then the HIP kernels against the oracle.

Tolerances.  Routing: ids exactly; a weight is at most a quotient of two sums of up to 1024 exponentials or a sigmoid, each exponential within
two units in the last place and each addition within half of one: (1024 / 2 + 8) 2^-23 relative at the worst; the sums' terms are positive.

Experts, per output, all bounds absolute: a sum of K products in FP32 is off by at most c(K) = (K/32 + 32 + 16) 2^-23 times the sum of its terms'
magnitudes (as many roundings as there are partial sums in a chain, the terms inside an instruction and the waves, each up to 2^-23).  So gate
and up are off by dg = c(H) |W1||x|, du = c(H) |W3||x|.  |act'| <= 1.13 for both activations, and act itself is computed to 2^-20 max(|g|, |act|).
h = act(g) u then is off by  dh = (1.13 dg + 2^-20 |g|) (|u| + du) + |act| du + 2^-16 |h|  (the last: two terms of eight bits, and the product's
rounding).  The second product adds  |weight| (|W2| dh + c(I) |W2| |h|), the sum over the experts 2^-23 (top_k + 16) of its terms,
the output half a unit in its last place: 2^-11 (FP16; 2^-25 at least) or 2^-8 (BF16).
"""
import os

import numpy as np
import pytest

from oracle import mx_oracle as mo

gpu = pytest.mark.gpu


# ---- the oracle's pins ----

def test_oracle_routes_worked_rows():
    nan, inf = np.nan, np.inf
    rows = [[1, 3, 3, 2], [-inf, 5, -inf, -inf], [-inf] * 4, [0.0, -0.0, 0.0, -0.0], [1, nan, 7, 2]]
    ids, w = mo.route(rows, 3)
    assert ids.tolist() == [[1, 2, 3], [1, -1, -1], [-1, -1, -1], [0, 1, 2], [1, 2, 3]]
    e = np.exp(-1.0)
    assert np.allclose(w[0], [1 / (2 + e), 1 / (2 + e), e / (2 + e)]) and w[1].tolist() == [1, 0, 0] and w[2].tolist() == [0, 0, 0]
    assert np.allclose(w[3], 1 / 3) and np.isnan(w[4]).all()
    _, all_ = mo.route(rows[:1], 3, renormalize=False, factor=2.0)
    assert np.allclose(all_[0], np.array([1, 1, e]) * 2 / (2 + e + np.exp(-2.0)))
    _, sig = mo.route(rows[:1], 2, sigmoid=True, renormalize=False)
    assert np.allclose(sig[0], 1 / (1 + np.exp(-3.0)))


def test_oracle_experts_by_hand():
    """One expert whose gate is 0 or large: SiLU is 0 or the identity."""
    W13 = np.zeros((2, 4, 2))
    W13[1] = [[1, 0], [0, 1], [2, 0], [0, 3]]   # gate rows, then up rows
    W2 = np.zeros((2, 2, 2))
    W2[1] = [[1, 1], [0, 1]]
    X = np.array([[50.0, 0.0], [0.0, 60.0], [50.0, 60.0]])
    ids = np.array([[1, -1], [1, 1], [0, 1]])
    w = np.array([[0.5, 9.0], [1.0, 2.0], [4.0, 1.0]])
    Y = mo.experts(X, ids, w, W13, W2)
    a, b = 50.0 * 100.0, 60.0 * 180.0
    assert np.allclose(Y, [[0.5 * a, 0.0], [3 * b, 3 * b], [a + b, b]])
    assert abs(mo.activate(np.float64(1.0), gelu=True) - 0.8411919906082768) < 1e-12


# ---- refusals ----

@pytest.fixture(scope="module")
def moe():
    from paper_2601_16536_amd import binding, build, moe
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    moe.lib()
    return moe


def test_header_functions_are_exported(moe):
    import re
    from paper_2601_16536_amd import binding
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "w4a16_mx.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(w4a16_moe_[a-z0-9_]+)\s*\(", text))
    assert declared == set(moe.EXPORTS)
    for name in declared:
        assert getattr(binding.lib(), name) is not None


def test_argument_checks_need_no_gpu(moe):
    from paper_2601_16536_amd import binding as b
    r = moe.lib().w4a16_moe_route

    def route(logits=16, dtype=2, T=1, E=8, ld=8, top_k=2, scoring=0, ids=16, weights=16):
        return r(logits, dtype, T, E, ld, top_k, scoring, 1, 1.0, ids, weights, 0)
    assert route(logits=0, T=0) == b.OK
    assert route(logits=0) == b.ERR_NULL and route(ids=0) == b.ERR_NULL and route(weights=0) == b.ERR_NULL
    assert route(dtype=3) == b.ERR_SHAPE and route(T=-1) == b.ERR_SHAPE and route(E=0, top_k=1) == b.ERR_SHAPE
    assert route(E=1025, ld=1025) == b.ERR_SHAPE and route(top_k=0) == b.ERR_SHAPE and route(top_k=9) == b.ERR_SHAPE
    assert route(E=64, ld=64, top_k=33) == b.ERR_SHAPE and route(T=2, ld=7) == b.ERR_SHAPE and route(scoring=2) == b.ERR_SHAPE
    assert route(logits=18) == b.ERR_ALIGN and route(ids=18) == b.ERR_ALIGN and route(logits=17, dtype=0) == b.ERR_ALIGN
    x = moe.lib().w4a16_moe_experts

    def experts(X=16, dtype=1, ldx=64, ids=16, weights=16, c13=16, s13=16, c2=16, s2=16, T=2, E=4, top_k=2, H=64, I=32, act=0, Y=16, ldy=64, ws=256,
                ws_bytes=2 * 2 * 96 * 4):
        return x(X, dtype, ldx, ids, weights, c13, s13, c2, s2, T, E, top_k, H, I, act, Y, ldy, ws, ws_bytes, 0)
    assert experts(X=0, T=0) == b.OK
    for name in ("X", "ids", "weights", "c13", "s13", "c2", "s2", "Y", "ws"):
        assert experts(**{name: 0}) == b.ERR_NULL
    for bad in (dict(dtype=2), dict(T=-1), dict(E=0), dict(E=1025), dict(top_k=0), dict(top_k=33), dict(H=40), dict(I=0), dict(I=48), dict(act=2),
                dict(ldx=32), dict(ldy=63)):
        assert experts(**bad) == b.ERR_SHAPE, bad
    for bad in (dict(X=24), dict(ids=18), dict(c13=24), dict(c2=20), dict(Y=17), dict(ws=128), dict(ldx=68)):
        assert experts(**bad) == b.ERR_ALIGN, bad
    assert experts(ws_bytes=2 * 2 * 96 * 4 - 1) == b.ERR_WORKSPACE
    assert experts(H=1 << 16, ldx=1 << 16, ldy=1 << 16, ws_bytes=1 << 40) == b.ERR_UNSUPPORTED
    assert moe.workspace_bytes(2, 2, 64, 32) == 1536 and moe.workspace_bytes(0, 2, 64, 32) == 0


# ---- the kernels ----

def _torch(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _exact(t):
    import torch
    return t.detach().to(torch.float64).cpu().numpy()


@gpu
@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("T,E,top_k", [(1, 1, 1), (1, 8, 2), (3, 64, 6), (5, 65, 8), (130, 128, 8), (7, 200, 1), (33, 256, 8), (4, 511, 32), (9, 1024, 5), (2, 7, 7)])
def test_route_matches_the_oracle(moe, kind, T, E, top_k):
    import torch
    rng = np.random.default_rng([T, E])
    big = _torch(1.5 * rng.standard_normal((T, E + 3))).to(getattr(torch, kind))
    for logits in (big[:, :E].contiguous(), big[:, 1:E + 1]):
        for scoring in ("softmax", "sigmoid"):
            for renormalize in (True, False):
                ids, w = moe.route(logits, top_k, scoring=scoring, renormalize=renormalize, factor=1.5)
                want, ww = mo.route(_exact(logits), top_k, scoring == "sigmoid", renormalize, 1.5)
                assert np.array_equal(ids.cpu().numpy(), want)
                assert np.all(np.abs(_exact(w) - ww) <= (1024 / 2 + 8) * 2.0 ** -23 * np.abs(ww) + 2.0 ** -126)


@gpu
def test_route_ties_and_special_values(moe):
    import torch
    inf, nan = np.inf, np.nan
    rng = np.random.default_rng(5)
    for E in (16, 130, 700):
        rows = np.zeros((12, E), np.float32)
        rows[1] = rng.integers(-1, 2, E)                 # many ties
        rows[2, ::2] = -0.0                              # zeros of both signs are equal
        rows[3] = -inf
        rows[4] = -inf
        rows[4, E - 1] = 3
        rows[5, 3] = nan
        rows[6, [2, 5]] = inf
        rows[7] = rng.choice([-inf, 1.0, 2.0], E)
        rows[8] = -3.4e38
        rows[8, 4] = 3.4e38
        rows[9] = 1e-45 * np.arange(E)                   # subnormal numbers in order
        rows[10] = -1e30
        rows[11, E - 1] = nan
        rows[11, 0] = nan
        for scoring in ("softmax", "sigmoid"):
            for renormalize in (True, False):
                ids, w = moe.route(_torch(rows), 4, scoring=scoring, renormalize=renormalize)
                want, ww = mo.route(rows, 4, scoring == "sigmoid", renormalize)
                assert np.array_equal(ids.cpu().numpy(), want)
                got = _exact(w)
                assert np.array_equal(np.isnan(got), np.isnan(ww))
                ok = np.isnan(ww) | (np.abs(got - ww) <= (1024 / 2 + 8) * 2.0 ** -23 * np.abs(ww) + 2.0 ** -126)
                assert ok.all()


def _random_mx(rng, lead, K, spread=2):
    codes = rng.integers(0, 256, (*lead, K // 2), dtype=np.uint8)
    middle = 127 - int(np.log2(K) / 2) - 2
    scales = rng.integers(middle - spread, middle + spread + 1, (*lead, K // 32)).astype(np.uint8)
    return codes, scales


def _bound(X, ids, w, W13, W2, gelu, top_k, dtype, Y):
    """The tolerance derived above, per output."""
    import torch
    H, I = W2.shape[1:]
    c = lambda K: (K / 32 + 32 + 16) * 2.0 ** -23
    D = np.zeros_like(X)
    terms = np.zeros_like(X)
    for t in range(X.shape[0]):
        for j in range(ids.shape[1]):
            e = ids[t, j]
            if not 0 <= e < W13.shape[0]:
                continue
            both, mags = W13[e] @ X[t], np.abs(W13[e]) @ np.abs(X[t])
            g, u = both[:I], both[I:]
            dg, du = c(H) * mags[:I], c(H) * mags[I:]
            act = np.abs(mo.activate(g, gelu))
            h = act * np.abs(u)
            dh = (1.13 * dg + 2.0 ** -20 * np.maximum(np.abs(g), act)) * (np.abs(u) + du) + act * du + 2.0 ** -16 * h
            a2 = np.abs(W2[e])
            D[t] += np.abs(w[t, j]) * (a2 @ dh + c(I) * (a2 @ (h + dh)))
            terms[t] += np.abs(w[t, j]) * (a2 @ (h + dh))
    D += 2.0 ** -23 * (top_k + 16) * terms
    half, least = (2.0 ** -11, 2.0 ** -25) if dtype == torch.float16 else (2.0 ** -8, 0.0)
    return D + half * (np.abs(Y) + D) + least


def check_layer(moe, rng, T, E, top_k, H, I, dtype, activation="silu", ids=None, ldx=0):
    import torch
    c13, s13 = _random_mx(rng, (E, 2 * I), H)
    c2, s2 = _random_mx(rng, (E, H), I)
    X = _torch(rng.standard_normal((T, H + ldx))).to(dtype)[:, :H]
    if ids is None:
        ids = np.stack([rng.choice(E, top_k, replace=False) for _ in range(T)])
    w = rng.random((T, top_k)).astype(np.float32)
    Y = moe.experts(X, _torch(ids.astype(np.int32)), _torch(w), _torch(c13), _torch(s13), _torch(c2), _torch(s2), activation=activation)
    W13, W2 = mo.values(c13, s13), mo.values(c2, s2)
    x = _exact(X)
    ref = mo.experts(x, ids, w.astype(np.float64), W13, W2, activation == "gelu")
    tol = _bound(x, ids, w.astype(np.float64), W13, W2, activation == "gelu", top_k, dtype, ref)
    bad = ~(np.abs(_exact(Y) - ref) <= tol)
    assert not bad.any(), "%d outputs off, first at %r" % (bad.sum(), np.argwhere(bad)[0].tolist())
    return Y


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("T,E,top_k,H,I", [(1, 1, 1, 32, 32), (1, 8, 2, 128, 96), (1, 64, 8, 512, 256), (2, 5, 5, 96, 160), (7, 16, 3, 288, 64), (16, 4, 2, 256, 128),
                                          (17, 3, 1, 160, 224), (40, 2, 2, 128, 64), (64, 32, 4, 64, 128), (65, 9, 2, 96, 96), (150, 6, 3, 64, 32)])
def test_experts_match_the_oracle(moe, kind, T, E, top_k, H, I):
    import torch
    check_layer(moe, np.random.default_rng([T, E, H]), T, E, top_k, H, I, getattr(torch, kind), ldx=8 * (T % 3))


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("T,E,top_k,H,I", [(66, 128, 1, 96, 64), (256, 5, 3, 96, 64), (257, 4, 2, 32, 96), (300, 40, 6, 288, 160), (130, 48, 32, 160, 32), (10, 4, 2, 6016, 64)])
def test_experts_of_long_batches(moe, kind, T, E, top_k, H, I):
    import torch
    check_layer(moe, np.random.default_rng([T, E, H]), T, E, top_k, H, I, getattr(torch, kind), ldx=8 * (T % 3))


@gpu
def test_gelu(moe):
    import torch
    for T in (1, 20):
        check_layer(moe, np.random.default_rng(T), T, 6, 2, 128, 160, torch.bfloat16, activation="gelu")


@gpu
def test_uneven_and_missing_experts(moe):
    """All tokens to one expert, tokens without any, ids out of range, an expert twice for one token, experts 0 and the last."""
    import torch
    rng = np.random.default_rng(3)
    T, E, top_k, H, I = 50, 300, 4, 96, 64
    ids = np.full((T, top_k), 7)
    ids[:, 1] = -1
    ids[:, 2] = E + 5
    ids[:, 3] = rng.integers(0, E, T)
    check_layer(moe, rng, T, E, top_k, H, I, torch.bfloat16, ids=ids)
    ids = np.full((T, top_k), -1)
    ids[3] = [0, E - 1, 0, 0]
    ids[9, 2] = E - 1
    Y = check_layer(moe, rng, T, E, top_k, H, I, torch.float16, ids=ids)
    empty = np.ones(T, bool)
    empty[[3, 9]] = False
    assert not _exact(Y)[empty].any()
    ids = np.stack([np.arange(32) + t for t in range(70)])  # top_k at its limit, more than a block of tokens
    check_layer(moe, rng, 70, 128, 32, 64, 32, torch.bfloat16, ids=ids)


@gpu
def test_weights_of_places_without_expert_are_not_read_and_nan_stays(moe):
    import torch
    rng = np.random.default_rng(4)
    T, E, H, I = 20, 4, 64, 64
    c13, s13 = map(_torch, _random_mx(rng, (E, 2 * I), H))
    c2, s2 = map(_torch, _random_mx(rng, (E, H), I))
    s2[2, 5] = 255                                     # row 5 of expert 2
    X = _torch(rng.standard_normal((T, H))).to(torch.bfloat16)
    X[4, 3] = float("nan")
    ids = torch.zeros(T, 2, dtype=torch.int32, device="cuda")
    ids[:, 1] = -1
    ids[9, 1] = 2
    w = torch.ones(T, 2, device="cuda")
    w[:, 1] = float("nan")
    w[9, 1] = 1.0
    Y = _exact(moe.experts(X, ids, w, c13, s13, c2, s2))
    want = np.zeros((T, H), bool)
    want[4] = True
    want[9, 5] = True
    assert np.array_equal(np.isnan(Y), want)


@gpu
@pytest.mark.parametrize("T", [1, 30, 100])
def test_reproducible_streams_graphs_and_canaries(moe, T):
    import torch
    from paper_2601_16536_amd import mx
    rng = np.random.default_rng(T)
    E, top_k, H, I = 16, 4, 256, 160
    W13, W2 = (_torch(rng.standard_normal(s)).float() * 0.1 for s in ((E, 2 * I, H), (E, H, I)))
    (c13, s13), (c2, s2) = mx.quantize(W13), mx.quantize(W2)
    assert c13.shape == (E, 2 * I, H // 2) and s2.shape == (E, H, I // 32)
    X = _torch(rng.standard_normal((T, H))).to(torch.bfloat16)
    logits = _torch(rng.standard_normal((T, E))).float()

    def layer(**kw):
        ids, w = moe.route(logits, top_k, stream=kw.get("stream"))
        return moe.experts(X, ids, w, c13, s13, c2, s2, **kw)
    want = layer()
    for _ in range(5):
        assert torch.equal(want, layer())
    need = moe.workspace_bytes(T, top_k, H, I)
    ws = torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda")
    flat = torch.full((16 + T * (H + 6),), 9.0, dtype=torch.bfloat16, device="cuda")
    out = flat[5:5 + T * (H + 6)].view(T, H + 6)[:, :H]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    layer(out=out, workspace=ws[256:256 + need], stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    out.fill_(9.0)
    assert bool((flat == 9.0).all()) and bool((ws[:256] == 255).all()) and bool((ws[256 + need:] == 255).all())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer()
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        torch.randn(1000, device="cuda").sum().item()


@gpu
def test_binding_refuses_what_does_not_fit(moe):
    import torch
    from paper_2601_16536_amd import mx
    assert moe.route(torch.empty(0, 8, device="cuda"), 2)[0].shape == (0, 2)
    x = torch.zeros(2, 64, dtype=torch.float16, device="cuda")
    (c13, s13), (c2, s2) = mx.quantize(torch.zeros(4, 64, 64, device="cuda")), mx.quantize(torch.zeros(4, 64, 32, device="cuda"))
    ids, w = moe.route(torch.zeros(2, 4, device="cuda"), 2)
    assert moe.experts(x, ids, w, c13, s13, c2, s2).shape == (2, 64)
    assert moe.experts(x[:0], ids[:0], w[:0], c13, s13, c2, s2).shape == (0, 64)
    with pytest.raises(ValueError):
        moe.route(torch.zeros(2, 4, device="cuda"), 5)
    with pytest.raises(TypeError):
        moe.route(torch.zeros(2, 4), 2)
    with pytest.raises(TypeError):
        moe.experts(x, ids.long(), w, c13, s13, c2, s2)
    with pytest.raises(ValueError):
        moe.experts(x, ids[:1], w[:1], c13, s13, c2, s2)
    with pytest.raises(ValueError):
        moe.experts(x, ids, w, c13, s13, c13, s13)
    with pytest.raises(ValueError):
        moe.experts(x, ids, w, c13, s13, c2, s2, activation="relu")
    with pytest.raises(ValueError):
        moe.experts(x, ids, w, c13, s13, c2, s2, stream=torch.cuda.Stream())
    with pytest.raises(Exception):
        moe.experts(x, ids, w, c13, s13, c2, s2, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))

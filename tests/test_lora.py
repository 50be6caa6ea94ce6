"""Low-rank adapters beside a shared projection: pins of the CPU oracle, refusals, then the HIP kernels against the oracle.

Tolerances, per output, all bounds absolute, |.| of a matrix its values' magnitudes.  H = s X A^T: 16-bit products are exact in FP32; at most K / 32 + 32 roundings in a chain
of matrix instructions, each of up to 32 products, and 36 where waves and slices of K meet, each below 2^-23 |s| |X| |A|^T; then the multiplication by s:
    dH = ((K / 32 + 68) 2^-23 + 2^-24) |s| |X| |A|^T,   dG the same with dY, B and N.
H B^T is summed over R; a value of H goes in as two or three 16-bit numbers whose sum is off by 2^-22 |H| at most, so there are at most 3 R products and roundings below 2^-23 |H| |B|^T each,
and what the sum is added to adds one more:
    out: dH |B|^T + 2^-23 (3 R + 3) |H| |B|^T + 2^-23 |out|, then half a unit in the last place.
dX the same with G and A.  dA = G^T X over n rows, a value of G as three bfloat16 numbers (two of eight bits each, off by 2^-16, for gradients in 16 bits), one of X as up to two: 6 n products
and roundings below 2^-23 |G|^T |X|, one after the other at the worst:
    dA: dG^T |X| + (2^-23 (6 n + 2) + 2^-16, or 2^-24 for FP32) |G|^T |X|, dB with H and dY; then half a unit in the last place of a 16-bit type.
"""
import math
import os

import numpy as np
import pytest

from oracle import grouped_oracle as go

gpu = pytest.mark.gpu
KINDS = ["float16", "bfloat16"]


# ---- the oracle's pins ----

def test_oracle_by_hand():
    A = np.array([[[1.0, 0.0, 1.0]], [[0.0, 2.0, 0.0]]])
    B = np.array([[[1.0], [2.0]], [[3.0], [0.0]]])
    X, Y = np.array([[1.0, 2.0, 3.0], [1.0, 1.0, 1.0], [5.0, 5.0, 5.0]]), np.ones((3, 2))
    out = go.lora_add(Y, X, A, B, [0, 1, -1], [0.5, 2.0])
    assert out.tolist() == [[1 + 0.5 * 4, 1 + 0.5 * 8], [1 + 2 * 6, 1], [1, 1]]


def test_oracle_gradients_are_differences():
    """The sum of C * out is linear in each of X, A and B."""
    rng = np.random.default_rng(1)
    M, L, R, K, N = 6, 3, 2, 5, 4
    Y, X, A, B, C = (rng.normal(size=s) for s in ((M, N), (M, K), (L, R, K), (L, N, R), (M, N)))
    ids, scaling = [2, 0, -1, 2, 3, 0], [1.0, 2.0, 0.5]
    base = rng.normal(size=(M, K))
    dX, dA, dB = go.lora_grad(C, X, A, B, ids, scaling, base)
    f = lambda x, a, b: (C * go.lora_add(Y, x, a, b, ids, scaling)).sum()
    for got, change in (((dX - base), lambda d: f(X + d, A, B) - f(X - d, A, B)), (dA, lambda d: f(X, A + d, B) - f(X, A - d, B)), (dB, lambda d: f(X, A, B + d) - f(X, A, B - d))):
        d = rng.normal(size=got.shape)
        assert math.isclose((got * d).sum(), change(d) / 2, rel_tol=1e-12)


# ---- refusals ----

@pytest.fixture(scope="module")
def lora():
    from paper_2601_16536_amd import binding, build, lora
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    lora.lib()
    return lora


def test_argument_checks_need_no_gpu(lora):
    from paper_2601_16536_amd import binding as b
    L = lora.lib()
    # Y, ldy, X, type, ldx, A, B, ids, scaling, M, L, R, K, N, out, ldo, workspace, bytes, stream
    good = dict(Y=16, ldy=32, X=16, type=0, ldx=64, A=16, B=16, ids=16, scaling=16, M=4, L=2, R=8, K=64, N=32, out=32, ldo=32, workspace=256, bytes=1 << 20, stream=0)

    def add(**change):
        return L.w4a16_lora_add(*dict(good, **change).values())
    assert add(M=0, Y=0, X=0, out=0, workspace=0) == b.OK
    for bad in (dict(type=2), dict(M=-1), dict(L=0), dict(L=1025), dict(R=0), dict(R=12), dict(R=136), dict(K=60), dict(N=4), dict(ldy=24), dict(ldx=56), dict(ldo=24),
                dict(out=16, ldo=40)):
        assert add(**bad) == b.ERR_SHAPE, bad
    for bad in (dict(Y=0), dict(X=0), dict(A=0), dict(B=0), dict(ids=0), dict(out=0), dict(workspace=0)):
        assert add(**bad) == b.ERR_NULL, bad
    for bad in (dict(Y=24), dict(X=24), dict(A=24), dict(B=24), dict(out=24), dict(ids=18), dict(scaling=18), dict(workspace=128), dict(ldx=68), dict(ldy=36), dict(ldo=36)):
        assert add(**bad) == b.ERR_ALIGN, bad
    for bad in (dict(K=(1 << 17) + 8, ldx=1 << 18), dict(N=(1 << 17) + 8, ldy=1 << 18, ldo=1 << 18), dict(M=(1 << 20) + 1), dict(ldx=1 << 23)):
        assert add(**bad) == b.ERR_UNSUPPORTED, bad
    need = lora.workspace_bytes(4, 2, 8, 64, 32)
    assert need > 0 and add(bytes=need - 1) == b.ERR_WORKSPACE
    # dY, ldy, X, type, ldx, A, B, ids, scaling, M, L, R, K, N, dX, lddx, dX_out, ldo, dA, dB, grad type, workspace, bytes, stream
    good2 = dict(dY=16, ldy=32, X=16, type=0, ldx=64, A=16, B=16, ids=16, scaling=0, M=4, L=2, R=8, K=64, N=32, dX=16, lddx=64, out=32, ldo=64, dA=16, dB=16, grad=2, workspace=256,
                 bytes=1 << 20, stream=0)

    def grad(**change):
        return L.w4a16_lora_grad(*dict(good2, **change).values())
    for bad in (dict(type=2), dict(grad=1), dict(M=-1), dict(L=0), dict(R=4), dict(K=60), dict(N=4), dict(ldy=24), dict(ldx=56), dict(lddx=56), dict(ldo=56), dict(out=16, ldo=72)):
        assert grad(**bad) == b.ERR_SHAPE, bad
    for bad in (dict(dY=0), dict(X=0), dict(A=0), dict(B=0), dict(ids=0), dict(out=0), dict(dA=0), dict(dB=0), dict(workspace=0), dict(M=0, dA=0)):
        assert grad(**bad) == b.ERR_NULL, bad
    for bad in (dict(dY=24), dict(X=24), dict(A=24), dict(B=24), dict(dX=24), dict(out=24), dict(dA=24), dict(dB=24), dict(ids=18), dict(workspace=128), dict(lddx=68)):
        assert grad(**bad) == b.ERR_ALIGN, bad
    need = lora.workspace_bytes(4, 2, 8, 64, 32, grad=True)
    assert need > 0 and grad(bytes=need - 1) == b.ERR_WORKSPACE


def test_every_size_has_a_workspace(lora):
    for M in (0, 1, 17, 64, 65, 1000, 1 << 20):
        for L in (1, 3, 64, 1024):
            for R in (8, 24, 128):
                for K, N in ((8, 8), (8192, 136), (1 << 17, 1 << 17)):
                    h = 0 if M == 0 else M * R * 4
                    assert lora.workspace_bytes(M, L, R, K, N) >= h and lora.workspace_bytes(M, L, R, K, N, grad=True) >= 2 * h + 4 * (L + 1 + M)
    assert lora.workspace_bytes(4, 2, 12, 64, 64) == 0


def test_binding_refuses_host_tensors(lora):
    import torch
    z = lambda *s: torch.zeros(*s, dtype=torch.float16)
    with pytest.raises(TypeError):
        lora.add(z(4, 32), z(4, 64), z(2, 8, 64), z(2, 32, 8), torch.zeros(4, dtype=torch.int32))


# ---- the kernels ----

def exact(t):
    import torch
    return t.detach().to(torch.float64).cpu().numpy()


def half_step(dtype):
    import torch
    return {torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 0.0), torch.float32: (0.0, 0.0)}[dtype]


def compare(got, ref, bound, where):
    half, least = half_step(got.dtype)
    g = exact(got)
    tol = bound + half * (np.abs(ref) + bound) + least
    bad = ~(np.abs(g - ref) <= tol)
    at = tuple(np.argwhere(bad)[0]) if bad.any() else None
    assert not bad.any(), "%s: %d of %d off, first at %r: %g for %g, tolerance %g" % (where, bad.sum(), bad.size, at, g[at], ref[at], tol[at])


def make(M, L, R, K, N, kind, seed, ids):
    """Y, X, A, B, ids, scaling, all on the GPU."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    v = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    dtype = getattr(torch, kind)
    rng = np.random.default_rng(seed)
    if ids == "each":
        ids = rng.permutation(max(L, M))[:M] % L
    elif ids == "mixed":
        ids = rng.integers(-1, L + 1, M)
    elif ids == "runs":
        ids = np.sort(rng.integers(0, L, M))[::-1].copy()
    elif ids == "one":
        ids = np.full(M, L // 2)
    else:
        ids = np.full(M, -1)
    return (v(M, N).to(dtype), v(M, K).to(dtype), (v(L, R, K) / K ** 0.5).to(dtype), (v(L, N, R) / R ** 0.5).to(dtype),
            torch.tensor(np.ascontiguousarray(ids), dtype=torch.int32, device="cuda"), 2.0 ** torch.randint(-1, 2, (L,), generator=gen, device="cuda").float())


def of_rows(ids, L, scaling):
    """(adapter, its rows, its scale) of every adapter with rows."""
    ids = ids.cpu().numpy()
    return [(a, np.nonzero(ids == a)[0], scaling[a]) for a in range(L) if (ids == a).any()]


def expected_add(Y, X, A, B, ids, scaling):
    out, bound = np.array(Y), np.zeros(Y.shape)
    R, K = A.shape[1:]
    for a, rows, s in of_rows(ids, len(A), scaling):
        x = X[rows]
        h, terms = s * (x @ A[a].T), abs(s) * (np.abs(x) @ np.abs(A[a]).T)
        dh = ((K / 32 + 68) * 2.0 ** -23 + 2.0 ** -24) * terms
        b = np.abs(B[a]).T
        out[rows] += h @ B[a].T
        bound[rows] = dh @ b + 2.0 ** -23 * ((3 * R + 3) * (np.abs(h) @ b) + np.abs(out[rows]))
    return out, bound


def expected_grad(dY, X, A, B, ids, scaling, dX, grads="float32"):
    L, R, K = A.shape
    N = B.shape[1]
    dX, ex = np.array(dX), np.zeros(dX.shape)
    dA, ea, dB, eb = np.zeros(A.shape), np.zeros(A.shape), np.zeros(B.shape), np.zeros(B.shape)
    split = 2.0 ** -24 if grads == "float32" else 2.0 ** -16
    for a, rows, s in of_rows(ids, L, scaling):
        x, y, n = X[rows], dY[rows], len(rows)
        h, g = s * (x @ A[a].T), s * (y @ B[a])
        dh = ((K / 32 + 68) * 2.0 ** -23 + 2.0 ** -24) * abs(s) * (np.abs(x) @ np.abs(A[a]).T)
        dg = ((N / 32 + 68) * 2.0 ** -23 + 2.0 ** -24) * abs(s) * (np.abs(y) @ np.abs(B[a]))
        dX[rows] += g @ A[a]
        ex[rows] = dg @ np.abs(A[a]) + 2.0 ** -23 * ((3 * R + 3) * (np.abs(g) @ np.abs(A[a])) + np.abs(dX[rows]))
        dA[a], dB[a] = g.T @ x, y.T @ h
        ea[a] = dg.T @ np.abs(x) + (2.0 ** -23 * (6 * n + 2) + split) * (np.abs(g).T @ np.abs(x))
        eb[a] = np.abs(y).T @ dh + (2.0 ** -23 * (6 * n + 2) + split) * (np.abs(y).T @ np.abs(h))
    return (dX, ex), (dA, ea), (dB, eb)


def check_add(lora, M, L, R, K, N, kind, ids, seed=1, scaled=True):
    import torch
    Y, X, A, B, who, scaling = make(M, L, R, K, N, kind, seed, ids)
    where = "M %d L %d R %d K %d N %d %s %s" % (M, L, R, K, N, kind, ids)
    ref, bound = expected_add(exact(Y), exact(X), exact(A), exact(B), who, exact(scaling) if scaled else np.ones(L))
    before = Y.clone()
    out = lora.add(Y, X, A, B, who, scaling if scaled else None)
    assert torch.equal(Y, before)
    compare(out, ref, bound, where)
    none = (who < 0) | (who >= L)
    assert torch.equal(out[none], Y[none])
    assert lora.add(Y, X, A, B, who, scaling if scaled else None, out=Y) is Y and torch.equal(Y, out), where


def check_grad(lora, M, L, R, K, N, kind, ids, grads="float32", seed=2, base=True):
    import torch
    dY, X, A, B, who, scaling = make(M, L, R, K, N, kind, seed, ids)
    where = "M %d L %d R %d K %d N %d %s %s" % (M, L, R, K, N, kind, ids)
    dX = torch.randn(M, K, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(X.dtype) if base else None
    dtype = torch.float32 if grads == "float32" else X.dtype
    got = lora.grad(dY, X, A, B, who, scaling, dX=dX, dtype=dtype)
    want = expected_grad(exact(dY), exact(X), exact(A), exact(B), who, exact(scaling), exact(dX) if base else np.zeros((M, K)), grads)
    assert got[0].dtype is X.dtype and got[1].dtype is dtype and got[2].dtype is dtype
    for g, (ref, bound), name in zip(got, want, ("dX", "dA", "dB")):
        compare(g, ref, bound, where + " " + name)
    if base:
        again = lora.grad(dY, X, A, B, who, scaling, dX=dX, out=(dX, torch.full_like(got[1], 7.0), torch.full_like(got[2], 7.0)))
        assert again[0] is dX and all(torch.equal(a, b) for a, b in zip(again, got)), where


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("ids", ["each", "mixed", "runs", "one", "none"])
@pytest.mark.parametrize("M,L", [(1, 1), (1, 9), (2, 1), (16, 1), (17, 2), (33, 40), (64, 64), (65, 3), (100, 1), (130, 200), (300, 4)])
def test_add_to_rows_of_every_mixture(lora, M, L, ids, kind):
    check_add(lora, M, L, 16, 264, 328, kind, ids)


@gpu
@pytest.mark.parametrize("R", [8, 16, 24, 32, 40, 64, 72, 96, 128])
@pytest.mark.parametrize("M", [5, 70, 200])
@pytest.mark.parametrize("K,N", [(8, 8), (136, 1000), (2056, 120)])
def test_add_of_every_rank(lora, M, R, K, N):
    check_add(lora, M, 3, R, K, N, "bfloat16", "mixed", scaled=R % 16 == 0)


@gpu
@pytest.mark.parametrize("M", [1, 3, 80, 600])
def test_add_of_long_rows(lora, M):
    check_add(lora, M, 4, 16, 8192, 5000, "float16", "mixed")
    check_add(lora, M, 4, 64, 20000, 264, "bfloat16", "runs")


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("ids", ["mixed", "runs", "one", "none"])
@pytest.mark.parametrize("M,L", [(1, 1), (1, 9), (17, 2), (64, 70), (65, 3), (130, 200), (300, 4), (1100, 2)])
def test_grad_of_rows_of_every_mixture(lora, M, L, ids, kind):
    check_grad(lora, M, L, 16, 264, 328, kind, ids, base=ids != "runs")


@gpu
@pytest.mark.parametrize("grads", ["same", "float32"])
@pytest.mark.parametrize("R", [8, 16, 24, 32, 40, 64, 72, 128])
@pytest.mark.parametrize("K,N", [(8, 8), (136, 1000), (2056, 120)])
def test_grad_of_every_rank(lora, R, K, N, grads):
    check_grad(lora, 90, 3, R, K, N, "float16" if R % 16 else "bfloat16", "mixed", grads)


@gpu
@pytest.mark.parametrize("M", [4096, 4097, 70000])
def test_many_rows(lora, M):
    """The rows' sort has another form from 4097 and from 65537 rows on."""
    check_add(lora, M, 5, 8, 16, 24, "bfloat16", "mixed")
    check_grad(lora, M, 5, 8, 16, 24, "float16", "mixed")


@gpu
@pytest.mark.parametrize("M,L,R,K,N", [(363, 1, 104, 1920, 1600), (363, 40, 104, 1920, 264), (2000, 3, 64, 264, 8200), (2000, 3, 128, 264, 4104), (2000, 3, 16, 264, 16392)])
def test_add_in_parts_and_whole(lora, M, L, R, K, N):
    """Tiles of 64 rows that the expanding product takes in four parts (up to 2047 waves), and whole."""
    check_add(lora, M, L, R, K, N, "bfloat16", "mixed")


@gpu
@pytest.mark.parametrize("grads", ["same", "float32"])
@pytest.mark.parametrize("R,kind", [(8, "float16"), (32, "bfloat16")])
def test_grad_of_many_adapters(lora, R, kind, grads):
    """So many columns of gradients that a workgroup has 128 of them at every rank."""
    check_grad(lora, 700, 130, R, 584, 600, kind, "mixed", grads)


@gpu
def test_strides(lora):
    import torch
    M, L, R, K, N = 75, 3, 24, 136, 200
    Y, X, A, B, ids, scaling = make(M, L, R, K, N, "bfloat16", 4, "mixed")

    def wide(t, ahead=8):
        big = torch.full((M, t.shape[1] + 48), math.nan, device="cuda", dtype=t.dtype)
        big[:, ahead:ahead + t.shape[1]] = t
        return big, big[:, ahead:ahead + t.shape[1]]
    (by, y), (bx, x), (bo, o) = wide(Y), wide(X, 16), wide(torch.zeros_like(Y), 24)
    assert torch.equal(lora.add(y, x, A, B, ids, scaling, out=o), lora.add(Y, X, A, B, ids, scaling))
    assert bool(bo[:, :24].isnan().all()) and bool(bo[:, 24 + N:].isnan().all())
    base = torch.randn(M, K, device="cuda").to(X.dtype)
    (bb, d), (bd, do) = wide(base), wide(torch.zeros_like(X), 16)
    want = lora.grad(Y, X, A, B, ids, scaling, dX=base)
    got = lora.grad(y, x, A, B, ids, scaling, dX=d, out=(do, torch.empty_like(A), torch.empty_like(B)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert bool(bd[:, :16].isnan().all()) and bool(bd[:, 16 + K:].isnan().all())


@gpu
def test_values_that_are_not_numbers_stay_in_their_rows(lora):
    import torch
    for M in (20, 90):
        Y, X, A, B, ids, scaling = make(M, 3, 8, 72, 136, "float16", 5, "mixed")
        A[2, 0, 0] = math.inf  # an adapter that no row has
        ids[ids == 2] = -1
        X[3, 5], X[4, 0], Y[6, 1] = math.nan, math.inf, math.nan
        ids[3], ids[4], ids[6] = 0, 1, -1
        out = exact(lora.add(Y, X, A, B, ids, scaling))
        assert np.isnan(out[3]).all() and not np.isfinite(out[4]).any() and np.isnan(out[6, 1]) and np.isfinite(np.delete(out, [3, 4, 6], 0)).all()
        dX, dA, dB = lora.grad(torch.nan_to_num(Y), X, A, B, ids, scaling)
        assert np.isfinite(exact(dX)).all() and np.isnan(exact(dA)[0][:, 5]).all() and np.isfinite(np.delete(exact(dA)[0], 5, 1)).all() and (exact(dA)[2] == 0).all()


@gpu
def test_gradients_are_differences_of_the_kernels_results(lora):
    """Whole numbers small enough that every value and sum is exact: the sum of C * out is linear in each of X, A and B."""
    import torch
    rng = np.random.default_rng(7)
    M, L, R, K, N = 70, 3, 8, 16, 24
    small = lambda *s: torch.tensor((rng.random(s) < 0.2) * rng.integers(-1, 2, s), dtype=torch.float16, device="cuda")
    X, A, B, C = small(M, K), small(L, R, K), small(L, N, R), small(M, N)
    ids = torch.tensor(rng.integers(-1, L, M), dtype=torch.int32, device="cuda")
    zero = torch.zeros_like(C)
    f = lambda x, a, b: (lora.add(zero, x, a, b, ids).double() * C.double()).sum()
    dX, dA, dB = lora.grad(C, X, A, B, ids, dtype=torch.float32)
    for got, change, like in ((dX, lambda d: f(X + d, A, B) - f(X - d, A, B), X), (dA, lambda d: f(X, A + d, B) - f(X, A - d, B), A), (dB, lambda d: f(X, A, B + d) - f(X, A, B - d), B)):
        d = small(*like.shape)
        assert float(change(d)) == 2 * float((got.double() * d.double()).sum())


@gpu
def test_no_rows(lora):
    import torch
    A, B = torch.ones(2, 8, 64, device="cuda").half(), torch.ones(2, 32, 8, device="cuda").half()
    X, Y, ids = torch.zeros(0, 64, device="cuda").half(), torch.zeros(0, 32, device="cuda").half(), torch.zeros(0, dtype=torch.int32, device="cuda")
    assert lora.add(Y, X, A, B, ids).shape == (0, 32)
    dX, dA, dB = lora.grad(Y, X, A, B, ids)
    assert dX.shape == (0, 64) and bool((dA == 0).all()) and bool((dB == 0).all())


@gpu
def test_binding_refuses_what_does_not_fit(lora):
    import torch
    Y, X, A, B, ids, scaling = make(4, 2, 8, 64, 32, "float16", 1, "one")
    for bad in (lambda: lora.add(Y[:3], X, A, B, ids), lambda: lora.add(Y, X, A[:1], B, ids), lambda: lora.add(Y, X, A, B, ids[:3]), lambda: lora.add(Y, X, A, B, ids, scaling[:1]),
                lambda: lora.add(Y, X, A, B, ids, out=X), lambda: lora.add(Y, X, A, B, ids, stream=torch.cuda.current_stream()), lambda: lora.grad(Y, X, A, B, ids, dX=Y),
                lambda: lora.grad(Y, X, A, B, ids, out=(X, B, A))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lora.add(Y, X.bfloat16(), A, B, ids), lambda: lora.add(Y, X, A, B.transpose(1, 2), ids), lambda: lora.add(Y, X, A, B, ids.long()),
                lambda: lora.add(Y, X, A, B, ids, scaling.half()), lambda: lora.grad(Y, X, A, B, ids, dtype=torch.bfloat16),
                lambda: lora.add(Y, X, A, B, ids, workspace=torch.empty(1 << 20, dtype=torch.uint8))):
        with pytest.raises((TypeError, ValueError)):
            bad()
    from paper_2601_16536_amd.binding import W4A16Error
    with pytest.raises(W4A16Error):
        lora.add(Y, X, A, B, ids, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(W4A16Error):
        lora.add(Y, X, torch.zeros(2, 12, 64, device="cuda").half(), torch.zeros(2, 32, 12, device="cuda").half(), ids)


@gpu
@pytest.mark.parametrize("M", [24, 100])
def test_replayed_graphs_and_other_streams_beside_a_shared_projection(lora, M):
    """MXFP4 projection, then the adapters, in place, as a server runs them."""
    import torch
    from paper_2601_16536_amd import mx
    L, R, K, N = 5, 16, 256, 136
    _, X, A, B, ids, scaling = make(M, L, R, K, N, "bfloat16", 8, "mixed")
    gen = torch.Generator(device="cuda").manual_seed(9)
    codes, scales = mx.quantize(torch.randn(N, K, generator=gen, device="cuda") / 16)

    def work():
        Y = mx.gemm(X, codes, scales)
        Y = lora.add(Y, X, A, B, ids, scaling, out=Y)
        return (Y,) + tuple(lora.grad(Y, X, A, B, ids, scaling))
    work()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = work()
    stream = torch.cuda.Stream()
    for i in range(3):
        X.copy_(torch.randn(M, K, generator=gen, device="cuda"))
        ids.copy_(torch.randint(-1, L, (M,), generator=gen, device="cuda", dtype=torch.int32))
        eager = work()
        graph.replay()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            other = work()
        torch.cuda.current_stream().wait_stream(stream)
        torch.cuda.synchronize()
        for a, b, c in zip(eager, captured, other):
            assert torch.equal(a, b) and torch.equal(a, c), i
    ref, bound = expected_add(exact(mx.gemm(X, codes, scales)), exact(X), exact(A), exact(B), ids, exact(scaling))
    compare(eager[0], ref, bound, "beside the projection")


@gpu
def test_rows_beyond_two_and_four_gib(lora):
    import torch
    M, L, R, K, N = 260000, 2, 8, 64, 8320  # Y: 4.3 GB
    gen = torch.Generator(device="cuda").manual_seed(10)
    Y = torch.zeros(M, N, device="cuda", dtype=torch.bfloat16)
    X = torch.randn(M, K, generator=gen, device="cuda").bfloat16()
    A, B = torch.randn(L, R, K, generator=gen, device="cuda").bfloat16(), torch.randn(L, N, R, generator=gen, device="cuda").bfloat16()
    ids = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    at = [0, 129040, 129060, 258100, 258120, M - 1]
    ids[at] = torch.tensor([0, 1, 0, 1, 0, 1], dtype=torch.int32, device="cuda")
    lora.add(Y, X, A, B, ids, out=Y)
    ref, bound = expected_add(np.zeros((6, N)), exact(X[at]), exact(A), exact(B), ids[at], np.ones(2))
    compare(Y[at], ref, bound, "large")
    got = lora.grad(Y, X, A, B, ids, dtype=torch.float32)
    want = expected_grad(exact(Y[at]), exact(X[at]), exact(A), exact(B), ids[at], np.ones(2), np.zeros((6, K)))
    compare(got[0][at], *want[0], "large dX")
    compare(got[1], *want[1], "large dA")
    compare(got[2], *want[2], "large dB")

"""Products of rows in groups: pins of the CPU oracle, refusals, then the HIP kernels against the oracle.

Tolerance of the products, per output, with A the sum of the terms' magnitudes and n the number of terms: 16-bit products are exact in FP32; an output is a chain of
ceil(n / 32) additions of a matrix instruction's 32 products, so at most ceil(n / 32) + 32 roundings, each below 2^-23 A (the instruction may truncate); then one
rounding to the output's type, half a unit in the last place: 2^-11 of an FP16 value or 2^-25 below its normal range, 2^-8 of a BF16 value, none for FP32.  What is
added to an output that was there adds one rounding, 2^-24 of the result.
"""
import math
import os

import numpy as np
import pytest

from oracle import grouped_oracle as go

gpu = pytest.mark.gpu
KINDS = ["float16", "bfloat16"]


# ---- the oracle's pins ----

def test_oracle_sorts_a_worked_example():
    offsets, order, place = go.sort([[2, 0], [-1, 2], [0, 5]], 3)
    assert offsets.tolist() == [0, 2, 2, 4] and order.tolist() == [1, 4, 0, 3, 2, 5] and place.tolist() == [2, 0, 4, 3, 1, 5]


def test_oracle_products_by_hand():
    X = np.array([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0]])
    W = np.array([[[1.0, 0.0], [0.0, 1.0], [1.0, 1.0]], [[2.0, 0.0], [0.0, 0.0], [0.0, -1.0]]])
    Y, terms, had = go.gemm(X, W, [0, 1, 2])
    assert Y.tolist() == [[1, 2, 3], [6, 0, -4], [0, 0, 0]] and terms[1].tolist() == [6, 0, 4] and had.tolist() == [True, True, False]
    Y, _, _ = go.gemm(X, W, [0, 2, 3], rows=[5, 0, -1], top_k=2)
    assert Y.tolist() == [[5, 6, 11], [1, 2, 3], [0, 0, 0]]
    dW, _, n = go.gemm_grad(np.array([[1.0, 0.0, 2.0], [0.0, 1.0, 0.0], [3.0, 0.0, 0.0]]), X, [0, 2, 3])
    assert dW[0].tolist() == [[1, 2], [3, 4], [2, 4]] and dW[1].tolist() == [[15, 18], [0, 0], [0, 0]] and n.tolist() == [2, 1]


def test_oracle_gradients_are_differences():
    """The sum of C * Y is linear in X and in W: differences of it are its gradients."""
    rng = np.random.default_rng(0)
    X, W, C, D = rng.normal(size=(7, 6)), rng.normal(size=(3, 5, 6)), rng.normal(size=(7, 5)), rng.normal(size=(3, 5, 6))
    offsets = [0, 2, 2, 6]
    C[6] = 0
    f = lambda x, w: (C * go.gemm(x, w, offsets)[0]).sum()
    dW, _, _ = go.gemm_grad(C, X, offsets)
    assert math.isclose((dW * D).sum(), (f(X, W + D) - f(X, W - D)) / 2, rel_tol=1e-12)
    dX, _, _ = go.gemm(C, W, offsets, transposed=True)
    E = rng.normal(size=X.shape)
    assert math.isclose((dX * E).sum(), (f(X + E, W) - f(X - E, W)) / 2, rel_tol=1e-12)


# ---- refusals ----

@pytest.fixture(scope="module")
def grouped():
    from paper_2601_16536_amd import binding, build, grouped
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    grouped.lib()
    return grouped


def test_header_functions_are_exported(grouped):
    import re
    from paper_2601_16536_amd import binding, lora
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "w4a16_grouped.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(w4a16_(?:grouped|lora)_[a-z0-9_]+)\s*\(", text))
    assert declared == set(grouped.EXPORTS) | set(lora.EXPORTS)
    for name in declared:
        assert getattr(binding.lib(), name) is not None


def test_argument_checks_need_no_gpu(grouped):
    from paper_2601_16536_amd import binding as b
    L = grouped.lib()
    s = L.w4a16_grouped_sort  # ids, count, E, offsets, order, place, workspace, bytes, stream
    assert s(16, 8, 0, 16, 16, 16, 0, 0, 0) == b.ERR_SHAPE
    assert s(16, 8, 1025, 16, 16, 16, 0, 0, 0) == b.ERR_SHAPE
    assert s(16, -1, 4, 16, 16, 16, 0, 0, 0) == b.ERR_SHAPE
    assert s(16, 1 << 30, 4, 16, 16, 16, 256, 1 << 40, 0) == b.ERR_UNSUPPORTED
    assert s(0, 8, 4, 16, 16, 16, 0, 0, 0) == b.ERR_NULL
    assert s(16, 8, 4, 0, 16, 16, 0, 0, 0) == b.ERR_NULL
    assert s(16, 8, 4, 16, 0, 16, 0, 0, 0) == b.ERR_NULL
    assert s(16, 8, 4, 18, 16, 16, 0, 0, 0) == b.ERR_ALIGN
    assert s(16, 1 << 20, 4, 16, 16, 16, 0, 0, 0) == b.ERR_NULL
    assert s(16, 1 << 20, 4, 16, 16, 16, 128, 1 << 30, 0) == b.ERR_ALIGN
    assert s(16, 1 << 20, 4, 16, 16, 16, 256, 16, 0) == b.ERR_WORKSPACE
    # X, type, x_rows, ldx, rows, top_k, W, stride_w, ldw, transposed, offsets, E, count, N, K, Y, ldy, fill, stream
    good = dict(X=16, type=0, x_rows=4, ldx=64, rows=0, top_k=1, W=16, stride_w=64 * 32, ldw=64, transposed=0, offsets=16, E=2, count=4, N=32, K=64, Y=16, ldy=32, fill=0, stream=0)

    def g(**change):
        return L.w4a16_grouped_gemm(*dict(good, **change).values())
    assert g(count=0, x_rows=0, X=0, W=0, Y=0) == b.OK
    for bad in (dict(type=2), dict(E=0), dict(E=1025), dict(count=-1), dict(N=0), dict(N=12), dict(K=0), dict(K=60), dict(x_rows=3), dict(rows=16, top_k=0), dict(rows=16, x_rows=0),
                dict(ldx=56), dict(ldy=24), dict(ldw=56), dict(stride_w=-8), dict(transposed=1, ldw=24)):
        assert g(**bad) == b.ERR_SHAPE, bad
    for bad in (dict(X=0), dict(W=0), dict(offsets=0), dict(Y=0)):
        assert g(**bad) == b.ERR_NULL, bad
    for bad in (dict(X=24), dict(W=24), dict(Y=24), dict(offsets=18), dict(rows=18), dict(ldx=68), dict(ldy=36), dict(ldw=68), dict(stride_w=64 * 32 + 4)):
        assert g(**bad) == b.ERR_ALIGN, bad
    for bad in (dict(count=1 << 30, x_rows=1 << 30), dict(K=(1 << 17) + 8, ldx=1 << 18, ldw=1 << 18), dict(N=(1 << 20) + 8, ldy=1 << 21), dict(ldx=(1 << 21) + 8), dict(ldy=1 << 23),
                dict(ldw=1 << 23)):
        assert g(**bad) == b.ERR_UNSUPPORTED, bad
    # dY, type, ldy, X, x_rows, ldx, rows, top_k, offsets, E, count, N, K, dW, grad type, accumulate, stream
    good2 = dict(dY=16, type=0, ldy=32, X=16, x_rows=4, ldx=64, rows=0, top_k=1, offsets=16, E=2, count=4, N=32, K=64, dW=16, grad=2, accumulate=0, stream=0)

    def w(**change):
        return L.w4a16_grouped_gemm_grad(*dict(good2, **change).values())
    for bad in (dict(type=2), dict(grad=1), dict(E=0), dict(N=12), dict(K=4), dict(x_rows=3), dict(ldy=24), dict(ldx=56), dict(rows=16, top_k=0)):
        assert w(**bad) == b.ERR_SHAPE, bad
    for bad in (dict(dY=0), dict(X=0), dict(offsets=0), dict(dW=0), dict(dW=0, count=0)):
        assert w(**bad) == b.ERR_NULL, bad
    for bad in (dict(dY=24), dict(X=24), dict(dW=24), dict(ldx=68), dict(ldy=36), dict(rows=18), dict(offsets=18)):
        assert w(**bad) == b.ERR_ALIGN, bad
    for bad in (dict(N=(1 << 17) + 8, ldy=1 << 18), dict(K=(1 << 17) + 8, ldx=1 << 18), dict(ldy=1 << 23)):
        assert w(**bad) == b.ERR_UNSUPPORTED, bad


def test_every_size_has_a_tile(grouped):
    for E in (1, 7, 64, 1024):
        for count in (1, 5, 300, 4096 * 8, (1 << 30) - 1):
            for N, K in ((8, 8), (136, 2056), (4096, 4096), (131072, 131072)):
                for kw in ({}, {"transposed": True}, {"grad": True}):
                    rows, cols = grouped.query_tile(E, count, N, K, **kw)
                    assert rows % 16 == 0 and cols % 16 == 0 and 16 <= rows <= 256 and 16 <= cols <= 256
    assert grouped.sort_workspace_bytes(4096, 1024) == 0 and grouped.sort_workspace_bytes(4097, 3) > 0


def test_binding_refuses_host_tensors_and_other_types(grouped):
    import torch
    ids = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        grouped.sort(ids, 4)
    x, w = torch.zeros(4, 64, dtype=torch.float16), torch.zeros(2, 32, 64, dtype=torch.float16)
    with pytest.raises(TypeError):
        grouped.gemm(x, w, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError):
        grouped.gemm(x.float(), w.float(), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError):
        grouped.gemm_grad(x, x, torch.zeros(3, dtype=torch.int32))


# ---- the kernels ----

def exact(t):
    import torch
    return t.detach().to(torch.float64).cpu().numpy()


def half_step(dtype):
    import torch
    return {torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 0.0), torch.float32: (0.0, 0.0)}[dtype]


def tolerance(dtype, ref, terms, n, added=0.0):
    half, least = half_step(dtype)
    sums = (np.ceil(n / 32) + 32) * 2.0 ** -23 * terms + added
    return sums + half * (np.abs(ref) + sums) + least


def compare(got, ref, tol, where):
    g = exact(got)
    bad = ~(np.abs(g - ref) <= tol)
    assert not bad.any(), "%s: %d of %d off, first at %r: %g for %g, tolerance %g" % (
        where, bad.sum(), bad.size, np.argwhere(bad)[0].tolist(), g[tuple(np.argwhere(bad)[0])], ref[tuple(np.argwhere(bad)[0])], np.broadcast_to(tol, g.shape)[tuple(np.argwhere(bad)[0])])


def ints(v):
    import torch
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def values(gen, shape, kind):
    import torch
    return torch.randn(*shape, generator=gen, device="cuda").to(getattr(torch, kind))


def generator(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


@gpu
@pytest.mark.parametrize("count", [0, 1, 2, 63, 64, 65, 255, 257, 4095, 4096, 4097, 20000, 65536, 65537, 300001])
@pytest.mark.parametrize("E", [1, 2, 3, 64, 256, 1000, 1024])
def test_sort_is_the_oracles(grouped, count, E):
    rng = np.random.default_rng(count * 2000 + E)
    for name, ids in (("even", rng.integers(0, E, count)), ("some without", rng.integers(-2, E + 2, count)),
                      ("skewed", np.minimum((E * rng.random(count) ** 6).astype(np.int64), E - 1)), ("one", np.full(count, E - 1)), ("none", np.full(count, -1))):
        got = grouped.sort(ints(ids), E)
        key = np.where((ids >= 0) & (ids < E), ids, E)
        order = np.argsort(key, kind="stable")
        want = (np.searchsorted(key[order], np.arange(E + 1)), order, np.argsort(order, kind="stable"))
        for g, w, what in zip(got, want, ("offsets", "order", "place")):
            assert np.array_equal(g.cpu().numpy(), w), "%s %s, %d ids, %d groups" % (name, what, count, E)


@gpu
def test_sort_is_what_the_lists_say_and_takes_any_shape(grouped):
    rng = np.random.default_rng(5)
    ids = rng.integers(-1, 12, (37, 6))
    for g, w in zip(grouped.sort(ints(ids), 11), go.sort(ids, 11)):
        assert np.array_equal(g.cpu().numpy(), w)


SIZES = {  # rows of each group
    "one_row": [1], "one_group": [37], "one_full": [128], "empty_ends": [0, 5, 0], "all_empty": [0, 0, 0], "ragged": [3, 0, 17, 64, 1, 0, 130, 16, 15], "tiles": [128, 256, 64, 16, 128],
    "large": [700, 0, 513, 255, 1], "many": [1, 0, 2] * 40, "very_many": ([0] * 9 + [1, 3]) * 93,
}


def group_case(grouped, sizes, N, K, kind, transposed, gather, seed, ahead=0, behind=0):
    """X, W, offsets, rows, top_k on the GPU."""
    import torch
    gen, rng = generator(seed), np.random.default_rng(seed)
    count = ahead + sum(sizes) + behind
    offsets = ahead + np.concatenate([[0], np.cumsum(sizes)])
    top_k = 3
    T = max(1, -(-count // top_k)) if gather else count
    X = values(gen, (T, K), kind)
    W = values(gen, (len(sizes),) + ((K, N) if transposed else (N, K)), kind)
    rows = rng.permutation(T * top_k)[:count] if gather else None
    return X, W, offsets, rows, top_k if gather else 1


def run_group_case(grouped, sizes, N, K, kind, transposed, gather, seed, ahead=0, behind=0, where=""):
    import torch
    X, W, offsets, rows, top_k = group_case(grouped, sizes, N, K, kind, transposed, gather, seed, ahead, behind)
    kw = {} if rows is None else {"rows": ints(rows), "top_k": top_k}
    ref, terms, had = go.gemm(exact(X), exact(W), offsets, rows, top_k, transposed)
    Y = grouped.gemm(X, W, ints(offsets), transposed=transposed, **kw)
    compare(Y, ref, tolerance(X.dtype, ref, terms, K), where)
    out = torch.full_like(Y, 7.0)
    assert grouped.gemm(X, W, ints(offsets), transposed=transposed, out=out, **kw) is out
    assert torch.equal(out[torch.from_numpy(had).cuda()], Y[torch.from_numpy(had).cuda()]) and bool((out[torch.from_numpy(~had).cuda()] == 7.0).all())


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("sizes", list(SIZES))
def test_gemm_of_every_raggedness(grouped, sizes, transposed, gather, kind):
    if sum(SIZES[sizes]) == 0 and gather:
        ahead, behind = 2, 3
    else:
        ahead, behind = (0, 0) if kind == "float16" else (5, 9)
    run_group_case(grouped, SIZES[sizes], 136, 200, kind, transposed, gather, 11, ahead, behind, "%s %s" % (sizes, kind))


@gpu
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("N,K", [(8, 8), (8, 64), (16, 72), (24, 120), (128, 128), (264, 56), (520, 320), (1000, 2056), (72, 8200)])
@pytest.mark.parametrize("sizes", ["one_row", "ragged", "large"])
def test_gemm_of_every_length(grouped, sizes, N, K, transposed):
    run_group_case(grouped, SIZES[sizes], N, K, "bfloat16", transposed, False, 12, where="N %d K %d" % (N, K))


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("K", [8, 328, 1032])
@pytest.mark.parametrize("sizes,N,tile", [([1, 0, 2] * 40, 400, (16, 128)), ([20, 0, 64, 65, 1, 33] * 6, 520, (64, 128)), ([100, 0, 129, 65, 128, 127, 300, 1, 200, 90] * 2, 520, (128, 128)),
                                          ([3, 0, 17, 1], 72, (16, 32)), ([37, 0, 64, 65, 130], 264, (64, 32))], ids=lambda v: "" if isinstance(v, list) else None)
def test_gemm_in_every_tile(grouped, sizes, N, tile, K, transposed, gather, kind):
    assert grouped.query_tile(len(sizes), sum(sizes) + 7, N, K, transposed) == tile
    run_group_case(grouped, sizes, N, K, kind, transposed, gather, 14, 3, 4, "K %d" % K)


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("K", [8, 64, 120, 128, 192, 256, 328, 448, 520, 1032])
def test_gemm_in_the_largest_tiles(grouped, K, transposed, gather, kind):
    """From one stage of 64 values to seventeen, whole and not; rows and columns that end inside a tile."""
    sizes, N = [300, 0, 257, 1, 700, 256, 2, 540], 4104
    assert grouped.query_tile(len(sizes), sum(sizes) + 13, N, K, transposed) == (256, 256)
    run_group_case(grouped, sizes, N, K, kind, transposed, gather, K, 5, 8, "K %d" % K)


@gpu
@pytest.mark.parametrize("transposed", [False, True])
def test_gemm_of_views(grouped, transposed):
    """X, W and out with strides, and NaN in between."""
    import torch
    gen = generator(3)
    sizes, N, K = [40, 0, 70, 5], 96, 136
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    count = offsets[-1]
    big = torch.full((count, K + 24), math.nan, device="cuda", dtype=torch.bfloat16)
    big[:, :K] = values(gen, (count, K), "bfloat16")
    rows, width = (K, N) if transposed else (N, K)
    W = torch.full((len(sizes), rows + 3, width + 16), math.nan, device="cuda", dtype=torch.bfloat16)
    W[:, 2:rows + 2, 8:width + 8] = values(gen, (len(sizes), rows, width), "bfloat16")
    out = torch.full((count, N + 40), 7.0, device="cuda", dtype=torch.bfloat16)
    X, W, Y = big[:, :K], W[:, 2:rows + 2, 8:width + 8], out[:, 16:N + 16]
    grouped.gemm(X, W, ints(offsets), transposed=transposed, out=Y)
    ref, terms, _ = go.gemm(exact(X), exact(W), offsets, transposed=transposed)
    compare(Y, ref, tolerance(X.dtype, ref, terms, K), "views")
    assert bool((out[:, :16] == 7.0).all()) and bool((out[:, N + 16:] == 7.0).all())


@gpu
def test_gemm_rows_that_are_not_there_and_values_that_are_not_numbers(grouped):
    import torch
    gen = generator(4)
    sizes, N, K = [20, 90], 64, 72
    offsets = np.array([0, 20, 110])
    X, W = values(gen, (50, K), "float16"), values(gen, (2, N, K), "float16")
    X[7, 3], X[9, 0], X[11, 5] = math.nan, math.inf, -math.inf
    rows = np.arange(110) % 100
    rows[[0, 25, 109]] = [-1, 100, 2 ** 31 - 1]
    Y = grouped.gemm(X, W, ints(offsets), rows=ints(rows), top_k=2)
    source = np.where((rows >= 0) & (rows < 100), rows // 2, -1)
    clean = exact(X)
    clean[[7, 9, 11]] = 0
    ref, terms, _ = go.gemm(clean, exact(W), offsets, rows, 2)
    odd = np.isin(source, [7, 9, 11])
    y = exact(Y)
    assert np.isnan(y[source == 7]).all() and not np.isfinite(y[odd]).any()
    assert (y[source == -1] == 0).all()
    keep = ~odd
    compare(Y[torch.from_numpy(keep).cuda()], ref[keep], tolerance(X.dtype, ref, terms, K)[keep], "the others")


@gpu
@pytest.mark.parametrize("transposed", [False, True])
def test_gemm_offsets_that_descend_touch_nothing_else(grouped, transposed):
    """Values of the rows concerned are undefined; what is around the tensors stays."""
    import torch
    gen = generator(5)
    X, W = values(gen, (64, 72), "bfloat16"), values(gen, (4, 72, 72), "bfloat16")
    out = torch.full((64 + 32, 72), 7.0, device="cuda", dtype=torch.bfloat16)
    for offsets in ([0, 50, 20, 60, 64], [-5, 3, 900, 2, 64], [64, 0, 0, 0, 0], [2 ** 31 - 1, -2 ** 31, 5, 6, 7]):
        grouped.gemm(X, W, ints(offsets), transposed=transposed, out=out[16:80])
        grouped.gemm(X, W, ints(offsets), transposed=transposed)
        dW = grouped.gemm_grad(X, X, ints(offsets))
        assert dW.shape == (4, 72, 72)
    assert bool((out[:16] == 7.0).all()) and bool((out[80:] == 7.0).all())


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("grads", ["same", "float32"])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("sizes", list(SIZES))
def test_gemm_grad_of_every_raggedness(grouped, sizes, gather, grads, kind):
    import torch
    N, K = (72, 136) if len(SIZES[sizes]) < 100 else (8, 24)
    X, W, offsets, rows, top_k = group_case(grouped, SIZES[sizes], N, K, kind, False, gather, 21, 5, 9)
    dY = values(generator(22), (offsets[-1] + 9, N), kind)
    if rows is not None:
        rows[[2, 8]] = [-3, 2 ** 31 - 1]
    kw = {} if rows is None else {"rows": ints(rows), "top_k": top_k}
    dtype = X.dtype if grads == "same" else torch.float32
    ref, terms, n = go.gemm_grad(exact(dY), exact(X), offsets, rows, top_k)
    n = n[:, None, None]
    # what is around the groups is not read
    dY[:5], dY[offsets[-1]:] = math.nan, math.nan
    dW = grouped.gemm_grad(dY, X, ints(offsets), dtype=dtype, **kw)
    assert dW.dtype is dtype
    compare(dW, ref, tolerance(dtype, ref, terms, n), sizes)
    old = values(generator(23), tuple(dW.shape), "float32").to(dtype)
    more = old.clone()
    assert grouped.gemm_grad(dY, X, ints(offsets), out=more, accumulate=True, **kw) is more
    both = ref + exact(old)
    compare(more, both, tolerance(dtype, both, terms, n, 2.0 ** -23 * (np.abs(both) + np.abs(exact(old)))), "added to")


@gpu
@pytest.mark.parametrize("N,K", [(8, 8), (16, 8), (120, 264), (1000, 520), (2056, 72)])
@pytest.mark.parametrize("sizes", ["one_row", "ragged", "large"])
def test_gemm_grad_of_every_width(grouped, sizes, N, K):
    import torch
    X, _, offsets, _, _ = group_case(grouped, SIZES[sizes], N, K, "bfloat16", False, False, 31)
    big = torch.full((X.shape[0], N + 24), math.nan, device="cuda", dtype=torch.bfloat16)
    big[:, 8:N + 8] = values(generator(32), (X.shape[0], N), "bfloat16")
    dY = big[:, 8:N + 8]
    ref, terms, n = go.gemm_grad(exact(dY), exact(X), offsets)
    compare(grouped.gemm_grad(dY, X, ints(offsets), dtype=torch.float32), ref, tolerance(torch.float32, ref, terms, n[:, None, None]), "N %d K %d" % (N, K))


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("grads", ["same", "float32"])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("N,K,tile", [(136, 328, 64), (1000, 520, 128)])
def test_gemm_grad_in_the_smaller_tiles(grouped, N, K, tile, gather, grads, kind):
    import torch
    sizes = [100, 0, 129, 65, 128, 127, 700, 1]
    assert grouped.query_tile(len(sizes), sum(sizes) + 7, N, K, grad=True) == (tile, tile)
    X, _, offsets, rows, top_k = group_case(grouped, sizes, 8, K, kind, False, gather, 51, 3, 4)
    dY = values(generator(52), (len(X) if rows is None else len(rows), N), kind)
    kw = {} if rows is None else {"rows": ints(rows), "top_k": top_k}
    dtype = X.dtype if grads == "same" else torch.float32
    ref, terms, n = go.gemm_grad(exact(dY), exact(X), offsets, rows, top_k)
    compare(grouped.gemm_grad(dY, X, ints(offsets), dtype=dtype, **kw), ref, tolerance(dtype, ref, terms, n[:, None, None]), "N %d K %d" % (N, K))


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("grads", ["same", "float32"])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("sizes", [[1, 63, 64, 65, 128, 500, 0, 129], [191, 192, 193, 0, 256, 257, 2, 3], [448, 320, 319, 321, 577, 640, 0, 8], [0, 0, 0, 5, 0, 0, 0, 0],
                                   [1, 0, 64, 65, 3, 0, 0, 16]])
def test_gemm_grad_in_the_largest_tiles(grouped, sizes, gather, grads, kind):
    import torch
    N, K = 2056, 1800
    behind = max(9, 96 * len(sizes) - sum(sizes))  # rows of no group
    assert grouped.query_tile(len(sizes), sum(sizes) + 5 + behind, N, K, grad=True) == (256, 256)
    X, W, offsets, rows, top_k = group_case(grouped, sizes, 8, K, kind, False, gather, 41, 5, behind)
    big = torch.full((offsets[-1] + behind, N + 24), math.nan, device="cuda", dtype=X.dtype)
    dY = big[:, 16:N + 16]
    dY[5:offsets[-1]] = values(generator(42), (sum(sizes), N), kind)
    if rows is not None:
        rows[[7, 300]] = [-1, 2 ** 31 - 1]
    kw = {} if rows is None else {"rows": ints(rows), "top_k": top_k}
    dtype = X.dtype if grads == "same" else torch.float32
    ref, terms, n = go.gemm_grad(np.nan_to_num(exact(dY)), exact(X), offsets, rows, top_k)
    tol = tolerance(dtype, ref, terms, n[:, None, None])
    dW = grouped.gemm_grad(dY, X, ints(offsets), dtype=dtype, **kw)
    compare(dW, ref, tol, sizes)
    if dtype == torch.float32:  # twice the sum, after one more rounding
        grouped.gemm_grad(dY, X, ints(offsets), out=dW, accumulate=True, **kw)
        compare(dW, 2 * ref, 2 * tol + 2 * np.abs(ref) * 2.0 ** -24, "added")


@gpu
def test_gradients_are_differences_of_the_kernels_products(grouped):
    """The sum of C * Y is linear in X and in W: its difference between W + D and W - D, whose values and results are whole numbers in BF16's and FP32's range,
    is twice the gradient times D, exactly."""
    import torch
    rng = np.random.default_rng(6)
    sizes, N, K = [9, 0, 20, 3], 40, 24
    offsets = ints(np.concatenate([[0], np.cumsum(sizes)]))
    small = lambda *shape: torch.tensor(rng.integers(-2, 3, shape), dtype=torch.bfloat16, device="cuda")
    X, W, D, C, E = small(32, K), small(4, N, K), small(4, N, K), small(32, N), small(32, K)
    f = lambda x, w: (grouped.gemm(x, w, offsets).double() * C.double()).sum()
    dW = grouped.gemm_grad(C, X, offsets, dtype=torch.float32)
    assert float(f(X, W + D) - f(X, W - D)) == 2 * float((dW.double() * D.double()).sum())
    dX = grouped.gemm(C, W, offsets, transposed=True)
    assert float(f(X + E, W) - f(X - E, W)) == 2 * float((dX.double() * E.double()).sum())


@gpu
def test_no_rows(grouped):
    import torch
    X, W = torch.zeros(0, 64, device="cuda", dtype=torch.float16), torch.zeros(3, 32, 64, device="cuda", dtype=torch.float16)
    offsets, order, place = grouped.sort(torch.zeros(0, dtype=torch.int32, device="cuda"), 3)
    assert offsets.tolist() == [0, 0, 0, 0] and order.numel() == place.numel() == 0
    assert grouped.gemm(X, W, offsets).shape == (0, 32)
    dW = torch.full((3, 32, 64), 7.0, device="cuda")
    grouped.gemm_grad(X[:, :32].contiguous(), X, offsets, out=dW)
    assert bool((dW == 0).all())


@gpu
def test_binding_refuses_what_does_not_fit(grouped):
    import torch
    z = lambda *s, dtype=torch.float16: torch.zeros(*s, dtype=dtype, device="cuda")
    X, W, o = z(4, 64), z(2, 32, 64), z(3, dtype=torch.int32)
    for bad in (lambda: grouped.gemm(X, W, z(4, dtype=torch.int32)), lambda: grouped.gemm(X, W, o, transposed=True), lambda: grouped.gemm(X, W, o, top_k=2),
                lambda: grouped.gemm(X, W, o, out=z(4, 40)), lambda: grouped.gemm(X, W, o, rows=z(4, dtype=torch.int32), top_k=0), lambda: grouped.gemm_grad(z(5, 32), X, o),
                lambda: grouped.gemm_grad(z(4, 32), X, o, out=z(2, 32, 56)), lambda: grouped.gemm_grad(z(4, 32), X, o, accumulate=True), lambda: grouped.sort(o, 0),
                lambda: grouped.gemm_grad(z(4, 32), X, o, rows=z(5, dtype=torch.int32)), lambda: grouped.sort(o, 4, out=(z(5, dtype=torch.int32), z(3, dtype=torch.int32), z(2, dtype=torch.int32))),
                lambda: grouped.sort(z(70000, dtype=torch.int32), 4, stream=torch.cuda.current_stream())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: grouped.gemm(X, W.bfloat16(), o), lambda: grouped.gemm(X, W.transpose(1, 2), o, transposed=True), lambda: grouped.gemm(X, W, o.long()),
                lambda: grouped.gemm_grad(z(4, 32), X, o, dtype=torch.bfloat16), lambda: grouped.gemm_grad(z(4, 32, dtype=torch.bfloat16), X, o), lambda: grouped.sort(o.long(), 4)):
        with pytest.raises(TypeError):
            bad()
    from paper_2601_16536_amd.binding import W4A16Error
    with pytest.raises(W4A16Error):
        grouped.gemm(z(4, 60), z(2, 32, 60), o)
    with pytest.raises(W4A16Error):
        grouped.gemm(z(4, 72)[:, 4:68], W, o)


@gpu
def test_rows_beyond_two_and_four_gib(grouped):
    """X, Y and the weights reach past 2^32 bytes."""
    import torch
    K = 4096
    X = torch.zeros(600000, K, device="cuda", dtype=torch.bfloat16)  # 4.9 GB
    gen = generator(7)
    at = [0, 262143, 262144, 524287, 524288, 599999]
    X[at] = values(gen, (len(at), K), "bfloat16")
    W = torch.zeros(300, 2048, K, device="cuda", dtype=torch.bfloat16)  # 5.0 GB
    W[299] = values(gen, (2048, K), "bfloat16")
    offsets = np.zeros(301, np.int64)
    offsets[300] = len(at)
    ref, terms, _ = go.gemm(exact(X[at]), exact(W[299:]), [0, len(at)])
    tol = tolerance(X.dtype, ref, terms, K)
    compare(grouped.gemm(X, W, ints(offsets), rows=ints(at)), ref, tol, "gathered")
    dY = values(gen, (len(at), 64), "bfloat16")
    dref, dterms, _ = go.gemm_grad(exact(dY), exact(X[at]), [0, len(at)])
    dW = grouped.gemm_grad(dY, X, ints(offsets), rows=ints(at), dtype=torch.float32)
    compare(dW[299:], dref, tolerance(torch.float32, dref, dterms, len(at)), "gathered gradient")
    offsets[:300], offsets[300] = 599990, 600000
    Y = torch.zeros(600000, 4096, device="cuda", dtype=torch.bfloat16)[:, :2048]  # rows to 4.9 GB
    grouped.gemm(X, W, ints(offsets), out=Y)
    compare(Y[599999:], ref[-1:], tol[-1:], "in place")


@gpu
@pytest.mark.parametrize("T,N,K,tile", [(50, 136, 264, 16), (3000, 2056, 2064, 256)])
def test_replayed_graphs_and_other_streams(grouped, T, N, K, tile):
    import torch
    gen = generator(8)
    E, top_k = 8, 2
    assert grouped.query_tile(E, T * top_k, N, K)[0] in (tile, 64) and grouped.query_tile(E, T * top_k, N, K, grad=True)[0] == max(tile, 64)
    ids = torch.randint(-1, E, (T, top_k), generator=gen, device="cuda", dtype=torch.int32)
    X, W = values(gen, (T, K), "bfloat16"), values(gen, (E, N, K), "bfloat16")

    def work():
        offsets, order, place = grouped.sort(ids, E)
        Y = grouped.gemm(X, W, offsets, rows=order, top_k=top_k)
        dW = grouped.gemm_grad(Y, X, offsets, rows=order, top_k=top_k, dtype=torch.float32)
        return offsets, order, place, Y, grouped.gemm(Y, W, offsets, transposed=True), dW
    work()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = work()
    stream = torch.cuda.Stream()
    for i in range(3):
        ids.copy_(torch.randint(-1, E, (T, top_k), generator=gen, device="cuda", dtype=torch.int32))
        X.copy_(values(gen, (T, K), "bfloat16"))
        eager = work()
        graph.replay()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            other = work()
        torch.cuda.current_stream().wait_stream(stream)
        torch.cuda.synchronize()
        for a, b, c in zip(eager, captured, other):
            assert torch.equal(a, b) and torch.equal(a, c), i


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_a_layer_of_experts_forward_and_backward(kind):
    """Route, sort, gate and up, down, and the gradients, as a training step runs them, against 64-bit automatic differentiation of the definition.

    A gradient passes up to three roundings to 16 bits and the sums between them: each value is held to 8 half steps of its type relative to the root mean square
    of its tensor beside its own size (three roundings of inputs to the products, one of the result, twice over for two products one behind the other)."""
    import torch
    from paper_2601_16536_amd import grouped, moe
    gen = generator(9)
    T, E, top_k, H, I = 61, 6, 2, 64, 96
    dtype = getattr(torch, kind)
    logits = values(gen, (T, E), kind)
    X = values(gen, (T, H), kind)
    W13 = (values(gen, (E, 2 * I, H), "float32") / H ** 0.5).to(dtype)
    W2 = (values(gen, (E, H, I), "float32") / I ** 0.5).to(dtype)
    dOut = values(gen, (T, H), kind)

    ids, weights = moe.route(logits, top_k)
    ids[5] = -1  # a token that goes nowhere
    offsets, order, place = grouped.sort(ids, E)
    both = grouped.gemm(X, W13, offsets, rows=order, top_k=top_k)
    gate, up = both.float().chunk(2, dim=1)
    hidden = (gate * torch.sigmoid(gate) * up).to(dtype)
    y = grouped.gemm(hidden, W2, offsets)
    out = (y[place.long()].view(T, top_k, H).float() * weights.unsqueeze(2)).sum(1)

    w_sorted = weights.flatten()[order.long()].unsqueeze(1)
    dy = (dOut[order.long() // top_k].float() * w_sorted).to(dtype)
    dW2 = grouped.gemm_grad(dy, hidden, offsets, dtype=torch.float32)
    dh = grouped.gemm(dy, W2, offsets, transposed=True).float()
    s = torch.sigmoid(gate)
    dboth = torch.cat([dh * up * s * (1 + gate * (1 - s)), dh * gate * s], dim=1).to(dtype)
    dW13 = grouped.gemm_grad(dboth, X, offsets, rows=order, top_k=top_k, dtype=torch.float32)
    dX = grouped.gemm(dboth, W13, offsets, transposed=True)[place.long()].view(T, top_k, H).float().sum(1)

    x, a, b = (t.double().cpu().requires_grad_() for t in (X, W13, W2))
    ref = torch.zeros(T, H, dtype=torch.float64)
    for t, (who, w) in enumerate(zip(ids.tolist(), weights.double().cpu())):
        for e, v in zip(who, w):
            if e >= 0:
                g, u = (a[e] @ x[t]).chunk(2)
                ref = ref + torch.nn.functional.one_hot(torch.tensor(t), T).double().unsqueeze(1) * (v * (b[e] @ (g * torch.sigmoid(g) * u)))
    ref.backward(dOut.double().cpu())
    assert bool((out[5] == 0).all()) and bool((dX[5] == 0).all())
    half = half_step(dtype)[0]
    for name, got, want in (("out", out, ref), ("dX", dX, x.grad), ("dW13", dW13, a.grad), ("dW2", dW2, b.grad)):
        w = want.detach().numpy()
        compare(got, w, 8 * half * (np.abs(w) + np.sqrt((w ** 2).mean())), name)

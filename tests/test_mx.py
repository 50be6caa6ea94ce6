"""Microscaled 4-bit floating point: pins of the CPU oracle, refusals, then the HIP kernels against the oracle.

Tolerance of the products, per output, with A = sum_k |x_k| |w_k|: the elements and scales enter exactly; an output is a chain of at most
K/32 + 16 additions of FP32 partial sums (16 waves), each of them a sum of 32 products (128 with MXFP4 X) inside one matrix instruction,
so at most K/32 + 16 + 128 roundings, each below 2^-23 A (the matrix instruction may truncate); then one rounding to the output's
type, half a unit in the last place: 2^-11 of an FP16 value (ten fraction bits) or 2^-25 below its normal range, 2^-8 of a BF16 value (seven).
"""
import math
import os

import numpy as np
import pytest

from oracle import mx_oracle as mo

gpu = pytest.mark.gpu


# ---- the oracle's pins ----

def test_elements_are_e2m1():
    for code in range(16):
        e, f = (code >> 1) & 3, code & 1
        v = f * 0.5 if e == 0 else (1 + 0.5 * f) * 2.0 ** (e - 1)
        assert mo.element(code) == (-v if code & 8 else v)


def test_oracle_quantizer_on_worked_blocks():
    x = np.zeros((4, 32))
    x[0, :9] = [6, -6, 5, 3.5, 2.5, 1.75, 1.25, 0.25, 0.26]    # ties: 5 -> 4, 3.5 -> 4, 2.5 -> 2, 1.75 -> 2, 1.25 -> 1, 0.25 -> 0
    x[1, 0], x[1, 1] = 7.9, -0.1                                # saturates at 6: 7.9 < 8 keeps exponent 0; -0.1 -> -0
    x[2, 0], x[2, 5] = 2.0 ** -130, 2.0 ** -128                 # the scale's lower end: 2^-127, of which 2^-128 is half
    x[3, 3] = np.inf
    codes, scales = mo.quantize(x)
    assert scales.tolist() == [[127], [127], [0], [255]]
    q = np.stack([codes & 15, codes >> 4], -1).reshape(4, 32)
    assert q[0, :9].tolist() == [7, 15, 6, 6, 4, 4, 2, 0, 1]
    assert q[1, :2].tolist() == [7, 8]
    assert q[2, 0] == 0 and q[2, 5] == 1
    assert not q[3].any()
    v = mo.values(codes, scales)
    assert v[0, :4].tolist() == [6, -6, 4, 4] and np.isnan(v[3]).all() and v[2, 5] == 2.0 ** -128


def test_oracle_values_survive_quantization():
    """A matrix of representable values whose blocks hold a 4 or a 6 is its own quantization."""
    rng = np.random.default_rng(3)
    q = rng.integers(0, 16, (5, 96))
    q[:, ::32] = 6
    s = rng.integers(1, 250, (5, 3))
    x = mo.element(q) * np.repeat(np.ldexp(1.0, s - 127), 32, axis=1)
    codes, scales = mo.quantize(x)
    assert np.array_equal(scales, s) and np.array_equal(mo.values(codes, scales), x)


# ---- refusals ----

@pytest.fixture(scope="module")
def mx():
    from paper_2601_16536_amd import binding, build, mx
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    mx.lib()
    return mx


def test_header_functions_are_exported(mx):
    import re
    from paper_2601_16536_amd import binding
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "w4a16_mx.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(w4a16_mx_[a-z0-9_]+)\s*\(", text))
    assert declared == set(mx.EXPORTS)
    for name in declared:
        assert getattr(binding.lib(), name) is not None


def test_argument_checks_need_no_gpu(mx):
    from paper_2601_16536_amd import binding as b
    L = mx.lib()
    for f in (lambda *a: L.w4a16_mx_quantize(*a), lambda X, t, r, K, ld, c, s, st: L.w4a16_mx_dequantize(c, s, r, K, X, t, ld, st)):
        assert f(0, 0, 0, 32, 32, 0, 0, 0) == b.OK                       # no rows
        assert f(0, 0, 1, 32, 32, 16, 16, 0) == b.ERR_NULL
        assert f(16, 0, 1, 32, 32, 16, 0, 0) == b.ERR_NULL
        assert f(16, 3, 1, 32, 32, 16, 16, 0) == b.ERR_SHAPE             # no such type
        assert f(16, 0, -1, 32, 32, 16, 16, 0) == b.ERR_SHAPE
        assert f(16, 0, 1, 48, 48, 16, 16, 0) == b.ERR_SHAPE
        assert f(16, 0, 1, 0, 0, 16, 16, 0) == b.ERR_SHAPE
        assert f(16, 0, 2, 64, 32, 16, 16, 0) == b.ERR_SHAPE             # rows overlap
        assert f(16, 0, 2, 32, 36, 16, 16, 0) == b.ERR_ALIGN             # the second row is not aligned
        assert f(16, 2, 2, 32, 34, 16, 16, 0) == b.ERR_ALIGN
        assert f(24, 0, 1, 32, 32, 16, 16, 0) == b.ERR_ALIGN
        assert f(16, 0, 1, 32, 32, 24, 16, 0) == b.ERR_ALIGN
    g = L.w4a16_mx_gemm  # X, type, ldx, codes, scales, M, N, K, Y, ldy, stream
    assert g(0, 0, 32, 0, 0, 0, 8, 32, 0, 8, 0) == b.OK
    assert g(16, 0, 32, 16, 16, 1, 8, 32, 0, 8, 0) == b.ERR_NULL
    assert g(16, 2, 32, 16, 16, 1, 8, 32, 16, 8, 0) == b.ERR_SHAPE       # FP32 X
    assert g(16, 0, 32, 16, 16, -1, 8, 32, 16, 8, 0) == b.ERR_SHAPE
    assert g(16, 0, 32, 16, 16, 1, 0, 32, 16, 8, 0) == b.ERR_SHAPE
    assert g(16, 0, 32, 16, 16, 1, 8, 40, 16, 8, 0) == b.ERR_SHAPE
    assert g(16, 0, 32, 16, 16, 2, 8, 32, 16, 7, 0) == b.ERR_SHAPE       # rows of Y overlap
    assert g(16, 0, 16, 16, 16, 2, 8, 32, 16, 8, 0) == b.ERR_SHAPE
    assert g(16, 0, 36, 16, 16, 2, 8, 32, 16, 8, 0) == b.ERR_ALIGN
    assert g(18, 0, 32, 16, 16, 1, 8, 32, 16, 8, 0) == b.ERR_ALIGN
    assert g(16, 0, 32, 18, 16, 1, 8, 32, 16, 8, 0) == b.ERR_ALIGN
    assert g(16, 0, 32, 16, 16, 1, 8, 32, 17, 8, 0) == b.ERR_ALIGN
    h = L.w4a16_mx_gemm_mx  # x codes, x scales, codes, scales, M, N, K, Y, type, ldy, stream
    assert h(0, 0, 0, 0, 0, 8, 32, 0, 0, 8, 0) == b.OK
    assert h(16, 0, 16, 16, 1, 8, 32, 16, 0, 8, 0) == b.ERR_NULL
    assert h(16, 16, 16, 16, 1, 8, 33, 16, 0, 8, 0) == b.ERR_SHAPE
    assert h(16, 16, 16, 16, 1, 8, 32, 16, 2, 8, 0) == b.ERR_SHAPE
    assert h(18, 16, 16, 16, 1, 8, 32, 16, 0, 8, 0) == b.ERR_ALIGN


def test_binding_refuses_host_tensors_and_other_types(mx):
    import torch
    x = torch.zeros(2, 64)
    with pytest.raises(TypeError):
        mx.quantize(x)
    with pytest.raises(TypeError):
        mx.quantize(x.to(torch.float64))
    with pytest.raises(TypeError):
        mx.gemm(x.half(), torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8))


# ---- the kernels ----

def _torch(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _exact(t):
    import torch
    return t.detach().to(torch.float64).cpu().numpy()


def _random_mx(rng, rows, K, lo=115, hi=132):
    codes = rng.integers(0, 256, (rows, K // 2), dtype=np.uint8)
    scales = rng.integers(lo, hi, (rows, K // 32), dtype=np.uint8)
    return codes, scales


def check(Y, ref, terms, K, where):
    """Y (torch) against the oracle's result and sum of magnitudes, by the tolerance derived above."""
    import torch
    y = _exact(Y)
    half, least = (2.0 ** -11, 2.0 ** -25) if Y.dtype == torch.float16 else (2.0 ** -8, 0.0)
    sums = (K / 32 + 16 + 128) * 2.0 ** -23 * terms
    tol = sums + half * (np.abs(ref) + sums) + least
    bad = ~(np.abs(y - ref) <= tol)
    assert not bad.any(), "%s: %d outputs off, first at %r: %g for %g, tolerance %g" % (
        where, bad.sum(), np.argwhere(bad)[0].tolist(), y[tuple(np.argwhere(bad)[0])], ref[tuple(np.argwhere(bad)[0])], tol[tuple(np.argwhere(bad)[0])])


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
def test_every_16_bit_value_quantizes_as_the_oracle_says(mx, kind):
    """All 65536 bit patterns, each the largest of its block and each beside a larger one."""
    import torch
    bits = np.arange(65536, dtype=np.int64).astype(np.uint16)
    rng = np.random.default_rng(1)
    alone = np.zeros((65536, 32), np.uint16)
    alone[np.arange(65536), rng.integers(0, 32, 65536)] = bits
    mixed = rng.permutation(bits).reshape(-1, 32)
    near = (rng.integers(0, 64, (4096, 32)) + rng.integers(0, 65536 - 64, (4096, 1))).astype(np.uint16)  # neighbours: ties and exponents' ends
    x = np.concatenate([alone, mixed, near])
    X = _torch(x.view(np.int16)).view(getattr(torch, kind))
    codes, scales = mx.quantize(X)
    with np.errstate(all="ignore"):
        wc, ws = mo.quantize(_exact(X))
    assert np.array_equal(scales.cpu().numpy(), ws)
    assert np.array_equal(codes.cpu().numpy(), wc)


@gpu
def test_fp32_quantizes_as_the_oracle_says(mx):
    import torch
    rng = np.random.default_rng(2)
    x = rng.integers(0, 2 ** 32, (20000, 32), dtype=np.uint64).astype(np.uint32)
    x[:10000] = (x[:10000] & 0x81FFFFFF) | (rng.integers(0, 255, (10000, 1)).astype(np.uint32) << 23)  # exponents near each other
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], np.float32)
    t = np.concatenate([np.nextafter(ties, np.float32(0)), ties, np.nextafter(ties, np.float32(9)), -ties]).astype(np.float32)
    x = np.concatenate([x.view(np.float32), t[None] * np.ldexp(np.float32(1), np.arange(-126, 120)).astype(np.float32)[:, None]])
    X = _torch(x)
    codes, scales = mx.quantize(X)
    with np.errstate(all="ignore"):
        wc, ws = mo.quantize(x.astype(np.float64))
    assert np.array_equal(scales.cpu().numpy(), ws) and np.array_equal(codes.cpu().numpy(), wc)


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "float32"])
def test_every_code_and_scale_reads_back(mx, kind):
    import torch
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(16, 16), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8), 16).reshape(-1, 1)
    out = mx.dequantize(_torch(codes), _torch(scales), dtype=getattr(torch, kind))
    want = torch.from_numpy(mo.values(codes, scales)).to(torch.float32)  # (exact but for overflow)
    want = want.to(getattr(torch, kind))
    got = out.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got, nan=0.0), torch.nan_to_num(want, nan=0.0))
    assert torch.equal(torch.signbit(got)[16:-16], torch.signbit(want)[16:-16])


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows,K,ld", [(1, 32, 32), (3, 96, 104), (7, 4128, 4128), (129, 32, 40), (1, 28672, 28672), (65, 1056, 2112)])
def test_shapes_and_strides_round_trip(mx, kind, rows, K, ld):
    import torch
    rng = np.random.default_rng([rows, K])
    big = _torch(rng.standard_normal((rows, ld)).astype(np.float32)).to(getattr(torch, kind))
    X = big[:, :K]
    codes, scales = mx.quantize(X)
    wc, ws = mo.quantize(_exact(X))
    assert np.array_equal(scales.cpu().numpy(), ws) and np.array_equal(codes.cpu().numpy(), wc)
    out = torch.full_like(big, 7.0)
    mx.dequantize(codes, scales, out=out[:, :K])
    assert torch.equal(out[:, :K].double().cpu(), torch.from_numpy(mo.values(wc, ws)).to(out.dtype).double())
    assert bool((out[:, K:] == 7.0).all())


@gpu
def test_offsets_beyond_32_bits(mx):
    """More than 2^32 values in, and weights of more than 4 GiB of codes in a product; the last rows are looked at."""
    import torch
    K = 65536
    rows = 2 ** 32 // K + 40
    X = torch.zeros(rows, K, dtype=torch.float16, device="cuda")
    rng = np.random.default_rng(4)
    X[-40:] = _torch(rng.standard_normal((40, K)).astype(np.float16))
    codes, scales = mx.quantize(X)
    tail = _exact(X[-40:])
    wc, ws = mo.quantize(tail)
    assert np.array_equal(scales[-40:].cpu().numpy(), ws) and np.array_equal(codes[-40:].cpu().numpy(), wc)
    X.fill_(1.0)
    mx.dequantize(codes, scales, out=X)
    assert np.array_equal(_exact(X[-40:]), mo.values(wc, ws).astype(np.float16).astype(np.float64)) and not bool(X[:1000].any())
    del X
    N = 2 ** 32 // (K // 2) + 21
    W = torch.zeros(N, K // 2, dtype=torch.uint8, device="cuda")
    S = torch.full((N, K // 32), 127, dtype=torch.uint8, device="cuda")
    W[-40:], S[-40:] = codes[-40:], scales[-40:]
    x = _torch(rng.standard_normal((2, K))).to(torch.bfloat16)
    ref, terms = mo.gemm(_exact(x), wc, ws)
    Y = mx.gemm(x, W, S)
    check(Y[:, -40:], ref, terms, K, "weights past 4 GiB")
    assert not bool(Y[:, :-40].any())


GEMM_SHAPES = [(1, 1, 32), (1, 17, 96), (2, 16, 128), (3, 33, 160), (16, 64, 4096), (17, 100, 1056), (5, 1000, 2080), (31, 48, 512),
               (33, 130, 288), (64, 257, 640), (65, 31, 1024), (100, 520, 1152), (129, 264, 416), (200, 1030, 2048), (257, 129, 4128)]


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "mx"])
@pytest.mark.parametrize("M,N,K", GEMM_SHAPES)
def test_products_match_the_oracle(mx, kind, M, N, K):
    import torch
    rng = np.random.default_rng([M, N, K])
    wc, ws = _random_mx(rng, N, K)
    if kind == "mx":
        xc, xs = _random_mx(rng, M, K)
        ref, terms = mo.gemm(mo.values(xc, xs), wc, ws)
        for dtype in (torch.bfloat16, torch.float16):
            scale = 2.0 ** -8 if dtype is torch.float16 else 1.0  # FP16's range
            xd = np.uint8(8) if dtype is torch.float16 else np.uint8(0)
            Y = mx.gemm_mx(_torch(xc), _torch(xs - xd), _torch(wc), _torch(ws), dtype=dtype)
            check(Y, ref * scale, terms * scale, K, "M=%d N=%d K=%d %s" % (M, N, K, dtype))
        return
    X = _torch(rng.standard_normal((M, K)) * (2.0 ** -4 if kind == "float16" else 1.0)).to(getattr(torch, kind))
    ref, terms = mo.gemm(_exact(X), wc, ws)
    check(mx.gemm(X, _torch(wc), _torch(ws)), ref, terms, K, "M=%d N=%d K=%d %s" % (M, N, K, kind))


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "mx"])
@pytest.mark.parametrize("M", [1, 20, 70, 300])
def test_whole_numbers_come_out_exactly(mx, kind, M):
    """Sums of whole numbers below 256 (BF16's exact range) have one answer."""
    import torch
    N, K = 200, 1024
    rng = np.random.default_rng(M)
    wq = rng.choice([0, 0, 0, 2, 10, 4, 12], (N, K)).astype(np.uint8)  # 0, +-1, +-2
    wc = wq[:, 0::2] | (wq[:, 1::2] << 4)
    ws = np.full((N, K // 32), 127, np.uint8)
    xq = np.zeros((M, K), np.uint8)
    for m in range(M):
        xq[m, rng.choice(K, 60, replace=False)] = rng.choice([2, 10, 4, 12], 60)
    xc = xq[:, 0::2] | (xq[:, 1::2] << 4)
    xs = np.full((M, K // 32), 127, np.uint8)
    ref = mo.element(xq) @ mo.element(wq).T
    assert np.abs(ref).max() <= 256
    if kind == "mx":
        Y = mx.gemm_mx(_torch(xc), _torch(xs), _torch(wc), _torch(ws))
    else:
        Y = mx.gemm(_torch(mo.element(xq)).to(getattr(torch, kind)), _torch(wc), _torch(ws))
    assert np.array_equal(_exact(Y), ref)


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "mx"])
@pytest.mark.parametrize("M", [1, 40, 150])
def test_not_a_number_stays_in_its_row_or_column(mx, kind, M):
    import torch
    N, K = 70, 288
    rng = np.random.default_rng(7)
    wc, ws = _random_mx(rng, N, K)
    ws[5, 8] = 255  # in the last block, behind the last whole step of four
    ws[66, 0] = 255
    xc, xs = _random_mx(rng, M, K)
    bad_row = M - 1 if M > 1 else None
    if kind == "mx":
        if bad_row is not None:
            xs[bad_row, 3] = 255
        Y = mx.gemm_mx(_torch(xc), _torch(xs), _torch(wc), _torch(ws))
    else:
        X = _torch(rng.standard_normal((M, K)) * 0.01).to(getattr(torch, kind))
        if bad_row is not None:
            X[bad_row, 287] = float("nan")
        Y = mx.gemm(X, _torch(wc), _torch(ws))
    want = np.zeros((M, N), bool)
    want[:, [5, 66]] = True
    if bad_row is not None:
        want[bad_row] = True
    assert np.array_equal(np.isnan(_exact(Y)), want)


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "mx"])
def test_extreme_scales(mx, kind):
    """Scales at both ends of their range: products of numbers that only FP32 sums can hold."""
    import torch
    M, N, K = 4, 32, 256
    rng = np.random.default_rng(9)
    wc, _ = _random_mx(rng, N, K)
    for s, factor in ((0, 120), (1, 120), (252, -120), (120, 0)):
        ws = np.full((N, K // 32), s, np.uint8)
        if kind == "mx":
            xc, _ = _random_mx(rng, M, K)
            xs = np.full((M, K // 32), 127 + factor, np.uint8)
            ref, terms = mo.gemm(mo.values(xc, xs), wc, ws)
            check(mx.gemm_mx(_torch(xc), _torch(xs), _torch(wc), _torch(ws)), ref, terms, K, "s=%d" % s)
        elif kind == "bfloat16":
            X = _torch(rng.standard_normal((M, K)) * 2.0 ** factor).to(torch.bfloat16)
            ref, terms = mo.gemm(_exact(X), wc, ws)
            check(mx.gemm(X, _torch(wc), _torch(ws)), ref, terms, K, "s=%d" % s)
        else:  # FP16: the smallest and largest X against scales far from 1 that bring the result back
            lo = {0: None, 1: None, 252: None, 120: 127 + 14}[s]
            if lo is None:
                continue
            ws = np.full((N, K // 32), lo, np.uint8)
            X = _torch(rng.integers(-1023, 1024, (M, K)) * 2.0 ** -24).to(torch.float16)  # subnormal numbers
            ref, terms = mo.gemm(_exact(X), wc, ws)
            check(mx.gemm(X, _torch(wc), _torch(ws)), ref, terms, K, "subnormal X")
            ws = np.full((N, K // 32), 127 - 40, np.uint8)
            X = _torch(rng.choice([-65504.0, 65504.0, 2.0 ** -24], (M, K))).to(torch.float16)
            ref, terms = mo.gemm(_exact(X), wc, ws)
            check(mx.gemm(X, _torch(wc), _torch(ws)), ref, terms, K, "largest X, elements below FP16's range")


@gpu
@pytest.mark.parametrize("M", [1, 9, 40, 130])
def test_strides_and_outputs_between_canaries(mx, M):
    import torch
    N, K = 100, 416
    rng = np.random.default_rng(M)
    wc, ws = _random_mx(rng, N, K)
    big = _torch(rng.standard_normal((M, 3 * K))).to(torch.bfloat16)
    X = big[:, K:2 * K]
    flat = torch.full((8 + M * (N + 5),), 9.0, dtype=torch.bfloat16, device="cuda")
    out = flat[3:3 + M * (N + 5)].view(M, N + 5)[:, :N]  # rows two-byte aligned
    scales = _torch(np.concatenate([np.zeros(1, np.uint8), ws.ravel()]))[1:].view(N, K // 32)  # not aligned
    Y = mx.gemm(X, _torch(wc), scales, out=out)
    assert Y.data_ptr() == out.data_ptr()
    ref, terms = mo.gemm(_exact(X), wc, ws)
    check(out, ref, terms, K, "strided")
    flat[3:3 + M * (N + 5)].view(M, N + 5)[:, :N] = 9.0
    assert bool((flat == 9.0).all())


@gpu
def test_bitwise_reproducible_and_row_independent(mx):
    import torch
    rng = np.random.default_rng(11)
    N, K = 300, 4096
    wc, ws = map(_torch, _random_mx(rng, N, K))
    X = _torch(rng.standard_normal((150, K))).to(torch.bfloat16)
    first = mx.gemm(X, wc, ws)
    for _ in range(5):
        assert torch.equal(first, mx.gemm(X, wc, ws))


@gpu
def test_other_streams_and_graphs(mx):
    import torch
    rng = np.random.default_rng(12)
    N, K = 264, 1024
    wc, ws = map(_torch, _random_mx(rng, N, K))
    for M in (1, 20, 150):
        X = _torch(rng.standard_normal((M, K))).to(torch.float16)
        want = mx.gemm(X, wc, ws)
        xc, xs = mx.quantize(X)
        want_mx = mx.gemm_mx(xc, xs, wc, ws)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        out = torch.empty_like(want)
        mx.gemm(X, wc, ws, out=out, stream=side)
        side.synchronize()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c, s = mx.quantize(X)
            y, ymx = mx.gemm(X, wc, ws), mx.gemm_mx(c, s, wc, ws)
        for _ in range(3):
            y.zero_(), ymx.zero_(), c.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want) and torch.equal(ymx, want_mx)
            torch.randn(1000, device="cuda").sum().item()


@gpu
def test_empty_batches(mx):
    import torch
    rng = np.random.default_rng(13)
    wc, ws = map(_torch, _random_mx(rng, 40, 64))
    assert mx.gemm(torch.empty(0, 64, dtype=torch.float16, device="cuda"), wc, ws).shape == (0, 40)
    c, s = mx.quantize(torch.empty(0, 64, device="cuda"))
    assert c.shape == (0, 32) and s.shape == (0, 2)
    assert mx.gemm_mx(c, s, wc, ws).shape == (0, 40) and mx.dequantize(c, s).shape == (0, 64)


@gpu
def test_binding_refuses_what_does_not_fit(mx):
    import torch
    X = torch.zeros(4, 64, dtype=torch.float16, device="cuda")
    c, s = mx.quantize(X)
    with pytest.raises(ValueError):
        mx.quantize(torch.zeros(4, 48, device="cuda"))
    with pytest.raises(TypeError):
        mx.quantize(torch.zeros(64, 4, dtype=torch.float16, device="cuda").t())
    with pytest.raises(ValueError):
        mx.gemm(X[:, :32], c, s)
    with pytest.raises(ValueError):
        mx.gemm(X, c, s[:, :1].contiguous())
    with pytest.raises(TypeError):
        mx.gemm(X.float(), c, s)
    with pytest.raises(TypeError):
        mx.gemm(X, c.t(), s)
    with pytest.raises(ValueError):
        mx.gemm(X, c, s, out=torch.empty(4, 5, dtype=torch.float16, device="cuda"))
    with pytest.raises(Exception):
        mx.gemm(torch.zeros(4, 65, dtype=torch.float16, device="cuda")[:, 1:], c, s)  # rows not aligned

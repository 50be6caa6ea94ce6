"""MXFP4 products over the whole range of sizes that the header names: what is planned, on the CPU, and the ends of the range on the GPU.  Tolerances
as derived in test_mx.py (16 waves at most, K/32 + 16 + 128 roundings: whatever the pieces that K comes in, a wave's sums are one chain)."""
import os
import subprocess
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


@pytest.mark.parametrize("kind", ["float16", "bfloat16", "mx"])
def test_the_largest_sizes_have_a_plan(mx, kind):
    most = 2 ** 31 - 1
    for M, N, K in ((most, 1, 32), (1, most, 32), (most, most, 32), (most, 1, 128), (most, 64, 1024), (16, most, 4096), (most, most, LONGEST)):
        lds, chunks = mx.query_lds(M, N, K, **_how(kind))
        assert 0 < lds <= LDS and chunks >= 1


@gpu
@pytest.mark.parametrize("kind", ["bfloat16", "mx"])
def test_more_columns_than_one_grid_has_threads_for(mx, kind):
    """Four threads to a column: 2^30 columns are 2^32 threads.  x is 1 at k = 0 alone, so Y is W's first column: elements 0 .. 6 in turn, with a scale of 1 or 2."""
    import torch
    N, K = 2 ** 30 + 37, 32
    codes = torch.zeros(N, K // 2, dtype=torch.uint8, device="cuda")
    scales = torch.full((N, 1), 127, dtype=torch.uint8, device="cuda")
    turn = torch.arange(N, dtype=torch.int32, device="cuda").remainder_(40).to(torch.uint8)
    codes[:, 0] = turn % 8
    scales[:, 0] += turn // 20
    values = torch.tensor(mo.MAGNITUDES, device="cuda", dtype=torch.bfloat16)[torch.arange(40, device="cuda") % 8] * (1 + torch.arange(40, device="cuda") // 20)
    if kind == "mx":
        xc = torch.zeros(1, K // 2, dtype=torch.uint8, device="cuda")
        xc[0, 0] = 2
        Y = mx.gemm_mx(xc, torch.full((1, 1), 127, dtype=torch.uint8, device="cuda"), codes, scales)
    else:
        x = torch.zeros(1, K, dtype=torch.bfloat16, device="cuda")
        x[0, 0] = 1
        Y = mx.gemm(x, codes, scales)
    for n in range(0, N, 2 ** 27):  # 40 divides no power of two: the pieces begin at places of their own
        here = Y[0, n:n + 2 ** 27]
        assert torch.equal(here, values[turn[n:n + 2 ** 27].int()])


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "mx"])
@pytest.mark.parametrize("K", [32, 160])
def test_many_rows(mx, kind, K):
    """More row blocks than a grid's second dimension is documented to hold, and pieces of rows: strided X and Y, every row with numbers of its own."""
    import torch
    M, N = 65535 * 16 + 21, 5
    rng = np.random.default_rng(K)
    wc, ws = tmx._random_mx(rng, N, K, 126, 129)
    W = torch.from_numpy(mo.values(wc, ws)).float().cuda()
    out = torch.full((M, N + 2), 9.0, dtype=torch.bfloat16 if kind == "mx" else getattr(torch, kind), device="cuda")
    x = torch.randint(-2, 3, (M, K + 8), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).float()[:, :K]
    if kind == "mx":
        xc, xs = mx.quantize(x.contiguous())
        mx.gemm_mx(xc, xs, tmx._torch(wc), tmx._torch(ws), out=out[:, :N])
    else:
        big = torch.zeros(M, K + 8, dtype=out.dtype, device="cuda")
        big[:, :K] = x
        mx.gemm(big[:, :K], tmx._torch(wc), tmx._torch(ws), out=out[:, :N])
    want = torch.stack([(x * W[n]).sum(1) for n in range(N)], 1).to(out.dtype)  # whole multiples of a quarter below 2^12: exact in FP32
    assert torch.equal(out[:, :N], want) and bool((out[:, N:] == 9.0).all())


def test_a_failing_call_leaves_no_error_behind(tmp_path):
    """A runtime whose hipFuncSetAttribute fails, in a child process: the call ends there, before anything is launched, and what the runtime keeps of it must not be the
    next caller's.  16 rows, K = N = 4096: a kernel that asks for more LDS than the default."""
    source, shim = tmp_path / "shim.c", tmp_path / "shim.so"
    source.write_text("static int last;\n"
                      "int hipFuncSetAttribute(const void *f, int a, int v) { (void)f; (void)a; (void)v; return last = 1; }\n"
                      "int hipGetLastError(void) { int e = last; last = 0; return e; }\n")
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-o", str(shim), str(source)])
    code = """if True:
        import ctypes, sys
        shim = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
        from paper_2601_16536_amd import binding, mx
        assert mx.lib().w4a16_mx_gemm(256, 1, 4096, 256, 256, 16, 4096, 4096, 256, 4096, 0) == binding.ERR_HIP
        assert "invalid argument" in binding.last_hip_error(), binding.last_hip_error()
        assert shim.hipGetLastError() == 0
        print("clean")
        """
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code, str(shim)], cwd=root, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and "clean" in r.stdout, r.stdout[-2000:]


# X in several pieces of K: 16 waves and 8 (N above 4096), K of whole steps and not, one piece short of whole pairs, all three types
CHUNKED = [("mx", 16, 100, 28672), ("mx", 16, 100, 28640), ("mx", 7, 4130, 20000), ("mx", 6, 4100, 21504), ("mx", 21, 40, 28672)]
CHUNKED += [(kind, *sizes) for kind in ("bfloat16", "float16") for sizes in ((8, 70, 16384), (11, 70, 16416), (3, 4130, 12512), (2, 4100, 18432), (1, 4099, 32960))]


def test_the_chunked_shapes_are_of_several_chunks(mx):
    for kind, M, N, K in CHUNKED:
        assert mx.query_tile(M, N, K, **_how(kind)) == (16, 16) and mx.query_lds(M, N, K, **_how(kind))[1] > 1, (kind, M, N, K)


@gpu
@pytest.mark.parametrize("kind,M,N,K", CHUNKED)
def test_x_in_chunks_matches_the_oracle(mx, kind, M, N, K):
    Y, ref, terms = _product(mx, kind, np.random.default_rng([M, N, K]), M, N, K)
    tmx.check(Y, ref, terms, K, "M=%d N=%d K=%d %s" % (M, N, K, kind))


@gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16", "mx"])
@pytest.mark.parametrize("M", [1, 40, 300])
def test_weights_beyond_fp32(mx, kind, M):
    """Rows 3 and 30 of W hold 6 2^126 and 2 2^127 in their first block, which no FP32 number is.  x is 2^-20, -2^-20 there, and the sum of the two 0; FP16 and MXFP4 X have
    that, and row 30's third value beside; with BF16 X such a weight is infinite, and the rows' outputs are no numbers.  The other outputs are as ever."""
    import torch
    N, K = 70, 288
    rng = np.random.default_rng(M)
    wc, ws = tmx._random_mx(rng, N, K)
    wc[[3, 30]] = 0
    ws[3, 0], ws[30, 0] = 253, 254
    wc[3, 0], wc[30, 0] = 0x77, 0x44
    wc[30, 16] = 2                                   # 1 at k = 32
    ws[30, 1] = 127
    xq = rng.integers(0, 16, (M, K)).astype(np.uint8)
    xq[:, 0], xq[:, 1], xq[:, 32] = 2, 10, 6         # 1, -1, 4, times the scale
    xc = xq[:, 0::2] | (xq[:, 1::2] << 4)
    xs = np.full((M, K // 32), 107, np.uint8)
    x = mo.values(xc, xs)
    if kind == "mx":
        Y = mx.gemm_mx(tmx._torch(xc), tmx._torch(xs), tmx._torch(wc), tmx._torch(ws))
    else:
        Y = mx.gemm(tmx._torch(x).to(getattr(torch, kind)), tmx._torch(wc), tmx._torch(ws))
    y = tmx._exact(Y)
    others = np.setdiff1d(np.arange(N), [3, 30])
    ref, terms = mo.gemm(x, wc[others], ws[others])
    tmx.check(Y[:, torch.from_numpy(others).cuda()], ref, terms, K, "beside weights beyond FP32")
    if kind == "bfloat16":
        assert not np.isfinite(y[:, [3, 30]]).any()
    else:
        assert not y[:, 3].any() and np.all(y[:, 30] == 4 * 2.0 ** -20)

"""The bindings of the products of rows in groups and of the adapters: sizes that 32 bits do not hold are refused, not taken modulo 2^32."""
import math

import pytest


class Tensor:
    """As much of a CUDA tensor as the checks look at."""
    is_cuda = True

    def __init__(self, shape, dtype):
        import torch
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", 0)

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def stride(self, i=None):
        strides = [math.prod(self.shape[j + 1:]) for j in range(len(self.shape))]
        return strides if i is None else strides[i]

    def is_contiguous(self):
        return True


def test_sizes_past_32_bits_are_refused():
    import torch
    from paper_2601_16536_amd import grouped, lora
    big, half, int32 = (1 << 32) + 8, torch.float16, torch.int32
    X, offsets, rows = Tensor((4, 8), half), Tensor((2,), int32), Tensor((4,), int32)
    for bad in (lambda: grouped.gemm(X, Tensor((1, big, 8), half), offsets), lambda: grouped.gemm(Tensor((4, big), half), Tensor((1, 8, big), half), offsets),
                lambda: grouped.gemm(X, Tensor((1, 8, 8), half), offsets, rows=rows, top_k=(1 << 32) + 2), lambda: grouped.gemm_grad(Tensor((4, big), half), X, offsets),
                lambda: grouped.gemm_grad(X, Tensor((4, big), half), offsets), lambda: lora.add(Tensor((4, 8), half), Tensor((4, 8), half), Tensor((big, 8, 8), half), Tensor((big, 8, 8), half), rows),
                lambda: lora.add(Tensor((big, 8), half), Tensor((big, 8), half), Tensor((1, 8, 8), half), Tensor((1, 8, 8), half), Tensor((big,), int32)),
                lambda: lora.grad(Tensor((4, 8), half), Tensor((4, 8), half), Tensor((1, big, 8), half), Tensor((1, 8, big), half), rows)):
        with pytest.raises(ValueError, match="past 32 bits"):
            bad()


def test_no_rows_of_an_x_without_rows_is_no_error():
    """A batch of no tokens, its (empty) list of rows in a buffer that has an address."""
    import os
    from paper_2601_16536_amd import binding as b, build, grouped
    if not os.path.exists(b.LIB_PATH):
        build.build(verbose=False)
    L = grouped.lib()
    # X, type, x_rows, ldx, rows, top_k, W, stride_w, ldw, transposed, offsets, E, count, N, K, Y, ldy, fill, stream
    for rows, top_k in ((0, 1), (64, 2), (64, 1)):
        assert L.w4a16_grouped_gemm(0, 0, 0, 64, rows, top_k, 16, 2048, 64, 0, 16, 2, 0, 32, 64, 0, 32, 1, 0) == b.OK
    assert L.w4a16_grouped_gemm(16, 0, 0, 64, 64, 2, 16, 2048, 64, 0, 16, 2, 4, 32, 64, 16, 32, 1, 0) == b.ERR_SHAPE

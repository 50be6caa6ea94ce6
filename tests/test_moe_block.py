"""The example block: its parts together against plain float64 operations on the values that its weights stand for."""
import numpy as np
import pytest

from oracle import mx_oracle as mo


@pytest.mark.gpu
@pytest.mark.parametrize("T,four", [(1, False), (3, True), (40, False)])
def test_block_matches_plain_operations(T, four):
    import torch
    from paper_2601_16536_amd.moe_block import random_block
    H, I, E, top_k = 256, 160, 8, 2
    block = random_block(H, I, E, top_k, four_bit_activations=four)
    gen = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, H, device="cuda", generator=gen).to(torch.bfloat16)
    o = torch.randn(T, H, device="cuda", generator=gen).to(torch.bfloat16)
    y = block(x, o)
    value = lambda pair: mo.values(*(t.cpu().numpy() for t in pair))
    f64 = lambda t: t.double().cpu().numpy()
    op = mo.values(*mo.quantize(f64(o))) if four else f64(o)
    bf16 = lambda a: f64(torch.from_numpy(a).to(torch.bfloat16))
    # BF16 is rounded where the block does: after each product and each sum; a sum whose terms are off by a rounding may round to the neighbour
    u = bf16(f64(x) + bf16(op @ value(block.o).T))
    logits = bf16(u @ value(block.router).T)
    ids, weights = mo.route(logits, top_k)
    want = u + mo.experts(u, ids, weights, value(block.w13), value(block.w2))
    got = f64(y)
    # per output: the layer's result, rounded, and the sum, rounded: 2^-8 of each; u, off by one neighbour (2^-8 of it) in a few places, passes through
    # two products of gain about one: compared in the norm of a token
    err = np.linalg.norm(got - want, axis=1) / np.linalg.norm(want, axis=1)
    assert (err <= 3 * 2.0 ** -8).all(), err
    assert np.array_equal(f64(block(x, o)), got)


@pytest.mark.gpu
def test_command_runs():
    from paper_2601_16536_amd import moe_block
    assert moe_block.main(["--tokens", "2", "--experts", "8", "--top-k", "2", "--hidden", "256", "--intermediate", "128", "--steps", "3"]) > 0

"""A mixture-of-experts block of a decoder on MXFP4 weights, as a serving program would run it for a few tokens:

    u = x + o W_o^T                       attention's output projection     mx.gemm (or mx.gemm_mx with `four_bit_activations`)
    logits = u W_r^T                      the router's product              mx.gemm
    ids, weights = choice of the top_k    moe.route
    y = u + experts(u)                    moe.experts

    python -m paper_2601_16536_amd.moe_block --tokens 4 --experts 64 --top-k 8 --hidden 4096 --intermediate 2048

runs it on random weights, recorded once as a HIP graph, and prints the time of a step.
"""
from __future__ import annotations

import argparse

from . import moe, mx


class MoeBlock:
    """Weights are quantized once (`mx.quantize`); a call enqueues on torch's current stream and allocates from torch's allocator, so it can be captured."""

    def __init__(self, W_o, W_router, W13, W2, top_k: int, activation: str = "silu", four_bit_activations: bool = False):
        self.o, self.router, self.w13, self.w2 = (mx.quantize(W) for W in (W_o, W_router, W13, W2))
        self.top_k, self.activation, self.four_bit_activations = top_k, activation, four_bit_activations

    def __call__(self, x, o):
        """x, o [T, H] float16 or bfloat16: the residual stream and attention's output.  Returns the new residual stream."""
        if self.four_bit_activations:
            u = x + mx.gemm_mx(*mx.quantize(o), *self.o, dtype=x.dtype)
        else:
            u = x + mx.gemm(o, *self.o)
        ids, weights = moe.route(mx.gemm(u, *self.router), self.top_k)
        return u + moe.experts(u, ids, weights, *self.w13, *self.w2, activation=self.activation)


def random_block(hidden: int, intermediate: int, experts: int, top_k: int, device="cuda", seed: int = 0, **options) -> MoeBlock:
    import torch
    gen = torch.Generator(device=device).manual_seed(seed)

    def weights(*shape):
        return torch.randn(*shape, device=device, generator=gen, dtype=torch.float32).mul_(shape[-1] ** -0.5).to(torch.bfloat16)
    return MoeBlock(weights(hidden, hidden), weights(experts, hidden), weights(experts, 2 * intermediate, hidden), weights(experts, hidden, intermediate),
                    top_k, **options)


def main(argv=None) -> float:
    import torch
    parser = argparse.ArgumentParser(description="times a mixture-of-experts block on MXFP4 weights")
    for name, value in (("--tokens", 4), ("--experts", 64), ("--top-k", 8), ("--hidden", 4096), ("--intermediate", 2048), ("--steps", 50)):
        parser.add_argument(name, type=int, default=value)
    parser.add_argument("--four-bit-activations", action="store_true", help="the output projection with MXFP4 activations")
    args = parser.parse_args(argv)
    block = random_block(args.hidden, args.intermediate, args.experts, args.top_k, four_bit_activations=args.four_bit_activations)
    x = torch.randn(args.tokens, args.hidden, device="cuda", dtype=torch.bfloat16)
    o = torch.randn_like(x)
    block(x, o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = block(x, o)
    graph.replay()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(args.steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    us = start.elapsed_time(end) / args.steps * 1e3
    print("%d tokens, %d experts, top %d, H = %d, I = %d: %.1f us a step, %.0f tokens/s, largest output %.3f" % (
        args.tokens, args.experts, args.top_k, args.hidden, args.intermediate, us, args.tokens / us * 1e6, float(y.abs().max())))
    return us


if __name__ == "__main__":
    main()

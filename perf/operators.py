"""Operators on microscaled 4-bit floating point weights whose speed counts: quantisation and its read-back, products with
16-bit and with 4-bit activations, and a mixture-of-experts layer's routing and experts.

Format (MXFP4 of the OCP microscaling specification): blocks of 32 values along a row share a power-of-two scale; an element is
a sign, two exponent bits and one fraction bit (0, 0.5, 1, 1.5, 2, 3, 4, 6).  codes: uint8 [rows, K/2], the even k in the low
nibble; scales: uint8 [rows, K/32], the exponent plus 127, 255 for a block that is not a number.

Operators:
  roundtrip  a matrix is quantised and read back in its own type
  gemm       Y = X W^T with 16-bit X [M, K] and MXFP4 W [N, K]
  gemm_mx    the same with X in MXFP4
  route      logits [T, E] -> the top_k experts of every token and their weights
  experts    y_t = sum_j weight_tj W2_e (silu(W1_e x_t) * (W3_e x_t)), e = id_tj, with MXFP4 weights

Activations are normal with one channel in a hundred 20 times larger (the outliers LLM layers show); weights are normal, scaled
by 1 / sqrt(K).
"""
import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
ELEMENTS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
MOST_WEIGHTS = 28672 * 8192           # of one product
MOST_PRODUCTS = 2048 * 8192 * 8192
MOST_EXPERT_WEIGHTS = 128 * 3 * 4096 * 2048


def _named(name, case):
    return dict(case, name=name) if name else case


def _roundtrip(name, rows, K, dtype):
    return _named(name, {"op": "roundtrip", "rows": rows, "K": K, "dtype": dtype})


def _gemm(name, M, K, N, dtype):
    return _named(name, {"op": "gemm", "M": M, "K": K, "N": N, "dtype": dtype})


def _gemm_mx(name, M, K, N, dtype):
    return _named(name, {"op": "gemm_mx", "M": M, "K": K, "N": N, "dtype": dtype})


def _route(name, T, E, top_k, dtype, scoring="softmax", renormalize=True):
    return _named(name, {"op": "route", "T": T, "E": E, "top_k": top_k, "dtype": dtype, "scoring": scoring,
                         "renormalize": renormalize})


def _experts(name, T, E, top_k, H, I, dtype):
    return _named(name, {"op": "experts", "T": T, "E": E, "top_k": top_k, "H": H, "I": I, "dtype": dtype})


def listed():
    return [
        # one token's activations on their way into a 4-bit product: latency is all
        _roundtrip("roundtrip_token", 1, 8192, "bf16"),
        # a large layer's weights prepared offline, and read back to look at the error
        _roundtrip("roundtrip_weights", 8192, 28672, "fp16"),
        # one token through one small projection: latency
        _gemm("gemm_1_small", 1, 4096, 1024, "bf16"),
        # one sequence, the largest down-projection: weights streamed once
        _gemm("gemm_1_large", 1, 28672, 8192, "fp16"),
        # a batch size nobody rounded, ragged in every dimension
        _gemm("gemm_37_ragged", 37, 10272, 4601, "bf16"),
        # a chunk of a prompt
        _gemm("gemm_2048", 2048, 8192, 8192, "bf16"),
        # a small server batch, activations in four bits as well
        _gemm_mx("gemm_mx_16", 16, 14336, 4096, "bf16"),
        # a chunk of a prompt in four bits throughout
        _gemm_mx("gemm_mx_2048", 2048, 8192, 8192, "bf16"),
        # one token's routing: latency
        _route("route_1", 1, 64, 6, "fp32"),
        # a chunk of a prompt through a router with many experts
        _route("route_4096", 4096, 256, 8, "bf16"),
        # one token through its experts: the weights of eight of 64 experts
        _experts("experts_1", 1, 64, 8, 4096, 2048, "bf16"),
        # a server batch that touches nearly all experts, a few rows each, unevenly
        _experts("experts_48", 48, 128, 8, 4096, 2048, "fp16"),
    ]


def _log_int(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n if n != 3072 else n - 1


def _blocks(rng, lo, hi):
    """A length of whole blocks; 1536 and 3072, the one the other's half, are left out."""
    n = 32 * _log_int(rng, lo, hi)
    return n if n not in (1536, 3072) else n - 32


def draw(rng):
    op = rng.choice(["roundtrip", "gemm", "gemm", "gemm_mx", "route", "experts", "experts"])
    if op == "roundtrip":
        K = _blocks(rng, 1, 896)
        return _roundtrip(None, _log_int(rng, 1, min(65536, MOST_WEIGHTS // K)), K, rng.choice(["fp16", "bf16", "fp32"]))
    if op in ("gemm", "gemm_mx"):
        K = _blocks(rng, 16, 896)
        N = _log_int(rng, 64, min(28672, MOST_WEIGHTS // K))
        M = _log_int(rng, 1, max(1, min(2048, MOST_PRODUCTS // (K * N))))
        return (_gemm if op == "gemm" else _gemm_mx)(None, M, K, N, rng.choice(["fp16", "bf16"]))
    if op == "route":
        E = _log_int(rng, 8, 512)
        return _route(None, _log_int(rng, 1, 4096), E, rng.randint(1, min(8, E)), rng.choice(["fp32", "fp16", "bf16"]),
                      rng.choice(["softmax", "softmax", "sigmoid"]), rng.random() < 0.7)
    H = _blocks(rng, 16, 224)
    I = _blocks(rng, 8, 128)
    E = _log_int(rng, 4, max(4, min(128, MOST_EXPERT_WEIGHTS // (3 * H * I))))
    return _experts(None, _log_int(rng, 1, 64), E, rng.randint(1, min(8, E)), H, I, rng.choice(["fp16", "bf16"]))


# ---- inputs ----

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(rows, K, dtype, gen):
    x = torch.randn(rows, K, device="cuda", generator=gen)
    big = torch.rand(K, device="cuda", generator=gen) < 0.01
    return torch.where(big, x * 20.0, x).to(dtype)


def _weights(lead, N, K, gen, powers):
    """MXFP4 weights [*lead, N, K], a slab at a time."""
    count = math.prod(lead)
    codes = torch.empty(count, N, K // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(count, N, K // 32, dtype=torch.uint8, device="cuda")
    for i in range(count):
        codes[i], scales[i] = _pack(*_quantize(torch.randn(N, K, device="cuda", generator=gen) / math.sqrt(K), powers))
    return codes.view(*lead, N, K // 2), scales.view(*lead, N, K // 32)


def prepare(case, seed):
    gen = _generator(seed)
    op = case["op"]
    dtype = DTYPES[case["dtype"]]
    state = {"case": case, "dtype": dtype, "pairs": _pair_table("cuda"), "powers": _power_table("cuda")}
    if op == "roundtrip":
        state["x"] = _activations(case["rows"], case["K"], dtype, gen)
    elif op in ("gemm", "gemm_mx"):
        x = _activations(case["M"], case["K"], dtype, gen)
        state["codes"], state["scales"] = _weights((), case["N"], case["K"], gen, state["powers"])
        if op == "gemm":
            state["x"] = x
        else:
            state["x_codes"], state["x_scales"] = _pack(*_quantize(x.float(), state["powers"]))
    elif op == "route":
        state["logits"] = (1.5 * torch.randn(case["T"], case["E"], device="cuda", generator=gen)).to(dtype)
    else:
        state["x"] = _activations(case["T"], case["H"], dtype, gen)
        state["codes13"], state["scales13"] = _weights((case["E"],), 2 * case["I"], case["H"], gen, state["powers"])
        state["codes2"], state["scales2"] = _weights((case["E"],), case["H"], case["I"], gen, state["powers"])
        logits = 1.5 * torch.randn(case["T"], case["E"], device="cuda", generator=gen)
        top = torch.topk(logits, case["top_k"], dim=1)
        state["ids"] = top.indices.to(torch.int32).contiguous()
        state["weights"] = torch.softmax(top.values, dim=1).contiguous()
    return state


# ---- one pass ----

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    from paper_2601_16536_amd import moe, mx
    case = state["case"]
    op = case["op"]
    if op == "roundtrip":
        codes, scales = mx.quantize(state["x"])
        return mx.dequantize(codes, scales, dtype=state["dtype"])
    if op == "gemm":
        return mx.gemm(state["x"], state["codes"], state["scales"])
    if op == "gemm_mx":
        return mx.gemm_mx(state["x_codes"], state["x_scales"], state["codes"], state["scales"], dtype=state["dtype"])
    if op == "route":
        return moe.route(state["logits"], case["top_k"], scoring=case["scoring"], renormalize=case["renormalize"])
    return moe.experts(state["x"], state["ids"], state["weights"], state["codes13"], state["scales13"], state["codes2"],
                       state["scales2"], activation="silu")


def _pair_table(device):
    signed = ELEMENTS + [-v for v in ELEMENTS]
    return torch.tensor([[signed[c & 15], signed[c >> 4]] for c in range(256)], dtype=torch.float32, device=device)


def _power_table(device):
    return torch.tensor([math.ldexp(1.0, s - 127) for s in range(255)] + [math.nan], dtype=torch.float32, device=device)


def _quantize(x, powers):
    """FP32 [rows, K] -> signed magnitudes as whole element values [rows, K/32, 32] and exponents [rows, K/32]
    (128 where the block is not a number)."""
    blocks = x.reshape(x.shape[0], -1, 32)
    most = blocks.abs().amax(dim=2)  # (a NaN is the largest)
    finite = torch.isfinite(most)
    exponent = (torch.frexp(torch.where(finite, most, 1.0)).exponent - 3).clamp(-127, 127)
    exponent = torch.where(most == 0, -127, exponent)
    y = torch.where(finite.unsqueeze(2), blocks, 0.0) * powers[127 - exponent].unsqueeze(2)
    a = y.abs()
    q = torch.where(a < 2, torch.round(a * 2) / 2, torch.where(a < 4, torch.round(a), torch.round(a / 2) * 2)).clamp(max=6.0)
    return torch.copysign(q, y), torch.where(finite, exponent, 128)


def _pack(q, exponent):
    a = q.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) + 8 * torch.signbit(q).to(torch.uint8)
    code = code.reshape(code.shape[0], -1)
    return code[:, 0::2] | (code[:, 1::2] << 4), (exponent + 127).to(torch.uint8)


def _values(state, codes, scales):
    """The FP32 values that codes [..., K/2] and scales [..., K/32] stand for."""
    v = state["pairs"][codes.int()].reshape(*scales.shape, 32)
    return (v * state["powers"][scales.int()].unsqueeze(-1)).flatten(-2)


def _run_plain(state):
    case, dtype = state["case"], state["dtype"]
    op = case["op"]
    if op == "roundtrip":
        q, exponent = _quantize(state["x"].float(), state["powers"])
        power = state["powers"][(exponent + 127)]
        return (q * power.unsqueeze(2)).reshape(state["x"].shape).to(dtype)
    if op == "gemm":
        return (state["x"].float() @ _values(state, state["codes"], state["scales"]).t()).to(dtype)
    if op == "gemm_mx":
        x = _values(state, state["x_codes"], state["x_scales"])
        return (x @ _values(state, state["codes"], state["scales"]).t()).to(dtype)
    if op == "route":
        return _plain_route(state["logits"].float(), case["top_k"], case["scoring"], case["renormalize"])
    return _plain_experts(state).to(dtype)


def _plain_route(logits, top_k, scoring, renormalize):
    ids = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :top_k]  # stable: ties to the lowest index
    if scoring == "softmax":
        score = torch.exp(logits - logits.amax(dim=1, keepdim=True))
        score = score / score.sum(dim=1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-logits))
    weights = torch.gather(score, 1, ids)
    if renormalize:
        weights = weights / weights.sum(dim=1, keepdim=True)
    return ids.to(torch.int32), weights


def _ffn(x, w13, w2):
    gate, up = (x @ w13.t()).chunk(2, dim=1)
    return (gate / (1.0 + torch.exp(-gate)) * up) @ w2.t()


def _plain_experts(state):
    x, ids, weights = state["x"].float(), state["ids"], state["weights"]
    T, top_k = ids.shape
    E = state["codes13"].shape[0]
    y = torch.zeros_like(x)
    if T * top_k <= E:  # each token's own experts
        for t in range(T):
            w13 = _values(state, state["codes13"][ids[t]], state["scales13"][ids[t]])
            w2 = _values(state, state["codes2"][ids[t]], state["scales2"][ids[t]])
            for j in range(top_k):
                y[t] += weights[t, j] * _ffn(x[t:t + 1], w13[j], w2[j])[0]
        return y
    share = torch.zeros(T, E, device=x.device).scatter_add_(1, ids.long(), weights)
    for e in range(E):  # every expert for all tokens
        w13 = _values(state, state["codes13"][e], state["scales13"][e])
        w2 = _values(state, state["codes2"][e], state["scales2"][e])
        y += share[:, e:e + 1] * _ffn(x, w13, w2)
    return y


# ---- the definition in 64 bits ----

def _exact_matrix(codes, scales):
    """float64 [..., K] from the bits: sign, two exponent bits, one fraction bit."""
    nibbles = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).to(torch.int16)
    power, fraction = (nibbles >> 1) & 3, (nibbles & 1).double()
    v = torch.where(power == 0, 0.5 * fraction, (1.0 + 0.5 * fraction) * (1 << (power - 1).clamp(min=0)).double())
    v = torch.where(nibbles >= 8, -v, v)
    return v * torch.exp2(scales.double() - 127.0).repeat_interleave(32, dim=-1)


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "roundtrip":
        parts = [_exact_roundtrip(part) for part in state["x"].split(1024)]
        return torch.cat(parts)
    if op == "gemm":
        x = state["x"].double()
    if op == "gemm_mx":
        x = _exact_matrix(state["x_codes"], state["x_scales"])
    if op in ("gemm", "gemm_mx"):
        parts = zip(state["codes"].split(1024), state["scales"].split(1024))
        return torch.cat([x @ _exact_matrix(c, s).t() for c, s in parts], dim=1)
    if op == "route":
        return _exact_route(state["logits"].double(), case)
    return _exact_experts(state)


def _exact_roundtrip(x):
    """The nearest element of each block's grid; of two as near the one with the even code."""
    b = x.double().reshape(x.shape[0], -1, 32)
    e = torch.floor(torch.log2(b.abs().amax(dim=2, keepdim=True).clamp(min=2.0 ** -125))) - 2
    power = torch.exp2(e)
    a = b.abs() / power
    q = torch.zeros_like(a)
    for code in range(1, 8):
        middle = (ELEMENTS[code - 1] + ELEMENTS[code]) / 2
        q[(a >= middle) if code % 2 == 0 else (a > middle)] = ELEMENTS[code]
    return (torch.where(b < 0, -q, q) * power).reshape(x.shape)


def _exact_route(logits, case):
    ids = torch.argsort(-logits, dim=1, stable=True)[:, :case["top_k"]]
    score = torch.softmax(logits, dim=1) if case["scoring"] == "softmax" else torch.sigmoid(logits)
    weights = score.gather(1, ids)
    if case["renormalize"]:
        weights = weights / weights.sum(dim=1, keepdim=True)
    return ids.to(torch.int32), weights


def _exact_experts(state):
    x, ids, weights = state["x"].double(), state["ids"].long().cpu(), state["weights"].double()
    y = torch.zeros_like(x)
    for e in sorted(set(ids.flatten().tolist())):
        t, j = (i.to(x.device) for i in torch.nonzero(ids == e, as_tuple=True))
        both = x[t] @ _exact_matrix(state["codes13"][e], state["scales13"][e]).t()
        half = both.shape[1] // 2
        h = both[:, :half] * torch.sigmoid(both[:, :half]) * both[:, half:]
        out = h @ _exact_matrix(state["codes2"][e], state["scales2"][e]).t()
        y.index_add_(0, t, weights[t, j].unsqueeze(1) * out)
    return y


# ---- what a pass cannot do without ----

def work(case):
    op = case["op"]
    size = torch.empty(0, dtype=DTYPES[case["dtype"]]).element_size()
    packed = lambda n: n * 17 // 32  # half a byte and a 32nd
    if op == "roundtrip":
        n = case["rows"] * case["K"]
        return {"bytes": 2 * size * n + 2 * packed(n), "flops": 4 * n}
    if op in ("gemm", "gemm_mx"):
        M, K, N = case["M"], case["K"], case["N"]
        x = size * M * K if op == "gemm" else packed(M * K)
        return {"bytes": x + packed(N * K) + size * M * N, "flops": 2 * M * N * K}
    if op == "route":
        T, E = case["T"], case["E"]
        return {"bytes": size * T * E + 8 * T * case["top_k"], "flops": 4 * T * E}
    T, E, top_k, H, I = (case[k] for k in ("T", "E", "top_k", "H", "I"))
    touched = E * (1.0 - (1.0 - top_k / E) ** T)  # experts that some token is expected to have chosen
    return {"bytes": int(touched * packed(3 * H * I)) + 2 * size * T * H + 8 * T * top_k, "flops": 6 * T * top_k * H * I}

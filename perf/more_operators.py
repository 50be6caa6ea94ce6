"""Products of rows in groups whose speed counts: experts on 16-bit weights with their gradients, and low-rank adapters of many
requests beside a shared projection with theirs.

Rows belong to groups (a token's experts, a request's adapter).  Operators:
  sort       ids [T, top_k] -> offsets [E + 1], order and place [T top_k]: the pairs by group, in their order inside one, those without
             a group (id -1) last; place is order's inverse
  gemm       y_i = W_e x_i for the rows offsets[e] <= i < offsets[e+1], W [E, N, K]; with `gather` x_i is row order[i] / top_k of X.
             `transposed`: W [E, K, N], y_i = x_i W_e, which is also the gradient of the first form's rows.  Rows without a group: 0
  gemm_grad  dW_e = sum over a group's rows of dy_i^T x_i
  lora       y_i + s_a B_a (A_a x_i), a the adapter of row i; rows without one as they are
  lora_grad  its gradients for rows (added to what the shared projection passed back), A and B

Activations are normal with one channel in a hundred 20 times larger (the outliers LLM layers show); weights are normal, scaled by
1 / sqrt(K); some experts are chosen far more often than others; gradients of outputs are normal, times 0.01.
"""
import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
MOST_WEIGHTS = 64 * 4096 * 4096            # of all experts of one layer
MOST_PRODUCTS = 4096 * 8 * 4096 * 4096     # of one pass
MOST_ADAPTERS = 16 * 64 * (8192 + 8192)    # values of all adapters of one layer
MOST_ROWS = 2048 * (8192 + 8192)           # values of the rows beside adapters
MOST_GRAD_ROWS = 4096 * (8192 + 8192)


def _named(name, case):
    return dict(case, name=name) if name else case


def _sort(name, T, E, top_k, drop=0.0):
    return _named(name, {"op": "sort", "T": T, "E": E, "top_k": top_k, "drop": drop})


def _gemm(name, T, E, top_k, K, N, dtype, gather=False, transposed=False, drop=0.0):
    return _named(name, {"op": "gemm", "T": T, "E": E, "top_k": top_k, "K": K, "N": N, "dtype": dtype, "gather": gather,
                         "transposed": transposed, "drop": drop})


def _gemm_grad(name, T, E, top_k, K, N, dtype, grads, gather=False, drop=0.0):
    return _named(name, {"op": "gemm_grad", "T": T, "E": E, "top_k": top_k, "K": K, "N": N, "dtype": dtype, "grads": grads,
                         "gather": gather, "drop": drop})


def _lora(name, M, requests, L, R, K, N, dtype):
    return _named(name, {"op": "lora", "M": M, "requests": requests, "L": L, "R": R, "K": K, "N": N, "dtype": dtype})


def _lora_grad(name, M, requests, L, R, K, N, dtype, grads):
    return _named(name, {"op": "lora_grad", "M": M, "requests": requests, "L": L, "R": R, "K": K, "N": N, "dtype": dtype,
                         "grads": grads})


def listed():
    return [
        # one token's experts: latency is all
        _sort("sort_1", 1, 64, 8),
        # a chunk of a prompt, many experts, some tokens padding
        _sort("sort_4096", 4096, 256, 8, drop=0.05),
        # one token through the gate and up projections of its eight experts
        _gemm("gemm_1", 1, 64, 8, 4096, 4096, "bf16", gather=True),
        # a server batch through the down projections of nearly all experts, a few rows each, unevenly
        _gemm("gemm_48", 48, 128, 8, 2048, 4096, "fp16"),
        # a training micro-batch, or a chunk of a prompt, through gate and up
        _gemm("gemm_4096", 4096, 64, 8, 4096, 4096, "bf16", gather=True),
        # the gradient of a ragged batch's rows
        _gemm("gemm_777_back", 777, 64, 6, 4096, 2048, "bf16", transposed=True, drop=0.05),
        # gradients of a small layer's weights, kept in 32 bits to be added up
        _gemm_grad("gemm_grad_300", 300, 8, 2, 2056, 1000, "fp16", "fp32"),
        # gradients of the micro-batch's gate and up weights
        _gemm_grad("gemm_grad_4096", 4096, 64, 8, 4096, 4096, "bf16", "bf16", gather=True),
        # a server batch: 32 requests with adapters of their own beside one projection
        _lora("lora_32", 32, 32, 64, 16, 8192, 8192, "bf16"),
        # prompts of a few requests, larger adapters
        _lora("lora_2048", 2048, 5, 16, 64, 8192, 8192, "bf16"),
        # a small adapter trained on a few short texts, beside the largest projections of the small layer
        _lora_grad("lora_grad_250", 250, 3, 3, 8, 4096, 11008, "fp16", "fp32"),
        # four adapters trained at once
        _lora_grad("lora_grad_4096", 4096, 4, 4, 32, 8192, 8192, "bf16", "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sort", "gemm", "gemm", "gemm", "gemm_grad", "gemm_grad", "lora", "lora", "lora_grad"])
    drop = rng.choice([0.0, 0.0, 0.1])
    dtype = rng.choice(["fp16", "bf16"])
    if op == "sort":
        E = _log_int(rng, 2, 512)
        return _sort(None, _log_int(rng, 1, 4096), E, rng.randint(1, min(8, E)), drop)
    if op in ("gemm", "gemm_grad"):
        E = _log_int(rng, 1, 256)
        K = 8 * _log_int(rng, 8, 1024)
        N = 8 * _log_int(rng, 8, max(8, min(1024, MOST_WEIGHTS // (8 * E * K))))
        top_k = rng.randint(1, min(8, E))
        T = _log_int(rng, 1, max(1, min(4096, MOST_PRODUCTS // (top_k * K * N))))
        if op == "gemm":
            return _gemm(None, T, E, top_k, K, N, dtype, rng.random() < 0.5, rng.random() < 0.4, drop)
        return _gemm_grad(None, T, E, top_k, K, N, dtype, rng.choice([dtype, "fp32"]), rng.random() < 0.5, drop)
    R = 8 * _log_int(rng, 1, 16)
    K, N = 8 * _log_int(rng, 64, 1792), 8 * _log_int(rng, 64, 1792)
    L = _log_int(rng, 1, max(1, min(128, MOST_ADAPTERS // (R * (K + N)))))
    M = _log_int(rng, 1, min(4096, (MOST_ROWS if op == "lora" else MOST_GRAD_ROWS) // (K + N)))
    requests = _log_int(rng, 1, M) if M <= 64 else _log_int(rng, 1, 64)
    if op == "lora":
        return _lora(None, M, requests, L, R, K, N, dtype)
    return _lora_grad(None, M, requests, L, R, K, N, dtype, rng.choice([dtype, "fp32"]))


# ---- inputs ----

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(rows, K, dtype, gen):
    x = torch.randn(rows, K, device="cuda", generator=gen)
    big = torch.rand(K, device="cuda", generator=gen) < 0.01
    return torch.where(big, x * 20.0, x).to(dtype)


def _weights(lead, rows, K, fan_in, dtype, gen):
    """Normal weights [lead, rows, K], a slab at a time."""
    w = torch.empty(lead, rows, K, dtype=dtype, device="cuda")
    for i in range(lead):
        w[i] = torch.randn(rows, K, device="cuda", generator=gen) / math.sqrt(fan_in)
    return w


def _choice(T, E, top_k, drop, gen):
    """ids int32 [T, top_k]: experts of uneven popularity; -1 for the tokens that are padding."""
    logits = 1.5 * torch.randn(T, E, device="cuda", generator=gen) + 0.7 * torch.randn(E, device="cuda", generator=gen)
    ids = torch.topk(logits, top_k, dim=1).indices.to(torch.int32)
    gone = torch.rand(T, 1, device="cuda", generator=gen) < drop
    return torch.where(gone, -1, ids).contiguous()


def prepare(case, seed):
    gen = _generator(seed)
    op = case["op"]
    state = {"case": case}
    if op in ("sort", "gemm", "gemm_grad"):
        T, E, top_k = case["T"], case["E"], case["top_k"]
        state["ids"] = _choice(T, E, top_k, case["drop"], gen)
        if op == "sort":
            return state
        state["offsets"], state["order"], _ = _plain_sort(state["ids"], E)
        state["bounds"] = state["offsets"].tolist()
        dtype, K, N = DTYPES[case["dtype"]], case["K"], case["N"]
        state["x"] = _activations(T if case["gather"] else T * top_k, K, dtype, gen)
        if op == "gemm":
            state["w"] = _weights(E, K, N, K, dtype, gen) if case["transposed"] else _weights(E, N, K, K, dtype, gen)
        else:
            state["dy"] = (0.01 * torch.randn(T * top_k, N, device="cuda", generator=gen)).to(dtype)
        return state
    M, L, R, K, N = (case[k] for k in ("M", "L", "R", "K", "N"))
    dtype = DTYPES[case["dtype"]]
    adapter = torch.randint(0, L, (case["requests"],), device="cuda", generator=gen)
    adapter = torch.where(torch.rand(case["requests"], device="cuda", generator=gen) < 0.1, -1, adapter)
    ends = torch.sort(torch.randperm(M - 1, device="cuda", generator=gen)[:case["requests"] - 1] + 1).values if M > 1 else None
    request = torch.bucketize(torch.arange(M, device="cuda"), ends, right=True) if M > 1 else torch.zeros(1, dtype=torch.long, device="cuda")
    state["ids"] = adapter[request].to(torch.int32)
    state["rows"] = [(a, torch.nonzero(state["ids"] == a).flatten()) for a in sorted(set(state["ids"].tolist()) - {-1})]
    state["x"] = _activations(M, K, dtype, gen)
    state["a"] = _weights(L, R, K, K, dtype, gen)
    state["b"] = _weights(L, N, R, 4 * R, dtype, gen)
    state["scaling"] = 2.0 ** torch.randint(-1, 2, (L,), device="cuda", generator=gen).float()
    if op == "lora":
        state["y"] = torch.randn(M, N, device="cuda", generator=gen).to(dtype)
    else:
        state["dy"] = (0.01 * torch.randn(M, N, device="cuda", generator=gen)).to(dtype)
        state["dx"] = (0.01 * torch.randn(M, K, device="cuda", generator=gen)).to(dtype)
    return state


# ---- one pass ----

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    from paper_2601_16536_amd import grouped, lora
    case = state["case"]
    op = case["op"]
    if op == "sort":
        return grouped.sort(state["ids"], case["E"])
    if op in ("gemm", "gemm_grad"):
        rows = {"rows": state["order"], "top_k": case["top_k"]} if case["gather"] else {}
        if op == "gemm":
            return grouped.gemm(state["x"], state["w"], state["offsets"], transposed=case["transposed"], **rows)
        return grouped.gemm_grad(state["dy"], state["x"], state["offsets"], dtype=DTYPES[case["grads"]], **rows)
    if op == "lora":
        return lora.add(state["y"], state["x"], state["a"], state["b"], state["ids"], state["scaling"])
    return lora.grad(state["dy"], state["x"], state["a"], state["b"], state["ids"], state["scaling"], dX=state["dx"],
                     dtype=DTYPES[case["grads"]])


def _plain_sort(ids, E):
    flat = ids.flatten().long()
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    order = torch.sort(key, stable=True).indices
    offsets = torch.searchsorted(key[order], torch.arange(E + 1, device=ids.device))
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=ids.device)
    return offsets.to(torch.int32), order.to(torch.int32), place.to(torch.int32)


def _run_plain(state):
    case, op = state["case"], state["case"]["op"]
    if op == "sort":
        return _plain_sort(state["ids"], case["E"])
    if op in ("gemm", "gemm_grad"):
        x, bounds = state["x"], state["bounds"]
        if case["gather"]:
            x = x[state["order"].long() // case["top_k"]]
        return _plain_gemm(state, x, bounds) if op == "gemm" else _plain_gemm_grad(state, x, bounds)
    return _plain_lora(state) if op == "lora" else _plain_lora_grad(state)


def _plain_gemm(state, x, bounds):
    w = state["w"]
    y = torch.zeros(x.shape[0], state["case"]["N"], dtype=x.dtype, device=x.device)
    for e in range(w.shape[0]):
        lo, hi = bounds[e], bounds[e + 1]
        if hi > lo:
            y[lo:hi] = x[lo:hi].float() @ (w[e].float() if state["case"]["transposed"] else w[e].float().t())
    return y


def _plain_gemm_grad(state, x, bounds):
    case, dy = state["case"], state["dy"]
    dw = torch.zeros(case["E"], case["N"], case["K"], dtype=DTYPES[case["grads"]], device=x.device)
    for e in range(case["E"]):
        lo, hi = bounds[e], bounds[e + 1]
        if hi > lo:
            dw[e] = dy[lo:hi].float().t() @ x[lo:hi].float()
    return dw


def _plain_lora(state):
    y = state["y"].float()
    for a, rows in state["rows"]:
        h = state["x"][rows].float() @ state["a"][a].float().t()
        y[rows] += state["scaling"][a] * (h @ state["b"][a].float().t())
    return y.to(state["y"].dtype)


def _plain_lora_grad(state):
    dx = state["dx"].float()
    grads = DTYPES[state["case"]["grads"]]
    da, db = torch.zeros_like(state["a"], dtype=grads), torch.zeros_like(state["b"], dtype=grads)
    for i, rows in state["rows"]:
        x, dy, s = state["x"][rows].float(), state["dy"][rows].float(), state["scaling"][i]
        a, b = state["a"][i].float(), state["b"][i].float()
        h, g = s * (x @ a.t()), s * (dy @ b)
        dx[rows] += g @ a
        da[i], db[i] = g.t() @ x, dy.t() @ h
    return dx.to(state["dx"].dtype), da, db


# ---- the definition in 64 bits ----

def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "sort":
        return _exact_sort(state["ids"], case["E"])
    if op in ("gemm", "gemm_grad"):
        return _exact_groups(state)
    x, ids, scaling = state["x"].double(), state["ids"], state["scaling"].double()
    touched = [a for a in range(case["L"]) if bool((ids == a).any())]
    mine = {a: (ids == a).double().unsqueeze(1) * scaling[a] for a in touched}
    if op == "lora":
        y = state["y"].double()
        for a in touched:  # all rows through every adapter, those of others times 0
            y += (mine[a] * x) @ state["a"][a].double().t() @ state["b"][a].double().t()
        return y
    dx, dy = state["dx"].double(), state["dy"].double()
    da, db = torch.zeros_like(state["a"], dtype=torch.float64), torch.zeros_like(state["b"], dtype=torch.float64)
    for i in touched:
        a, b = state["a"][i].double(), state["b"][i].double()
        dx += (mine[i] * dy) @ b @ a
        da[i] = b.t() @ (dy.t() @ (mine[i] * x))
        db[i] = (dy.t() @ (mine[i] * x)) @ a.t()
    return dx, da, db


def _exact_sort(ids, E):
    groups = [[] for _ in range(E + 1)]
    for pair, e in enumerate(ids.flatten().tolist()):
        groups[e if 0 <= e < E else E].append(pair)
    offsets, order = [0], []
    for e in range(E):
        order += groups[e]
        offsets.append(len(order))
    order += groups[E]
    place = [0] * len(order)
    for at, pair in enumerate(order):
        place[pair] = at
    return tuple(torch.tensor(v, dtype=torch.int32) for v in (offsets, order, place))


def _exact_groups(state):
    case = state["case"]
    E, top_k = case["E"], case["top_k"]
    offsets, order, _ = _exact_sort(state["ids"], E)
    K, N = case["K"], case["N"]
    if case["op"] == "gemm":
        y = torch.zeros(case["T"] * top_k, N, dtype=torch.float64, device="cuda")
    else:
        dw = torch.zeros(E, N, K, dtype=torch.float64, device="cuda")
    for e in range(E):
        at = torch.arange(int(offsets[e]), int(offsets[e + 1]))
        if at.numel() == 0:
            continue
        source = (torch.div(order[at], top_k, rounding_mode="floor") if case["gather"] else at).long().cuda()
        x, at = state["x"][source].double(), at.cuda()
        if case["op"] == "gemm":
            w = state["w"][e].double()
            y[at] = x @ w if case["transposed"] else (w @ x.t()).t()
        else:
            dw[e] = (x.t() @ state["dy"][at].double()).t()
    return y if case["op"] == "gemm" else dw


# ---- what a pass cannot do without ----

def work(case):
    op = case["op"]
    size = lambda name: torch.empty(0, dtype=DTYPES[name]).element_size()
    if op == "sort":
        P = case["T"] * case["top_k"]
        return {"bytes": 12 * P + 4 * (case["E"] + 1), "flops": 0}
    if op in ("gemm", "gemm_grad"):
        T, E, top_k, K, N = (case[k] for k in ("T", "E", "top_k", "K", "N"))
        kept = 1.0 - case["drop"]
        P = T * top_k
        x = (T if case["gather"] else P) * K
        touched = E * (1.0 - (1.0 - top_k / E) ** (T * kept))  # experts that some token is expected to have chosen
        flops = int(2 * kept * P * N * K)
        if op == "gemm":
            return {"bytes": int(size(case["dtype"]) * (kept * x + touched * N * K + P * N)), "flops": flops}
        return {"bytes": int(size(case["dtype"]) * kept * (x + P * N) + size(case["grads"]) * E * N * K), "flops": flops}
    M, requests, L, R, K, N = (case[k] for k in ("M", "requests", "L", "R", "K", "N"))
    touched = L * (1.0 - (1.0 - 0.9 / L) ** requests)
    adapters = touched * R * (K + N)
    if op == "lora":
        return {"bytes": int(size(case["dtype"]) * (0.9 * M * K + 2 * M * N + adapters)), "flops": int(0.9 * 2 * M * R * (K + N))}
    return {"bytes": int(size(case["dtype"]) * (M * (3 * K + N) + adapters) + size(case["grads"]) * L * R * (K + N)),
            "flops": int(0.9 * M * R * (6 * K + 4 * N))}

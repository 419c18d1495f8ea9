"""MXFP4 linear layers, dense and by expert, as a list of cases with their inputs, one pass of each through the public entry
points, a plain form in elementary torch operations, and the definition in 64 bits.

MXFP4: E2M1 elements (0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives), one power of two as the scale of 32 channels,
2^(floor(log2 of the largest magnitude) - 2).  A case is a dict of plain values.  `kind` says which operator it takes:

  quantize  rows of activations are quantized and the stored values read back as bf16;
  linear    rows of activations are quantized and multiplied with quantized weights, with a bias or without;
  experts   tokens are quantized, and the rows that each expert gets are multiplied with its weights: rows of one token go to
            `k` experts (`gather`), or every row is there already in the experts' order;
  route     every token's `k` largest of the router's logits: experts, weights, and the order of the rows by expert;
  combine   the weighted sum of the rows that a token's experts made of it, on top of an addend or not.
"""
import math

import torch

DEV = "cuda"
BLOCK = 32

own = False


def listed():
    return [
        # ---- quantize
        # the tokens of one decode step: latency counts
        dict(name="quantize_tokens", kind="quantize", M=3, K=2560, pad=0),
        # a batch of prompts, a slice of wider rows
        dict(name="quantize_prompts", kind="quantize", M=8211, K=5120, pad=64),
        # ---- linear
        # one new token: the weights are all there is to read
        dict(name="linear_token", kind="linear", M=1, N=6144, K=4096, bias=False),
        # a decode step of a batch of conversations
        dict(name="linear_batch", kind="linear", M=56, N=12288, K=4096, bias=True),
        # one prompt of odd length, sizes that are no multiples of a tile
        dict(name="linear_ragged", kind="linear", M=1777, N=4008, K=2016, bias=True),
        # the largest: prompts of a full server's batch
        dict(name="linear_prompts", kind="linear", M=8192, N=12288, K=8192, bias=False),
        # ---- experts
        # a decode step of a batch, some twelve rows an expert, in the experts' order already (the second product of a layer)
        dict(name="experts_batch", kind="experts", T=192, k=8, E=128, N=1536, K=2560, gather=False, bias=True),
        # prompts: long groups of uneven lengths, rows gathered from their tokens (the first product of a layer)
        dict(name="experts_prompts", kind="experts", T=8191, k=8, E=64, N=2816, K=2048, gather=True, bias=False),
        # ---- route
        # one decode step's tokens: latency counts
        dict(name="route_tokens", kind="route", T=7, E=64, k=6, dtype="float32", renormalize=True, padded=0),
        # prompts, the last rows padding that goes nowhere
        dict(name="route_prompts", kind="route", T=16381, E=256, k=8, dtype="bfloat16", renormalize=False, padded=200),
        # ---- combine
        # one decode step's tokens
        dict(name="combine_tokens", kind="combine", T=7, k=4, N=2560, addend=False, padded=0),
        # prompts, on top of what all tokens share
        dict(name="combine_prompts", kind="combine", T=8191, k=8, N=5120, addend=True, padded=100),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "linear", "experts", "experts", "route", "combine"])
    while True:
        if kind == "quantize":
            case = dict(kind=kind, M=_log(rng, 1, 20000), K=BLOCK * _log(rng, 8, 400), pad=8 * rng.randrange(0, 9))
            if case["M"] * case["K"] <= 42e6:
                return case
        elif kind == "linear":
            case = dict(kind=kind, M=_log(rng, 1, 12000), N=_log(rng, 200, 16000), K=BLOCK * _log(rng, 8, 400), bias=rng.random() < 0.5)
            if case["M"] * case["N"] * case["K"] <= 8192 * 12288 * 8192:
                return case
        elif kind == "experts":
            E = _log(rng, 2, 256)
            case = dict(kind=kind, T=_log(rng, 1, 10000), k=rng.randrange(1, min(E, 10) + 1), E=E, N=_log(rng, 200, 6000),
                        K=BLOCK * _log(rng, 8, 160), gather=rng.random() < 0.5, bias=rng.random() < 0.5)
            if E * case["N"] * case["K"] <= 510e6 and case["T"] * case["k"] * max(case["N"], case["K"]) * case["K"] <= 400e9:
                return case
        elif kind == "route":
            E = _log(rng, 4, 512)
            case = dict(kind=kind, T=_log(rng, 1, 30000), E=E, k=rng.randrange(1, min(E, 12) + 1), dtype=rng.choice(["float32", "bfloat16"]),
                        renormalize=rng.random() < 0.5, padded=0)
            case["padded"] = rng.randrange(0, case["T"] // 8 + 1)
            if case["T"] * E <= 4.3e6:
                return case
        else:
            case = dict(kind=kind, T=_log(rng, 1, 20000), k=rng.randrange(1, 11), N=8 * _log(rng, 32, 900), addend=rng.random() < 0.5, padded=0)
            case["padded"] = rng.randrange(0, case["T"] // 8 + 1)
            if case["T"] * case["k"] * case["N"] <= 336e6:
                return case


# ------------------------------------------------------------------------ inputs

def _rng(seed, salt):
    return torch.Generator(device=DEV).manual_seed(seed * 16 + salt)


def _randn(rows, width, g, scale):
    """bf16 [rows, width] of normal values times scale[width], made in pieces."""
    out = torch.empty(rows, width, dtype=torch.bfloat16, device=DEV)
    step = max(1, (1 << 27) // width)
    for r0 in range(0, rows, step):
        out[r0:r0 + step] = torch.randn(min(step, rows - r0), width, generator=g, device=DEV) * scale
    return out


def _activations(rows, K, pad, seed):
    """Rows of a layer's input: channels of uneven sizes, a few far larger; a slice of wider rows where pad > 0."""
    g = _rng(seed, 1)
    s = torch.exp(0.5 * torch.randn(K + pad, generator=g, device=DEV))
    s[torch.randint(0, K, (max(1, K // 128),), generator=g, device=DEV)] *= 20.0
    return _randn(rows, K + pad, g, s)[:, :K]


def _weights(rows, K, seed):
    g = _rng(seed, 2)
    return _randn(rows, K, g, 0.02 * torch.exp(0.3 * torch.randn(K, generator=g, device=DEV)))


def _bias(rows, N, seed):
    return (0.5 * torch.randn(rows, N, generator=_rng(seed, 3), device=DEV)).to(torch.bfloat16)


def _assignment(case, seed):
    """(token of each row in the experts' order, rows of each expert): every token goes to k of E experts, some of them
    asked for more often than others, as a router's are."""
    g = _rng(seed, 4)
    T, E, k = case["T"], case["E"], case["k"]
    popular = torch.randn(E, generator=g, device=DEV)
    ids = (torch.randn(T, E, generator=g, device=DEV) + 0.7 * popular).topk(k, dim=1).indices.reshape(-1)
    order = torch.argsort(ids, stable=True)
    return (order // k).to(torch.int32), torch.bincount(ids, minlength=E)


def _logits(case, seed):
    g = _rng(seed, 5)
    x = 1.5 * torch.randn(case["T"], case["E"], generator=g, device=DEV) + 0.5 * torch.randn(case["E"], generator=g, device=DEV)
    x = x.to(getattr(torch, case["dtype"]))
    if case["padded"]:
        x[case["T"] - case["padded"]:] = -math.inf
    return x


def _made(case, seed):
    """(rows that the experts made, place of each token's rows among them, their weights, addend)."""
    g = _rng(seed, 6)
    T, k, N = case["T"], case["k"], case["N"]
    y = _randn(T * k, N, g, torch.ones(N, device=DEV))
    positions = torch.randperm(T * k, generator=g, device=DEV).to(torch.int32).reshape(T, k)
    weights = torch.softmax(torch.randn(T, k, generator=g, device=DEV), 1)
    if case["padded"]:
        positions[T - case["padded"]:] = -1
        weights[T - case["padded"]:] = 0.0
    return y, positions, weights, _randn(T, N, g, torch.ones(N, device=DEV)) if case["addend"] else None


def _stored(w):
    """Codes [rows, K / 2] and scale bytes [rows, K / 32] of quantized rows, as a checkpoint holds them, made in pieces."""
    rows, K = w.shape
    codes = torch.empty(rows, K // 2, dtype=torch.uint8, device=DEV)
    scales = torch.empty(rows, K // BLOCK, dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 26) // K)
    for r0 in range(0, rows, step):
        q, e = _quantized(w[r0:r0 + step])
        a = q.abs()
        idx = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) + 8 * torch.signbit(q).to(torch.uint8)
        idx = idx.reshape(-1, K)
        codes[r0:r0 + step] = idx[:, 0::2] + 16 * idx[:, 1::2]
        scales[r0:r0 + step] = (e + 127).to(torch.uint8).reshape(-1, K // BLOCK)
    return codes, scales


def prepare(case, seed):
    kind = case["kind"]
    if kind == "quantize":
        x = _activations(case["M"], case["K"], case["pad"], seed)
        state = dict(case=case, x=x)
    elif kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        state = dict(case=case, x=_activations(M, K, 0, seed), bias=_bias(1, N, seed)[0] if case["bias"] else None)
        state["codes"], state["scales"] = _stored(_weights(N, K, seed))
    elif kind == "experts":
        E, N, K = case["E"], case["N"], case["K"]
        tokens, sizes = _assignment(case, seed)
        state = dict(case=case, x=_activations(case["T"] if case["gather"] else tokens.numel(), K, 0, seed),
                     tokens=tokens if case["gather"] else None, sizes=sizes.tolist(),
                     offsets=torch.cat([sizes.new_zeros(1), sizes.cumsum(0)]).to(torch.int32),
                     bias=_bias(E, N, seed) if case["bias"] else None)
        state["codes"], state["scales"] = _stored(_weights(E * N, K, seed))
    elif kind == "route":
        state = dict(case=case, logits=_logits(case, seed))
    else:
        y, positions, weights, addend = _made(case, seed)
        state = dict(case=case, y=y, positions=positions, weights=weights, addend=addend)
    if own:
        _keep(state)
    return state


def _keep(state):
    """What a program that uses the library keeps: weights in the product's layout, buffers of activations, a workspace."""
    from paper_2605_09503_amd import pq
    case = state["case"]
    kind, K = case["kind"], case.get("K")
    state["pq"] = pq
    if kind == "quantize":
        state["codes"], state["scales"] = pq.alloc_quantized(pq.FMT_MXFP4, BLOCK, case["M"], K)
    elif kind == "linear":
        state["w"] = pq.pq_pack_operand(pq.FMT_MXFP4, BLOCK, state.pop("codes"), state.pop("scales"))
    elif kind == "experts":
        state["w"] = pq.pack_experts(state.pop("codes"), state.pop("scales"), case["E"])
    elif kind == "route":
        state["out"] = pq.alloc_route(case["T"], case["E"], case["k"])
        state["workspace"] = pq.pq_moe_route_workspace(case["T"], case["E"], case["k"])
    if kind in ("linear", "experts"):
        rows = state["x"].shape[0]
        state["operand"] = torch.empty(pq.pq_operand_bytes(pq.FMT_MXFP4, BLOCK, rows, K), dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------------------ one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    case, pq = state["case"], state["pq"]
    kind = case["kind"]
    if kind == "quantize":
        pq.pq_quantize_act(pq.FMT_MXFP4, BLOCK, state["x"], None, None, state["codes"], state["scales"])
        return pq.pq_dequantize(pq.FMT_MXFP4, BLOCK, state["codes"], state["scales"])
    if kind == "route":
        r = pq.pq_moe_route(state["logits"], case["k"], case["renormalize"], out=state["out"], workspace=state["workspace"])
        return r.ids, r.weights, r.offsets, r.rows, r.positions
    if kind == "combine":
        return pq.pq_moe_combine(state["y"], state["positions"], state["weights"], addend=state["addend"])
    N, K = case["N"], case["K"]
    a = pq.pq_quantize_act_packed(pq.FMT_MXFP4, BLOCK, state["x"], None, state["operand"])
    M = case["M"] if kind == "linear" else case["T"] * case["k"]
    y = torch.empty(M, (N + 7) // 8 * 8, dtype=torch.bfloat16, device=DEV)[:, :N]
    if kind == "experts":
        pq.pq_qgemm_grouped(pq.FMT_MXFP4, BLOCK, a, state["x"].shape[0], state["w"], state["offsets"], y, N, K, rows=state["tokens"],
                            bias=state["bias"])
    elif case["bias"]:
        pq.pq_qgemm_packed_bias(pq.FMT_MXFP4, BLOCK, a, None, state["w"], None, state["bias"], y, M, N, K)
    else:
        pq.pq_qgemm_packed(pq.FMT_MXFP4, BLOCK, a, None, state["w"], None, y, M, N, K)
    return y


# ---- plain form: elementary torch operations in 32 bits, rounded once at the end

def _quantized(x):
    """(E2M1 values with their signs [rows, blocks, 32], exponents of the scales [rows, blocks, 1]) of bf16 x."""
    x = x.float().unflatten(1, (-1, BLOCK))
    amax = x.abs().amax(2, keepdim=True)
    e = (torch.frexp(amax).exponent - 3).clamp(-127, 127)
    e = torch.where(amax == 0, torch.full_like(e, -127), e)
    v = torch.ldexp(x, -e)
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign(((a / step).round() * step).clamp(max=6.0), v), e


def _values(x):
    q, e = _quantized(x)
    return torch.ldexp(q, e).flatten(1)


def _read(codes, scales):
    """fp32 values of stored codes and scales."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    table = torch.cat([table, -table])
    v = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], 2).reshape(codes.shape[0], -1, BLOCK)
    return torch.ldexp(v, scales.unsqueeze(2).int() - 127).flatten(1)


def _run_plain(state):
    case = state["case"]
    kind = case["kind"]
    if kind == "quantize":
        return _values(state["x"]).to(torch.bfloat16)
    if kind == "linear":
        y = _values(state["x"]) @ _read(state["codes"], state["scales"]).T
        return (y if state["bias"] is None else y + state["bias"].float()).to(torch.bfloat16)
    if kind == "experts":
        x, N = _values(state["x"]), case["N"]
        if state["tokens"] is not None:
            x = x[state["tokens"].long()]
        y = torch.empty(x.shape[0], N, dtype=torch.bfloat16, device=DEV)
        at = 0
        for e, n in enumerate(state["sizes"]):
            if n:
                part = x[at:at + n] @ _read(state["codes"][e * N:(e + 1) * N], state["scales"][e * N:(e + 1) * N]).T
                y[at:at + n] = part if state["bias"] is None else part + state["bias"][e].float()
                at += n
        return y
    if kind == "route":
        return _route_plain(state["logits"].float(), case["k"], case["renormalize"])
    w, pos = state["weights"], state["positions"].long()
    out = state["addend"].float() if case["addend"] else torch.zeros(case["T"], case["N"], device=DEV)
    for j in range(case["k"]):
        out = out + torch.where(pos[:, j:j + 1] >= 0, w[:, j:j + 1] * state["y"][pos[:, j].clamp(min=0)].float(), 0.0)
    return out.to(torch.bfloat16)


def _route_plain(x, k, renormalize):
    """An expert whose logit is -inf is not chosen: -1 stands in its place, with weight 0."""
    T, E = x.shape
    top, ids = torch.sort(x, dim=1, descending=True, stable=True)
    top, ids = top[:, :k], ids[:, :k]
    there = top > -math.inf
    shift = torch.where(there[:, :1], top[:, :1], 0.0)
    p = torch.exp(top - shift)
    total = (p if renormalize else torch.exp(x - shift)).sum(1, keepdim=True)
    weights = torch.where(there, p / total, 0.0)
    flat = torch.where(there, ids, E).reshape(-1)
    order = torch.argsort(flat, stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device=x.device)
    offsets = torch.searchsorted(flat[order], torch.arange(E + 1, device=x.device))
    rows = torch.where(flat[order] < E, order // k, -1)
    return (torch.where(there, ids, -1).to(torch.int32), weights, offsets.to(torch.int32), rows.to(torch.int32),
            torch.where(there, place.reshape(T, k), -1).to(torch.int32))


# ------------------------------------------------------------------------ the definition in 64 bits

def _exact_values(x):
    """fp64 values of quantized bf16 x: the exponent from the bits of the largest magnitude, the element by its place among
    the midpoints of neighbouring E2M1 values (a tie goes to the one with the even code)."""
    bits = (x.contiguous().view(torch.int16).int() & 0x7FFF).unflatten(1, (-1, BLOCK)).amax(2, keepdim=True)
    field = bits >> 7
    e = (torch.where(field > 0, field - 127, -127) - 2).clamp(min=-127)
    scale = torch.ones_like(e, dtype=torch.float64) * torch.pow(torch.tensor(2.0, dtype=torch.float64, device=DEV), e.double())
    v = x.double().unflatten(1, (-1, BLOCK)) / scale
    a, code = v.abs(), torch.zeros_like(v, dtype=torch.int64)
    for i, mid in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (a > mid) if i % 2 == 0 else (a >= mid)
    value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)[code]
    return (torch.copysign(value, v) * scale).flatten(1)


def exact(case, seed):
    kind = case["kind"]
    if kind == "quantize":
        return _exact_values(_activations(case["M"], case["K"], case["pad"], seed))
    if kind == "linear":
        y = _exact_values(_activations(case["M"], case["K"], 0, seed)) @ _exact_values(_weights(case["N"], case["K"], seed)).T
        return y + _bias(1, case["N"], seed).double() if case["bias"] else y
    if kind == "experts":
        N = case["N"]
        tokens, sizes = _assignment(case, seed)
        x = _exact_values(_activations(case["T"] if case["gather"] else tokens.numel(), case["K"], 0, seed))
        w = _weights(case["E"] * N, case["K"], seed)
        bias = _bias(case["E"], N, seed).double() if case["bias"] else None
        y = torch.empty(tokens.numel(), N, dtype=torch.float64, device=DEV)
        at = 0
        for e, n in enumerate(sizes.tolist()):
            rows = x[tokens[at:at + n].long()] if case["gather"] else x[at:at + n]
            y[at:at + n] = rows @ _exact_values(w[e * N:(e + 1) * N]).T
            if bias is not None:
                y[at:at + n] += bias[e]
            at += n
        return y
    if kind == "route":
        return _exact_route(_logits(case, seed).double(), case["k"], case["renormalize"])
    y, positions, weights, addend = _made(case, seed)
    out = addend.double() if addend is not None else torch.zeros(case["T"], case["N"], dtype=torch.float64, device=DEV)
    for j in range(case["k"]):
        there = (positions[:, j] >= 0).nonzero()[:, 0]
        out[there] += weights[there, j, None].double() * y[positions[there, j].long()].double()
    return out


def _exact_route(x, k, renormalize):
    """The largest k one after another; rows placed by counting those of smaller experts and of earlier tokens."""
    T, E = x.shape
    left, ids = x.clone(), torch.full((T, k), -1, dtype=torch.int64, device=DEV)
    column = torch.arange(E, device=DEV)
    for j in range(k):
        best = left.amax(1, keepdim=True)
        first = torch.where(left == best, column, E).amin(1)
        ids[:, j] = torch.where(best[:, 0] > -math.inf, first, -1)
        left[torch.arange(T, device=DEV), first] = -math.inf
    there = ids >= 0
    chosen = torch.where(there, x.gather(1, ids.clamp(min=0)), -math.inf)
    over = chosen if renormalize else x
    weights = torch.where(there, torch.exp(chosen - torch.logsumexp(over, 1, keepdim=True)), 0.0)
    took = torch.zeros(T, E + 1, dtype=torch.int64, device=DEV).scatter_(1, torch.where(there, ids, E), 1)[:, :E]
    counts = took.sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    earlier = took.cumsum(0) - took
    positions = torch.where(there, offsets[:E][ids.clamp(min=0)] + earlier.gather(1, ids.clamp(min=0)), -1)
    rows = torch.full((T * k + 1,), -1, dtype=torch.int64, device=DEV)
    rows[torch.where(there, positions, T * k)] = torch.arange(T, device=DEV)[:, None].expand(T, k)
    rows = rows[:T * k]
    return ids.to(torch.int32), weights, offsets.to(torch.int32), rows.to(torch.int32), positions.to(torch.int32)


# ------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    kind = case["kind"]
    stored = 0.5 + 1 / BLOCK
    if kind == "quantize":
        return {"bytes": 4 * case["M"] * case["K"], "flops": 2 * case["M"] * case["K"]}
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": int(2 * M * K + stored * N * K + 2 * M * N + 2 * N * case["bias"]), "flops": 2 * M * N * K}
    if kind == "experts":
        E, N, K, R = case["E"], case["N"], case["K"], case["T"] * case["k"]
        reached = E * (1 - (1 - case["k"] / E) ** case["T"])          # experts that some token goes to, were all alike
        x = 2 * K * (case["T"] if case["gather"] else R)
        return {"bytes": int(x + reached * (stored * N * K + 2 * N * case["bias"]) + 2 * R * N + 4 * R * case["gather"] + 4 * E),
                "flops": 2 * R * N * K}
    if kind == "route":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": T * E * (4 if case["dtype"] == "float32" else 2) + 16 * T * k + 4 * E, "flops": T * E}
    T, k, N = case["T"] - case["padded"], case["k"], case["N"]
    return {"bytes": 2 * T * k * N + 8 * case["T"] * k + 2 * case["T"] * N * (1 + case["addend"]), "flops": 2 * T * k * N}

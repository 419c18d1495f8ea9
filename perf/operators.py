"""The key-value cache of a transformer's attention in the library's per-group formats, and the attention of one new token a
sequence over it, as a list of cases with their inputs, one pass of each through the public entry points, a plain form in
elementary torch operations, and the definition in 64 bits.

A case is a dict of plain values.  `kind` says which operator it takes:

  write   tokens' keys and values, slices of the rows of a fused QKV projection, are quantized into the cache's pages, and
          the sequences they belong to are read back as bf16;
  read    sequences that the cache holds are read back as bf16 (what attention over a prompt's cached prefix starts with);
  attn    one new token a sequence attends to the tokens that the cache holds of it.

Formats (`fmt`): NVFP4 with groups of 16, INT4 with groups of 32 .. head_dim, BF16 (the values as they are).
Sequences are ragged: `lens(case)` gives each one's tokens, the first has the most.  Their pages lie in any order.
"""
import math

import torch

NVFP4, INT4, BF16 = 0, 1, 3
DEV = "cuda"

own = False


def listed():
    return [
        # ---- write
        # one decode step's tokens of a batch that has just begun: latency counts
        dict(name="append_int4", kind="write", fmt=INT4, group=64, kv_heads=8, head_dim=128, page=64, seqs=16, max_len=61, new=1),
        # a batch of prompts, odd lengths, from the rows of the fused projection
        dict(name="prompts_int4", kind="write", fmt=INT4, group=32, kv_heads=8, head_dim=128, page=64, seqs=7, max_len=2051, new=2051),
        # the largest: a long document's pages
        dict(name="document_nvfp4", kind="write", fmt=NVFP4, group=16, kv_heads=8, head_dim=128, page=128, seqs=2, max_len=40009, new=40009),
        # ---- read
        # a short prefix that several requests share
        dict(name="prefix_nvfp4", kind="read", fmt=NVFP4, group=16, kv_heads=8, head_dim=128, page=32, seqs=3, max_len=311),
        # prefixes of a batch, narrow heads
        dict(name="prefixes_int4", kind="read", fmt=INT4, group=32, kv_heads=4, head_dim=64, page=128, seqs=12, max_len=9001),
        # ---- attn
        # the first tokens of a single answer: latency counts
        dict(name="first_tokens_int4", kind="attn", fmt=INT4, group=64, kv_heads=8, q_heads=32, head_dim=128, page=64, seqs=1, max_len=19, window=0, lse=False),
        # a batch of conversations
        dict(name="conversations_nvfp4", kind="attn", fmt=NVFP4, group=16, kv_heads=8, q_heads=64, head_dim=128, page=64, seqs=32, max_len=4099, window=0, lse=False),
        # one long context: the cache's length is all there is to split
        dict(name="long_context_int4", kind="attn", fmt=INT4, group=128, kv_heads=8, q_heads=32, head_dim=128, page=128, seqs=1, max_len=131071, window=0, lse=False),
        # the cache as it was, a head of keys for each head of queries; the statistics go to another part of the context
        dict(name="unquantized_bf16", kind="attn", fmt=BF16, group=0, kv_heads=24, q_heads=24, head_dim=128, page=32, seqs=8, max_len=4608, window=0, lse=True),
        # narrow heads, an odd number of query heads a key head, the finest groups
        dict(name="narrow_heads_int4", kind="attn", fmt=INT4, group=32, kv_heads=2, q_heads=14, head_dim=64, page=256, seqs=48, max_len=5003, window=0, lse=False),
        # wide heads, a sliding window over longer sequences
        dict(name="window_int4", kind="attn", fmt=INT4, group=128, kv_heads=4, q_heads=16, head_dim=256, page=64, seqs=24, max_len=6007, window=1024, lse=False),
        # the largest: a full server's batch
        dict(name="full_batch_int4", kind="attn", fmt=INT4, group=64, kv_heads=8, q_heads=32, head_dim=128, page=64, seqs=64, max_len=24001, window=0, lse=False),
    ]


def lens(case):
    """Tokens of each sequence after the pass, from a quarter of the longest up."""
    n, top = case["seqs"], case["max_len"]
    return [max(1, top - (top * 3 // 4) * ((i * 7) % n) // max(n, 1)) for i in range(n)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _token_bytes(case):
    """Bytes of one token of one key head in the cache, keys and values."""
    D, g = case["head_dim"], case["group"]
    return 4 * D if case["fmt"] == BF16 else 2 * (D // 2 + D // 16) if case["fmt"] == NVFP4 else 2 * (D // 2 + D // g * 2)


def _attended(case):
    w = case.get("window", 0)
    return [min(n, w) if w else n for n in lens(case)]


def draw(rng):
    kind = rng.choice(["write", "read", "attn", "attn"])
    while True:
        D = rng.choice([64, 128, 128, 256])
        fmt = rng.choice([NVFP4, INT4, INT4, BF16])
        group = 16 if fmt == NVFP4 else 0 if fmt == BF16 else rng.choice([g for g in (32, 64, 128, 256) if g <= D])
        case = dict(kind=kind, fmt=fmt, group=group, kv_heads=_log(rng, 1, 24), head_dim=D, page=rng.choice([32, 64, 128, 256]))
        if kind == "attn":
            case["q_heads"] = case["kv_heads"] * rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16, 20])
            case.update(seqs=_log(rng, 1, 96), max_len=_log(rng, 1, 120000), window=rng.choice([0, 0, 0, _log(rng, 16, 5000)]),
                        lse=rng.random() < 0.5)
            read = sum(_attended(case)) * case["kv_heads"]
            # no more bytes than the largest listed case, nor more of the plain form's products, nor a larger cache
            if (read * _token_bytes(case) <= 900e6 and read * D * (1 + case["q_heads"] // case["kv_heads"] / 8) <= 1.2e9
                    and sum(lens(case)) * case["kv_heads"] * D <= 2.5e9):
                return case
        else:
            case.update(seqs=_log(rng, 1, 32), max_len=_log(rng, 4, 30000))
            if kind == "write":
                case["new"] = rng.choice([1, case["max_len"], max(1, case["max_len"] // 3)])
            if sum(lens(case)) * case["kv_heads"] * D <= 50e6:
                return case


# ------------------------------------------------------------------------ inputs

def _rng(seed, salt):
    return torch.Generator(device=DEV).manual_seed(seed * 16 + salt)


def _channels(case, g):
    """Channel sizes of a head's keys: most alike, a few far larger."""
    s = torch.exp(0.4 * torch.randn(case["kv_heads"], case["head_dim"], generator=g, device=DEV))
    s[:, :: case["head_dim"] // 4] *= 4.0
    return s


def _tokens(case, n, seed):
    """Keys and values of n tokens as slices of the rows of a fused projection, [n, heads, dim] each."""
    H, D = case["kv_heads"], case["head_dim"]
    g = _rng(seed, 1)
    chan = _channels(case, g)
    width = 3 * H * D if case["kind"] == "write" else 2 * H * D
    rows = torch.empty(n, width, dtype=torch.bfloat16, device=DEV)
    step = max(1, (1 << 28) // width)
    for r0 in range(0, n, step):
        part = torch.randn(min(step, n - r0), width, generator=g, device=DEV)
        part[:, -2 * H * D:-H * D] *= chan.reshape(-1)
        rows[r0:r0 + step] = part
    return rows[:, -2 * H * D:-H * D].unflatten(1, (H, D)), rows[:, -H * D:].unflatten(1, (H, D))


def _tables(case, seed):
    """(page table [seqs, pages of the longest], pages in all, slots of every token, sequence by sequence)."""
    n, page = lens(case), case["page"]
    counts = [(m + page - 1) // page for m in n]
    total = sum(counts)
    order = torch.randperm(total, generator=_rng(seed, 2), device=DEV).to(torch.int32)
    table = torch.full((len(n), max(counts)), -1, dtype=torch.int32, device=DEV)
    slots, at = [], 0
    for i, (m, c) in enumerate(zip(n, counts)):
        table[i, :c] = order[at:at + c]
        at += c
        pos = torch.arange(m, device=DEV)
        slots.append(table[i].long()[pos // page] * page + pos % page)
    return table, total, torch.cat(slots)


def _fresh(case):
    """Which of the tokens, sequence by sequence, the pass writes: the last `new` of each sequence."""
    return torch.cat([torch.arange(m, device=DEV) >= m - case["new"] for m in lens(case)])


def _tensor_scales(k, v):
    return [(t.abs().amax().double() / 2688.0).float().reshape(1) for t in (k, v)]


def _query(case, seed):
    return torch.randn(case["seqs"], case["q_heads"], case["head_dim"], generator=_rng(seed, 3), device=DEV).to(torch.bfloat16)


def _empty_plain(case, slots, ts):
    """The plain form's cache: a code and a group's scale for every slot, keys and values."""
    H, D, g = case["kv_heads"], case["head_dim"], case["group"]
    code = torch.bfloat16 if case["fmt"] == BF16 else torch.int8
    make = lambda: (torch.zeros(slots, H, D, dtype=code, device=DEV),
                    None if case["fmt"] == BF16 else torch.zeros(slots, H, D // g, device=DEV))
    return make() + make() + tuple(ts)


def prepare(case, seed):
    n_slots_used = sum(lens(case))
    table, pages, slots = _tables(case, seed)
    k, v = _tokens(case, n_slots_used, seed)
    ts = _tensor_scales(k, v) if case["fmt"] == NVFP4 else [None, None]
    st = dict(case=case, table=table, slots=slots)
    if own:
        from paper_2605_09503_amd import pq
        cache = pq.alloc_kv_cache(case["fmt"], case["group"], case["kv_heads"], case["head_dim"], case["page"], pages, *ts)
        write = lambda k_, v_, s_: pq.pq_kv_write(cache, k_, v_, s_)
    else:
        cache = _empty_plain(case, pages * case["page"], ts)
        write = lambda k_, v_, s_: _plain_write(case, cache, k_, v_, s_)
    st["cache"] = cache
    if case["kind"] == "write":
        new = _fresh(case)
        if not bool(new.all()):
            write(k[~new], v[~new], slots[~new])
            rows = torch.cat([k.flatten(1), k.flatten(1), v.flatten(1)], 1)[new]      # the new tokens' rows of the projection
            HD = case["kv_heads"] * case["head_dim"]
            k, v = rows[:, HD:2 * HD].unflatten(1, k.shape[1:]), rows[:, 2 * HD:].unflatten(1, k.shape[1:])
        st.update(k=k, v=v, new_slots=slots[new])
    else:
        step = max(1, (1 << 27) // (case["kv_heads"] * case["head_dim"]))
        for r0 in range(0, n_slots_used, step):
            write(k[r0:r0 + step], v[r0:r0 + step], slots[r0:r0 + step])
    if case["kind"] == "attn":
        st["q"] = _query(case, seed)
        st["lengths"] = torch.tensor(lens(case), dtype=torch.int32, device=DEV)
        st["scale"] = case["head_dim"] ** -0.5
        if own:
            st["workspace"] = pq.pq_attn_decode_workspace(cache, case["seqs"], case["q_heads"], case["max_len"], case["window"])
    return st


# ------------------------------------------------------------------------ one pass

def run(st):
    return _own(st) if own else _plain(st)


def _own(st):
    from paper_2605_09503_amd import pq
    case, cache = st["case"], st["cache"]
    if case["kind"] == "write":
        pq.pq_kv_write(cache, st["k"], st["v"], st["new_slots"])
        return pq.pq_kv_read(cache, st["slots"])
    if case["kind"] == "read":
        return pq.pq_kv_read(cache, st["slots"])
    lse = torch.empty(case["seqs"], case["q_heads"], device=DEV) if case["lse"] else None
    out = pq.pq_attn_decode(cache, st["q"], st["table"], st["lengths"], case["max_len"], st["scale"], lse=lse,
                            window=case["window"], workspace=st["workspace"])
    return [out, lse] if case["lse"] else [out]


def _plain(st):
    case, cache = st["case"], st["cache"]
    if case["kind"] == "write":
        _plain_write(case, cache, st["k"], st["v"], st["new_slots"])
        return _plain_read(case, cache, st["slots"])
    if case["kind"] == "read":
        return _plain_read(case, cache, st["slots"])
    return _plain_attention(st)


def _normal(s):
    return (s >= 2.0 ** -126) & torch.isfinite(s)


def _quantize(case, x, T):
    """Codes (NVFP4: twice the value) and scales of [n, heads, dim]: every step one binary32 operation."""
    D, g = case["head_dim"], case["group"]
    x = x.float().unflatten(2, (D // g, g))
    amax = x.abs().amax(3)
    if case["fmt"] == INT4:
        s = (amax.double() / 7.0).float()
        inv = torch.where(_normal(s), (1.0 / s.double()).float(), torch.zeros_like(s))
        z = torch.round(x * inv.unsqueeze(3)).clamp(-7.0, 7.0)
        return z.flatten(2).to(torch.int8), s
    enc = torch.where(_normal(T), (1.0 / T.double()).float(), torch.zeros_like(T))
    t = ((amax * enc).double() / 6.0).float().clamp(max=448.0)
    s = t.to(torch.float8_e4m3fn).float()
    d = s * T
    inv = torch.where(_normal(d), (1.0 / d.double()).float(), torch.zeros_like(d))
    a = (x * inv.unsqueeze(3)).abs()
    twice = torch.zeros_like(a)
    for border, tie_up, step in ((0.25, False, 1), (0.75, True, 1), (1.25, False, 1), (1.75, True, 1), (2.5, False, 2),
                                 (3.5, True, 2), (5.0, False, 4)):
        twice += step * ((a >= border) if tie_up else (a > border))
    return (twice * torch.sign(x)).flatten(2).to(torch.int8), s


def _plain_write(case, cache, k, v, slots):
    kc, ks, vc, vs, kt, vt = cache
    if case["fmt"] == BF16:
        kc[slots], vc[slots] = k, v
        return
    step = max(1, (1 << 27) // (case["kv_heads"] * case["head_dim"]))
    for r0 in range(0, slots.numel(), step):
        at = slots[r0:r0 + step]
        kc[at], ks[at] = _quantize(case, k[r0:r0 + step], kt)
        vc[at], vs[at] = _quantize(case, v[r0:r0 + step], vt)


def _values(case, codes, scales, T):
    """fp32 values of codes [.., heads, dim]; NVFP4's still without the tensor scale."""
    if case["fmt"] == BF16:
        return codes.float()
    x = codes.float().unflatten(-1, (-1, case["group"])) * scales.unsqueeze(-1)
    return (x * 0.5 if case["fmt"] == NVFP4 else x).flatten(-2)


def _plain_read(case, cache, slots):
    kc, ks, vc, vs, kt, vt = cache
    out = []
    for codes, scales, T in ((kc, ks, kt), (vc, vs, vt)):
        x = _values(case, codes[slots], None if scales is None else scales[slots], T)
        out.append((x if T is None else x * T).to(torch.bfloat16))
    return tuple(out)


def _plain_attention(st):
    case = st["case"]
    kc, ks, vc, vs, kt, vt = st["cache"]
    B, Hq, D = st["q"].shape
    H, page, G = case["kv_heads"], case["page"], st["q"].shape[1] // case["kv_heads"]
    L = min(case["max_len"], case["window"] or case["max_len"])
    out = torch.empty(B, Hq, D, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(B, Hq, device=DEV)
    step = max(1, (1 << 29) // (L * H * D))
    for b in range(0, B, step):
        n = st["lengths"][b:b + step].long().unsqueeze(1)
        pos = n - n.clamp(max=L) + torch.arange(L, device=DEV)                  # the attended tokens, then what is masked
        alive = pos < n
        pos = torch.where(alive, pos, torch.zeros_like(pos))
        slots = torch.gather(st["table"][b:b + step].long(), 1, pos // page) * page + pos % page
        q = st["q"][b:b + step].float().unflatten(1, (H, G))                    # [b, H, G, D]
        k = _values(case, kc[slots], None if ks is None else ks[slots], kt)     # [b, L, H, D]
        s = torch.matmul(k.permute(0, 2, 1, 3), q.transpose(2, 3).contiguous()) * st["scale"]      # [b, H, L, G]
        if kt is not None:
            s = s * kt
        s = torch.where(alive[:, None, :, None], s, torch.full_like(s, -math.inf))
        m = s.amax(2, keepdim=True)
        p = torch.exp(s - m)
        total = p.sum(2, keepdim=True)
        v = _values(case, vc[slots], None if vs is None else vs[slots], vt)
        o = torch.matmul((p / total).transpose(2, 3).contiguous(), v.permute(0, 2, 1, 3))          # [b, H, G, D]
        out[b:b + step] = (o if vt is None else o * vt).flatten(1, 2).to(torch.bfloat16)
        lse[b:b + step] = (m + torch.log(total)).flatten(1)
    return [out, lse] if case["lse"] else [out]


# ------------------------------------------------------------------------ the definition in 64 bits

def _fl32(x):
    return x.float().double()


def _e4m3(t):
    """The nearest E4M3 value (ties to even) of t >= 0, at most 448."""
    t = t.clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -6))) - 3)
    return torch.round(t / step) * step


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_values(case, x, T):
    """What the cache holds of bf16 values [n, heads, dim], in 64 bits."""
    if case["fmt"] == BF16:
        return x.double()
    tiny = 2.0 ** -126
    y = x.double().reshape(x.shape[0], x.shape[1], -1, case["group"])
    top = y.abs().max(3, keepdim=True).values
    if case["fmt"] == INT4:
        s = _fl32(top / 7.0)
        r = _fl32(1.0 / s.clamp(min=tiny)) * (s >= tiny)
        return (torch.round(_fl32(y * r)).clamp(-7, 7) * s).reshape(x.shape)
    T = T.double()
    e = _fl32(1.0 / T.clamp(min=tiny)) * (T >= tiny)
    s = _e4m3(_fl32(_fl32(top * e) / 6.0))
    d = _fl32(s * T)
    r = _fl32(1.0 / d.clamp(min=tiny)) * (d >= tiny)
    a = _fl32(y * r).abs()
    table = torch.tensor(_E2M1, dtype=torch.float64, device=DEV)
    mid = (table[1:] + table[:-1]) / 2
    low = torch.bucketize(a, mid)                      # a tie stays below
    up = torch.bucketize(a, mid, right=True)           # a tie goes up
    index = torch.where(low % 2 == 0, low, up)         # to the even index
    return (torch.copysign(table[index], y) * s * T).reshape(x.shape)


def exact(case, seed):
    n = lens(case)
    k, v = _tokens(case, sum(n), seed)
    kt, vt = _tensor_scales(k, v) if case["fmt"] == NVFP4 else (None, None)
    if case["kind"] != "attn":
        return _exact_values(case, k, kt), _exact_values(case, v, vt)
    H, D, w = case["kv_heads"], case["head_dim"], case["window"]
    q = _query(case, seed).double().reshape(len(n), H, -1, D)
    out, lse, at = [], [], 0
    for i, m in enumerate(n):
        first = at + (max(0, m - w) if w else 0)
        at += m
        kk = _exact_values(case, k[first:at], kt)
        vv = _exact_values(case, v[first:at], vt)
        s = torch.matmul(q[i], kk.permute(1, 2, 0).contiguous()) * D ** -0.5     # [H, G, tokens]
        weights = torch.softmax(s, 2)
        out.append(torch.matmul(weights, vv.permute(1, 0, 2).contiguous()).reshape(-1, D))
        lse.append(torch.logsumexp(s, 2).reshape(-1))
    out, lse = torch.stack(out), torch.stack(lse)
    return [out, lse] if case["lse"] else [out]


# ------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    H, D, n = case["kv_heads"], case["head_dim"], lens(case)
    stored = _token_bytes(case) * H
    if case["kind"] == "attn":
        tokens, Hq = sum(_attended(case)), case["q_heads"]
        return {"bytes": tokens * stored + case["seqs"] * Hq * (4 * D + (4 if case["lse"] else 0)), "flops": 4 * tokens * Hq * D}
    read = sum(n)
    new = sum(min(m, case["new"]) for m in n) if case["kind"] == "write" else 0
    return {"bytes": new * (4 * H * D + stored) + read * (stored + 4 * H * D), "flops": 4 * H * D * (new + read)}

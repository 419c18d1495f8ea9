"""The key-value cache and the attention over it against the oracle in 64 bits.

Tolerances.  Reading back is bit-exact.  Attention: scores are sums of D exact products in fp32, so a score is off by at most
(D + 16) 2^-24 of the largest sum of |scale q k|, and a weight by e to that power; weights are rounded once to fp16 (2^-11), the
output once to bf16 (2^-8).  The sums over tokens add 2^-24 a token of what they add up.  An fp16 weight (with its value's scale) is
at least 2^6 where the largest is, and below 2^-14 of steps of 2^-24: it may be off by 2^-31 of the largest weight times scale, which
is what is left of an element whose tokens of any weight hold zeros."""
import numpy as np
import pytest
import torch

from oracle import formats as OF
from oracle import kv as OK
from paper_2605_09503_amd import pq

pytestmark = pytest.mark.gpu
DEV = "cuda"
NV, I4, BF = pq.FMT_NVFP4, pq.FMT_INT4, pq.FMT_BF16
FORMATS = [(NV, 16, 64), (NV, 16, 128), (NV, 16, 256), (I4, 32, 64), (I4, 64, 64), (I4, 32, 128), (I4, 64, 128), (I4, 128, 128),
           (I4, 32, 256), (I4, 64, 256), (I4, 128, 256), (I4, 256, 256), (BF, 0, 64), (BF, 0, 128), (BF, 0, 256)]


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def f64(t):
    return OF.bf16_bits_to_f64(bits(t))


def rows(rng, n, heads, dim, gap=8):
    """bf16 [n, heads, dim], a slice of wider rows; channel sizes differ, some groups are far smaller than others."""
    x = rng.standard_normal((n, heads * dim)) * np.exp(rng.standard_normal(heads * dim))
    x *= np.where(rng.random((n, heads * dim)) < 0.02, 20.0, 1.0)
    wide = np.full((n, heads * dim + 2 * gap), 7.0)
    wide[:, gap:-gap] = x
    t = pq.bf16_from_bits(OF.f64_to_bf16_bits_rne(wide), DEV)
    return t[:, gap:-gap].unflatten(1, (heads, dim))


def make_cache(fmt, group, heads, dim, page, pages, k, v, garbage=True):
    ts = [torch.full((1,), np.float32(np.abs(f64(t)).max(initial=1.0) / 2688).item(), device=DEV) for t in (k, v)]
    cache = pq.alloc_kv_cache(fmt, group, heads, dim, page, pages, *(ts if fmt == NV else ()))
    cache.data.fill_(0xFF if garbage else 0)            # scales and bf16 values of all ones are NaN
    return cache, [t.item() for t in ts]


def same_bits(got, want):
    """equal as values: a zero's sign does not count"""
    a, b = (np.where(x == 0x8000, 0, x) for x in (bits(got), want))
    assert np.array_equal(a, b)


@pytest.mark.parametrize("fmt,group,dim", FORMATS)
@pytest.mark.parametrize("n,heads,page", [(1, 1, 32), (37, 3, 64), (130, 2, 256)])
def test_write_then_read(fmt, group, dim, n, heads, page):
    rng = np.random.default_rng(100 + n)
    pages = (n + 40) // page + 2
    k, v = rows(rng, n, heads, dim), rows(rng, n, heads, dim)
    cache, (kt, vt) = make_cache(fmt, group, heads, dim, page, pages, k, v)
    want = [OK.read_back(fmt, group, f64(t), s) for t, s in ((k, kt), (v, vt))]
    slots = torch.from_numpy(rng.permutation(pages * page)[:n]).to(DEV)
    first = n // 2                                       # in two calls: the second leaves the first's tokens alone
    pq.pq_kv_write(cache, k[:first], v[:first], slots[:first])
    pq.pq_kv_write(cache, k[first:], v[first:], slots[first:])
    for got, w in zip(pq.pq_kv_read(cache, slots), want):
        same_bits(got, w)
    order = torch.from_numpy(rng.permutation(n)).to(DEV)
    out = torch.full((n, heads, 2 * dim), 3.0, dtype=torch.bfloat16, device=DEV)      # k and v side by side, repeated slots
    again = torch.cat([order[:n // 2], order[:n - n // 2]])
    got = pq.pq_kv_read(cache, slots[again], out[:, :, :dim], out[:, :, dim:])
    for g, w in zip(got, want):
        same_bits(g, w[again.cpu().numpy()])


@pytest.mark.parametrize("fmt,group,dim", FORMATS)
def test_runs_of_slots(fmt, group, dim):
    # whole blocks and their edges, in order, as a prompt writes and reads them
    rng = np.random.default_rng(3)
    n, heads, page = 150, 2, 64
    k, v = rows(rng, n, heads, dim), rows(rng, n, heads, dim)
    cache, (kt, vt) = make_cache(fmt, group, heads, dim, page, 4, k, v)
    want = [OK.read_back(fmt, group, f64(t), s) for t, s in ((k, kt), (v, vt))]
    for start in (0, 32, 5):
        slots = torch.arange(start, start + n, device=DEV)
        pq.pq_kv_write(cache, k, v, slots)
        for got, w in zip(pq.pq_kv_read(cache, slots), want):
            same_bits(got, w)


@pytest.mark.parametrize("fmt,group,dim", [(NV, 16, 128), (I4, 32, 64), (BF, 0, 256)])
def test_slots_outside(fmt, group, dim):
    rng = np.random.default_rng(4)
    k, v = rows(rng, 40, 2, dim), rows(rng, 40, 2, dim)
    cache, (kt, vt) = make_cache(fmt, group, 2, dim, 32, 2, k, v, garbage=False)
    slots = torch.arange(40, device=DEV)
    slots[3], slots[20], slots[33] = -1, 64, 1 << 40
    pq.pq_kv_write(cache, k, v, slots)
    got = pq.pq_kv_read(cache, slots)
    inside = np.ones(40, bool)
    inside[[3, 20, 33]] = False
    for g, t, s in zip(got, (k, v), (kt, vt)):
        want = OK.read_back(fmt, group, f64(t), s)
        want[~inside] = 0
        same_bits(g, want)


def test_values_at_the_quantizer_s_edges():
    # groups of zeros, of one magnitude, of ties, of bf16's smallest and largest; beyond the tensor scale
    for fmt, group in ((NV, 16), (I4, 32), (I4, 128)):
        x = np.zeros((8, 1, 128))
        x[1] = 3.0
        x[2, 0, :64] = np.arange(64) / 8 - 4
        x[3, 0, ::3] = 2.0 ** -133
        x[4, 0, ::5] = 2.0 ** -126
        x[5, 0, ::7] = 1e30
        x[6, 0, :] = np.where(np.arange(128) % 2, 3.5, -7.0)
        x[7, 0, 5] = -1.0
        t = pq.bf16_from_bits(OF.f64_to_bf16_bits_rne(x), DEV)
        ts = torch.full((1,), 0.01, device=DEV)
        cache = pq.alloc_kv_cache(fmt, group, 1, 128, 32, 1, *((ts, ts) if fmt == NV else ()))
        slots = torch.arange(8, device=DEV)
        pq.pq_kv_write(cache, t, t, slots)
        want = OK.read_back(fmt, group, f64(t), ts.item())
        for got in pq.pq_kv_read(cache, slots):
            same_bits(got, want)


def test_nothing_to_write():
    cache = pq.alloc_kv_cache(I4, 64, 2, 64, 32, 1)
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    slots = torch.empty(0, dtype=torch.int64, device=DEV)
    pq.pq_kv_write(cache, none, none, slots)
    k, v = pq.pq_kv_read(cache, slots)
    assert k.shape == v.shape == (0, 2, 64)


def test_the_largest_launch():
    # 2^24 - 1 workgroups but for a few; every head of every token is the same row, and all but two tokens are padding
    heads, n, dim = 4095, 4097 * 32, 64
    x = torch.randn(2, dim, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    k, v = (t.expand(n, heads, dim) for t in x)
    cache = pq.alloc_kv_cache(I4, 32, heads, dim, 32, 1)
    slots = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    slots[1], slots[n - 1] = 30, 4
    pq.pq_kv_write(cache, k, v, slots)
    for got, row in zip(pq.pq_kv_read(cache, torch.tensor([4, 30], device=DEV)), x):
        want = OK.read_back(I4, 32, f64(row))
        assert np.array_equal(np.where(bits(got) == 0x8000, 0, bits(got)), np.broadcast_to(np.where(want == 0x8000, 0, want), got.shape))


def test_outputs_that_memory_cannot_hold():
    # what a program catches to give memory back and try again
    cache = pq.alloc_kv_cache(BF, 0, 4095, 256, 32, 1)
    slots = torch.full((4097 * 32,), -1, dtype=torch.int64, device=DEV)
    torch.cuda.empty_cache()
    torch.cuda.set_per_process_memory_fraction(0.1)
    try:
        with pytest.raises(torch.OutOfMemoryError):
            pq.pq_kv_read(cache, slots)                       # 275 GB
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)


# ------------------------------------------------------------------------ attention

def check(got, got_lse, q64, ks, vs, scale, label=""):
    """one sequence's outputs and lse (or None) against the oracle over the attended tokens, within the tolerance above"""
    want, wlse, mag, top = OK.attention(q64, ks, vs, scale)
    n, dim = ks.shape[0], q64.shape[1]
    ds, sums = (dim + 16) * 2.0 ** -24 * top, n * 2.0 ** -24
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2 * ds[:, None] + 2 * sums) * mag * (1 + 2.0 ** -7) + 1e-38
    if n:
        tol = tol + n * 2.0 ** -31 * np.abs(vs).max()
    worst = (np.abs(got - want) - tol).max()
    assert worst <= 0, "%s: off by %g over the tolerance" % (label, worst)
    if got_lse is not None:
        if n == 0:
            assert np.all(got_lse == -np.inf), label
        else:
            off = (np.abs(got_lse - wlse) - (ds + sums + 2.0 ** -22 * (1 + np.abs(wlse)))).max()
            assert off <= 0, "%s: lse off by %g over the tolerance" % (label, off)


def run_case(fmt, group, dim, lengths, heads=2, per=4, page=32, window=0, scale=None, seed=0, lse=True, noise=True, big=None,
             q_scale=1.0, max_len=None):
    """One call checked against the oracle; the cache is full of NaN behind every sequence, and in front of its window."""
    rng = np.random.default_rng(seed)
    seqs, Hq = len(lengths), heads * per
    scale = dim ** -0.5 if scale is None else scale
    n = [max(0, m) for m in lengths]
    top = max(n + [1]) if max_len is None else max_len
    per_seq = (top + page - 1) // page
    pages = seqs * per_seq + 3
    table = np.full((seqs, per_seq + 1), -1, dtype=np.int32)
    order = rng.permutation(pages)[:seqs * per_seq].reshape(seqs, per_seq)
    for b, m in enumerate(n):
        table[b, :(m + page - 1) // page] = order[b, :(m + page - 1) // page]
    k, v = rows(rng, sum(n), heads, dim), rows(rng, sum(n), heads, dim)
    if big is not None:
        v = v * big
    cache, (kt, vt) = make_cache(fmt, group, heads, dim, page, pages, k, v)
    pos = [np.arange(m) for m in n]
    slots = np.concatenate([table[b][p // page].astype(np.int64) * page + p % page for b, p in enumerate(pos)] or [np.zeros(0, np.int64)])
    keep = np.concatenate([p >= OK.attended(m, window).start for p, m in zip(pos, n)] or [np.zeros(0, bool)])
    if not noise:
        keep[:] = True
    sl = np.where(keep, slots, -1)                       # what the window leaves out stays NaN
    pq.pq_kv_write(cache, k, v, torch.from_numpy(sl).to(DEV))
    wide = torch.randn(seqs, Hq + 1, dim, generator=torch.Generator().manual_seed(seed)) * q_scale
    q = wide.to(torch.bfloat16).to(DEV)[:, 1:]
    lse_t = torch.full((seqs, Hq), 5.0, device=DEV) if lse else None
    wide_table = torch.from_numpy(np.concatenate([table, table], 1)).to(DEV)[:, :per_seq + 1]
    lens = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    ws = pq.pq_attn_decode_workspace(cache, seqs, Hq, top, window)
    out = pq.pq_attn_decode(cache, q, wide_table, lens, top, scale, lse=lse_t, window=window, workspace=ws)
    out2 = torch.full((seqs, 2, Hq, dim), 9.0, dtype=torch.bfloat16, device=DEV)
    assert pq.pq_attn_decode(cache, q, wide_table, lens, top, scale, out=out2[:, 1], window=window, workspace=ws).data_ptr() \
        == out2[:, 1].data_ptr()
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), out2[:, 1].contiguous().view(torch.int16)), "not the same bits from call to call"
    assert bool((out2[:, 0] == 9.0).all())
    assert int(ws[:pq.ATTN_DECODE_ZERO_BYTES].max()) == 0
    ks, vs = OK.stored(fmt, group, f64(k), kt), OK.stored(fmt, group, f64(v), vt)
    got, q64, at = f64(out), f64(q), 0
    for b, m in enumerate(n):
        r = OK.attended(m, window)
        sel = slice(at + r.start, at + m)
        at += m
        check(got[b], lse_t[b].cpu().numpy().astype(np.float64) if lse else None, q64[b], ks[sel], vs[sel], scale,
              "sequence %d, %d tokens" % (b, m))
    return out


@pytest.mark.parametrize("fmt,group,dim", FORMATS)
def test_lengths(fmt, group, dim):
    run_case(fmt, group, dim, [0, 1, 2, 31, 32, 33, 63, 64, 65, 96, 97, 250, -4, 129])


@pytest.mark.parametrize("fmt,group,dim", FORMATS)
def test_long_sequences(fmt, group, dim):
    run_case(fmt, group, dim, [2500, 1, 777], page=64, seed=1)


@pytest.mark.parametrize("per", [1, 2, 3, 5, 7, 8, 12, 15, 16, 17, 20, 31, 32, 33, 48, 70])
@pytest.mark.parametrize("fmt,group,dim", [(I4, 64, 128), (NV, 16, 64), (BF, 0, 256), (I4, 32, 256)])
def test_queries_a_head(fmt, group, dim, per):
    run_case(fmt, group, dim, [70, 5, 300], heads=2 if per < 20 else 1, per=per, seed=per)


@pytest.mark.parametrize("fmt,group,dim", [(I4, 32, 64), (I4, 128, 128), (NV, 16, 256), (NV, 16, 128), (BF, 0, 128)])
@pytest.mark.parametrize("window", [1, 15, 32, 33, 100, 400, 5000])
def test_windows(fmt, group, dim, window):
    run_case(fmt, group, dim, [0, 1, 33, 64, 100, 401, 1030], window=window, page=64, seed=window)


@pytest.mark.parametrize("page", [32, 64, 128, 256, 512, 1024])
def test_pages(page):
    run_case(I4, 64, 128, [40, 1500, 3], page=page, seed=page)
    run_case(NV, 16, 64, [40, 1500, 3], page=page, seed=page, heads=3, per=1)


@pytest.mark.parametrize("fmt,group,dim", [(I4, 64, 128), (NV, 16, 128), (BF, 0, 64)])
def test_many_sequences(fmt, group, dim):
    rng = np.random.default_rng(9)
    run_case(fmt, group, dim, [int(m) for m in rng.integers(0, 200, 150)], heads=1, per=2)
    run_case(fmt, group, dim, [int(m) for m in rng.integers(0, 20, 700)], heads=1, per=1, lse=False)


@pytest.mark.parametrize("fmt,group,dim", [(I4, 64, 128), (NV, 16, 128), (BF, 0, 128)])
def test_one_long_sequence(fmt, group, dim):
    run_case(fmt, group, dim, [30011], heads=1, per=4, page=256)


@pytest.mark.parametrize("fmt,group,dim", [(I4, 64, 64), (NV, 16, 128), (BF, 0, 256)])
def test_one_long_sequence_of_many_queries(fmt, group, dim):
    run_case(fmt, group, dim, [40003], heads=1, per=11, page=1024)


@pytest.mark.parametrize("per", [3, 16])                   # sixteen parts joined at a time, and eight
@pytest.mark.parametrize("fmt,group,dim", [(I4, 64, 128), (NV, 16, 64), (BF, 0, 64), (I4, 128, 256)])
def test_parts_joined_over_levels(fmt, group, dim, per):
    # up to 64 parts a pair: sums of parts are joined again, out of the slots that they were read from
    rng = np.random.default_rng(41)
    lengths, heads, page = [20011, 9000], 3, 256
    per_seq = (max(lengths) + page - 1) // page
    k, v = rows(rng, sum(lengths), heads, dim), rows(rng, sum(lengths), heads, dim)
    cache, (kt, vt) = make_cache(fmt, group, heads, dim, page, 2 * per_seq, k, v)
    table = torch.arange(2 * per_seq, dtype=torch.int32, device=DEV).reshape(2, per_seq)
    slots = torch.cat([b * per_seq * page + torch.arange(n) for b, n in enumerate(lengths)]).to(DEV)
    pq.pq_kv_write(cache, k, v, slots)
    q = torch.randn(2, heads * per, dim, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).to(DEV)
    lens, ws = torch.tensor(lengths, dtype=torch.int32, device=DEV), pq.pq_attn_decode_workspace(cache, 2, heads * per, max(lengths))
    results = []
    for _ in range(100):
        lse = torch.empty(2, heads * per, device=DEV)
        results.append((pq.pq_attn_decode(cache, q, table, lens, max(lengths), dim ** -0.5, lse=lse, workspace=ws), lse))
    out, lse = results[0]
    for o, l in results[1:]:
        assert torch.equal(o.view(torch.int16), out.view(torch.int16)) and torch.equal(l, lse)
    ks, vs = OK.stored(fmt, group, f64(k), kt), OK.stored(fmt, group, f64(v), vt)
    got, q64, at = f64(out), f64(q), 0
    for b, n in enumerate(lengths):
        check(got[b], lse[b].cpu().numpy().astype(np.float64), q64[b], ks[at:at + n], vs[at:at + n], dim ** -0.5, "sequence %d" % b)
        at += n


@pytest.mark.parametrize("fmt,group,dim", [(I4, 32, 64), (NV, 16, 64), (BF, 0, 64), (I4, 128, 128)])
def test_more_pairs_than_workgroups(fmt, group, dim):
    # sequences of a server's batch: workgroups that end one pair and begin the next
    rng = np.random.default_rng(21)
    run_case(fmt, group, dim, [int(m) for m in rng.integers(1, 1500, 130)] + [1500], heads=4, per=2, page=64)
    # many pairs, one of them long: a workgroup each
    run_case(fmt, group, dim, [1200] + [int(m) for m in rng.integers(0, 70, 89)], heads=24, per=1, page=64, lse=False)


@pytest.mark.parametrize("fmt,group,dim", [(I4, 32, 64), (NV, 16, 64), (BF, 0, 64), (I4, 64, 128)])
def test_shares_of_pairs(fmt, group, dim):
    # three pairs a sequence (33 queries of one key head)
    rng = np.random.default_rng(33)
    some = lambda lo, hi, n: [int(m) for m in rng.integers(lo, hi, n)]
    run_case(fmt, group, dim, some(300, 1500, 133), heads=1, per=33, page=64)              # fewer pairs than workgroups, each whole
    run_case(fmt, group, dim, some(300, 1000, 132) + [4000], heads=1, per=33, page=64)     # one much longer: equal parts of pairs
    run_case(fmt, group, dim, [6000] + some(900, 1700, 200), heads=1, per=33, page=64, lse=False)    # blocks in a row
    run_case(fmt, group, dim, some(0, 60, 180) + [3000], heads=1, per=33, page=64, lse=False)        # many short ones


@pytest.mark.parametrize("fmt,group,dim", [(I4, 64, 128), (NV, 16, 64), (BF, 0, 128)])
def test_short_sequences_of_a_large_capacity(fmt, group, dim):
    run_case(fmt, group, dim, [0, 900, 1, 33, 400], max_len=20000, page=64)
    run_case(fmt, group, dim, [900, 70], max_len=20000, page=1024, window=300)
    rng = np.random.default_rng(34)
    run_case(fmt, group, dim, [int(m) for m in rng.integers(0, 200, 300)], heads=2, per=1, max_len=2000, page=64, lse=False)


def test_blocks_near_the_limit_of_a_call():
    # 262 140 pairs of 2501 blocks, over 2^29 in all (sequences that share their pages): numbers of idle waves would pass 31 bits
    rng = np.random.default_rng(35)
    n, seqs, heads = 2500 * 32 + 5, 65535, 4
    k, v = rows(rng, n, heads, 64), rows(rng, n, heads, 64)
    cache, _ = make_cache(I4, 64, heads, 64, 1024, 79, k, v)
    pq.pq_kv_write(cache, k, v, torch.arange(n, device=DEV))
    table = torch.arange(79, dtype=torch.int32, device=DEV).repeat(seqs, 1)
    q = torch.randn(1, heads, 64, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    lengths = torch.full((seqs,), n, dtype=torch.int32, device=DEV)
    out = pq.pq_attn_decode(cache, q.repeat(seqs, 1, 1), table, lengths, n, 0.125)
    assert torch.equal(out, out[:1].expand_as(out))
    ks, vs = OK.stored(I4, 64, f64(k[:, :2]), None), OK.stored(I4, 64, f64(v[:, :2]), None)
    check(f64(out[0, :2]), None, f64(q[0, :2]), ks, vs, 0.125)


@pytest.mark.parametrize("fmt,group,dim", [(I4, 64, 128), (NV, 16, 128), (BF, 0, 128)])
def test_sharp_and_flat_scores(fmt, group, dim):
    run_case(fmt, group, dim, [500, 33], scale=1.0, q_scale=4.0)            # one token takes nearly all
    run_case(fmt, group, dim, [500, 33], scale=0.0)                         # the mean
    run_case(fmt, group, dim, [500, 33], scale=-0.05)
    run_case(fmt, group, dim, [500, 33], q_scale=1e-30, scale=1e28)
    run_case(fmt, group, dim, [500, 33], q_scale=1e18, scale=1e-20)


@pytest.mark.parametrize("fmt,group,dim", [(I4, 64, 128), (I4, 32, 64), (BF, 0, 128)])
@pytest.mark.parametrize("big", [1e30, 1e-25, 3e5])
def test_sizes_of_values(fmt, group, dim, big):
    # fp16 weights carry the groups' scales: neither overflow nor underflow may come of it
    run_case(fmt, group, dim, [500, 33, 1], big=big)


@pytest.mark.parametrize("fmt,group,dim", [(I4, 64, 128), (I4, 256, 256), (NV, 16, 128), (BF, 0, 64)])
@pytest.mark.parametrize("exponent", [-70, 78])            # values of rows() lie some 2^10 to both sides
def test_ends_of_the_values_range(fmt, group, dim, exponent):
    run_case(fmt, group, dim, [20011, 33, 1], big=2.0 ** exponent, page=256, heads=1)
    run_case(fmt, group, dim, [900], big=2.0 ** exponent, scale=0.0)


@pytest.mark.parametrize("fmt,group,dim", [(I4, 64, 128), (NV, 16, 128), (BF, 0, 128)])
def test_pages_outside_are_left_out(fmt, group, dim):
    rng = np.random.default_rng(12)
    n, page = 200, 32
    k, v = rows(rng, n, 1, dim), rows(rng, n, 1, dim)
    cache, (kt, vt) = make_cache(fmt, group, 1, dim, page, 8, k, v)
    slots = np.arange(n)
    pq.pq_kv_write(cache, k, v, torch.from_numpy(slots).to(DEV))
    table = np.arange(8, dtype=np.int32)[None].repeat(2, 0)
    table[0, 2], table[0, 5], table[1, :7] = -1, 8, 1 << 30
    q = torch.randn(2, 4, dim, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    lse = torch.empty(2, 4, device=DEV)
    out = pq.pq_attn_decode(cache, q, torch.from_numpy(table).to(DEV), torch.tensor([n, n], dtype=torch.int32, device=DEV), n, 0.1, lse=lse)
    inside = np.ones(n, bool)
    inside[64:96] = inside[160:192] = False
    check(f64(out)[0], lse[0].cpu().numpy().astype(np.float64), f64(q)[0], OK.stored(fmt, group, f64(k), kt)[inside],
          OK.stored(fmt, group, f64(v), vt)[inside], 0.1)
    assert np.all(f64(out)[1] == 0) and bool((lse[1] == -np.inf).all())


@pytest.mark.parametrize("n", [5, 120, 4000])              # tokens a sequence: within a block, a workgroup a pair, parts that join
@pytest.mark.parametrize("fmt,group", [(I4, 64), (NV, 16), (BF, 0)])
def test_nan_stays_in_its_row(fmt, group, n):
    rng = np.random.default_rng(14)
    heads, per, pages = 2, 3, 2 * ((n + 63) // 64)
    k, v = rows(rng, 2 * n, heads, 128), rows(rng, 2 * n, heads, 128)
    cache, _ = make_cache(fmt, group, heads, 128, 64, pages, k, v)
    table = torch.arange(pages, dtype=torch.int32, device=DEV).reshape(2, -1)
    slots = torch.cat([torch.arange(n), pages // 2 * 64 + torch.arange(n)]).to(DEV)
    pq.pq_kv_write(cache, k, v, slots)
    q = torch.randn(2, heads * per, 128, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(DEV)
    lens = torch.full((2,), n, dtype=torch.int32, device=DEV)

    def call(q):
        lse = torch.empty(2, heads * per, device=DEV)
        return pq.pq_attn_decode(cache, q, table, lens, n, 0.09, lse=lse), lse
    want, want_lse = call(q)
    q[0, 4, 17] = float("nan")
    got, lse = call(q)
    assert bool(got[0, 4].isnan().all()) and bool(lse[0, 4].isnan())       # a part of a context that is NaN may not weigh nothing
    hit = torch.zeros(2, heads * per, dtype=torch.bool, device=DEV)
    hit[0, 4] = True
    assert torch.equal(got[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])


@pytest.mark.parametrize("n", [5, 120, 4000, 20011])
def test_nan_in_a_key_of_a_bf16_cache(n):
    # all queries of its key head, in its sequence, and no others; across parts that join
    rng = np.random.default_rng(15)
    heads, per, pages = 2, 3, 2 * ((n + 63) // 64)
    k, v = rows(rng, 2 * n, heads, 128), rows(rng, 2 * n, heads, 128)
    cache, _ = make_cache(BF, 0, heads, 128, 64, pages, k, v)
    table = torch.arange(pages, dtype=torch.int32, device=DEV).reshape(2, -1)
    slots = torch.cat([torch.arange(n), pages // 2 * 64 + torch.arange(n)]).to(DEV)
    pq.pq_kv_write(cache, k, v, slots)
    q = torch.randn(2, heads * per, 128, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).to(DEV)
    lens = torch.full((2,), n, dtype=torch.int32, device=DEV)

    def call():
        lse = torch.empty(2, heads * per, device=DEV)
        return pq.pq_attn_decode(cache, q, table, lens, n, 0.09, lse=lse), lse
    want, want_lse = call()
    at = n + n // 2                                            # a token of the second sequence
    bad = k[at:at + 1].clone()
    bad[0, 0, 5] = float("nan")
    pq.pq_kv_write(cache, bad, v[at:at + 1], slots[at:at + 1])
    got, lse = call()
    hit = torch.zeros(2, heads * per, dtype=torch.bool, device=DEV)
    hit[1, :per] = True
    assert bool(got[hit].isnan().all()) and bool(lse[hit].isnan().all())
    assert torch.equal(got[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])


def test_lengths_beyond_max_len_are_cut():
    rng = np.random.default_rng(13)
    k, v = rows(rng, 96, 1, 64), rows(rng, 96, 1, 64)
    cache, _ = make_cache(I4, 32, 1, 64, 32, 3, k, v)
    pq.pq_kv_write(cache, k, v, torch.arange(96, device=DEV))
    table = torch.arange(3, dtype=torch.int32, device=DEV)[None]
    q = torch.randn(1, 2, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    call = lambda n, top: pq.pq_attn_decode(cache, q, table, torch.tensor([n], dtype=torch.int32, device=DEV), top, 0.1)
    assert torch.equal(call(50, 96), call(1 << 30, 50))


def test_no_sequences():
    cache = pq.alloc_kv_cache(I4, 64, 2, 64, 32, 1)
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    out = pq.pq_attn_decode(cache, q, torch.empty((0, 1), dtype=torch.int32, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV), 32, 0.1)
    assert out.shape == (0, 4, 64)


@pytest.mark.parametrize("n", [120, 4000])                 # one workgroup a pair; several that join
@pytest.mark.parametrize("fmt,group", [(I4, 64), (NV, 16), (BF, 0)])
def test_graph_replays_and_other_streams(fmt, group, n):
    """A decode step (write, attention) captured once: replays follow the lengths and slots in device memory, and a second stream
    with a workspace of its own gives the same."""
    rng = np.random.default_rng(14)
    dim, heads, page = 128, 2, 32
    pages = (n + 40) // page
    k, v = rows(rng, n, heads, dim), rows(rng, n, heads, dim)
    cache, (kt, vt) = make_cache(fmt, group, heads, dim, page, pages, k, v)
    pq.pq_kv_write(cache, k, v, torch.arange(n, device=DEV))
    q = torch.randn(1, 8, dim, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    lengths, slot = torch.tensor([n - 4], dtype=torch.int32, device=DEV), torch.tensor([n - 5], device=DEV)
    kn, vn = k[:1].clone(), v[:1].clone()
    ws = pq.pq_attn_decode_workspace(cache, 1, 8, n + 8)
    out = torch.empty_like(q)
    other = torch.cuda.Stream()

    def step(o, w):
        pq.pq_kv_write(cache, kn, vn, slot)
        pq.pq_attn_decode(cache, q, table, lengths, n + 8, 0.1, out=o, workspace=w)

    step(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, ws)
    ws2 = pq.pq_attn_decode_workspace(cache, 1, 8, n + 8)
    for i in range(4):
        kn.copy_(k[10 + i:11 + i])
        vn.copy_(v[20 + i:21 + i])
        slot.fill_(n - 5 + i)
        lengths.fill_(n - 4 + i)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        eager = torch.empty_like(q)
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            step(eager, ws2)
        torch.cuda.current_stream().wait_stream(other)
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.int16), eager.view(torch.int16))
        rk, rv = pq.pq_kv_read(cache, slot)
        same_bits(rk, OK.read_back(fmt, group, f64(kn), kt))
        same_bits(rv, OK.read_back(fmt, group, f64(vn), vt))


def example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_cache.py")
    spec = importlib.util.spec_from_file_location("decode_cache", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("fmt", ["nvfp4", "int4", "bf16"])
def test_attention_of_the_example(fmt):
    """Every write and attention of the example, of its cache and the unquantized one, against the oracle over what was written."""
    module, steps = example(), 3
    held, calls = {}, []

    class Watched:
        def __getattr__(self, name):
            return getattr(pq, name)

        def pq_kv_write(self, cache, k, v, slots):
            pq.pq_kv_write(cache, k, v, slots)
            parts = held.setdefault(id(cache), {})
            ts = [t.item() if cache.fmt == NV else None for t in (cache.k_tensor_scale, cache.v_tensor_scale)]
            ks, vs = (OK.stored(cache.fmt, cache.group, f64(t), s) for t, s in zip((k, v), ts))
            parts.update((int(s), (ks[i], vs[i])) for i, s in enumerate(slots.tolist()))

        def pq_attn_decode(self, cache, q, table, lengths, max_len, scale, workspace):
            out = pq.pq_attn_decode(cache, q, table, lengths, max_len, scale, workspace=workspace)
            calls.append(cache.fmt)
            got, q64, parts = f64(out), f64(q), held[id(cache)]
            for b, n in enumerate(lengths.tolist()):
                slots = [int(table[b, t // cache.page]) * cache.page + t % cache.page for t in range(n)]
                ks, vs = (np.stack([parts[s][i] for s in slots]) for i in (0, 1))
                check(got[b], None, q64[b], ks, vs, scale, "sequence %d of %d tokens" % (b, n))
            return out

    module.pq = Watched()
    module.run(fmt, steps=steps)
    assert len(calls) == 2 * steps and calls.count(BF) == (2 if fmt == "bf16" else 1) * steps


@pytest.mark.parametrize("fmt", ["nvfp4", "int4", "bf16"])
def test_example(fmt):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_cache.py")
    spec = importlib.util.spec_from_file_location("decode_cache", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    worst, x = module.run(fmt, steps=3)
    assert bool(torch.isfinite(x.float()).all())
    # 4-bit keys and values of normal variates: codes are off by up to a seventh of a group's largest, some 2.5 standard deviations,
    # so an output may be off by as much as it is large; the unquantized cache gives the same bits
    assert worst <= (0.0 if fmt == "bf16" else 2.0)

"""MXFP4 quantizers and products, routing and the weighted sum against the oracle in 64 bits.

Tolerances.  Codes, scales and read-back values are exact.  A product's terms are exact; a 32 x 32 x 64 instruction adds 64 of them to
an fp32 sum, and each of its additions is taken to lose at most 2^-23 of the terms' absolute sum (2^-24 rounded, twice that cut off): K / 64
instructions in turn and some 8 additions that join parts give (K / 64 + 8) 2^-23 of sum |terms|.  A bias is one of the terms: the sum may
begin with it.  bf16 outputs are rounded once (2^-8 of themselves).  Weights: e^x of an argument that is off by 2^-24 of itself (|x| < 100) and a few
roundings in sum and quotient: 1e-5.  The weighted sum: k + 1 fused steps of 2^-24 of the terms' absolute sum, then bf16's 2^-8."""
import numpy as np
import pytest
import torch

from oracle import formats as OF
from oracle import mx
from oracle import quantize as OQ
from paper_2605_09503_amd import pq

pytestmark = pytest.mark.gpu
DEV = "cuda"
MX = pq.FMT_MXFP4


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def f64(t):
    return OF.bf16_bits_to_f64(bits(t)) if t.dtype == torch.bfloat16 else t.cpu().double().numpy()


def rows_of(rng, rows, K, gap=0, odd=True):
    """bf16 [rows, K], a slice of wider rows where gap > 0: channels of uneven sizes, zeros, groups of subnormals and of huge values."""
    x = rng.standard_normal((rows, K)) * np.exp(rng.standard_normal(K))
    x[rng.random((rows, K)) < 0.02] *= 30.0
    if odd:
        x[rng.random((rows, K)) < 0.05] = 0.0
        g = x.reshape(rows, K // 32, 32)
        g[rng.random(g.shape[:2]) < 0.03] = 0.0
        g[rng.random(g.shape[:2]) < 0.03] *= 2.0 ** -20
    wide = np.full((rows, K + 2 * gap), 7.0)
    wide[:, gap:gap + K] = x
    return pq.bf16_from_bits(OF.f64_to_bf16_bits_rne(wide), DEV)[:, gap:gap + K]


def stored(q):
    return torch.from_numpy(mx.packed_codes(q)).to(DEV), torch.from_numpy(q.scale).to(DEV)


def operand(x):
    return pq.pq_quantize_act_packed(MX, 32, x, None)


def bound(K, mag):
    return (K / 64 + 8) * 2.0 ** -23 * mag


def close(got, ref, err, rounding=2.0 ** -8):
    got = f64(got)
    nan = np.isnan(ref)
    assert np.array_equal(np.isnan(got), nan)
    off, allowed = np.abs(got - ref)[~nan], (err + rounding * (np.abs(ref) + err) + 2.0 ** -133)[~nan]
    worst = (off / allowed).max(initial=0.0)
    assert worst <= 1.0, worst


EXTREMES = [0.0, -0.0, 2.0 ** -133, -2.0 ** -126, 2.0 ** -127, 2.0 ** -120, 1.0, -1.75, 3.5, 5.0, -7.0, 7.96875, 2.0 ** 120, -2.0 ** 127 * 1.9921875]


# ------------------------------------------------------------------------ quantizers

@pytest.mark.parametrize("rows,K,gap", [(1, 32, 0), (3, 96, 8), (64, 256, 0), (37, 288, 16), (129, 2016, 8), (5, 10240, 0)])
def test_quantize_stored(rows, K, gap):
    rng = np.random.default_rng(rows + K)
    x = rows_of(rng, rows, K, gap)
    want = mx.quantize(f64(x))
    codes, scales = pq.alloc_quantized(MX, 32, rows, K)
    pq.pq_quantize_act(MX, 32, x, None, None, codes, scales)
    assert np.array_equal(codes.cpu().numpy(), mx.packed_codes(want)) and np.array_equal(scales.cpu().numpy(), want.scale)
    y = pq.pq_dequantize(MX, 32, codes, scales)
    assert np.array_equal(f64(y), mx.dequantize(want))
    wide = torch.full((rows, K + 24), 3.0, dtype=torch.bfloat16, device=DEV)
    pq.pq_dequantize(MX, 32, codes, scales, y=wide[:, 8:8 + K])
    assert torch.equal(wide[:, 8:8 + K], y) and bool((wide[:, :8] == 3).all()) and bool((wide[:, 8 + K:] == 3).all())
    perm = torch.from_numpy(rng.permutation(K).astype(np.int32)).to(DEV)
    pq.pq_quantize_act(MX, 32, x, perm, None, codes, scales)
    want = mx.quantize(f64(x)[:, perm.cpu().numpy()])
    assert np.array_equal(codes.cpu().numpy(), mx.packed_codes(want)) and np.array_equal(scales.cpu().numpy(), want.scale)
    one = torch.zeros(1, device=DEV)
    codes.zero_()
    pq.pq_quantize_weights(MX, 32, x.contiguous(), perm, codes, scales, one)
    assert np.array_equal(codes.cpu().numpy(), mx.packed_codes(want)) and one.item() == 1.0


def test_every_bf16_value():
    # each finite value as the largest of its group, with a spread of smaller ones, and next to infinities and NaN
    rng = np.random.default_rng(7)
    values = np.arange(65536, dtype=np.uint16)
    x = rng.permutation(np.tile(values, 8))                    # 16384 groups of any values: most hold one that is not finite
    lone = np.zeros((65536, 32), dtype=np.uint16)
    lone[:, 3] = values
    e = OF.f64_to_bf16_bits_rne(np.ldexp(rng.standard_normal((40, 32 * 32)), np.repeat(rng.integers(-140, 127, (40, 32)), 32, axis=1)).clip(-3e38, 3e38))
    for b in (x.reshape(128, -1), lone.reshape(1024, -1), e):
        t = pq.bf16_from_bits(b, DEV)
        want = mx.quantize(f64(t))
        codes, scales = pq.alloc_quantized(MX, 32, *t.shape)
        pq.pq_quantize_act(MX, 32, t, None, None, codes, scales)
        assert np.array_equal(scales.cpu().numpy(), want.scale)
        ok = np.repeat(want.scale != 255, 16, axis=1)            # codes of a NaN group do not matter
        assert np.array_equal(codes.cpu().numpy()[ok], mx.packed_codes(want)[ok])
        got, ref = f64(pq.pq_dequantize(MX, 32, codes, scales)), mx.dequantize(want)
        assert np.array_equal(got, ref, equal_nan=True)


@pytest.mark.parametrize("rows,K,gap", [(1, 32, 0), (3, 96, 8), (64, 256, 0), (37, 288, 16), (129, 2016, 8), (300, 544, 0)])
def test_operand_is_the_packed_stored_form(rows, K, gap):
    rng = np.random.default_rng(rows * K)
    x = rows_of(rng, rows, K, gap)
    want = mx.quantize(f64(x))
    codes, scales = stored(want)
    need = pq.pq_operand_bytes(MX, 32, rows, K)
    a, b = (torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(2))
    got_codes, got_scales = pq.alloc_quantized(MX, 32, rows, K)
    pq.pq_pack_operand(MX, 32, codes, scales, a)
    pq.pq_quantize_act_packed(MX, 32, x, None, b, got_codes, got_scales)
    assert torch.equal(got_codes, codes) and torch.equal(got_scales, scales)
    # what lies between the parts to make them multiples of 256 bytes is nobody's
    panels = (K + 127) // 128
    at = (panels * rows * 64 + 255) // 256 * 256
    for part in (slice(0, panels * rows * 64), slice(at, at + panels * rows * 4)):
        assert torch.equal(a[part], b[part])


@pytest.mark.parametrize("fmt,group", [(pq.FMT_NVFP4, 16), (pq.FMT_INT4, 32), (pq.FMT_INT4, 128), (pq.FMT_INT3, 64)])
def test_dequantize_other_formats(fmt, group):
    rng = np.random.default_rng(11)
    x = rows_of(rng, 19, 384)
    ts = torch.full((1,), float(np.float32(np.abs(f64(x)).max() / 2688)), device=DEV)
    codes, scales = pq.alloc_quantized(fmt, group, 19, 384)
    pq.pq_quantize_act(fmt, group, x, None, ts, codes, scales)
    q = OQ.quantize(fmt, group, f64(x), np.float32(ts.item()))
    want = OF.f64_to_bf16_bits_rne(OF.fl32(OQ.dequantize(fmt, group, q)))
    got = bits(pq.pq_dequantize(fmt, group, codes, scales, ts))
    assert np.array_equal(np.where(got == 0x8000, 0, got), np.where(want == 0x8000, 0, want))


def test_dequantize_refuses_tensors_that_do_not_fit():
    codes, scales = pq.alloc_quantized(MX, 32, 4, 64)
    out = lambda *shape, **kw: torch.empty(shape, device=DEV, **{"dtype": torch.bfloat16, **kw})
    for args, kw in [((codes, scales[:3]), {}), ((codes, scales.float()), {}), ((codes, scales.cpu()), {}), ((codes, scales), dict(y=out(3, 64))),
                     ((codes, scales), dict(y=out(4, 64, dtype=torch.float32))), ((codes, scales), dict(y=out(64, 4).T)),
                     ((codes, scales), dict(y=out(1, 64).expand(4, 64))), ((codes, scales), dict(y=out(4, 60)))]:
        with pytest.raises(pq.PQError):
            pq.pq_dequantize(MX, 32, *args, **kw)
    with pytest.raises(pq.PQError):
        pq.pq_dequantize(pq.FMT_NVFP4, 16, codes, torch.zeros(4, 4, dtype=torch.uint8, device=DEV), torch.ones(1, dtype=torch.float64, device=DEV))
    y = out(1, 64)
    pq.pq_dequantize(MX, 32, codes[:1].zero_(), scales[:1].zero_(), y=y)
    assert not y.any()


# ------------------------------------------------------------------------ products

SHAPES = [(1, 1, 32), (1, 8, 96), (1, 300, 4096), (2, 517, 1056), (16, 64, 256), (17, 40, 288), (31, 136, 512), (33, 1000, 544), (64, 257, 2016), (65, 128, 1024),
          (100, 333, 800), (128, 128, 128), (129, 200, 2560), (250, 512, 768), (257, 260, 320), (300, 1030, 1312), (777, 520, 640), (1025, 515, 2080)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(M, N, K):
    rng = np.random.default_rng(M * 7 + N + K)
    x, w = rows_of(rng, M, K, 8), rows_of(rng, N, K)
    xq, wq = (mx.dequantize(mx.quantize(f64(t))) for t in (x, w))
    ref, mag = xq @ wq.T, np.abs(xq) @ np.abs(wq).T
    a, b = operand(x), pq.pq_pack_operand(MX, 32, *stored(mx.quantize(f64(w))))
    ldy = (N + 7) // 8 * 8 + 8
    y = torch.full((M + 1, ldy), 5.0, device=DEV)
    pq.pq_qgemm_packed_f32(MX, 32, a, None, b, None, y[:M], M, N, K)
    close(y[:M, :N], ref, bound(K, mag), 0.0)
    assert bool((y[M:] == 5).all()) and bool((y[:, N:] == 5).all())
    y = torch.full((M + 1, ldy), 5.0, dtype=torch.bfloat16, device=DEV)
    pq.pq_qgemm_packed(MX, 32, a, None, b, None, y[:M], M, N, K)
    close(y[:M, :N], ref, bound(K, mag))
    assert bool((y[M:] == 5).all()) and bool((y[:, N:] == 5).all())
    bias = rows_of(rng, 1, (N + 31) // 32 * 32, odd=False)[0, :N].clone()
    pq.pq_qgemm_packed_bias(MX, 32, a, None, b, None, bias, y[:M], M, N, K)
    close(y[:M, :N], ref + f64(bias[None]), bound(K, mag + np.abs(f64(bias[None]))))
    assert bool((y[M:] == 5).all()) and bool((y[:, N:] == 5).all())


@pytest.mark.parametrize("M,N,K", [(5, 70, 288), (200, 300, 512), (600, 700, 320)])
def test_product_of_extremes(M, N, K):
    # the largest and smallest scales; a group with an infinity or a NaN makes its row (or column) NaN and nothing else
    rng = np.random.default_rng(M)
    x, w = rows_of(rng, M, K), rows_of(rng, N, K)
    x[0, :32] = torch.tensor(EXTREMES + [0.0] * (32 - len(EXTREMES)), dtype=torch.bfloat16)
    x[M // 2] *= 2.0 ** 100
    w[1] *= 2.0 ** -110
    x[1, 33] = float("inf")
    x[M - 1, K - 1] = float("nan")
    w[N - 2, 5] = -float("inf")
    w[0, :32] = 0.0                                                       # what meets the extremes of row 0: fp32 holds the rest
    w[1:, :32] = torch.where(w[1:, :32].abs() > 1, torch.zeros_like(w[1:, :32]), w[1:, :32])
    xq, wq = (mx.dequantize(mx.quantize(f64(t))) for t in (x, w))
    with np.errstate(invalid="ignore", over="ignore"):
        ref, mag = xq @ wq.T, np.abs(xq) @ np.abs(wq).T
    keep = np.isnan(ref) | (np.abs(mag) < 2.0 ** 120)
    y = torch.empty(M, (N + 7) // 8 * 8, device=DEV)
    pq.pq_qgemm_packed_f32(MX, 32, operand(x), None, operand(w), None, y, M, N, K)
    got = y[:, :N].cpu().double().numpy()
    assert np.array_equal(np.isnan(got)[keep], np.isnan(ref)[keep])
    fine = keep & ~np.isnan(ref)
    assert (np.abs(got - ref)[fine] <= (bound(K, mag) + 2.0 ** -126)[fine]).all()


def big(rows, K, seed, scale=1.0):
    """bf16 [rows, K] and its quantized values in float64, both on the GPU (the quantizers have tests of their own)."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = (torch.randn(rows, K, generator=g, device=DEV) * scale * torch.exp(torch.randn(K, generator=g, device=DEV))).to(torch.bfloat16)
    codes, scales = pq.alloc_quantized(MX, 32, rows, K)
    pq.pq_quantize_act(MX, 32, x, None, None, codes, scales)
    return x, codes, scales, pq.pq_dequantize(MX, 32, codes, scales).double()


def close_big(got, ref, err):
    assert bool((torch.isnan(got) == torch.isnan(ref)).all())
    worst = ((got.double() - ref).abs() / (err + 2.0 ** -8 * (ref.abs() + err) + 2.0 ** -133)).nan_to_num(0.0).max().item()
    assert worst <= 1.0, worst


# several tiles for every workgroup, with one to seven panels of 128 channels each: the loads of a tile begin in the one before it, or
# three before it; edges in both directions, rows that end inside eight columns
@pytest.mark.parametrize("M,N,K,tile", [(5757, 2618, 32, 128), (3153, 3068, 160, 128), (3018, 3480, 384, 128), (3179, 3592, 512, 128), (3955, 4469, 640, 128),
                                        (2650, 5944, 672, 128), (4063, 4060, 256, 256), (7352, 8877, 288, 256), (5692, 5624, 480, 256), (4999, 5733, 512, 256), (4522, 6360, 608, 256),
                                        (4423, 6544, 1184, 256), (45, 9001, 2080, 64), (150, 3001, 96, 32), (90, 2000, 512, 32), (333, 1000, 4128, 32),
                                        (1, 12345, 8192, 32), (200, 4099, 8192, 32), (200, 4090, 8192, 64), (700, 905, 1056, 64), (64, 12288, 96, 64), (61, 9002, 32, 64)])
@pytest.mark.parametrize("bias", [False, True])
def test_product_of_many_tiles(M, N, K, tile, bias):
    assert pq.pq_qgemm_tile(MX, 32, M, N, K)[0] == tile
    x, _, _, xq = big(M, K, 1)
    _, codes, scales, wq = big(N, K, 2, 0.02)
    b = torch.randn(N, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).to(torch.bfloat16)
    a, w = operand(x), pq.pq_pack_operand(MX, 32, codes, scales)
    ldy = (N + 7) // 8 * 8 + 8
    y = torch.full((M + 1, ldy), 5.0, dtype=torch.bfloat16, device=DEV)
    if bias:
        pq.pq_qgemm_packed_bias(MX, 32, a, None, w, None, b, y[:M], M, N, K)
    else:
        pq.pq_qgemm_packed(MX, 32, a, None, w, None, y[:M], M, N, K)
    ref, mag = xq @ wq.T, xq.abs() @ wq.T.abs()
    if bias:
        ref, mag = ref + b.double(), mag + b.double().abs()
    close_big(y[:M, :N], ref, (K / 64 + 8) * 2.0 ** -23 * mag)
    assert bool((y[M:] == 5).all()) and bool((y[:, N:] == 5).all())


def test_product_repeats_its_bits():
    rng = np.random.default_rng(1)
    for M, N, K in ((3, 700, 4096), (70, 900, 2048), (700, 900, 1024)):
        a, b = operand(rows_of(rng, M, K)), operand(rows_of(rng, N, K))
        y = [torch.empty(M, (N + 7) // 8 * 8, device=DEV) for _ in range(3)]
        for t in y:
            pq.pq_qgemm_packed_f32(MX, 32, a, None, b, None, t, M, N, K)
        assert torch.equal(y[0][:, :N], y[1][:, :N]) and torch.equal(y[0][:, :N], y[2][:, :N])


# ------------------------------------------------------------------------ products by expert

def experts_case(rng, sizes, a_rows, N, K, gather, bias, first=0, behind=0):
    E, M = len(sizes), first + sum(sizes) + behind
    x, w = rows_of(rng, a_rows, K), rows_of(rng, E * N, K)
    xq, wq = mx.dequantize(mx.quantize(f64(x))), mx.dequantize(mx.quantize(f64(w)))
    rows = rng.integers(0, a_rows, M).astype(np.int32) if gather else None
    b = rng.standard_normal((E, N)) if bias else np.zeros((E, N))
    b = OF.bf16_bits_to_f64(OF.f64_to_bf16_bits_rne(b))
    offsets = first + np.concatenate([[0], np.cumsum(sizes)])
    ref, err = np.full((M, N), 5.0), np.zeros((M, N))
    for e in range(E):
        for i in range(offsets[e], offsets[e + 1]):
            r = rows[i] if gather else i
            part = wq[e * N:(e + 1) * N]
            ref[i] = part @ xq[r] + b[e]
            err[i] = bound(K, np.abs(part) @ np.abs(xq[r]) + np.abs(b[e]))
    t = lambda v: None if v is None else torch.from_numpy(np.ascontiguousarray(v)).to(DEV)
    codes, scales = stored(mx.quantize(f64(w)))
    return dict(a=operand(x), w=pq.pack_experts(codes, scales, E), offsets=t(offsets.astype(np.int32)), rows=t(rows),
                bias=pq.bf16_from_bits(OF.f64_to_bf16_bits_rne(b), DEV) if bias else None, ref=ref, err=err, M=M)


def grouped(c, a_rows, N, K, **kw):
    y = torch.full((c["M"], (N + 7) // 8 * 8 + 8), 5.0, dtype=torch.bfloat16, device=DEV)
    pq.pq_qgemm_grouped(MX, 32, c["a"], a_rows, c["w"], c["offsets"], y[:, :N], N, K, rows=kw.get("rows", c["rows"]), bias=c["bias"])
    assert bool((y[:, N:] == 5).all())
    return y[:, :N]


@pytest.mark.parametrize("sizes,a_rows,N,K,gather,bias", [
    ([1], 1, 8, 32, True, False), ([0, 0, 3, 0], 5, 40, 288, True, True), ([5, 1, 0, 33, 2], 41, 72, 512, False, True),
    ([1] * 70, 9, 33, 96, True, True), ([0] * 130 + [17] + [0] * 65, 17, 64, 256, False, False), ([64, 0, 128, 31, 200], 50, 260, 544, True, True),
    ([300, 1, 257, 0, 512], 1100, 264, 320, False, False), ([700, 30], 300, 520, 1056, True, True), ([3, 4, 2, 7, 0, 1, 5, 2], 8, 1000, 2016, True, False),
    ([20] * 40, 200, 136, 640, True, True)])
def test_grouped(sizes, a_rows, N, K, gather, bias):
    rng = np.random.default_rng(len(sizes) + a_rows + N)
    c = experts_case(rng, sizes, a_rows, N, K, gather, bias, first=0 if gather is False else 2, behind=0 if gather is False else 3)
    close(grouped(c, a_rows, N, K), c["ref"], c["err"])


# experts of all lengths by every kernel: few and many panels, an index or none, more experts than the kernels keep a table of
@pytest.mark.parametrize("E,M,a_rows,N,K,gather,bias,few_experts", [
    (64, 9000, 1500, 2056, 640, True, True, 0), (64, 9000, 1500, 2056, 544, True, False, 0), (64, 9000, 1500, 2050, 512, True, True, 0), (64, 9000, 1500, 2056, 96, True, True, 0),
    (8, 30000, 30000, 1288, 704, False, True, 0), (8, 30000, 7000, 1288, 672, True, True, 0), (8, 30000, 7000, 1285, 256, True, False, 0), (8, 40000, 9000, 2056, 1152, True, True, 3),
    (300, 2400, 300, 520, 1056, True, True, 0), (300, 2400, 300, 515, 160, True, False, 0), (100, 4500, 500, 1032, 576, True, True, 0), (100, 4500, 4500, 1032, 320, False, True, 9),
    (1500, 3000, 400, 264, 288, True, True, 0), (1100, 60000, 4000, 512, 640, True, False, 0), (1100, 60000, 60000, 512, 128, False, True, 0), (3, 90, 40, 1000, 2080, True, True, 0),
    (4, 300, 90, 1000, 2080, True, True, 0), (8, 200, 200, 1502, 2080, False, True, 0), (4, 200, 50, 2500, 672, True, True, 0), (4, 200, 200, 2501, 672, False, False, 2),
    (8, 100, 30, 2001, 96, True, False, 0)])
def test_grouped_of_all_lengths(E, M, a_rows, N, K, gather, bias, few_experts):
    rng = np.random.default_rng(E + M + K)
    share = np.exp(rng.standard_normal(E))
    share[rng.random(E) < 0.2] = 0.0
    if few_experts:
        share[rng.permutation(E)[:E - few_experts]] = 0.0                 # all rows go to a few of them
    sizes = np.floor(share / share.sum() * (M - 5)).astype(np.int64)      # the last rows are nobody's
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    x, _, _, xq = big(a_rows, K, 1)
    _, codes, scales, wq = big(E * N, K, 2, 0.02)
    b = torch.randn(E, N, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).to(torch.bfloat16)
    rows = torch.from_numpy(rng.integers(0, a_rows, M).astype(np.int32)).to(DEV) if gather else None
    if gather:
        rows[7::97] = -1
        rows[11::101] = a_rows
    y = torch.full((M, (N + 7) // 8 * 8 + 8), 5.0, dtype=torch.bfloat16, device=DEV)
    pq.pq_qgemm_grouped(MX, 32, operand(x), a_rows, pq.pack_experts(codes, scales, E), torch.from_numpy(offsets.astype(np.int32)).to(DEV), y[:, :N], N, K,
                        rows=rows, bias=b if bias else None)
    assert bool((y[:, N:] == 5).all()) and bool((y[offsets[-1]:] == 5).all())
    for e in range(E):
        if sizes[e] == 0:
            continue
        at = slice(offsets[e], offsets[e + 1])
        index = rows[at].long() if gather else torch.arange(offsets[e], offsets[e + 1], device=DEV)
        known = (index >= 0) & (index < a_rows)
        part, aq = wq[e * N:(e + 1) * N], xq[index.clamp(0, a_rows - 1)]
        ref, mag = aq @ part.T, aq.abs() @ part.T.abs()
        if bias:
            ref, mag = ref + b[e].double(), mag + b[e].double().abs()
        ref, mag = torch.where(known[:, None], ref, 5.0), torch.where(known[:, None], mag, 0.0)
        close_big(y[at, :N], ref, (K / 64 + 8) * 2.0 ** -23 * mag)


def test_grouped_leaves_other_rows():
    rng = np.random.default_rng(3)
    a_rows, N, K = 20, 48, 288
    c = experts_case(rng, [4, 0, 40, 3], a_rows, N, K, True, True, first=1, behind=2)
    rows = c["rows"].clone()
    rows[6], rows[11], rows[44] = -1, a_rows, 1 << 30                     # unknown rows: left as they were
    ref = c["ref"].copy()
    ref[[6, 11, 44]] = 5.0
    err = c["err"].copy()
    err[[6, 11, 44]] = 0.0
    close(grouped(c, a_rows, N, K, rows=rows), ref, err)
    # offsets beyond M and below 0 are cut
    c["offsets"] = torch.tensor([-7, 5, 5, 45, 1 << 30], dtype=torch.int32, device=DEV)
    y = grouped(c, a_rows, N, K)
    close(y[1:48], c["ref"][1:48], c["err"][1:48])
    assert not bool((y[0] == 5).all()) and not bool((y[48:] == 5).all())
    # nothing at all
    c["offsets"] = torch.full((5,), 9, dtype=torch.int32, device=DEV)
    assert bool((grouped(c, a_rows, N, K) == 5).all())
    c["M"] = 0
    c["rows"] = c["rows"][:0]
    assert grouped(c, a_rows, N, K).numel() == 0


@pytest.mark.parametrize("E,M,N,K", [(4, 48, 48, 288), (70, 700, 264, 640), (70, 20, 40, 96), (1100, 5000, 264, 288)])
def test_grouped_of_offsets_that_go_up_and_down(E, M, N, K):
    # rows in them may be computed or not, others are not touched
    x, _, _, _ = big(M, K, 1)
    _, codes, scales, _ = big(E * N, K, 2)
    offsets = torch.tensor(([0, M - 1] * E)[:E + 1], dtype=torch.int32, device=DEV)
    y = torch.full((M + 1, (N + 7) // 8 * 8 + 8), 5.0, dtype=torch.bfloat16, device=DEV)
    pq.pq_qgemm_grouped(MX, 32, operand(x), M, pq.pack_experts(codes, scales, E), offsets, y[:M, :N], N, K)
    assert bool((y[M - 1:] == 5).all()) and bool((y[:, N:] == 5).all())


def test_grouped_of_one_expert_is_the_product():
    rng = np.random.default_rng(4)
    for M, N, K in ((3, 100, 512), (90, 300, 800), (520, 520, 256)):
        x, w = rows_of(rng, M, K), rows_of(rng, N, K)
        a, b = operand(x), operand(w)
        y, z = (torch.empty(M, (N + 7) // 8 * 8, dtype=torch.bfloat16, device=DEV)[:, :N] for _ in range(2))
        pq.pq_qgemm_packed(MX, 32, a, None, b, None, y, M, N, K)
        pq.pq_qgemm_grouped(MX, 32, a, M, b[None], torch.tensor([0, M], dtype=torch.int32, device=DEV), z, N, K)
        ref = mx.dequantize(mx.quantize(f64(x))) @ mx.dequantize(mx.quantize(f64(w))).T
        mag = np.abs(mx.dequantize(mx.quantize(f64(x)))) @ np.abs(mx.dequantize(mx.quantize(f64(w)))).T
        close(y, ref, bound(K, mag))
        close(z, ref, bound(K, mag))


# ------------------------------------------------------------------------ routing, weighted sum

def check_route(r, want, exact_weights=False):
    for name in ("ids", "offsets", "rows", "positions"):
        assert np.array_equal(getattr(r, name).cpu().numpy(), getattr(want, name)), name
    assert np.abs(r.weights.cpu().double().numpy() - want.weights).max(initial=0.0) <= 1e-5


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 6), (5, 3, 3), (7, 65, 8), (64, 16, 2), (65, 128, 4), (200, 300, 10), (130, 1024, 32), (90, 100, 20), (64, 256, 16), (1000, 256, 8)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("renormalize", [True, False])
def test_route(T, E, k, dtype, renormalize):
    rng = np.random.default_rng(T + E)
    x = rng.standard_normal((T, E)) * 2
    x[rng.random((T, E)) < 0.1] = -np.inf
    x[rng.random((T, E)) < 0.02] = np.nan
    x[rng.random(T) < 0.1] = -np.inf                                      # padding
    x[rng.random(T) < 0.1, :min(E, 7)] = 3.0                              # ties
    wide = torch.full((T, E + 5), 1e30, dtype=dtype, device=DEV)
    wide[:, 3:3 + E] = torch.from_numpy(x).to(dtype)
    logits = wide[:, 3:3 + E]
    r = pq.alloc_route(T, E, k)
    for t in r:
        t.fill_(77)
    pq.pq_moe_route(logits, k, renormalize, out=r)
    check_route(r, mx.route(logits.double().cpu().numpy(), k, renormalize))
    # again, and from rows that may be read in wider pieces: contiguous ones, and those of rows behind which other values stand
    aligned = torch.full((T, E + 8 + (-E) % 8), 1e30, dtype=dtype, device=DEV)
    aligned[:, :E] = logits
    for other in (logits, logits.contiguous(), aligned[:, :E]):
        assert all(torch.equal(a, b) for a, b in zip(r, pq.pq_moe_route(other, k, renormalize)))


def test_route_no_tokens_and_no_choices():
    r = pq.pq_moe_route(torch.empty(0, 9, device=DEV), 2)
    assert r.offsets.tolist() == [0] * 10 and r.rows.numel() == 0
    r = pq.pq_moe_route(torch.full((70, 9), -float("inf"), device=DEV), 2)
    assert r.offsets.tolist() == [0] * 10 and bool((r.rows == -1).all()) and bool((r.ids == -1).all()) and bool((r.weights == 0).all())
    big = torch.zeros(3, 4, device=DEV)
    big[:, 1] = 3e38
    big[:, 2] = -3e38
    r = pq.pq_moe_route(big, 4)
    assert r.ids.tolist() == [[1, 0, 3, 2]] * 3 and r.weights.tolist() == [[1.0, 0.0, 0.0, 0.0]] * 3


@pytest.mark.parametrize("T,E,k", [(33000, 8, 2), (70001, 33, 3), (1025, 1000, 7), (4099, 200, 12), (9000, 600, 20), (16385, 64, 4), (33, 256, 8), (9, 1024, 4), (17, 500, 32)])
def test_route_of_many_tokens(T, E, k):
    # more tokens than one pass of all workgroups
    x = torch.randn(T, E, generator=torch.Generator(device=DEV).manual_seed(T), device=DEV)
    r = pq.pq_moe_route(x, k)
    ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(r.ids.long(), ids)
    order = torch.argsort(ids.reshape(-1), stable=True)
    assert torch.equal(r.rows.long(), order // k)
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device=DEV)
    assert torch.equal(r.positions.long().reshape(-1), place)
    assert torch.equal(r.offsets.long()[1:], torch.bincount(ids.reshape(-1), minlength=E).cumsum(0))


@pytest.mark.parametrize("T,k,N", [(1, 1, 1), (3, 2, 8), (7, 4, 13), (50, 8, 264), (33, 32, 100), (4, 3, 5000)])
@pytest.mark.parametrize("addend", [False, True])
def test_combine(T, k, N, addend):
    rng = np.random.default_rng(T * k + N)
    R = T * k + 2
    bf = lambda a: pq.bf16_from_bits(OF.f64_to_bf16_bits_rne(a), DEV)
    y = rng.standard_normal((R, N + 9))
    y[R - 1] = np.nan                                                     # no token's
    y = bf(y)
    ld = (N + 7) // 8 * 8 + 8
    wide = torch.full((R, ld), 9.0, dtype=torch.bfloat16, device=DEV)
    wide[:, :N] = y[:, :N]
    pos = rng.integers(-1, R - 1, (T, k)).astype(np.int32)                # the same row twice among them
    pos[rng.random((T, k)) < 0.1] = R + 3
    pos[0] = -1
    weights = rng.standard_normal((T, k)).astype(np.float32)
    add = torch.full((T, ld), 4.0, dtype=torch.bfloat16, device=DEV)
    add[:, :N] = bf(rng.standard_normal((T, N)))
    out = torch.full((T + 1, ld), 6.0, dtype=torch.bfloat16, device=DEV)
    args = (wide[:, :N], torch.from_numpy(pos).to(DEV), torch.from_numpy(weights).to(DEV), add[:, :N] if addend else None)
    pq.pq_moe_combine(*args, out=out[:T, :N])
    ref, mag = mx.combine(f64(wide[:, :N]), pos, weights, f64(add[:, :N]) if addend else None)
    close(out[:T, :N], ref, (k + 1) * 2.0 ** -24 * mag)
    assert bool((out[T:] == 6).all()) and bool((out[:, N:] == 6).all())
    assert torch.equal(pq.pq_moe_combine(*args), out[:T, :N])
    if addend:                                                            # on top of the addend itself
        pq.pq_moe_combine(*args, out=add[:, :N])
        assert torch.equal(add[:, :N], out[:T, :N]) and bool((add[:, N:] == 4).all())


# ------------------------------------------------------------------------ what lies more than 2^32 bytes from where it begins

def test_far_rows_of_quantizers_and_products():
    M, N, K = 1 << 20, 2304, 2304                              # x and y 4.8 GB
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([0, 5, M // 2 + 77, M - 130, M - 1], device=DEV)
    x[at] = torch.randn(len(at), K, generator=g, device=DEV).to(torch.bfloat16)
    codes, scales = pq.alloc_quantized(MX, 32, M, K)
    pq.pq_quantize_act(MX, 32, x, None, None, codes, scales)
    few, few_scales = pq.alloc_quantized(MX, 32, len(at), K)
    pq.pq_quantize_act(MX, 32, x[at], None, None, few, few_scales)
    assert torch.equal(codes[at], few) and torch.equal(scales[at], few_scales) and int((scales != 0).sum()) == few_scales.count_nonzero()
    xq = pq.pq_dequantize(MX, 32, few, few_scales).double()
    y = pq.pq_dequantize(MX, 32, codes, scales)
    assert torch.equal(y[at].double(), xq) and int(y.count_nonzero()) == xq.count_nonzero()
    _, wc, ws, wq = big(N, K, 2, 0.02)
    a = operand(x)
    del x
    pq.pq_qgemm_packed(MX, 32, a, None, pq.pq_pack_operand(MX, 32, wc, ws), None, y, M, N, K)
    close_big(y[at], xq @ wq.T, (K / 64 + 8) * 2.0 ** -23 * (xq.abs() @ wq.T.abs()))
    other = torch.ones(M, dtype=torch.bool, device=DEV)
    other[at] = False
    assert not y[other].any()


def test_far_experts_rows_and_tokens():
    # weights of 150 experts 4.9 GB, tokens' operand 4.6 GB; then rows 5 GB
    E, N, K, a_rows = 150, 15360, 4096, 2200000
    g = torch.Generator(device=DEV).manual_seed(2)
    w = torch.zeros(E, pq.pq_operand_bytes(MX, 32, N, K), dtype=torch.uint8, device=DEV)
    _, wc, ws, wq = big(N, K, 3, 0.02)
    w[E - 1] = pq.pq_pack_operand(MX, 32, wc, ws)
    x = torch.zeros(a_rows, K, dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([a_rows - 1, 3, a_rows - 200, a_rows // 2 + 1], dtype=torch.int32, device=DEV)
    x[at.long()] = torch.randn(len(at), K, generator=g, device=DEV).to(torch.bfloat16)
    a = operand(x)
    few, few_scales = pq.alloc_quantized(MX, 32, len(at), K)
    pq.pq_quantize_act(MX, 32, x[at.long()], None, None, few, few_scales)
    xq = pq.pq_dequantize(MX, 32, few, few_scales).double()
    del x
    offsets = torch.full((E + 1,), 0, dtype=torch.int32, device=DEV)
    for M in (len(at), 300):                                   # small tiles, large ones
        offsets[E] = M
        index = at.repeat((M + len(at) - 1) // len(at))[:M].contiguous()
        y = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
        pq.pq_qgemm_grouped(MX, 32, a, a_rows, w, offsets, y, N, K, rows=index)
        ref, mag = xq @ wq.T, xq.abs() @ wq.T.abs()
        for i in range(0, M, len(at)):
            n = min(len(at), M - i)
            close_big(y[i:i + n], ref[:n], ((K / 64 + 8) * 2.0 ** -23 * mag)[:n])
    del a, w
    rows, tokens, width = 2500000, 2400000, 1024
    z = torch.zeros(rows, width, dtype=torch.bfloat16, device=DEV)
    z[-2:] = torch.randn(2, width, generator=g, device=DEV).to(torch.bfloat16)
    positions = torch.full((tokens, 2), -1, dtype=torch.int32, device=DEV)
    positions[-1] = torch.tensor([rows - 1, rows - 2], dtype=torch.int32)
    weights = torch.full((tokens, 2), 0.5, device=DEV)
    out = pq.pq_moe_combine(z, positions, weights)
    assert torch.equal(out[-1], (0.5 * z[-1].float() + 0.5 * z[-2].float()).to(torch.bfloat16)) and not out[:-1].any()


def test_far_logits():
    T, E = 1200000, 1024                                       # 4.9 GB
    x = torch.zeros(T, E, device=DEV)
    x[torch.arange(T, device=DEV), torch.arange(T, device=DEV) % E] = 1.0
    r = pq.pq_moe_route(x, 1)
    assert torch.equal(r.ids[:, 0], (torch.arange(T, device=DEV) % E).int())
    assert torch.equal(r.rows.long(), torch.arange(T, device=DEV).reshape(-1)[torch.argsort(r.ids[:, 0], stable=True)])


# ------------------------------------------------------------------------ together

class Layer:
    """A layer of experts as a program holds it: two products an expert, the rows weighted and summed on top of the input."""

    def __init__(self, rng, T, D, H, E, k):
        self.k, self.D, self.H, self.E, self.T = k, D, H, E, T
        self.w1, self.w2, self.router = rows_of(rng, E * H, D, odd=False), rows_of(rng, E * D, H, odd=False), rows_of(rng, E, D, odd=False)
        pack = lambda w: pq.pack_experts(*stored(mx.quantize(f64(w))), E)
        self.p1, self.p2 = pack(self.w1), pack(self.w2)
        self.route = pq.alloc_route(T, E, k)
        self.ws = pq.pq_moe_route_workspace(T, E, k)
        self.a1 = torch.empty(pq.pq_operand_bytes(MX, 32, T, D), dtype=torch.uint8, device=DEV)
        self.a2 = torch.empty(pq.pq_operand_bytes(MX, 32, T * k, H), dtype=torch.uint8, device=DEV)
        self.h, self.z = (torch.zeros(T * k, n, dtype=torch.bfloat16, device=DEV) for n in (H, D))
        self.out = torch.empty(T, D, dtype=torch.bfloat16, device=DEV)

    def __call__(self, x, logits):
        r = pq.pq_moe_route(logits, self.k, out=self.route, workspace=self.ws)
        pq.pq_quantize_act_packed(MX, 32, x, None, self.a1)
        pq.pq_qgemm_grouped(MX, 32, self.a1, self.T, self.p1, r.offsets, self.h, self.H, self.D, rows=r.rows)
        pq.pq_quantize_act_packed(MX, 32, torch.relu(self.h), None, self.a2)
        pq.pq_qgemm_grouped(MX, 32, self.a2, self.T * self.k, self.p2, r.offsets, self.z, self.D, self.H)
        return pq.pq_moe_combine(self.z, r.positions, r.weights, x, self.out)

    def check(self, x, logits):
        """Step by step, each step's input as the step before left it."""
        want = mx.route(logits.double().cpu().numpy(), self.k, True)
        check_route(self.route, want)
        value = lambda t: mx.dequantize(mx.quantize(f64(t)))
        total = want.offsets[-1]
        for a, w, y, n, rows in ((value(x), value(self.w1), self.h, self.H, want.rows), (value(torch.relu(self.h)), value(self.w2), self.z, self.D, np.arange(self.T * self.k))):
            for e in range(self.E):
                at = slice(want.offsets[e], want.offsets[e + 1])
                part, rr = w[e * n:(e + 1) * n], rows[at]
                close(y[at.start:at.stop], a[rr] @ part.T, bound(a.shape[1], np.abs(a[rr]) @ np.abs(part).T))
        ref, mag = mx.combine(f64(self.z), want.positions, self.route.weights.cpu().numpy(), f64(x))
        close(self.out, ref, (self.k + 1) * 2.0 ** -24 * mag)
        return total


@pytest.mark.parametrize("T,D,H,E,k", [(1, 64, 96, 8, 2), (40, 288, 160, 6, 3), (300, 512, 544, 16, 4)])
def test_layer_of_experts(T, D, H, E, k):
    rng = np.random.default_rng(T)
    layer = Layer(rng, T, D, H, E, k)
    x = rows_of(rng, T, D, odd=False)
    logits = torch.from_numpy(rng.standard_normal((T, E))).float().to(DEV)
    logits[T // 2 + 1:T // 2 + 3] = -float("inf")                          # padding
    layer(x, logits)
    layer.check(x, logits)


def test_layer_in_graphs_and_streams():
    rng = np.random.default_rng(8)
    T, D, H, E, k = 30, 256, 288, 8, 2
    layers = [Layer(rng, T, D, H, E, k) for _ in range(2)]
    inputs = [(rows_of(rng, T, D, odd=False), torch.from_numpy(rng.standard_normal((T, E))).float().to(DEV)) for _ in range(4)]
    x, logits = inputs[0][0].clone(), inputs[0][1].clone()
    for layer in layers:
        layer(x, logits)
    torch.cuda.synchronize()
    graphs = []
    for layer in layers:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            layer(x, logits)
        graphs.append(g)
    for new_x, new_logits in inputs[1:]:
        x.copy_(new_x)
        logits.copy_(new_logits)
        for layer, g in zip(layers, graphs):
            g.replay()
            torch.cuda.synchronize()
            layer.check(x, logits)
            got = layer.out.clone()
            assert torch.equal(layer(x, logits), got)                     # eager work between the replays
    streams = [torch.cuda.Stream() for _ in layers]
    want = [layer.out.clone() for layer in layers]
    for layer in layers:
        layer.out.zero_()
    torch.cuda.synchronize()
    for layer, st in zip(layers, streams):
        with torch.cuda.stream(st):
            for _ in range(5):
                layer(x, logits)
    torch.cuda.synchronize()
    for layer, w in zip(layers, want):
        assert torch.equal(layer.out, w)


# ------------------------------------------------------------------------ every kernel of the products by expert

def by_expert(sizes, a_rows, N, K, gather, bias, first=0, behind=3):
    """One call and its check against float64: experts of these sizes, rows in front of and behind theirs that are nobody's."""
    E, M = len(sizes), first + int(sum(sizes)) + behind
    offsets = first + np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    x, _, _, xq = big(a_rows, K, 1)
    _, codes, scales, wq = big(E * N, K, 2, 0.02)
    g = torch.Generator(device=DEV).manual_seed(3)
    b = torch.randn(E, N, generator=g, device=DEV).to(torch.bfloat16) if bias else None
    rows = torch.randint(0, a_rows, (M,), generator=g, device=DEV, dtype=torch.int32) if gather else None
    if gather:
        rows[7::97] = -1
        rows[11::101] = a_rows
    y = torch.full((M, (N + 7) // 8 * 8 + 8), 5.0, dtype=torch.bfloat16, device=DEV)
    pq.pq_qgemm_grouped(MX, 32, operand(x), a_rows, pq.pack_experts(codes, scales, E), torch.from_numpy(offsets.astype(np.int32)).to(DEV), y[:, :N], N, K,
                        rows=rows, bias=b)
    assert bool((y[:, N:] == 5).all()) and bool((y[:first] == 5).all()) and bool((y[offsets[-1]:] == 5).all())
    for e in range(E):
        if sizes[e] == 0:
            continue
        at = slice(offsets[e], offsets[e + 1])
        index = rows[at].long() if gather else torch.arange(offsets[e], offsets[e + 1], device=DEV)
        known = ((index >= 0) & (index < a_rows))[:, None]
        part, aq = wq[e * N:(e + 1) * N], xq[index.clamp(0, a_rows - 1)]
        ref, mag = aq @ part.T, aq.abs() @ part.T.abs()
        if bias:
            ref, mag = ref + b[e].double(), mag + b[e].double().abs()
        close_big(y[at, :N], torch.where(known, ref, 5.0), (K / 64 + 8) * 2.0 ** -23 * torch.where(known, mag, 0.0))


# the table of experts in LDS: its last word stands behind lanes that are all taken, behind idle ones, and at the table's end; tiles of 128 rows, of
# 256, and waves with tiles of 32 and 64 rows
@pytest.mark.parametrize("E,each,N,K", [(1, 5500, 264, 2048), (63, 100, 1032, 2048), (64, 100, 1032, 2048), (65, 100, 1032, 2048), (127, 100, 1032, 2048), (129, 100, 1032, 2048),
                                        (3, 2000, 2048, 2048), (65, 1000, 2048, 2048),
                                        (63, 20, 1032, 64), (65, 20, 1032, 64), (1000, 5, 264, 512), (1023, 5, 264, 512), (1024, 5, 264, 512),
                                        (63, 64, 1032, 512), (129, 70, 1032, 512), (1000, 64, 520, 256)])
@pytest.mark.parametrize("last", ["full", "empty"])
def test_grouped_last_expert(E, each, N, K, last):
    sizes = [each] * E
    if last == "empty":
        sizes[-1] = 0
    by_expert(sizes, 3000, N, K, True, True, first=1)


def skewed(E, total, seed):
    """Sizes of E experts, uneven, some of them empty; all of total."""
    rng = np.random.default_rng(seed)
    share = np.exp(rng.standard_normal(E))
    if E > 2:
        share[rng.random(E) < 0.2] = 0.0
        share[rng.integers(E)] = 1.0
    sizes = np.floor(share / share.sum() * total).astype(np.int64)
    sizes[np.argmax(sizes)] += total - sizes.sum()
    return sizes


# each kernel by expert, the large tiles with one to four panels (their index and bias are read as they are needed) and more (loaded ahead), with whole
# pieces of eight columns and without, and with more experts than the kernels keep a table of
BY_EXPERT = [(66, 2330, 261, 32, 128, 128), (66, 2330, 264, 64, 128, 128), (8, 3300, 261, 160, 128, 128), (8, 3300, 264, 160, 128, 128), (3, 3300, 261, 384, 128, 128),
             (3, 3300, 264, 384, 128, 128), (11, 3150, 261, 512, 128, 128), (8, 16384, 4096, 512, 128, 128), (66, 2300, 261, 640, 128, 128), (66, 2300, 264, 640, 128, 128),
             (1030, 185000, 264, 2048, 128, 128), (1030, 176000, 261, 2048, 128, 128),
             (2, 5300, 2816, 512, 256, 256), (8, 40000, 2816, 512, 256, 256), (2, 5200, 6003, 512, 256, 256), (2, 3000, 4096, 640, 256, 256), (3, 6000, 2048, 1152, 256, 256),
             (20, 30000, 2045, 1152, 256, 256), (1030, 3200000, 256, 512, 256, 256), (1030, 840000, 256, 1024, 256, 256),
             (63, 1300, 1029, 96, 32, 128), (1100, 5000, 261, 640, 32, 128), (63, 5000, 1029, 512, 64, 128), (1030, 200000, 520, 256, 64, 128),
             (8, 400, 1032, 64, 64, 64), (8, 300, 1032, 64, 32, 64), (8, 300, 261, 2048, 32, 32)]


@pytest.mark.parametrize("E,M,N,K,tile_m,tile_n,gather,bias", [c + f for c in BY_EXPERT for f in ((True, True), (True, False), (False, True), (False, False))
                                                               if c[1] < 100000 or f[0] == f[1]])
def test_grouped_by_every_kernel(E, M, N, K, tile_m, tile_n, gather, bias):
    assert pq.pq_qgemm_grouped_tile(MX, 32, E, M, N, K) == (tile_m, tile_n)
    first = 5
    by_expert(skewed(E, M - first - 3, E + K), 1500 if gather else M, N, K, gather, bias, first=first)


# ------------------------------------------------------------------------ the large tiles: sums, values that are not finite, repeated and captured calls

LARGE = [(2100, 1029, 32, 128), (2100, 1029, 384, 128), (1700, 1030, 640, 128), (1777, 4008, 2016, 128), (4063, 4060, 256, 256), (4423, 6541, 1184, 256)]


@pytest.mark.parametrize("M,N,K,tile", LARGE)
def test_sums_of_large_tiles(M, N, K, tile):
    assert pq.pq_qgemm_tile(MX, 32, M, N, K) == (tile, tile)
    x, _, _, xq = big(M, K, 1)
    _, codes, scales, wq = big(N, K, 2, 0.02)
    ldy = (N + 7) // 8 * 8 + 8
    y = torch.full((M + 1, ldy), 5.0, device=DEV)
    pq.pq_qgemm_packed_f32(MX, 32, operand(x), None, pq.pq_pack_operand(MX, 32, codes, scales), None, y[:M], M, N, K)
    off = (y[:M, :N].double() - xq @ wq.T).abs()
    assert bool((off <= (K / 64 + 8) * 2.0 ** -23 * (xq.abs() @ wq.T.abs()) + 2.0 ** -133).all())
    assert bool((y[M:] == 5).all()) and bool((y[:, N:] == 5).all())


def odd_values(x, w):
    """Puts values that are not finite, the largest and the smallest scales into some rows of x and of w."""
    M, K = x.shape
    x[0] *= 2.0 ** -100
    x[M // 2] *= 2.0 ** 60
    x[3, 5] = float("inf")
    x[M - 1, K - 1] = float("nan")
    x[M // 3, :32] = -float("inf")
    x[7] = 0.0
    w[1] *= 2.0 ** -100
    w[w.shape[0] - 1, K - 2] = float("nan")
    w[2] *= 2.0 ** 50


def quantized(t):
    codes, scales = pq.alloc_quantized(MX, 32, *t.shape)
    pq.pq_quantize_act(MX, 32, t, None, None, codes, scales)
    return codes, scales, pq.pq_dequantize(MX, 32, codes, scales).double()


@pytest.mark.parametrize("M,N,K,tile", LARGE)
@pytest.mark.parametrize("f32", [False, True])
def test_values_not_finite_in_large_tiles(M, N, K, tile, f32):
    # a group with one of them makes its row or its column NaN and nothing else; scales from far below to far above 1 beside it
    x, w = big(M, K, 1)[0], big(N, K, 2, 0.02)[0]
    odd_values(x, w)
    (_, _, xq), (codes, scales, wq) = quantized(x), quantized(w)
    ref, mag = xq @ wq.T, xq.abs() @ wq.T.abs()
    assert int(torch.isnan(ref).all(dim=1).sum()) == 3 and int(torch.isnan(ref).all(dim=0).sum()) == 1
    y = torch.empty(M, (N + 7) // 8 * 8, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV)
    assert pq.pq_qgemm_tile(MX, 32, M, N, K) == (tile, tile)
    (pq.pq_qgemm_packed_f32 if f32 else pq.pq_qgemm_packed)(MX, 32, operand(x), None, pq.pq_pack_operand(MX, 32, codes, scales), None, y, M, N, K)
    got = y[:, :N].double()
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    # a sum below what binary32 holds whole may be cut to zero at every step
    allowed = (K / 64 + 8) * 2.0 ** -23 * mag * (1 + 2.0 ** -8) + (0 if f32 else 2.0 ** -8) * ref.abs() + (K / 64 + 8) * 2.0 ** -126
    assert bool(((got - ref).abs() <= allowed)[~torch.isnan(ref)].all())


@pytest.mark.parametrize("E,M,N,K,tile_m,tile_n", [c for c in BY_EXPERT if c[1] < 10000])
def test_grouped_values_not_finite(E, M, N, K, tile_m, tile_n):
    assert pq.pq_qgemm_grouped_tile(MX, 32, E, M, N, K) == (tile_m, tile_n)
    a_rows = 700
    x, w = big(a_rows, K, 1)[0], big(E * N, K, 2, 0.02)[0]
    odd_values(x, w)
    (_, _, xq), (codes, scales, wq) = quantized(x), quantized(w)
    sizes = skewed(E, M, E + K)
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    rows = torch.randint(0, a_rows, (M,), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV, dtype=torch.int32)
    y = torch.full((M, (N + 7) // 8 * 8), 5.0, dtype=torch.bfloat16, device=DEV)
    pq.pq_qgemm_grouped(MX, 32, operand(x), a_rows, pq.pack_experts(codes, scales, E), torch.from_numpy(offsets.astype(np.int32)).to(DEV), y[:, :N], N, K, rows=rows)
    for e in np.nonzero(sizes)[0]:
        at = slice(offsets[e], offsets[e + 1])
        part, aq = wq[e * N:(e + 1) * N], xq[rows[at].long()]
        ref, mag, got = aq @ part.T, aq.abs() @ part.T.abs(), y[at, :N].double()
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        allowed = (K / 64 + 8) * 2.0 ** -23 * mag * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs() + (K / 64 + 8) * 2.0 ** -126
        assert bool(((got - ref).abs() <= allowed)[~torch.isnan(ref)].all())


def test_large_products_repeat_their_bits_and_replay():
    # every kernel, dense and by expert: call after call, captured into graphs that are replayed with other inputs, eager calls between them
    calls = []
    for M, N, K, tile in LARGE:
        w = pq.pq_pack_operand(MX, 32, *big(N, K, 2, 0.02)[1:3])
        x = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
        a, y = operand(x), torch.zeros(M, (N + 7) // 8 * 8, dtype=torch.bfloat16, device=DEV)

        def dense(x=x, a=a, w=w, y=y, M=M, N=N, K=K):
            pq.pq_quantize_act_packed(MX, 32, x, None, a)
            pq.pq_qgemm_packed(MX, 32, a, None, w, None, y, M, N, K)
        calls.append((dense, x, y[:, :N]))
    for E, M, N, K, tile_m, tile_n in [c for c in BY_EXPERT if c[1] < 7000]:
        w = pq.pack_experts(*big(E * N, K, 2, 0.02)[1:3], E)
        x = torch.zeros(900, K, dtype=torch.bfloat16, device=DEV)
        a, y = operand(x), torch.zeros(M, (N + 7) // 8 * 8, dtype=torch.bfloat16, device=DEV)
        offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(skewed(E, M, E + K))]).astype(np.int32)).to(DEV)
        rows = torch.randint(0, 900, (M,), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV, dtype=torch.int32)

        def by(x=x, a=a, w=w, y=y, N=N, K=K, offsets=offsets, rows=rows):
            pq.pq_quantize_act_packed(MX, 32, x, None, a)
            pq.pq_qgemm_grouped(MX, 32, a, 900, w, offsets, y[:, :N], N, K, rows=rows)
        calls.append((by, x, y[:, :N]))
    for call, x, y in calls:
        call()                                                 # before a capture: what a kernel's first launch sets
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        for seed in range(3):
            x.copy_(big(*x.shape, 10 + seed)[0])
            call()
            want = y.clone()
            for _ in range(2):
                y.fill_(4.0)
                call()
                assert torch.equal(y, want)
                y.fill_(6.0)
                g.replay()
                torch.cuda.synchronize()
                assert torch.equal(y, want)


# ------------------------------------------------------------------------ routing's weights, relative to themselves

def routed(x, k, renormalize):
    """What pq_moe_route leaves for logits x, by sorting and float64; with each choice's logit less the largest."""
    T, E = x.shape
    v = x.double()
    v = torch.where(torch.isnan(v), -float("inf"), v)
    value, ids = torch.sort(v, dim=1, descending=True, stable=True)
    value, ids = value[:, :k], torch.where(value[:, :k] == -float("inf"), -1, ids[:, :k])
    top = torch.where(value[:, :1] == -float("inf"), 0.0, value[:, :1])
    total = torch.exp((value if renormalize else v) - top).sum(dim=1, keepdim=True)
    weights = torch.where(ids >= 0, torch.exp(value - top) / total, 0.0)
    chosen = (ids.reshape(-1) >= 0).nonzero()[:, 0]
    order = chosen[torch.argsort(ids.reshape(-1)[chosen], stable=True)]
    rows, positions = torch.full((T * k,), -1, device=DEV), torch.full((T * k,), -1, device=DEV)
    rows[:len(order)] = order // k
    positions[order] = torch.arange(len(order), device=DEV)
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=DEV)
    offsets[1:] = torch.bincount(ids.reshape(-1)[chosen], minlength=E).cumsum(0)
    return ids, weights, offsets, rows, positions.reshape(T, k), torch.where(ids >= 0, value - top, 0.0)


# One launch and two, one step of a workgroup's tokens and several, sixteen lanes a token and a wave; few and many experts a lane.
# Units of 2^-24 of a weight: the difference of two logits is rounded (|x|), e^x is off by at most two; of the sum's terms every one by the difference and
# the product with log2 e (2.3 |x| of it with the constant's own rounding; over all terms 2.3 ln E at most, the entropy's bound) and by two, its at most
# 15 + 6 additions by one each; the quotient by one.
@pytest.mark.parametrize("T,E,k", [(1, 8, 2), (7, 64, 6), (64, 64, 8), (33, 256, 8), (16, 1024, 4), (17, 1024, 8), (300, 60, 4), (1000, 256, 8), (2500, 300, 20), (16385, 64, 4),
                                   (20000, 130, 12), (33000, 256, 8), (9000, 600, 20), (9001, 1000, 7), (70001, 33, 3)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("spread", [0.3, 6.0])
def test_route_weights(T, E, k, dtype, renormalize, spread):
    g = torch.Generator(device=DEV).manual_seed(T + E)
    x = (torch.randn(T, E, generator=g, device=DEV) * spread).to(dtype)
    odd = torch.rand(T, E, generator=g, device=DEV)
    x[odd < 0.05] = -float("inf")
    x[odd > 0.98] = float("nan")
    x[torch.rand(T, generator=g, device=DEV) < 0.02] = -float("inf")
    r = pq.pq_moe_route(x, k, renormalize)
    ids, weights, offsets, rows, positions, below = routed(x, k, renormalize)
    for got, want in ((r.ids, ids), (r.offsets, offsets), (r.rows, rows), (r.positions, positions)):
        assert torch.equal(got.long(), want.long())
    allowed = (below.abs() + 2.3 * float(np.log(E)) + 27) * 2.0 ** -24 * weights + 2.0 ** -126
    assert bool(((r.weights.double() - weights).abs() <= allowed).all())


# ------------------------------------------------------------------------ every value under every scale; reading back the other formats

def test_every_bf16_value_under_every_scale():
    # every finite value beside a largest one that sets the scale, for each scale under which it is not itself larger
    for byte in range(253):
        largest = (byte + 2) << 7                                          # 2^(byte - 125)
        magnitudes = np.arange(largest + 128, dtype=np.uint16)             # those up to the next power of two set the same scale
        values = np.concatenate([magnitudes, magnitudes | 0x8000])
        b = np.full((-(-len(values) // 31), 32), largest, dtype=np.uint16)
        b[:, :31] = np.resize(values, (len(b), 31))
        t = pq.bf16_from_bits(b, DEV)
        codes, scales = pq.alloc_quantized(MX, 32, *t.shape)
        pq.pq_quantize_act(MX, 32, t, None, None, codes, scales)
        want = mx.quantize(OF.bf16_bits_to_f64(b))
        assert bool((want.scale == byte).all()) and bool((scales == byte).all()), byte
        assert np.array_equal(codes.cpu().numpy(), mx.packed_codes(want)), byte


def test_every_code_under_every_scale():
    code = np.tile(np.arange(16, dtype=np.uint8), (256, 2))
    q = mx.MxQuant(code, np.arange(256, dtype=np.uint8)[:, None])
    want = mx.dequantize(q)
    held = ~(np.abs(want) >= 2.0 ** 128)                                   # bf16 has no larger ones; NaN among them
    got = f64(pq.pq_dequantize(MX, 32, *stored(q)))
    assert np.array_equal(got[held], want[held], equal_nan=True)


@pytest.mark.parametrize("rows,K,gap", [(1, 256, 0), (19, 768, 8), (65, 5376, 0), (300, 512, 16)])
@pytest.mark.parametrize("fmt,group", [(pq.FMT_NVFP4, 16)] + [(f, g) for f in (pq.FMT_INT4, pq.FMT_INT3) for g in (32, 64, 128, 256)])
def test_dequantize_all_formats(fmt, group, rows, K, gap):
    rng = np.random.default_rng(rows + K)
    x = rows_of(rng, rows, K)
    ts = torch.full((1,), float(np.float32(np.abs(f64(x)).max() / 2688)), device=DEV)
    codes, scales = pq.alloc_quantized(fmt, group, rows, K)
    pq.pq_quantize_act(fmt, group, x, None, ts, codes, scales)
    q = OQ.quantize(fmt, group, f64(x), np.float32(ts.item()))
    want = OF.f64_to_bf16_bits_rne(OF.fl32(OQ.dequantize(fmt, group, q)))
    wide = torch.full((rows + 1, K + 2 * gap), 3.0, dtype=torch.bfloat16, device=DEV)
    pq.pq_dequantize(fmt, group, codes, scales, ts, y=wide[:rows, gap:gap + K])
    got = bits(wide[:rows, gap:gap + K])
    assert np.array_equal(np.where(got == 0x8000, 0, got), np.where(want == 0x8000, 0, want))       # a zero has no sign in the oracle
    assert bool((wide[rows:] == 3).all()) and bool((wide[:, :gap] == 3).all()) and bool((wide[:, gap + K:] == 3).all())

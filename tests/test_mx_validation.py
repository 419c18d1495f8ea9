"""Refusals of the MXFP4 and routing entry points: every check is the host's, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2605_09503_amd import pq
from test_kv_python_binding import python  # noqa: F401
from test_abi import FAKE, PQ_ERR_FORMAT, PQ_ERR_NULL, PQ_ERR_SHAPE, PQ_ERR_WORKSPACE, lib  # noqa: F401

ODD = C.c_void_p(0x1008)
ODD2 = C.c_void_p(0x1002)
MX = pq.FMT_MXFP4


def test_operand_bytes(lib):  # noqa: F811
    f = pq.pq_operand_bytes
    assert f(MX, 32, 64, 128) == 64 * (64 + 4)
    assert f(MX, 32, 64, 160) == 2 * 64 * (64 + 4)                # panels of 128 channels
    assert f(MX, 32, 3, 32) == 256 + 256                          # 192 and 12 bytes, each to a multiple of 256
    assert f(MX, 32, 1 << 24, 1 << 24) == (1 << 17) * (1 << 24) * 68
    for bad in [(MX, 16, 64, 256), (MX, 64, 64, 256), (MX, 32, 0, 256), (MX, 32, 64, 0), (MX, 32, 64, 48), (MX, 32, (1 << 24) + 1, 32),
                (MX, 32, 1, (1 << 24) + 32), (5, 32, 64, 256)]:
        assert f(*bad) == 0, bad


def test_quantizers(lib):  # noqa: F811
    qa = lambda fmt=MX, g=32, x=FAKE, M=4, K=64, ld=64, perm=None, codes=FAKE, s=FAKE: lib.pq_quantize_act(fmt, g, x, M, K, ld, perm, None, codes, s, None)
    assert qa(x=None) == qa(codes=None) == qa(s=None) == PQ_ERR_NULL
    assert qa(g=16) == qa(g=64) == qa(fmt=5) == PQ_ERR_FORMAT
    assert qa(K=48, ld=48) == qa(K=0) == qa(M=0) == qa(ld=56) == qa(ld=68) == qa(x=ODD) == qa(codes=ODD) == qa(s=ODD) == qa(perm=ODD) == PQ_ERR_SHAPE
    assert qa(M=1 << 40, K=1 << 12, ld=1 << 12) == qa(M=1 << 62) == qa(M=1 << 60, K=1 << 58, ld=1 << 58) == PQ_ERR_SHAPE
    qp = lambda g=32, x=FAKE, M=4, K=64, ld=64, op=FAKE, size=1 << 20, codes=None, s=None: lib.pq_quantize_act_packed(MX, g, x, M, K, ld, None, op, size, codes, s, None)
    assert qp(x=None) == qp(op=None) == qp(codes=FAKE) == qp(s=FAKE) == PQ_ERR_NULL
    assert qp(g=16) == PQ_ERR_FORMAT
    assert qp(M=0) == qp(K=48, ld=48) == qp(ld=60) == qp(op=ODD) == qp(M=(1 << 24) + 1) == PQ_ERR_SHAPE
    assert qp(size=pq.pq_operand_bytes(MX, 32, 4, 64) - 1) == PQ_ERR_WORKSPACE
    pk = lambda g=32, codes=FAKE, s=FAKE, rows=4, K=64, op=FAKE, size=1 << 20: lib.pq_pack_operand(MX, g, codes, s, rows, K, op, size, None)
    assert pk(codes=None) == pk(s=None) == pk(op=None) == PQ_ERR_NULL
    assert pk(g=48) == PQ_ERR_FORMAT
    assert pk(rows=0) == pk(K=48) == pk(codes=ODD) == pk(s=ODD) == PQ_ERR_SHAPE
    assert pk(size=100) == PQ_ERR_WORKSPACE
    qw = lambda g=32, w=FAKE, N=4, K=64, codes=FAKE, s=FAKE, ts=FAKE, perm=None: lib.pq_quantize_weights(MX, g, w, N, K, perm, codes, s, ts, None)
    assert qw(w=None) == qw(ts=None) == PQ_ERR_NULL and qw(g=16) == PQ_ERR_FORMAT and qw(N=0) == qw(K=33) == qw(w=ODD) == qw(perm=ODD) == PQ_ERR_SHAPE


def test_products(lib):  # noqa: F811
    g = lambda fmt=MX, gr=32, a=FAKE, w=FAKE, M=8, N=8, K=64, y=FAKE, ldy=8: lib.pq_qgemm_packed(fmt, gr, a, None, w, None, M, N, K, y, ldy, None)
    assert g(a=None) == g(w=None) == g(y=None) == PQ_ERR_NULL
    assert g(gr=16) == PQ_ERR_FORMAT
    assert g(M=0) == g(N=0) == g(K=48) == g(ldy=4) == g(ldy=12) == g(a=ODD) == g(y=ODD) == g(M=(1 << 24) + 1) == PQ_ERR_SHAPE
    assert g(M=1 << 24, N=1 << 24, ldy=1 << 24) == g(ldy=(1 << 24) + 8) == PQ_ERR_SHAPE      # more tiles than a launch has
    assert lib.pq_qgemm_packed_bias(MX, 32, FAKE, None, FAKE, None, 8, 8, 64, None, FAKE, 8, None) == PQ_ERR_NULL
    assert lib.pq_qgemm_packed_f32(MX, 32, FAKE, None, FAKE, None, 8, 8, 64, FAKE, 4, None) == PQ_ERR_SHAPE


def test_tile(lib):  # noqa: F811
    assert pq.pq_qgemm_tile(MX, 32, 1, 4096, 4096) == (32, 32)
    assert pq.pq_qgemm_tile(MX, 32, 16, 12288, 8192) == (32, 64)
    assert pq.pq_qgemm_tile(MX, 32, 60, 12288, 4096) == (64, 64)
    assert pq.pq_qgemm_tile(MX, 32, 2000, 4096, 2048) == (128, 128)
    assert pq.pq_qgemm_tile(MX, 32, 8192, 12288, 8192) == (256, 256)
    for bad in [(MX, 16, 8, 8, 64), (MX, 32, 0, 8, 64), (MX, 32, 8, 8, 48)]:
        with pytest.raises(pq.PQError):
            pq.pq_qgemm_tile(*bad)


def test_calls_that_do_not_offer_it(lib):  # noqa: F811
    assert lib.pq_qgemm(MX, 32, FAKE, FAKE, None, FAKE, FAKE, None, 8, 8, 64, FAKE, 8, FAKE, 1 << 20, None) == PQ_ERR_FORMAT
    assert "MXFP4" in pq.pq_last_error()
    assert lib.pq_hadamard_quantize_act_packed(None, MX, 32, FAKE, 8, 64, 64, None, FAKE, 1 << 20, None, 0, None) == PQ_ERR_FORMAT
    p = pq.NormParams(0, None, None, None, None, 0, 1e-6)
    assert lib.pq_norm_quantize_act_packed(C.byref(p), MX, 32, FAKE, 8, 64, 64, None, FAKE, 1 << 20, None, 0, None) == PQ_ERR_FORMAT
    assert lib.pq_quant_error(MX, 32, FAKE, 8, 64, None, 1.0, FAKE, FAKE, 1 << 20, None) == PQ_ERR_FORMAT
    assert pq.pq_kv_cache_bytes(MX, 32, 8, 128, 64, 1) == 0


def test_dequantize(lib):  # noqa: F811
    f = lambda fmt=MX, g=32, codes=FAKE, s=FAKE, ts=None, rows=4, K=64, y=FAKE, ldy=64: lib.pq_dequantize(fmt, g, codes, s, ts, rows, K, y, ldy, None)
    assert f(codes=None) == f(s=None) == f(y=None) == f(fmt=pq.FMT_NVFP4, g=16) == PQ_ERR_NULL
    assert f(g=16) == f(fmt=pq.FMT_INT4, g=16) == f(fmt=pq.FMT_BF16, g=0) == PQ_ERR_FORMAT
    assert f(rows=0) == f(K=48) == f(ldy=56) == f(ldy=68) == f(y=ODD) == f(codes=ODD) == f(rows=(1 << 24) + 1) == PQ_ERR_SHAPE


def test_grouped(lib):  # noqa: F811
    def g(fmt=MX, gr=32, a=FAKE, a_rows=8, w=FAKE, experts=4, off=FAKE, rows=FAKE, M=16, N=8, K=64, bias=None, y=FAKE, ldy=8):
        return lib.pq_qgemm_grouped(fmt, gr, a, a_rows, w, experts, off, rows, M, N, K, bias, y, ldy, None)
    assert g(a=None) == g(w=None) == g(off=None) == g(y=None) == PQ_ERR_NULL
    assert g(fmt=pq.FMT_INT4) == g(fmt=pq.FMT_NVFP4, gr=16) == g(gr=64) == PQ_ERR_FORMAT
    assert g(experts=0) == g(experts=65537) == g(M=-1) == g(a_rows=-1) == g(N=0) == g(K=48) == g(ldy=12) == g(ldy=0) == PQ_ERR_SHAPE
    assert g(a=ODD) == g(w=ODD) == g(y=ODD) == g(bias=ODD) == g(off=ODD2) == g(rows=ODD2) == PQ_ERR_SHAPE
    assert g(rows=None) == PQ_ERR_SHAPE                                              # 8 rows cannot make 16 in order
    assert g(M=1 << 24, N=1 << 24, ldy=1 << 24) == g(ldy=(1 << 24) + 8) == PQ_ERR_SHAPE
    assert g(M=0) == 0 and g(a_rows=0) == 0 and g(M=0, a=None, y=None) == 0          # nothing to do, nothing launched


def test_route(lib):  # noqa: F811
    assert pq.pq_moe_route_workspace_bytes(0, 4, 2) > 0
    need = [pq.pq_moe_route_workspace_bytes(t, 257, 8) for t in (0, 1, 64, 65, 4000, 32768, 32769, 70000, 1 << 24)]
    assert need == sorted(need) and need[-1] >= 512 * 257 * 2           # one for more tokens serves fewer
    for bad in [(-1, 4, 2), (4, 0, 1), (4, 1025, 2), (4, 4, 0), (4, 4, 5), (4, 64, 33), ((1 << 24) + 1, 4, 2)]:
        assert pq.pq_moe_route_workspace_bytes(*bad) == 0
        with pytest.raises(pq.PQError):
            pq.pq_moe_route_workspace(*bad, device="cpu")

    def r(type=0, x=FAKE, T=4, E=8, ld=8, k=2, ids=FAKE, w=FAKE, off=FAKE, rows=FAKE, pos=FAKE, ws=FAKE, size=1 << 20):
        return lib.pq_moe_route(type, x, T, E, ld, k, 1, ids, w, off, rows, pos, ws, size, None)
    assert r(type=2) == PQ_ERR_FORMAT
    assert r(x=None) == r(ids=None) == r(w=None) == r(off=None) == r(rows=None) == r(pos=None) == PQ_ERR_NULL
    assert r(T=-1) == r(E=0) == r(E=1025, ld=1025) == r(k=0) == r(k=9) == r(ld=7) == r(x=ODD2) == r(ids=ODD2) == r(ws=ODD) == PQ_ERR_SHAPE
    assert r(ws=None) == r(size=16) == PQ_ERR_WORKSPACE


def test_combine(lib):  # noqa: F811
    def f(y=FAKE, rows=8, yl=64, pos=FAKE, w=FAKE, T=4, k=2, N=60, add=None, al=0, out=FAKE, ol=64):
        return lib.pq_moe_combine(y, rows, yl, pos, w, T, k, N, add, al, out, ol, None)
    assert f(y=None) == f(pos=None) == f(w=None) == f(out=None) == PQ_ERR_NULL
    assert f(T=-1) == f(rows=-1) == f(k=0) == f(k=33) == f(N=0) == f(yl=56) == f(yl=60) == f(ol=56) == f(add=FAKE, al=56) == PQ_ERR_SHAPE
    assert f(y=ODD) == f(out=ODD) == f(add=ODD, al=64) == f(pos=ODD2) == f(w=ODD2) == PQ_ERR_SHAPE
    assert f(T=0) == 0 and f(T=0, y=None, out=None) == 0


@pytest.mark.parametrize("native", [True, False])
def test_python_arguments(lib, python, native):  # noqa: F811
    # the native calls, and the functions of pq.py that stand in for them; tensors in host memory never reach a kernel
    m = pq if native else python
    z = lambda *shape, dtype=torch.uint8: torch.zeros(shape, dtype=dtype)
    need = pq.pq_operand_bytes(MX, 32, 8, 64)
    y, off = z(4, 8, dtype=torch.bfloat16), z(3, dtype=torch.int32)

    def refused(call, match=None):
        with pytest.raises(Exception, match=match) as e:
            call()
        assert type(e.value).__name__ == "PQError" and e.value.code == PQ_ERR_SHAPE

    for call in (lambda: m.pq_qgemm_grouped(MX, 32, z(need), 4, z(2, need), off, y, 8, 64),
                 lambda: m.pq_moe_route(z(4, 8, dtype=torch.float32), 2),
                 lambda: m.pq_dequantize(MX, 32, z(4, 32), z(4, 2)),
                 lambda: m.pq_moe_combine(y, z(2, 2, dtype=torch.int32), z(2, 2, dtype=torch.float32))):
        refused(call, "GPU")
    for call in (lambda: m.pq_qgemm_grouped(MX, 32, z(need), 4, z(2, need + 256), off, y, 8, 64),
                 lambda: m.pq_qgemm_grouped(MX, 32, z(need), 4, z(2 * need), off, y, 8, 64),
                 lambda: m.pq_qgemm_grouped(MX, 32, z(need), 4, z(2, need), off, y.float(), 8, 64),
                 lambda: m.pq_qgemm_grouped(MX, 32, z(need), 4, z(2, need), off, y[:, :4], 8, 64),
                 lambda: m.pq_moe_route(z(4, 8, dtype=torch.float64), 2),
                 lambda: m.pq_moe_route(z(8, dtype=torch.float32), 2),
                 lambda: m.pq_moe_route(z(8, 4, dtype=torch.float32).T, 2),
                 lambda: m.pq_moe_combine(y.float(), z(2, 2, dtype=torch.int32), z(2, 2, dtype=torch.float32)),
                 lambda: m.pq_moe_combine(y, z(2, dtype=torch.int32), z(2, 2, dtype=torch.float32)),
                 lambda: m.pq_dequantize(MX, 32, z(4, 32, dtype=torch.int8), z(4, 2)),
                 lambda: m.pq_dequantize(MX, 32, z(4 * 32), z(4, 2)),
                 lambda: m.pq_dequantize(MX, 32, z(4, 64)[:, :32], z(4, 2)),
                 lambda: m.pack_experts(z(9, 32), z(9, 2), 4),
                 lambda: m.pack_experts(z(8, 32), z(8, 4), 4),
                 lambda: m.pack_experts(z(8, 32), z(8, 2), 4)):
        refused(call)


@pytest.mark.parametrize("name", ["pq_dequantize", "pq_qgemm_grouped", "pq_moe_route", "pq_moe_combine"])
def test_native_and_python_signatures(lib, python, name):  # noqa: F811
    import inspect
    native = getattr(pq, name)
    assert inspect.isbuiltin(native)
    want = inspect.signature(getattr(python, name))
    got = inspect.signature(native)
    assert [(p.name, p.default) for p in got.parameters.values()] == [(p.name, p.default) for p in want.parameters.values()]


def test_weights_too_large_are_refused_before_a_launch(lib):  # noqa: F811
    qw = lambda N, K: lib.pq_quantize_weights(MX, 32, FAKE, N, K, None, FAKE, FAKE, FAKE, None)
    assert qw(1 << 40, 1 << 12) == qw(1 << 62, 64) == qw(1 << 60, 1 << 58) == PQ_ERR_SHAPE


def test_grouped_tile(lib):  # noqa: F811
    f = lambda *a: pq.pq_qgemm_grouped_tile(MX, 32, *a)
    assert f(8, 16, 512, 2048) == (32, 32)
    assert f(8, 300, 1032, 64) == (32, 64)
    assert f(8, 400, 1032, 64) == (64, 64)
    assert f(128, 1536, 1536, 2560) == (32, 128)
    assert f(63, 5000, 1032, 512) == (64, 128)
    assert f(8, 4000, 264, 64) == (128, 128)
    assert f(64, 65528, 2816, 2048) == (256, 256)
    f = lambda fmt=MX, g=32, E=4, M=8, N=8, K=64: lib.pq_qgemm_grouped_tile(fmt, g, E, M, N, K, C.byref(C.c_int()), C.byref(C.c_int()))
    assert f() == 0
    assert lib.pq_qgemm_grouped_tile(MX, 32, 4, 8, 8, 64, None, C.byref(C.c_int())) == PQ_ERR_NULL
    assert f(fmt=pq.FMT_INT4) == f(g=16) == PQ_ERR_FORMAT
    assert f(E=0) == f(E=65537) == f(M=0) == f(M=(1 << 24) + 1) == f(N=0) == f(K=48) == f(K=0) == PQ_ERR_SHAPE


def test_calls_past_the_largest_grid(lib):  # noqa: F811
    c = lambda T, N: lib.pq_moe_combine(FAKE, 8, 1 << 24, FAKE, FAKE, T, 2, N, None, 0, FAKE, 1 << 24, None)
    assert c(1 << 24, 1025) == c((1 << 23) + 1, 4096) == c(1 << 11, 1 << 24) == PQ_ERR_SHAPE
    d = lambda rows, K: lib.pq_dequantize(MX, 32, FAKE, FAKE, None, rows, K, FAKE, 1 << 24, None)
    assert d(1 << 24, 1 << 13) == d(1 << 13, 1 << 24) == d(1 << 24, 1 << 24) == PQ_ERR_SHAPE
    qp = lambda M, K: lib.pq_quantize_act_packed(MX, 32, FAKE, M, K, K, None, FAKE, 1 << 60, None, None, None)
    assert qp(1 << 24, 1 << 13) == qp(1 << 13, 1 << 24) == PQ_ERR_SHAPE
    g = lambda E, M, N: lib.pq_qgemm_grouped(MX, 32, FAKE, 1 << 24, FAKE, E, FAKE, FAKE, M, N, 32, None, FAKE, 1 << 24, None)
    assert g(128, 512, 1 << 24) == g(1, 1 << 24, 1 << 24) == PQ_ERR_SHAPE
    assert lib.pq_qgemm_packed(MX, 32, FAKE, None, FAKE, None, 46340, 5931641, 32, FAKE, 1 << 24, None) == PQ_ERR_SHAPE

"""Refusals of the cache's entry points: every check is the host's, before anything is launched (no GPU needed)."""
import ast
import ctypes as C

import pytest
import torch

from paper_2605_09503_amd import pq
from test_abi import FAKE, PQ_ERR_FORMAT, PQ_ERR_NULL, PQ_ERR_SHAPE, PQ_ERR_WORKSPACE, lib  # noqa: F401

ODD = C.c_void_p(0x1008)


def test_cache_bytes(lib):  # noqa: F811
    f = pq.pq_kv_cache_bytes
    tokens = 8 * 64 * 10
    assert f(pq.FMT_NVFP4, 16, 8, 128, 64, 10) == tokens * 2 * (64 + 8)
    assert f(pq.FMT_INT4, 64, 8, 128, 64, 10) == tokens * 2 * (64 + 4)
    assert f(pq.FMT_INT4, 256, 8, 256, 64, 10) == tokens * 2 * (128 + 2)
    assert f(pq.FMT_BF16, 0, 8, 64, 64, 10) == tokens * 256
    assert f(pq.FMT_INT4, 32, 1, 64, 1024, (1 << 26) - 1) == ((1 << 26) - 1) * 1024 * 72
    for bad in [(pq.FMT_INT3, 32, 8, 128, 64, 1), (pq.FMT_NVFP4, 32, 8, 128, 64, 1), (pq.FMT_INT4, 16, 8, 128, 64, 1),
                (pq.FMT_INT4, 128, 8, 64, 64, 1), (pq.FMT_BF16, 16, 8, 64, 64, 1), (pq.FMT_INT4, 32, 0, 64, 64, 1),
                (pq.FMT_INT4, 32, 8, 96, 64, 1), (pq.FMT_INT4, 32, 8, 64, 48, 1), (pq.FMT_INT4, 32, 8, 64, 16, 1),
                (pq.FMT_INT4, 32, 8, 64, 2048, 1), (pq.FMT_INT4, 32, 8, 64, 64, 0), (pq.FMT_INT4, 32, 8, 64, 64, 1 << 31), (pq.FMT_INT4, 32, 1, 64, 1024, 1 << 26),
                (9, 32, 8, 64, 64, 1)]:
        assert f(*bad) == 0, bad
        assert "pq_kv_cache_bytes" in pq.pq_last_error()
        with pytest.raises(pq.PQError):
            pq.alloc_kv_cache(*bad, device="cpu")


def cache(**kw):
    a = dict(fmt=1, group=64, kv_heads=2, head_dim=128, page=64, pages=4, data=0x1000, k_tensor_scale=None, v_tensor_scale=None)
    a.update(kw)
    return C.byref(pq._KVCacheStruct(*a.values()))


def test_cache_argument(lib):  # noqa: F811
    calls = [lambda c: lib.pq_kv_write(c, FAKE, 256, 128, FAKE, 256, 128, FAKE, 1, None),
             lambda c: lib.pq_kv_read(c, FAKE, 1, FAKE, 256, 128, FAKE, 256, 128, None),
             lambda c: lib.pq_attn_decode(c, FAKE, 512, 128, FAKE, 4, FAKE, 1, 4, 64, 0, 1.0, FAKE, 512, 128, None, FAKE, 0, None)]
    for f in calls:
        assert f(None) == PQ_ERR_NULL
        assert f(cache(data=None)) == PQ_ERR_NULL
        assert f(cache(fmt=0, group=16)) == PQ_ERR_NULL                      # NVFP4 without tensor scales
        assert f(cache(fmt=0, group=16, k_tensor_scale=0x1000)) == PQ_ERR_NULL
        assert f(cache(fmt=2, group=32)) == PQ_ERR_FORMAT
        assert f(cache(group=48)) == PQ_ERR_FORMAT
        assert f(cache(group=256)) == PQ_ERR_SHAPE                           # longer than a head
        assert f(cache(head_dim=80)) == PQ_ERR_SHAPE
        assert f(cache(page=40)) == PQ_ERR_SHAPE
        assert f(cache(pages=0)) == PQ_ERR_SHAPE
        assert f(cache(kv_heads=-1)) == PQ_ERR_SHAPE
        assert f(cache(data=0x1004)) == PQ_ERR_SHAPE


def test_rows(lib):  # noqa: F811
    w = lambda k=FAKE, kl=256, kh=128, v=FAKE, vl=256, vh=128, s=FAKE, n=3: lib.pq_kv_write(cache(), k, kl, kh, v, vl, vh, s, n, None)
    r = lambda k=FAKE, kl=256, kh=128, v=FAKE, vl=256, vh=128, s=FAKE, n=3: lib.pq_kv_read(cache(), s, n, k, kl, kh, v, vl, vh, None)
    for f in (w, r):
        assert f(k=None) == PQ_ERR_NULL and f(v=None) == PQ_ERR_NULL and f(s=None) == PQ_ERR_NULL
        assert f(n=-1) == PQ_ERR_SHAPE and f(n=1 << 31) == PQ_ERR_SHAPE
        assert f(k=ODD) == PQ_ERR_SHAPE and f(v=ODD) == PQ_ERR_SHAPE
        assert f(kl=260) == PQ_ERR_SHAPE and f(vh=132) == PQ_ERR_SHAPE
        assert f(n=0) == 0 and f(n=0, k=None, v=None, s=None) == 0           # nothing to do, nothing launched
    assert r(kl=128) == PQ_ERR_SHAPE and r(vh=64) == PQ_ERR_SHAPE            # rows that overlap are not written
    assert "overlap" in pq.pq_last_error()


def test_attention(lib):  # noqa: F811
    def call(c=None, q=FAKE, ql=512, qh=128, table=FAKE, tl=4, lengths=FAKE, seqs=3, heads=4, top=200, window=0, scale=1.0, out=FAKE,
             ol=512, oh=128, lse=None, ws=FAKE, size=1 << 40):
        return lib.pq_attn_decode(c or cache(), q, ql, qh, table, tl, lengths, seqs, heads, top, window, scale, out, ol, oh, lse, ws, size, None)
    for name in ("q", "table", "lengths", "out"):
        assert call(**{name: None}) == PQ_ERR_NULL
    assert call(seqs=-1) == PQ_ERR_SHAPE and call(seqs=65536) == PQ_ERR_SHAPE
    assert call(heads=3) == PQ_ERR_SHAPE and call(heads=0) == PQ_ERR_SHAPE
    assert call(top=-1) == PQ_ERR_SHAPE and call(top=257) == PQ_ERR_SHAPE    # four pages of 64
    assert call(window=-1) == PQ_ERR_SHAPE
    assert call(scale=float("nan")) == PQ_ERR_SHAPE and call(scale=float("inf")) == PQ_ERR_SHAPE
    assert call(q=ODD) == PQ_ERR_SHAPE and call(out=ODD) == PQ_ERR_SHAPE and call(ql=500) == PQ_ERR_SHAPE
    assert call(ol=256) == PQ_ERR_SHAPE and call(oh=64) == PQ_ERR_SHAPE
    assert call(table=C.c_void_p(0x1002)) == PQ_ERR_SHAPE and call(lse=C.c_void_p(0x1002)) == PQ_ERR_SHAPE
    assert call(ws=None) == PQ_ERR_WORKSPACE and call(size=100) == PQ_ERR_WORKSPACE
    assert call(ws=ODD) == PQ_ERR_SHAPE
    assert call(seqs=0) == 0 and call(seqs=0, q=None, ws=None) == 0
    size = lambda *a: lib.pq_attn_decode_workspace_bytes(cache(), *a)
    assert size(3, 4, 200, 0) >= pq.ATTN_DECODE_ZERO_BYTES and size(0, 4, 0, 0) >= pq.ATTN_DECODE_ZERO_BYTES
    assert size(3, 3, 200, 0) == 0 and size(-1, 4, 200, 0) == 0 and size(3, 4, 200, -1) == 0
    assert lib.pq_attn_decode_workspace_bytes(None, 3, 4, 200, 0) == 0
    # a workspace for more serves for less
    for seqs in (1, 7, 300):
        for top in (1, 33, 5000, 100000):
            for window in (0, 100):
                assert size(seqs, 4, top, window) <= size(seqs + 1, 4, top + 1, 0)


def python_binding():
    """pq.py alone, as it serves where the native module is not built."""
    import importlib.util
    spec = importlib.util.spec_from_file_location("pq_python", pq.__file__)
    module = importlib.util.module_from_spec(spec)
    import sys
    sys.modules["pq_python"] = module
    spec.loader.exec_module(module)
    pq.load()
    module.load()                            # binds the native module, one a process, to this copy's helpers, and its calls here
    if pq._calls:
        pq._calls.bind(pq._raise, pq._new_operand, pq._new_workspace, pq._refuse, pq._new_attn_workspace)
    for name in ("pq_kv_write", "pq_kv_read", "pq_attn_decode"):
        with open(pq.__file__) as f:
            tree = ast.parse(f.read())
        f = next(n for n in tree.body if isinstance(n, ast.FunctionDef) and n.name == name)
        exec(compile(ast.Module([f], []), pq.__file__, "exec"), module.__dict__)
    return module


@pytest.mark.parametrize("native", [True, False])
def test_binding_refuses_other_tensors(lib, native):  # noqa: F811
    pq = globals()["pq"] if native else python_binding()
    c = pq.alloc_kv_cache(pq.FMT_INT4, 64, 2, 128, 64, 4, device="cpu")
    t = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    slots = torch.zeros(3, dtype=torch.int64)

    def refused(f, *a, **kw):
        with pytest.raises(pq.PQError) as e:
            f(*a, **kw)
        assert e.value.code == PQ_ERR_SHAPE
    for bad in (t.float(), t[:2], t[:, :1], t.transpose(1, 2), t[..., ::2], t[0], t.expand(3, 2, 128)[:, :, :64]):
        refused(pq.pq_kv_write, c, bad, t, slots)
        refused(pq.pq_kv_write, c, t, bad, slots)
        refused(pq.pq_kv_read, c, slots, bad, t)
        refused(pq.pq_kv_read, c, slots, t, bad)
    for bad in (slots.int(), slots[None], torch.zeros(6, dtype=torch.int64)[::2]):
        refused(pq.pq_kv_write, c, t, t, bad)
        refused(pq.pq_kv_read, c, bad)
    q, table, lengths = torch.zeros(3, 4, 128, dtype=torch.bfloat16), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    refused(pq.pq_attn_decode, c, q.half(), table, lengths, 200, 1.0, workspace=ws)
    refused(pq.pq_attn_decode, c, q[0], table, lengths, 200, 1.0, workspace=ws)
    refused(pq.pq_attn_decode, c, q[:, :3], table, lengths, 200, 1.0, workspace=ws)
    refused(pq.pq_attn_decode, c, q[..., :64], table, lengths, 200, 1.0, workspace=ws)
    refused(pq.pq_attn_decode, c, q, table.long(), lengths, 200, 1.0, workspace=ws)
    refused(pq.pq_attn_decode, c, q, table[:2], lengths, 200, 1.0, workspace=ws)
    refused(pq.pq_attn_decode, c, q, table, lengths, 257, 1.0, workspace=ws)
    refused(pq.pq_attn_decode, c, q, table[:, :3], lengths, 200, 1.0, workspace=ws)       # the view's columns count, not its stride
    refused(pq.pq_attn_decode, c, q, table, lengths.long(), 200, 1.0, workspace=ws)
    refused(pq.pq_attn_decode, c, q, table, lengths[:2], 200, 1.0, workspace=ws)
    refused(pq.pq_attn_decode, c, q, table, lengths, 200, 1.0, out=q[:, :2], workspace=ws)
    refused(pq.pq_attn_decode, c, q, table, lengths, 200, 1.0, lse=torch.zeros(3, 4, dtype=torch.float64), workspace=ws)
    refused(pq.pq_attn_decode, c, q, table, lengths, 200, 1.0, lse=torch.zeros(4, 3), workspace=ws)
    refused(pq.pq_attn_decode, c, q, table, lengths, 200, 1.0, workspace=ws)                # all fits, in host memory
    refused(pq.pq_kv_write, c, t, t, slots)
    refused(pq.pq_kv_read, c, slots)
    for kw in (dict(data=c.data[:100]), dict(data=c.data.view(torch.int8)), dict(fmt=0, group=16), dict(page=33), dict(fmt=2, group=32)):
        with pytest.raises(pq.PQError):
            pq.KVCache(**{**{f: getattr(c, f) for f in ("fmt", "group", "kv_heads", "head_dim", "page", "pages", "data")}, **kw})


@pytest.mark.parametrize("native", [True, False])
def test_binding_refuses_other_workspaces(lib, native):  # noqa: F811
    # a strided one would be written past its end, one in host memory from the GPU
    pq = globals()["pq"] if native else python_binding()
    c = pq.alloc_kv_cache(pq.FMT_INT4, 64, 2, 128, 64, 4, device="cpu")
    q, table, lengths = torch.zeros(3, 4, 128, dtype=torch.bfloat16), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for ws in (torch.zeros(1 << 21, dtype=torch.uint8)[::2], torch.zeros(1 << 20, dtype=torch.uint8, device="meta")):
        with pytest.raises(pq.PQError, match="workspace"):
            pq.pq_attn_decode(c, q, table, lengths, 200, 1.0, workspace=ws)


SIGNATURES = {
    "pq_kv_write": "(cache, k, v, slots)",
    "pq_kv_read": "(cache, slots, k=None, v=None)",
    "pq_attn_decode": "(cache, q, table, lengths, max_len, scale, out=None, lse=None, window=0, workspace=None)",
}


@pytest.mark.parametrize("name", sorted(SIGNATURES))
def test_native_and_python_signatures(lib, name):  # noqa: F811
    import inspect
    assert str(inspect.signature(getattr(pq, name))) == SIGNATURES[name]
    python = inspect.signature(getattr(python_binding(), name))
    assert [str(p.replace(annotation=p.empty)) for p in python.parameters.values()] == SIGNATURES[name][1:-1].split(", ")


def test_more_than_a_launch_takes(lib):  # noqa: F811
    # 2^24 workgroups of 256 threads are refused by name (the largest that are not go on to the next check)
    for heads, n in ((1, (1 << 29) - 32), (8, (1 << 26) - 32), (4095, 4097 * 32)):
        c = cache(kv_heads=heads)
        w = lambda n: lib.pq_kv_write(c, None, 256, 128, None, 256, 128, None, n, None)
        r = lambda n: lib.pq_kv_read(c, None, n, None, 256, 128, None, 256, 128, None)
        for f in (w, r):
            assert f(n) == PQ_ERR_NULL
            assert f(n + 1) == PQ_ERR_SHAPE and "2^24" in pq.pq_last_error()
    size = lambda kv, q, seqs=65535: lib.pq_attn_decode_workspace_bytes(cache(kv_heads=kv), seqs, q, 31, 0)
    assert size(256, 256) > 0 and size(1, 512) > 0
    assert size(257, 257) == 0 and "2^24" in pq.pq_last_error()
    assert size(129, 129 * 3, 65535) > 0 and size(300, 300, 60000) == 0


def test_rows_that_overlap(lib):  # noqa: F811
    # tokens of a head that overlap each other, however far apart the heads lie; heads outermost is a layout like another
    def read(ld, head, n=3, heads=2):
        return lib.pq_kv_read(cache(kv_heads=heads), FAKE, n, FAKE, ld, head, ODD, 4096, 512, None)      # v's address ends those that pass
    for bad in ((64, 1024), (0, 1024), (120, 4096)):
        assert read(*bad) == PQ_ERR_SHAPE and "rows of k overlap" in pq.pq_last_error(), bad
    for bad in ((64, 1024), (0, 1 << 20)):
        assert read(*bad, heads=1) == PQ_ERR_SHAPE and "rows of k overlap" in pq.pq_last_error(), bad
    for good in ((256, 128), (128, 384), (264, 136), (128, 1024)):
        assert read(*good) == PQ_ERR_SHAPE and "v must be 16-byte aligned" in pq.pq_last_error(), good
    assert read(128, 0, heads=1) == read(0, 128, n=1) == PQ_ERR_SHAPE and "v must be 16-byte aligned" in pq.pq_last_error()
    assert lib.pq_attn_decode(cache(), FAKE, 512, 128, FAKE, 4, FAKE, 3, 4, 200, 0, 1.0, FAKE, 64, 4096, None, FAKE, 1 << 40, None) == PQ_ERR_SHAPE
    assert "rows of out overlap" in pq.pq_last_error()


def test_what_is_no_cache(lib):  # noqa: F811
    # read as an address and not asked whether it is one, these ended the process
    import types
    t, i = torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    for address in ("no address", None, 0, 1.5):
        c = types.SimpleNamespace(_address=address, data=torch.zeros(1, dtype=torch.uint8))
        for f in (lambda: pq.pq_kv_write(c, t, t, i), lambda: pq.pq_kv_read(c, i),
                  lambda: pq.pq_attn_decode(c, t, i[None].int(), i.int(), 3, 1.0)):
            with pytest.raises((TypeError, AttributeError)):
                f()
    for c in (None, t):
        with pytest.raises(AttributeError):
            pq.pq_kv_write(c, t, t, i)

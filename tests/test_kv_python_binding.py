"""The cache's calls as pq.py serves them where the native module is not built or was built for another torch: the functions that
Python finds under their names, with the refusals of the native ones (no GPU needed, nothing is launched)."""
import ast
import collections
import importlib.machinery
import importlib.util
import sys
import types
import warnings

import pytest
import torch

from paper_2605_09503_amd import pq
from test_abi import PQ_ERR_SHAPE, lib  # noqa: F401


@pytest.fixture
def python(lib, monkeypatch):  # noqa: F811
    """pq.py as a module of its own for which the native one cannot be loaded."""
    def no_module(*_):
        raise ImportError("built for another torch")
    spec = importlib.util.spec_from_file_location("pq_without_native", pq.__file__)
    module = importlib.util.module_from_spec(spec)
    sys.modules[spec.name] = module
    try:
        with monkeypatch.context() as m, warnings.catch_warnings():
            warnings.simplefilter("ignore", RuntimeWarning)          # that the native binding cannot be used
            m.setattr(importlib.machinery, "ExtensionFileLoader", no_module)
            spec.loader.exec_module(module)
            module.load()
        for name in ("pq_kv_write", "pq_kv_read", "pq_attn_decode"):
            assert isinstance(getattr(module, name), types.FunctionType)
        yield module
    finally:
        del sys.modules[spec.name]


def test_every_name_is_defined_once():
    with open(pq.__file__) as f:
        tree = ast.parse(f.read())
    names = []
    for node in tree.body:
        if isinstance(node, (ast.FunctionDef, ast.ClassDef)):
            names.append(node.name)
        elif isinstance(node, ast.Assign):
            names += [n.id for t in node.targets for n in ast.walk(t) if isinstance(n, ast.Name)]
    declare = next(n for n in tree.body if isinstance(n, ast.FunctionDef) and n.name == "_declare")
    names += [ast.unparse(t) for n in declare.body if isinstance(n, ast.Assign) for t in n.targets]
    assert [name for name, count in collections.Counter(names).items() if count > 1] == []


def refused(f, *a, match=None, **kw):
    with pytest.raises(Exception, match=match) as e:
        f(*a, **kw)
    assert type(e.value).__name__ == "PQError" and e.value.code == PQ_ERR_SHAPE


def host_cache(m):
    return m.alloc_kv_cache(m.FMT_INT4, 64, 2, 128, 64, 4, device="cpu")


def test_host_memory_is_refused(python):
    c, t, slots = host_cache(python), torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    refused(python.pq_kv_write, c, t, t, slots, match="GPU memory")
    refused(python.pq_kv_read, c, slots, match="GPU memory")
    q, table = torch.zeros(3, 4, 128, dtype=torch.bfloat16), torch.zeros(3, 4, dtype=torch.int32)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    refused(python.pq_attn_decode, c, q, table, table[:, 0].contiguous(), 200, 1.0, workspace=ws, match="GPU memory")


def test_other_workspaces_are_refused(python):
    c, q, table = host_cache(python), torch.zeros(3, 4, 128, dtype=torch.bfloat16), torch.zeros(3, 4, dtype=torch.int32)
    lengths = torch.zeros(3, dtype=torch.int32)
    for ws in (torch.zeros(1 << 21, dtype=torch.uint8)[::2], torch.zeros(1, dtype=torch.uint8).expand(1 << 20),
               torch.zeros(1 << 20, dtype=torch.uint8, device="meta")):
        refused(python.pq_attn_decode, c, q, table, lengths, 200, 1.0, workspace=ws, match="workspace")


def test_other_tensors_are_refused(python):
    c, t, slots = host_cache(python), torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    for bad in (t.float(), t[:2], t[:, :1], t.transpose(1, 2), t[..., ::2], t[0]):
        refused(python.pq_kv_write, c, bad, t, slots)
        refused(python.pq_kv_write, c, t, bad, slots)
        refused(python.pq_kv_read, c, slots, bad, t)
        refused(python.pq_kv_read, c, slots, t, bad)
    q, table, lengths = torch.zeros(3, 4, 128, dtype=torch.bfloat16), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    for a in ((q.half(), table, lengths, 200), (q[0], table, lengths, 200), (q, table.long(), lengths, 200), (q, table[:2], lengths, 200),
              (q, table, lengths, 257), (q, table, lengths[:2], 200)):
        refused(python.pq_attn_decode, c, *a, 1.0, workspace=ws)
    refused(python.pq_attn_decode, c, q, table, lengths, 200, 1.0, lse=torch.zeros(4, 3), workspace=ws)
    refused(python.pq_attn_decode, c, q, table, lengths, 200, 1.0, out=q[:, :2], workspace=ws)

"""Calls whose buffers are not where, or not of the shape that, the kernels would take them for are refused before anything is
launched: a cache of another head_dim than the queries', outputs and workspaces of another device.

Without a GPU the tensors are fake ones, which claim a device and have no memory: a call that is not refused fails when it asks
for their addresses, with another error."""

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2503_05096_amd as pkg
from paper_2503_05096_amd import binding
from tests.test_fastcall_host import ENTRIES, ints, module  # noqa: F401  (fixture)
from tests.test_fastcall_pages import MORE, Stubs


def _int(*shape, dev="cuda"):
    return torch.zeros(shape, dtype=torch.int32, device=dev)


def _attn(d=64, out=None, ws=None, device="cuda", **kw):
    """verify_attn of heads of 64 channels on a cache of heads of d"""
    q, kv = torch.zeros((2, 2, 64), device=device), torch.zeros((3, 2, 16, d), device=device)
    return pkg.verify_attn(q, kv, kv, _int(1, 2), _int(1), _int(1), out, max_spec_len=1, workspace=ws, **kw)


FORMS = [dict(), dict(path="vector"), dict(window=8), dict(window=8, sinks=2, path="vector"), dict(window=8, plan="reuse")]
BAD = {
    "cache of smaller heads": (lambda **kw: _attn(d=32, ws=_ws(), **kw), AssertionError, None),
    "cache of larger heads": (lambda **kw: _attn(d=128, ws=_ws(), **kw), AssertionError, None),
    "out on the host": (lambda **kw: _attn(out=torch.zeros((2, 2, 64)), ws=_ws(), **kw), ValueError, "^out is on cpu"),
    "workspace on the host": (lambda **kw: _attn(ws=_ws("cpu"), **kw), ValueError, "^workspace= is on cpu"),
}
PAGES = {
    "remap": lambda: pkg.kv_remap(_int(1, 2), _int(3), _int(1), _int(1), _int(1), workspace=_ws("cpu")),
    "compact": lambda: pkg.kv_compact_pages(_int(1, 2), _int(3), workspace=_ws("cpu")),
}


def _ws(dev="cuda"):
    return torch.zeros(1 << 16, dtype=torch.uint8, device=dev)


@pytest.fixture
def fake(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 0)
    with FakeTensorMode():
        yield


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("what", BAD)
def test_refused_on_the_host(fake, what, form):
    f, error, message = BAD[what]
    with pytest.raises(error, match=message):
        f(**form)


@pytest.mark.parametrize("what", PAGES)
def test_pages_refused_on_the_host(fake, what):
    with pytest.raises(ValueError, match="^workspace= is on cpu"):
        PAGES[what]()


def test_any_workspace_of_another_device():
    for device in ("cuda:0", "cuda:1"):
        with pytest.raises(ValueError, match=f"cpu, the call's tensors are on {device}"):
            binding._workspace(256, torch.device(device), torch.zeros(256, dtype=torch.uint8), "pages")
    ws = torch.zeros(256, dtype=torch.uint8)
    assert binding._workspace(256, torch.device("cpu"), ws, "pages") is ws


def test_left_to_python(module):  # noqa: F811
    stubs = Stubs(module, ENTRIES + MORE)
    q, bt = torch.zeros((4, 2, 64), device="meta"), ints(1, 2)
    for d, out, ws in ((64, None, None), (32, None, None), (128, None, None), (64, torch.zeros((4, 2, 64)), None),
                       (64, None, torch.zeros(512, dtype=torch.uint8))):
        kv = torch.zeros((2, 2, 16, d), device="meta")
        stubs.calls.clear()
        a = module.verify_attn_window(q, kv, kv, bt, ints(1), ints(1), out, 3, 0.0, None, "run", ws, None, 8, 0)
        b = module.verify_attn(q, kv, kv, bt, ints(1), ints(1), out, 3, 0.0, None, "run", ws, None, None)
        good = d == 64 and out is None and ws is None
        assert ((a is NotImplemented), (b is NotImplemented)) == (not good, not good)
        assert stubs.calls == (["window", "attn"] if good else [])


@pytest.mark.gpu
@pytest.mark.parametrize("form", FORMS[:4], ids=str)
@pytest.mark.parametrize("what", BAD)
def test_refused_with_memory(what, form):
    f, error, message = BAD[what]
    with pytest.raises(error, match=message):
        f(**form)
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_pages_refused_with_memory():
    for f in PAGES.values():
        with pytest.raises(ValueError, match="^workspace= is on cpu"):
            f()
    torch.cuda.synchronize()

"""The native call path of windowed attention and of the cache's pages: against the Python one it stands in for, and, where no
GPU is needed, on a build of it that takes meta tensors, with functions of this file in the place of the library's."""
import ctypes as C
import types

import pytest
import torch

import paper_2503_05096_amd as pkg
from paper_2503_05096_amd import binding
from tests.test_fastcall_host import ENTRIES, ERR_DIM, ERR_HIP, OK, ints, module  # noqa: F401  (fixture)

NAMES = ("verify_attn_window", "kv_remap", "kv_compact_pages", "kv_copy_pages")
MORE = [("window_ws", C.c_size_t, 3), ("window", C.c_int, 13), ("remap_ws", C.c_size_t, 1), ("remap", C.c_int, 14),
        ("compact_ws", C.c_size_t, 1), ("compact", C.c_int, 12), ("copy_pages", C.c_int, 7)]


class Stubs:
    def __init__(self, module, entries):  # noqa: F811
        self.calls, self.status, self.keep = [], OK, []
        for name, res, n in entries:
            self.keep.append(C.CFUNCTYPE(res, *[C.c_void_p] * n)(
                (lambda *a: 512) if res is C.c_size_t else (lambda *a, name=name: self.calls.append(name) or self.status)))
        module.setup(tuple(C.cast(f, C.c_void_p).value for f in self.keep),
                     lambda nbytes, device, given, family: torch.empty(nbytes, dtype=torch.uint8, device=device), lambda dev: 0, lambda: 0,
                     binding.AdaspecError)


def every_call(module, **kw):  # noqa: F811
    q, kv, bt = torch.zeros((4, 2, 64), device="meta"), torch.zeros((2, 2, 16, 64), device="meta"), ints(1, 2)
    a = dict(out=None, table=bt, refs=ints(9), ctx=ints(1), window=100, moves=4, plan="run", src=ints(3))
    a.update(kw)
    return {"verify_attn_window": lambda: module.verify_attn_window(q, kv, kv, a["table"], a["ctx"], ints(1), a["out"], 3, 0.0, None, a["plan"], None, None,
                                                                    a["window"], 4),
            "kv_remap": lambda: module.kv_remap(a["table"], a["refs"], a["src"], a["ctx"], ints(3), a["window"], 0, 16, a["out"], *[None] * 6),
            "kv_compact_pages": lambda: module.kv_compact_pages(a["table"], a["refs"], a["moves"], 16, a["out"], *[None] * 7),
            "kv_copy_pages": lambda: module.kv_copy_pages(kv, kv, a["src"], ints(3), None)}


def test_statuses_of_the_library(module):  # noqa: F811
    stubs = Stubs(module, ENTRIES + MORE)
    for name, f in every_call(module).items():
        stubs.status = OK
        assert f() is not NotImplemented, name
        stubs.status = ERR_DIM
        assert f() is NotImplemented, name
        stubs.status = ERR_HIP
        stubs.calls.clear()
        with pytest.raises(binding.AdaspecError, match=f"^adaspec_{name}: ") as e:
            f()
        assert e.value.status == ERR_HIP and len(stubs.calls) == 1, name


def test_what_is_not_plain_is_left_to_python(module):  # noqa: F811
    stubs = Stubs(module, ENTRIES + MORE)
    cpu = torch.zeros((1, 2), dtype=torch.int32)
    refused = {"verify_attn_window": (dict(table=cpu), dict(ctx=ints(2)), dict(ctx=ints(1).long()), dict(window=1 << 31), dict(window=2.0),
                                      dict(plan="build"), dict(plan="reuse"), dict(out=torch.zeros((4, 2, 32), device="meta")),
                                      dict(out=torch.zeros((4, 2, 64), device="meta").half())),
               "kv_remap": (dict(table=cpu), dict(table=ints(1, 2).long()), dict(refs=ints(3, 3)), dict(ctx=ints(2)), dict(src=ints(2)),
                            dict(out=ints(2, 2)), dict(out=ints(3, 2).long()), dict(window=-(1 << 40))),
               "kv_compact_pages": (dict(table=cpu), dict(refs=ints(2, 2)), dict(moves=1 << 40), dict(out=ints(2, 2))),
               "kv_copy_pages": (dict(src=ints(2)), dict(src=ints(3).long()), dict(src=ints(3, 1)))}
    for name, kws in refused.items():
        for kw in kws:
            assert every_call(module, **kw)[name]() is NotImplemented, (name, kw)
    module.set_meta_index(1)                              # tensors of another device than the current one
    try:
        for name, f in every_call(module).items():
            assert f() is NotImplemented, name
    finally:
        module.set_meta_index(0)
    for n in NAMES:
        assert getattr(module, n)() is NotImplemented
    assert stubs.calls == []


def test_new_outputs_share_an_allocation_and_nothing_else(module):  # noqa: F811
    Stubs(module, ENTRIES + MORE)
    given = ints(9)
    for shape in ((1, 2), (0, 2), (1, 0), (70, 3)):
        table, lens = ints(*shape), ints(shape[0])
        remap = module.kv_remap(table, ints(9), ints(3), lens, ints(3), 0, 0, 16, None, given, *[None] * 5)
        compact = module.kv_compact_pages(table, given, 65, 16, None, None, None, None, None, None, None, None)
        assert remap[1] is given
        assert [tuple(t.shape) for t in remap] == [(3, shape[1]), (9,), (3,), (3,), (2,)]
        assert [tuple(t.shape) for t in compact] == [shape, (9,), (9,), (65,), (65,), (2,)]
        for out in (remap[:1] + remap[2:], compact):
            spans = sorted((t.storage_offset(), t.storage_offset() + t.numel()) for t in out if t.numel())
            assert all(a % 64 == 0 and t.is_contiguous() and t.dtype == torch.int32 for t in out for a in (t.storage_offset(),))
            assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
            assert spans[-1][1] * 4 <= out[-1].untyped_storage().nbytes()


def test_entry_points_that_are_not_there(module):  # noqa: F811
    """A library without them: the older calls work, these are left to Python."""
    stubs = Stubs(module, ENTRIES)
    for name, f in every_call(module).items():
        assert f() is NotImplemented, name
    assert stubs.calls == []
    with pytest.raises(ValueError, match="entry points"):
        Stubs(module, ENTRIES + MORE[:3])


@pytest.fixture
def python_only(monkeypatch):
    """call(f): f() with the native path switched off"""
    off = types.SimpleNamespace(**{n: lambda *a: NotImplemented for n in NAMES})

    def call(f):
        with monkeypatch.context() as m:
            m.setattr(binding, "_fast", off)
            return f()
    return call


@pytest.mark.gpu
def test_native_calls_equal_python_calls(python_only):
    gen = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn((7, 8, 128), generator=gen, device="cuda").bfloat16()
    k, v = (torch.randn((40, 2, 16, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    table = torch.randperm(40, generator=gen, device="cuda").to(torch.int32)[:36].view(3, 12).contiguous()
    dev = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")                         # noqa: E731
    ctx, spec, refs = dev(150, 33, 190), dev(2, 0, 1), torch.zeros(40, dtype=torch.int32, device="cuda")
    refs[table.reshape(-1).long()] = 1
    at = (q[:6].contiguous(), k, v, table, ctx, spec)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def copied(**kw):
        kp, vp = k.clone(), v.clone()
        pkg.kv_copy_pages(kp, vp, dev(3, -1, 4), dev(7, 8, 9), **kw)
        return kp, vp
    calls = {
        "window": lambda: pkg.verify_attn(*at, max_spec_len=2, window=50, sinks=4),
        "window f32 out": lambda: pkg.verify_attn(*at, max_spec_len=2, window=50, out_dtype=0, scale=0.1, workspace=ws),
        "window huge": lambda: pkg.verify_attn(*at, max_spec_len=2, window=1 << 40, sinks=1 << 50),
        "window out given": lambda: pkg.verify_attn(*at, torch.empty_like(at[0]), max_spec_len=2, window=50),
        "window stream": lambda: pkg.verify_attn(*at, max_spec_len=2, window=50, workspace=ws, stream=side),
        "remap": lambda: pkg.kv_remap(table, refs, dev(2, 0, -1, 2), ctx, dev(192, 160, 20, 190), window=60, sinks=4),
        "remap no window": lambda: pkg.kv_remap(table, refs, dev(2, 0), ctx, dev(192, 160), status=dev(0, 0), workspace=ws, stream=side),
        "compact": lambda: pkg.kv_compact_pages(table, refs),
        "compact some": lambda: pkg.kv_compact_pages(table, refs, max_moves=1, page_map=torch.empty_like(refs)),
        "copy": copied, "copy of layers": lambda: (pkg.kv_copy_pages(k[None].clone(), v[None].clone(), dev(1), dev(2)),)[1:],
    }
    for name, f in calls.items():
        a, b = f(), None
        torch.cuda.synchronize()
        b = python_only(f)
        torch.cuda.synchronize()
        a, b = (list(x) if isinstance(x, tuple) else [x] for x in (a, b))
        assert len(a) == len(b), name
        for x, y in zip(a, b):
            assert x.dtype == y.dtype and x.shape == y.shape and torch.equal(x, y), name


@pytest.mark.gpu
def test_native_calls_raise_what_python_calls_raise(python_only):
    q, kv = torch.zeros((2, 2, 64), device="cuda"), torch.zeros((3, 2, 16, 64), device="cuda")
    dev = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")                         # noqa: E731
    table, refs = dev(0, 1).view(1, 2), dev(1, 1, 0)
    at = (q, kv, kv, table, dev(20), dev(1))
    bad = {
        "window of none": lambda: pkg.verify_attn(*at, max_spec_len=1, window=0),
        "negative sinks": lambda: pkg.verify_attn(*at, max_spec_len=1, window=4, sinks=-1),
        "window of many lengths": lambda: pkg.verify_attn(*at[:4], dev(20, 21), dev(1, 1), max_spec_len=1, window=4),
        "window output of another type": lambda: pkg.verify_attn(*at, q.half(), max_spec_len=1, window=4),
        "window plan without workspace": lambda: pkg.verify_attn(*at, max_spec_len=1, window=4, plan="reuse"),
        "small workspace": lambda: pkg.kv_remap(table, refs, dev(0), dev(20), dev(21), workspace=torch.empty(64, dtype=torch.uint8, device="cuda")),
        "overlap": lambda: pkg.kv_remap(table, refs, dev(0), dev(20), dev(21), out_table=table),
        "too many moves": lambda: pkg.kv_compact_pages(table, refs, max_moves=4),
        "no moves": lambda: pkg.kv_compact_pages(table, refs, max_moves=0),
        "page size": lambda: pkg.kv_remap(table, refs, dev(0), dev(20), dev(21), page_size=0),
        "odd head dim": lambda: pkg.kv_copy_pages(kv[..., :3].contiguous(), kv[..., :3].contiguous(), dev(0), dev(2)),
    }
    for name, f in bad.items():
        with pytest.raises(Exception) as a:
            f()
        with pytest.raises(type(a.value)) as b:
            python_only(f)
        assert str(a.value) == str(b.value), name

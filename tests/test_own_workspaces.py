"""Calls of the cache's pages, and windowed calls that are cut into parts, without a workspace of the caller's: several of them at
once, on streams, threads and in graphs, do not meet in memory."""
import threading

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from oracle.pages import kv_compact_pages, kv_remap
from paper_2503_05096_amd import binding
from tests.test_fastcall_host import ENTRIES, ints, module  # noqa: F401  (fixture)
from tests.test_fastcall_pages import MORE, Stubs, every_call
from tests.test_gpu_kv_pages import dev, state
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)


class Stream:
    cuda_stream = 0


def test_native_calls_do_not_ask_for_the_default_workspace(module):  # noqa: F811
    stubs = Stubs(module, ENTRIES + MORE)
    shared = []
    ask = lambda nbytes, device, given, family: shared.append(family) or torch.empty(nbytes, dtype=torch.uint8, device=device)    # noqa: E731
    setup = tuple(binding.C.cast(f, binding.C.c_void_p).value for f in stubs.keep)
    module.setup(setup, ask, lambda dev: 0, lambda: 0, binding.AdaspecError)
    for name, f in every_call(module).items():          # (the stand-ins ask for 512 bytes: the windowed call is cut into parts)
        assert f() is not NotImplemented, name
    given = [ints(3, 2), ints(9), ints(3), ints(3), ints(2)]
    assert module.kv_remap(ints(1, 2), ints(9), ints(3), ints(1), ints(3), 0, 0, 16, *given, None, None) is not NotImplemented
    assert shared == []
    q, kv, bt = torch.zeros((4, 2, 64), device="meta"), torch.zeros((2, 2, 16, 64), device="meta"), ints(1, 2)
    assert module.verify_attn(q, kv, kv, bt, ints(1), ints(1), None, 3, 0.0, None, "run", None, None, None) is not NotImplemented
    assert shared == ["attn"]
    # a stream that is none of torch's: left to Python
    stubs.calls.clear()
    assert module.kv_remap(ints(1, 2), ints(9), ints(3), ints(1), ints(3), 0, 0, 16, *[None] * 6, Stream()) is NotImplemented
    assert stubs.calls == []


def test_results_and_workspace_of_one_allocation(module):  # noqa: F811
    Stubs(module, ENTRIES + MORE)
    for out in (module.kv_remap(ints(1, 2), ints(9), ints(3), ints(1), ints(3), 0, 0, 16, *[None] * 7),
                module.kv_compact_pages(ints(1, 2), ints(9), 4, 16, *[None] * 8)):
        end = max(t.storage_offset() + t.numel() for t in out)
        assert out[0].untyped_storage().nbytes() >= (end + 63) // 64 * 256 + 512


def test_python_calls_do_not_ask_for_the_default_workspace(monkeypatch):
    asked, own = [], []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 0)
    monkeypatch.setattr(binding, "_workspace", lambda *a: asked.append(a) or torch.zeros(1 << 20, dtype=torch.uint8))
    if hasattr(binding, "_scratch"):
        monkeypatch.setattr(binding, "_scratch", lambda n, *a: own.append(n) or torch.zeros(n, dtype=torch.uint8, device="cuda"))
    none = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")                 # noqa: E731
    with FakeTensorMode():
        q, kv = torch.zeros((3, 8, 128), device="cuda"), torch.zeros((200, 2, 16, 128), device="cuda")
        for f in (lambda: binding.kv_remap(none(1, 2), none(3), none(1), none(1), none(1)),
                  lambda: binding.kv_compact_pages(none(1, 2), none(3)),
                  lambda: binding.verify_attn(q, kv, kv, none(1, 200), none(1), none(1), max_spec_len=2, window=2000)):
            with pytest.raises(binding.AdaspecError):   # (tensors without addresses)
                f()
    assert asked == [] and len(own) == 3 and own[2] > 256


def _jobs(pkg, seed, n):  # noqa: F811
    """(call, reference) of remaps of both forms, compactions of both forms, and windowed attention in parts"""
    r = np.random.default_rng(seed)
    out = []
    for k in range(n):
        old, B, width, slack = ((130, 140, 400, 9000), (40, 60, 30, 4000))[k % 2]
        table, refs, held = state(r, old, width, 16, slack)
        lens = np.minimum(r.integers(0, width * 16 + 1, old), held * 16)
        sources = r.integers(-1, old, B)
        new_lens = np.where(sources >= 0, lens[np.clip(sources, 0, old - 1)], 0) + r.integers(1, 60, B)
        args = [dev(x) for x in (table, refs, sources, lens, new_lens)]
        out.append((lambda args=args, **kw: pkg.kv_remap(*args, **kw), kv_remap(table, refs, sources, lens, new_lens)))
        out.append((lambda args=args, **kw: pkg.kv_compact_pages(*args[:2], **kw), kv_compact_pages(table, refs, max(1, len(refs) // 2))))
        g = torch.Generator(device="cuda").manual_seed(seed + k)
        q, kp, vp = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((4, 8, 128), (256, 2, 16, 128), (256, 2, 16, 128)))
        at = (q, kp, vp, torch.randperm(256, generator=g, device="cuda").to(torch.int32)[None].contiguous(), dev([4000 - k]), dev([3]))
        kw = dict(max_spec_len=3, window=3000, sinks=4)
        ws = torch.empty(4 << 20, dtype=torch.uint8, device="cuda")
        dims = pkg.attn_dims(q, kp, at[3], max_spec_len=3)
        assert pkg.lib().adaspec_verify_attn_window_workspace_bytes(binding.C.byref(dims), 3000, 4) > 256
        ref = (pkg.verify_attn(*at, **kw, workspace=ws).view(torch.int16).cpu().numpy(),)
        out.append((lambda at=at, kw=kw, **more: (pkg.verify_attn(*at, **kw, **more).view(torch.int16),), ref))
    torch.cuda.synchronize()
    return out


def _check(results, what):
    torch.cuda.synchronize()
    for k, (got, ref) in enumerate(results):
        for a, b in zip(got, ref):
            assert np.array_equal(a.cpu().numpy(), b), (what, k)


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("form", ["under streams", "stream=", "raw stream="])
def test_streams(form, native, pkg, monkeypatch):  # noqa: F811
    jobs = _jobs(pkg, 1, 3)
    if not native:
        monkeypatch.setattr(binding, "_fast", binding._PythonOnly())
    streams = [torch.cuda.Stream() for _ in range(3)]
    print(f"[case] {form} native={native}", flush=True)
    for _ in range(6):
        results = []
        for k in range(3 * len(jobs)):
            call, ref = jobs[k % len(jobs)]
            s = streams[(k + k // len(jobs)) % 3]
            if form == "under streams":
                with torch.cuda.stream(s):
                    results.append((call(), ref))
            else:
                raw = type("Raw", (), {"cuda_stream": s.cuda_stream})
                results.append((call(stream=s if form == "stream=" else raw), ref))
        _check(results, form)


@pytest.mark.gpu
def test_threads(pkg):  # noqa: F811
    """Threads on one stream: their calls' launches come in any order."""
    jobs, done = _jobs(pkg, 2, 2), {}

    def work(t):
        done[t] = [(call(), ref) for _ in range(8) for call, ref in jobs[t:] + jobs[:t]]
    threads = [threading.Thread(target=work, args=(t,)) for t in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert sorted(done) == [0, 1, 2, 3]
    for t in done:
        _check(done[t], t)


@pytest.mark.gpu
def test_graphs_replayed_at_once(pkg):  # noqa: F811
    """Two graphs captured on the same stream, replayed on two others with eager calls between."""
    jobs = _jobs(pkg, 3, 2)
    capture, streams, graphs = torch.cuda.Stream(), [torch.cuda.Stream() for _ in range(2)], []
    capture.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(capture):
        for call, _ in jobs:
            call()
    torch.cuda.synchronize()
    for half in (jobs[:3], jobs[3:]):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=capture):
            results = [(call(), ref) for call, ref in half]
        graphs.append((g, results))
    torch.cuda.synchronize()
    for n in range(5):
        for g, results in graphs:
            for got, _ in results:
                for t in got:
                    t.fill_(-7)
        torch.cuda.synchronize()
        eager = []
        for (g, _), s, (call, ref) in zip(graphs, streams, jobs):
            with torch.cuda.stream(s):
                g.replay()
            eager.append((call(), ref))
        _check(eager, n)
        for g, results in graphs:
            _check(results, n)

"""What the calls of positions and of the cache in 8 bits refuse, on the host: no call of this file gets as far as a kernel."""
import ctypes as C

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2503_05096_amd as pkg
from paper_2503_05096_amd import binding
from paper_2503_05096_amd.binding import BF16, F16, F32, CopyDims, RopeDims
from tests.test_abi import PTR, _attn_dims
from tests.test_fastcall_host import ENTRIES, ERR_DIM, ERR_HIP, OK, ints, module  # noqa: F401  (fixture)
from tests.test_fastcall_pages import MORE, Stubs

FAR = 1 << 40           # addresses that are never looked at, far apart


def _dims(**kw):
    base = dict(batch=2, total_q=5, max_spec_len=3, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, num_pages=64,
                max_pages_per_req=8, dtype=BF16, rot_dim=128, interleaved=0, attn_factor=1.0, reserved=0, q_row_stride=1024,
                k_row_stride=256, v_row_stride=256, q_out_row_stride=1024)
    base.update(kw)
    return RopeDims(**base)


def _append(d, scales=False, **ptrs):
    names = ["q", "k", "v", "freq", "q_out", "k_pages", "v_pages", "k_scales", "v_scales", "table", "ctx", "spec", "parents"]
    p = {n: FAR * (i + 1) for i, n in enumerate(names)}
    p["parents"] = None
    if not scales:
        p["k_scales"] = p["v_scales"] = None
    p.update(ptrs)
    return pkg.lib().adaspec_kv_append_rope(*[p[n] for n in names], C.byref(d), None)


def _rope(d, **ptrs):
    p = dict(x=FAR, freq=2 * FAR, out=3 * FAR, ctx=4 * FAR, spec=5 * FAR, parents=None)
    p.update(ptrs)
    return pkg.lib().adaspec_rope(*p.values(), C.byref(d), None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), -2), (dict(total_q=1), -2), (dict(total_q=9), -2), (dict(max_spec_len=-1), -2), (dict(n_q_heads=0), -2),
    (dict(head_dim=0), -2), (dict(head_dim=100), -6), (dict(head_dim=264, q_row_stride=1 << 20, q_out_row_stride=1 << 20), -6),
    (dict(dtype=3), -3), (dict(dtype=-1), -3), (dict(rot_dim=0), -2), (dict(rot_dim=127), -2), (dict(rot_dim=130), -2),
    (dict(rot_dim=-2), -2), (dict(interleaved=2), -2), (dict(attn_factor=-1.0), -2), (dict(attn_factor=float("inf")), -2),
    (dict(attn_factor=float("nan")), -2), (dict(q_row_stride=1016), -2), (dict(q_out_row_stride=0), -2), (dict(q_row_stride=1028), -4),
    (dict(batch=1 << 23, total_q=1 << 23, max_spec_len=0), -6), (dict(batch=1 << 12, total_q=1 << 12, max_spec_len=1 << 16), -6),
    (dict(n_q_heads=1 << 17, q_row_stride=1 << 24, q_out_row_stride=1 << 24), -6),
])
def test_bad_dims(kw, code):
    d = _dims(**kw)
    assert _rope(d) == code
    if "q" not in next(iter(kw)) or "n_q" in next(iter(kw)):
        assert _append(_dims(**{**dict(k_row_stride=1 << 20, v_row_stride=1 << 20), **kw})) == code


def test_too_many_heads():
    wide = dict(head_dim=8, rot_dim=8, q_row_stride=1 << 20, q_out_row_stride=1 << 20, k_row_stride=1 << 20, v_row_stride=1 << 20)
    assert _rope(_dims(n_q_heads=65536, **wide)) == -6
    for scales in (False, True):
        assert _append(_dims(n_q_heads=65536, n_kv_heads=65536, **wide), scales=scales) == -6
        assert _append(_dims(n_q_heads=0, n_kv_heads=65536, **wide), scales=scales, q=None, q_out=None) == -6
        assert _append(_dims(n_q_heads=512, n_kv_heads=2, **wide), scales=scales) == -6


@pytest.mark.parametrize("kw,code", [
    (dict(n_kv_heads=3), -2), (dict(n_kv_heads=0), -2), (dict(page_size=32), -6), (dict(page_size=0), -2), (dict(num_pages=0), -2),
    (dict(max_pages_per_req=0), -2), (dict(k_row_stride=248), -2), (dict(v_row_stride=128), -2), (dict(v_row_stride=260), -4),
])
def test_bad_dims_of_an_append(kw, code):
    assert _append(_dims(**kw)) == code and _append(_dims(**kw), scales=True) == code


def test_pointers_and_alignment():
    d = _dims()
    assert pkg.lib().adaspec_rope(*[PTR] * 6, None, None) == -1 and pkg.lib().adaspec_kv_append_rope(*[PTR] * 13, None, None) == -1
    for n in ("x", "freq", "out", "ctx", "spec"):
        assert _rope(d, **{n: None}) == -1
    for n in ("x", "out"):
        assert _rope(d, **{n: 3 * FAR + 8}) == -4
    assert _rope(d, freq=2 * FAR + 2) == -4
    for n in ("k", "v", "freq", "q_out", "k_pages", "v_pages", "table", "ctx", "spec"):
        assert _append(d, **{n: None}) == -1, n
    for n in ("q", "k", "v", "q_out", "k_pages", "v_pages"):
        assert _append(d, **{n: 99 * FAR + 8}) == -4, n
    for n in ("k_scales", "v_scales"):
        assert _append(d, scales=True, **{n: None}) == -1 and _append(d, scales=True, **{n: 99 * FAR + 2}) == -4
    assert _append(_dims(max_spec_len=64), parents=99 * FAR) == -6 and _rope(_dims(max_spec_len=64), parents=99 * FAR) == -6
    # nothing to do
    assert _rope(_dims(batch=0, total_q=0), x=None) == 0 or _rope(_dims(batch=0, total_q=0)) == 0
    assert _append(_dims(batch=0, total_q=0)) == 0


def test_what_may_lie_over_what():
    d = _dims()
    # 5 rows of 2 KB; out a row further, or over the frequencies, is refused
    assert _rope(d, out=FAR + 2048) == -2 and _rope(d, out=FAR - 16) == -2 and _rope(d, freq=3 * FAR + 64) == -2
    assert _rope(d, ctx=3 * FAR + 4096) == -2
    assert _rope(_dims(q_out_row_stride=2048), out=FAR) == -2          # the same rows, apart
    fused = _dims(q_row_stride=1536, q_out_row_stride=1536, k_row_stride=1536, v_row_stride=1536)
    assert _append(fused, q=FAR, k=FAR + 2048, v=FAR + 2560, q_out=FAR + 2048) == -2      # over the keys
    assert _append(fused, q=FAR, k=FAR + 2048, v=FAR + 2560, q_out=FAR + 1024) == -2
    assert _append(d, k_pages=FAR) == -2 and _append(d, v_pages=6 * FAR + 4096) == -2 and _append(d, k_pages=10 * FAR) == -2
    assert _append(d, scales=True, k_scales=6 * FAR) == -2 and _append(d, scales=True, v_scales=8 * FAR + 256) == -2
    assert _append(d, scales=True, k_scales=12 * FAR) == -2


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), -2), (dict(total_q=1), -2), (dict(n_kv_heads=3), -2), (dict(num_pages=0), -2), (dict(dtype=3), -3),
    (dict(out_dtype=1), -3), (dict(page_size=32), -6), (dict(head_dim=100), -6), (dict(head_dim=512), -6), (dict(path=3), -2),
    (dict(scale=-1.0), -2), (dict(plan_mode=3), -2), (dict(path=2, head_dim=96), -6), (dict(path=2, dtype=F32, out_dtype=F32), -6),
])
def test_attention_refuses(kw, code):
    d, L = _attn_dims(**kw), pkg.lib()
    assert L.adaspec_verify_attn_scaled(*[PTR] * 8, None, PTR, C.byref(d), PTR, 1 << 40, None) == code
    assert L.adaspec_verify_attn_scaled_workspace_bytes(C.byref(d)) == 0


def test_attention_pointers_and_workspace():
    d, L = _attn_dims(), pkg.lib()

    def call(dims=d, ws=PTR, ws_bytes=1 << 40, **at):
        p = [PTR] * 8 + [None, PTR]
        for k, v in at.items():
            p[int(k[1:])] = v
        return L.adaspec_verify_attn_scaled(*p, C.byref(dims), ws, ws_bytes, None)
    for k in (0, 1, 2, 3, 4, 5, 6, 7, 9):
        assert call(**{f"a{k}": None}) == -1, k
    for k in (0, 1, 2, 9):
        assert call(**{f"a{k}": PTR + 8}) == -4
    for k in (3, 4):
        assert call(**{f"a{k}": PTR + 2}) == -4
    assert call(ws=None) == -1 and call(ws=PTR + 64) == -4
    assert call(dims=_attn_dims(max_spec_len=64, total_q=60), a8=PTR) == -6
    for dims in (d, _attn_dims(head_dim=64, path=2), _attn_dims(head_dim=96), _attn_dims(dtype=F32, out_dtype=F32), _attn_dims(dtype=F16, out_dtype=F32),
                 _attn_dims(batch=1, total_q=3, max_pages_per_req=4096)):
        need = L.adaspec_verify_attn_scaled_workspace_bytes(C.byref(dims))
        assert need > 0 and need % 256 == 0 and call(dims=dims, ws_bytes=need - 1) == -5


def test_pages_refuse():
    L = pkg.lib()
    copy = lambda d, n=3, p=(PTR,) * 6: L.adaspec_kv_copy_pages_scaled(*p, n, C.byref(d), None)               # noqa: E731
    good = dict(layers=1, num_pages=8, n_kv_heads=2, page_size=16, head_dim=64, dtype=BF16)
    for kw, code in ((dict(layers=-1), -2), (dict(num_pages=0), -2), (dict(head_dim=60), -6), (dict(page_size=8), -6), (dict(n_kv_heads=0), -2)):
        assert copy(CopyDims(**{**good, **kw})) == code
    for k in range(6):
        p = [PTR] * 6
        p[k] = None
        assert copy(CopyDims(**good), p=p) == -1
        p[k] = PTR + (8 if k < 2 else 2)
        if k < 4:
            assert copy(CopyDims(**good), p=p) == -4
    assert copy(CopyDims(**good), n=0) == 0 and copy(CopyDims(**good), n=-1) == -2 and copy(CopyDims(**{**good, "layers": 0})) == 0
    path = lambda d, stride=4, p=(PTR,) * 9: L.adaspec_kv_compact_path_scaled(*p, C.byref(d), stride, None)    # noqa: E731
    for kw, code in ((dict(batch=-1), -2), (dict(head_dim=100), -6), (dict(page_size=32), -6), (dict(max_spec_len=64), -2), (dict(n_kv_heads=0), -2)):
        assert path(_attn_dims(**kw)) == code
    assert path(_attn_dims(max_spec_len=64), 65) == -6 and path(_attn_dims(), 3) == -2 and path(_attn_dims(batch=70000)) == -6
    for k in range(9):
        p = [PTR] * 9
        p[k] = None
        assert path(_attn_dims(), p=p) == -1
    assert path(_attn_dims(batch=0)) == 0


# ---- the binding's own checks, on tensors that claim a device and have no memory -------------------------------------------
def _z(*shape, dtype=torch.bfloat16, dev="cuda"):
    return torch.zeros(shape, dtype=dtype, device=dev)


def _i(*shape, dev="cuda"):
    return _z(*shape, dtype=torch.int32, dev=dev)


E8 = torch.float8_e4m3fn


def _binding_append(dev="cuda", **kw):
    a = dict(q=_z(4, 8, 64), k=_z(4, 2, 64), v=_z(4, 2, 64), f=_z(32, dtype=torch.float32), kp=_z(9, 2, 16, 64, dtype=E8), vp=_z(9, 2, 16, 64, dtype=E8),
             ks=_z(9, 2, dtype=torch.float32), vs=_z(9, 2, dtype=torch.float32), out=None, parents=None, table=_i(2, 3), gain=1.0)
    a.update(kw)
    return pkg.kv_append_rope(a["q"], a["k"], a["v"], a["f"], a["kp"], a["vp"], a["table"], _i(2), _i(2), max_spec_len=1, k_scales=a["ks"],
                              v_scales=a["vs"], parents=a["parents"], q_out=a["out"], attn_factor=a["gain"])


def _binding_attn(**kw):
    a = dict(q=_z(4, 8, 64), kp=_z(9, 2, 16, 64, dtype=E8), vp=_z(9, 2, 16, 64, dtype=E8), ks=_z(9, 2, dtype=torch.float32),
             vs=_z(9, 2, dtype=torch.float32), out=None, parents=None, table=_i(2, 3))
    a.update(kw)
    more = {k: v for k, v in kw.items() if k in ("window", "sinks", "plan", "workspace")}
    return pkg.verify_attn(a["q"], a["kp"], a["vp"], a["table"], _i(2), _i(2), a["out"], max_spec_len=1, k_scales=a["ks"], v_scales=a["vs"],
                           parents=a["parents"], **more)


REFUSED = [
    (_binding_append, dict(gain=0.0), ValueError), (_binding_append, dict(f=None), ValueError), (_binding_append, dict(ks=None), ValueError),
    (_binding_append, dict(q=None, out=lambda: _z(4, 8, 64)), ValueError),
    (_binding_append, dict(kp=lambda: _z(9, 2, 16, 64)), AssertionError), (_binding_append, dict(ks=lambda: _z(9, 3, dtype=torch.float32)), AssertionError),
    (_binding_append, dict(vs=lambda: _z(9, 2)), AssertionError), (_binding_append, dict(k=lambda: _z(4, 2, 32)), AssertionError),
    (_binding_append, dict(q=lambda: _z(5, 8, 64)), AssertionError), (_binding_append, dict(q=lambda: _z(4, 8, 128)[..., ::2]), AssertionError),
    (_binding_append, dict(out=lambda: _z(4, 8, 64, dev="cpu")), ValueError), (_binding_append, dict(out=lambda: _z(4, 4, 64)), AssertionError),
    (_binding_append, dict(parents=lambda: _i(3)), AssertionError), (_binding_append, dict(table=lambda: _i(3, 3)), AssertionError),
    (_binding_append, dict(f=lambda: _z(32)), AssertionError),
    (_binding_attn, dict(window=100), ValueError), (_binding_attn, dict(sinks=1), ValueError), (_binding_attn, dict(ks=None), ValueError),
    (_binding_attn, dict(kp=lambda: _z(9, 2, 16, 64)), AssertionError), (_binding_attn, dict(vs=lambda: _z(8, 2, dtype=torch.float32)), AssertionError),
    (_binding_attn, dict(q=lambda: _z(4, 8, 128)), AssertionError), (_binding_attn, dict(out=lambda: _z(4, 8, 64, dev="cpu")), ValueError),
    (_binding_attn, dict(out=lambda: _z(4, 8, 32)), AssertionError), (_binding_attn, dict(plan="reuse"), ValueError),
    (_binding_attn, dict(parents=lambda: _i(5)), AssertionError), (_binding_attn, dict(workspace=lambda: _z(1 << 22, dtype=torch.uint8, dev="cpu")), ValueError),
]


@pytest.mark.parametrize("f,kw,error", REFUSED, ids=lambda x: getattr(x, "__name__", None) or (next(iter(x)) if isinstance(x, dict) else ""))
def test_binding_refuses(f, kw, error, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 0)
    with FakeTensorMode():
        with pytest.raises(error):
            f(**{k: v() if callable(v) else v for k, v in kw.items()})


# ---- the native call path ----------------------------------------------------------------------------------------------------
SCALED = [("rope", C.c_int, 8), ("append_rope", C.c_int, 15), ("scaled_ws", C.c_size_t, 1), ("scaled", C.c_int, 14)]
NAMES = ("rope", "kv_append_rope", "verify_attn_scaled")


def _native(m, **kw):
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="meta")                          # noqa: E731
    f32 = torch.float32
    a = dict(q=z(4, 8, 64), k=z(4, 2, 64), f=z(32, dtype=f32), p=z(9, 2, 16, 64, dtype=E8), s=z(9, 2, dtype=f32), table=ints(2, 3), ctx=ints(2), gain=1.0,
             out=None, parents=None, plan="run")
    a.update(kw)
    return {"rope": lambda: m.rope(a["q"], a["f"], a["ctx"], ints(2), 1, False, a["gain"], a["parents"], a["out"], None),
            "kv_append_rope": lambda: m.kv_append_rope(a["q"], a["k"], a["k"], a["f"], a["p"], a["p"], a["table"], a["ctx"], ints(2), 1, a["s"], a["s"],
                                                       False, a["gain"], a["parents"], a["out"], None),
            "verify_attn_scaled": lambda: m.verify_attn_scaled(a["q"], a["p"], a["p"], a["s"], a["s"], a["table"], a["ctx"], ints(2), a["out"], 1, 0.0,
                                                               None, a["plan"], None, None, a["parents"])}


def test_native_calls(module):  # noqa: F811
    stubs = Stubs(module, ENTRIES + MORE + SCALED)
    for name, f in _native(module).items():
        stubs.status = OK
        assert f().shape == (4, 8, 64), name
        stubs.status = ERR_DIM
        assert f() is NotImplemented
        stubs.status = ERR_HIP
        with pytest.raises(binding.AdaspecError):
            f()
    stubs.status = OK
    assert module.kv_append_rope(None, *[torch.zeros((4, 2, 64), device="meta")] * 2, None, *[torch.zeros((9, 2, 16, 64), device="meta")] * 2, ints(2, 3),
                                 ints(2), ints(2), 1, None, None, False, 1.0, None, None, None) is None
    stubs.calls.clear()
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="meta")                          # noqa: E731
    for kw, names in ((dict(gain=0.0), NAMES[:2]), (dict(gain=1), NAMES[:2]), (dict(f=z(32)), NAMES[:2]), (dict(ctx=ints(3)), NAMES), (dict(parents=ints(3)), NAMES),
                      (dict(out=z(4, 8, 32)), NAMES), (dict(q=z(4, 8, 128)[..., ::2]), NAMES), (dict(p=z(9, 2, 16, 64)), NAMES[1:]),
                      (dict(s=z(9, 3, dtype=torch.float32)), NAMES[1:]), (dict(table=ints(3, 3)), NAMES[1:]), (dict(k=z(5, 2, 64)), NAMES[1:2]),
                      (dict(plan="reuse"), NAMES[2:]), (dict(plan="build"), NAMES[2:])):
        for n in names:
            assert _native(module, **kw)[n]() is NotImplemented, (kw.keys(), n)
    assert stubs.calls == []
    # slices of wider rows
    wide = z(4, 12 * 64)
    assert _native(module, q=wide[:, :512].unflatten(1, (8, 64)), k=wide[:, 512:640].unflatten(1, (2, 64)))["kv_append_rope"]().is_contiguous()


def test_native_calls_of_a_library_without_them(module):  # noqa: F811
    stubs = Stubs(module, ENTRIES + MORE)
    for name, f in _native(module).items():
        assert f() is NotImplemented, name
    assert stubs.calls == []
    with pytest.raises(ValueError, match="entry points"):
        Stubs(module, ENTRIES + MORE + SCALED[:2])


def test_native_calls_do_not_ask_for_the_default_workspace(module):  # noqa: F811
    shared = []
    stubs = Stubs(module, ENTRIES + MORE + SCALED)
    module.setup(tuple(C.cast(f, C.c_void_p).value for f in stubs.keep), lambda *a: shared.append(a), lambda dev: 0, lambda: 0, binding.AdaspecError)
    for name, f in _native(module).items():
        assert f() is not NotImplemented
    assert shared == []

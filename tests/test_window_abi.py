"""What adaspec_verify_attn_window refuses, on the host: no call of this file gets as far as a kernel."""
import ctypes as C

import pytest

import paper_2503_05096_amd as pkg
from paper_2503_05096_amd.binding import BF16, F32
from tests.test_abi import PTR, _attn_dims


def _call(dims, window=100, sinks=4, ptrs=None, ws=PTR, ws_bytes=1 << 40):
    p = [PTR] * 7 if ptrs is None else ptrs
    return pkg.lib().adaspec_verify_attn_window(*p, C.byref(dims), window, sinks, ws, ws_bytes, None)


def _bytes(dims, window=100, sinks=4):
    return pkg.lib().adaspec_verify_attn_window_workspace_bytes(C.byref(dims), window, sinks)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), -2), (dict(total_q=1), -2), (dict(n_kv_heads=3), -2), (dict(num_pages=0), -2), (dict(dtype=7), -3),
    (dict(out_dtype=1), -3), (dict(page_size=32), -6), (dict(head_dim=100), -6), (dict(head_dim=512), -6), (dict(path=3), -2),
    (dict(scale=-1.0), -2), (dict(plan_mode=3), -2), (dict(max_spec_len=-1), -2),
    (dict(max_pages_per_req=(1 << 26) + 1, batch=1, total_q=1, max_spec_len=0), -6),            # more than 2^30 tokens in a row
    # units that do not fit the grid: 16384 requests of 8192 rows with 1024 kv heads
    (dict(batch=1 << 14, total_q=1 << 14, max_spec_len=8191, n_q_heads=1024, n_kv_heads=1024, max_pages_per_req=1), -6),
    (dict(batch=1 << 20, total_q=1 << 20, max_spec_len=1023, n_q_heads=1, n_kv_heads=1, max_pages_per_req=1), -6),
    (dict(n_q_heads=65536, n_kv_heads=65536), -6), (dict(n_q_heads=(1 << 16) + 2, n_kv_heads=2), -6),
])
def test_bad_dims(kw, code):
    d = _attn_dims(**kw)
    assert _call(d) == code and _bytes(d) == 0


@pytest.mark.parametrize("window,sinks", [(0, 0), (-5, 0), (-(1 << 31), 0), (1, -1), (16, -(1 << 31))])
def test_bad_windows(window, sinks):
    assert _call(_attn_dims(), window, sinks) == -2 and _bytes(_attn_dims(), window, sinks) == 0
    L = pkg.lib()
    assert L.adaspec_check_window_inputs(PTR, PTR, PTR, C.byref(_attn_dims()), window, sinks, PTR, None) == -2


def test_pointers_alignment_and_workspace():
    d = _attn_dims()
    assert pkg.lib().adaspec_verify_attn_window(*[PTR] * 7, None, 100, 4, PTR, 1 << 30, None) == -1
    for k in range(7):
        p = [PTR] * 7
        p[k] = None
        assert _call(d, ptrs=p) == -1
    assert _call(d, ws=None) == -1
    for k in (0, 1, 2, 6):
        p = [PTR] * 7
        p[k] = PTR + 8
        assert _call(d, ptrs=p) == -4
    assert _call(d, ws=PTR + 64) == -4
    for dims in (d, _attn_dims(head_dim=64), _attn_dims(dtype=F32, out_dtype=F32), _attn_dims(out_dtype=F32),
                 _attn_dims(batch=1, total_q=3, max_pages_per_req=4096)):
        for window in (1, 100, 5000, (1 << 31) - 1):
            need = _bytes(dims, window, (1 << 31) - 1 if window == 100 else 0)
            assert need > 0 and need % 256 == 0
            assert _call(dims, window, (1 << 31) - 1 if window == 100 else 0, ws_bytes=need - 1) == -5
    for k in range(3):
        p = [PTR] * 3
        p[k] = None
        assert pkg.lib().adaspec_check_window_inputs(*p, C.byref(d), 100, 4, PTR, None) == -1
    assert pkg.lib().adaspec_check_window_inputs(PTR, PTR, PTR, C.byref(d), 100, 4, None, None) == -1


def test_calls_that_enqueue_nothing():
    L = pkg.lib()
    empty = _attn_dims(batch=0, total_q=0)
    assert L.adaspec_verify_attn_window(*[None] * 7, C.byref(empty), 100, 4, None, 0, None) == 0
    build = _attn_dims(plan_mode=1)
    assert L.adaspec_verify_attn_window(None, None, None, PTR, PTR, PTR, None, C.byref(build), 100, 4, PTR, 1 << 40, None) == 0
    assert L.adaspec_verify_attn_window(None, None, None, None, PTR, PTR, None, C.byref(build), 100, 4, PTR, 1 << 40, None) == -1
    assert L.adaspec_verify_attn_window(None, None, None, PTR, PTR, PTR, None, C.byref(build), 100, 4, PTR, 0, None) == -5


def test_python_refusals():
    import torch
    q = torch.zeros(2, 2, 64)
    kv, bt, one = torch.zeros(1, 2, 16, 64), torch.zeros(1, 1, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="sinks"):
        pkg.verify_attn(q, kv, kv, bt, one, one, max_spec_len=1, sinks=4)
    with pytest.raises(ValueError, match="sinks"):
        pkg.check_ragged_inputs(bt, one, one, _attn_dims(), sinks=4)
    with pytest.raises(ValueError, match="trees"):
        pkg.verify_attn(q, kv, kv, bt, one, one, max_spec_len=1, window=8, parents=one)
    with pytest.raises(AssertionError):                             # tensors that are not on a GPU
        pkg.verify_attn(q, kv, kv, bt, one, one, max_spec_len=1, window=8)
    assert BF16 == 2

"""The oracle of windowed attention (oracle/window.py): against the oracle of plain verification attention, and by hand."""
import numpy as np
import pytest

import workloads as W
from oracle.window import hidden_tokens, verify_attn_window, visible


def test_a_window_over_everything_is_plain_attention(oracle_mod):
    st = W.make_custom_step(71, ctx_lens=[1, 17, 40, 70], spec_lens=[0, 3, 1, 5], n_q_heads=4, n_kv_heads=2, head_dim=32, dtype="bf16",
                            acceptance=False)
    ref, _ = oracle_mod.verify_attn(st.q, st.k_pages, st.v_pages, st.block_table, st.ctx_lens, st.spec_lens, dtype=st.dtype)
    for window, sinks in ((70, 0), (1 << 30, 0), (1, 70), (30, 40)):
        out = verify_attn_window(st.q, st.k_pages, st.v_pages, st.block_table, st.ctx_lens, st.spec_lens, window=window, sinks=sinks,
                                 dtype=st.dtype)
        assert np.abs(out - ref).max() < 1e-12


def test_by_hand():
    # one head of two channels, scores 0: the mean of the values a row sees
    k = np.zeros((3, 1, 16, 2), np.float32)
    v = np.zeros_like(k)
    v[0, 0, :, 0] = np.arange(16)                                   # tokens 0..15
    v[2, 0, :, 0] = 16 + np.arange(16)                              # tokens 16..31
    q = np.zeros((2, 1, 2), np.float32)
    out = verify_attn_window(q, k, v, np.array([[0, 2]]), [20], [1], window=3, sinks=2, dtype="f32")
    assert np.allclose(out[0, 0], [(0 + 1 + 16 + 17 + 18) / 5, 0]) and np.allclose(out[1, 0], [(0 + 1 + 17 + 18 + 19) / 5, 0])
    out = verify_attn_window(q, k, v, np.array([[0, 2]]), [20], [1], window=1, sinks=0, dtype="f32")
    assert out[0, 0, 0] == 18 and out[1, 0, 0] == 19


@pytest.mark.parametrize("L,n,window,sinks", [(50, 4, 7, 3), (5, 5, 1, 0), (20, 1, 100, 2), (33, 2, 16, 40)])
def test_hidden_tokens_are_those_that_no_row_sees(L, n, window, sinks):
    seen = set()
    for j in range(n):
        t = set(visible(L - n + j, window, sinks).tolist())
        assert t == {x for x in range(L - n + j + 1) if x > L - n + j - window or x < sinks}
        seen |= t
    assert set(hidden_tokens(L, n, window, sinks).tolist()) == set(range(L)) - seen

"""Arguments of the calls of positions at the ends of their ranges. No GPU: tensors that claim a device and have no memory."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2503_05096_amd as pkg
from paper_2503_05096_amd import binding


@pytest.mark.parametrize("gain", [0.0, -1.0, float("nan"), 1e-60, 5e-324], ids=str)
def test_a_factor_that_is_nothing_in_fp32_is_refused(gain, monkeypatch):
    """1e-60 is 0 as the library sees it, and 0 stands for 1 there."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 0)
    with FakeTensorMode():
        z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")                   # noqa: E731
        x, kv, f = z(4, 8, 64), z(4, 2, 64), z(32, dtype=torch.float32)
        lens, table, pages = z(2, dtype=torch.int32), z(2, 3, dtype=torch.int32), z(9, 2, 16, 64)
        with pytest.raises(ValueError):
            pkg.rope(x, f, lens, lens, max_spec_len=1, attn_factor=gain)
        with pytest.raises(ValueError):
            pkg.kv_append_rope(x, kv, kv, f, pages, pages, table, lens, lens, max_spec_len=1, attn_factor=gain)


def test_frequencies_on_a_device_by_its_number():
    with FakeTensorMode():
        freq, _ = pkg.rope_frequencies(16, device=0)
    assert freq.device == torch.device("cuda", 0)
    assert pkg.rope_frequencies(16)[0].device.type == "cpu" and pkg.rope_frequencies(16, device="meta")[0].device.type == "meta"

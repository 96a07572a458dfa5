"""A refused reset() or resume() leaves the object with the context that it had."""
import pytest
import torch

from paper_2412_05693_amd import batchmax as bmx

SHAPE = dict(b=2, s=64, kv_max=32, block=16, max_gen=8, n_heads=4, n_kv_heads=2, head_dim=64, device="cpu",
             init=False)


@pytest.mark.parametrize("cls", [bmx.PDAttentionKV4, bmx.PDAttention])
def test_a_state_that_is_not_reachable(cls):
    a = cls(**SHAPE)
    a.resume(3, 70)
    for bad in ((5, 1), (49, 60), (3, 73), (-1, 3)):
        with pytest.raises(bmx.BatchMaxError):
            a.resume(*bad)
        assert (a.length, a.next_pos) == (3, 70)
    a.resume(4, 71)
    assert (a.length, a.next_pos) == (4, 71)


def test_another_current_device(monkeypatch):
    a = bmx.PDAttentionKV4(**SHAPE)
    a.resume(3, 70)
    a._dev_index = 0
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        a.reset()
    assert (a.length, a.next_pos) == (3, 70)

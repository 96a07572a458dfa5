"""Refusals of the calls that move rows into and out of a 4-bit cache (no device work)."""
import pytest
import torch

from paper_2412_05693_amd import batchmax as bmx

SHAPE = dict(b=2, s=64, kv_max=32, block=16, max_gen=8, n_heads=4, n_kv_heads=2, head_dim=64, device="cpu",
             init=False)


@pytest.fixture
def att(monkeypatch):
    monkeypatch.setattr(bmx.PDAttentionKV4, "_stream", lambda self: 0)
    return bmx.PDAttentionKV4(**SHAPE)


@pytest.mark.parametrize("slot0", [2**31, 2**32, 2**32 + 5, -(2**32)])
def test_a_slot_beyond_32_bits_is_refused(att, slot0):
    """(no rows: a call that took slot0 modulo 2^32 would pass without device work)"""
    x = torch.zeros(2, 2, 0, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="32 bits"):
        att.write_rows(slot0, x, x.clone())
    with pytest.raises(ValueError, match="32 bits"):
        att.read_rows(slot0, 0, x, x.clone())


@pytest.mark.parametrize("state", [(2**32 + 3, 70), (3, 2**32 + 70)])
def test_a_state_beyond_32_bits_is_refused(att, state):
    with pytest.raises(ValueError, match="32 bits"):
        att.resume(*state)

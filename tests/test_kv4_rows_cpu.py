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


def test_a_read_into_one_tensor_is_refused(att):
    x = torch.zeros(2, 2, 5, 64, dtype=torch.bfloat16)
    with pytest.raises(bmx.BatchMaxError, match="overlap"):
        att.read_rows(0, 5, x, x)


@pytest.mark.parametrize("seq_ld,n,rows_apart", [(8, 4, 0), (8, 4, 3), (8, 4, -3), (8, 4, 5), (8, 4, 8), (8, 4, -24),
                                                 (8, 5, 4), (8, 8, 7), (4, 4, 15)])
def test_overlapping_rows_of_one_buffer(seq_ld, n, rows_apart):
    """k at row 0 and v `rows_apart` rows behind it: rows that both would write."""
    d = bmx.make_dims(**{x: SHAPE[x] for x in SHAPE if x not in ("device", "init")}, dtype="bf16")
    fake = 0x7000000000
    c = bmx.bm_kv4_cache(*(fake + i * 0x1000000 for i in range(8)), bmx.bm_kv4_workspace_bytes(d))
    units = range(4)
    k_rows = {u * seq_ld + r for u in units for r in range(n)}
    both = k_rows & {u * seq_ld + r + rows_apart for u in units for r in range(n)}
    assert both                        # (a pair that is not refused would reach the device)
    k = 0x7100000000
    with pytest.raises(bmx.BatchMaxError, match="overlap"):
        bmx.bm_kv4_read(d, c, 0, n, k, k + rows_apart * 64 * 2, seq_ld, 0)

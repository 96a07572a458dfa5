"""A cache in the caller's own tensors: which types are taken, and as what."""
import pytest
import torch

from paper_2412_05693_amd import batchmax as bmx

SHAPE = dict(b=2, s=64, kv_max=32, block=16, max_gen=8, n_heads=4, n_kv_heads=2, head_dim=64)


def buffers_of(cls, **kw):
    a = cls(**SHAPE, init=False, **kw)
    names = [*a._buffers(), "work"]
    return names, [getattr(a, n) for n in names]


@pytest.mark.parametrize("name,other", [("k", torch.int8), ("v_scale", torch.bool), ("score", torch.int32),
                                        ("pos", torch.float32), ("len", torch.float32), ("score", torch.float64),
                                        ("k", torch.int16)])
def test_a_4_bit_cache_takes_its_own_types_alone(name, other):
    names, parts = buffers_of(bmx.PDAttentionKV4, device="cpu")
    bmx.PDAttentionKV4(**SHAPE, device="cpu", init=False, buffers=parts)
    i = names.index(name)
    with pytest.raises(ValueError, match=f"buffer {name}"):
        bmx.PDAttentionKV4(**SHAPE, device="cpu", init=False,
                           buffers=[*parts[:i], torch.zeros(parts[i].shape, dtype=other), *parts[i + 1:]])

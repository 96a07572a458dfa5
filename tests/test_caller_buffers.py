"""A cache in the caller's own tensors: which types are taken, and as what."""
import warnings

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


WIDER = {"k": torch.float32, "v": torch.float16, "score": torch.float64, "pos": torch.int64, "len": torch.float32}


def test_a_wider_tensor_is_raw_storage():
    names, parts = buffers_of(bmx.PDAttention, device="cpu")
    for name, other in WIDER.items():
        i = names.index(name)
        wide = torch.zeros(parts[i].shape, dtype=other)
        with pytest.warns(UserWarning, match=f"buffer {name}"):
            a = bmx.PDAttention(**SHAPE, device="cpu", init=False, buffers=[*parts[:i], wide, *parts[i + 1:]])
        x = getattr(a, name)
        assert x.dtype == parts[i].dtype and x.shape == parts[i].shape and x.is_contiguous()
        assert x.data_ptr() == wide.data_ptr() == getattr(a.cache, name)
        assert all(getattr(a, n) is y for n, y in zip(names, parts) if n != name)
    # its own types: the tensors themselves, and nothing said
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        a = bmx.PDAttention(**SHAPE, device="cpu", init=False, buffers=parts)
    assert all(getattr(a, n) is x for n, x in zip(names, parts))


@pytest.mark.gpu
def test_wider_storage_changes_no_result():
    g = torch.Generator().manual_seed(3)
    b, hk, h, d, t = 2, 2, 4, 64, 72
    q, o = (torch.randn((b, h, t, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    k, v = (torch.randn((b, hk, t, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    names, parts = buffers_of(bmx.PDAttention)
    wide = [torch.zeros(x.shape, dtype=WIDER.get(n, x.dtype), device="cuda") for n, x in zip(names, parts)]
    with pytest.warns(UserWarning):
        other = bmx.PDAttention(**SHAPE, buffers=wide)
    got = []
    for a in (bmx.PDAttention(**SHAPE), other):
        o.zero_()
        a.run_prefill(q, k, v, o)
        a.run_decode(q, k, v, o)
        n = a.length
        got.append([o.clone(), *(getattr(a, x)[:, :, :n].clone() for x in ("k", "v", "score", "pos")), a.len.clone()])
    assert all(torch.equal(x, y) for x, y in zip(*got))

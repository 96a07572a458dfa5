"""The 4-bit cache's calls without a GPU: every refusal comes before any device work
(placeholder addresses are never followed), and sizes follow the format."""
import pytest
import torch

from kv4_reference import stored
from paper_2412_05693_amd import batchmax as bmx
from test_abi_cpu import FAKE, dims, status_of

BAD, UNSUP, CAP, ORDER = (bmx.BM_ERR_INVALID_ARG, bmx.BM_ERR_UNSUPPORTED, bmx.BM_ERR_CAPACITY,
                          bmx.BM_ERR_ORDER)


def fake(d, **kw):
    c = bmx.bm_kv4_cache(*(FAKE + i * 0x1000000 for i in range(8)), bmx.bm_kv4_workspace_bytes(d))
    for name, x in kw.items():
        setattr(c, name, x)
    return c


def test_workspace_holds_the_cached_rows():
    for dtype, es in (("bf16", 2), ("f32", 4)):
        d = dims(dtype=dtype)
        rows = 2 * 2 * (128 + 64) * 128 * es          # units, slots, head size
        assert bmx.bm_kv4_workspace_bytes(d) >= bmx.bm_workspace_bytes(d) + 2 * rows
        assert bmx.bm_kv4_workspace_bytes(d) <= bmx.bm_workspace_bytes(d) + 2 * rows + 1024
    assert bmx.bm_kv4_workspace_bytes(dims(head_dim=96)) == 0


def test_slots_are_whole_groups_of_64():
    assert bmx.bm_kv4_slots(dims()) == 192
    assert bmx.bm_kv4_slots(dims(kv_max=129)) == 256
    assert bmx.bm_kv4_slots(dims(b=0)) == -1


def test_context_pointer_checks():
    d = dims()
    resume = lambda c, n=0, pos=0: status_of(bmx.bm_kv4_resume, d, c, n, pos)    # noqa: E731
    for name in ("k", "v", "k_scale", "v_scale", "score", "pos", "len", "work"):
        assert resume(fake(d, **{name: 0})) == BAD, name
    for name in ("k", "v", "k_scale", "v_scale", "work"):
        assert resume(fake(d, **{name: FAKE + 8})) == BAD, name
    for name in ("score", "pos", "len"):
        assert resume(fake(d, **{name: FAKE + 2})) == BAD, name
    # the workspace of batchmax.h alone is too small
    assert resume(fake(d, work_bytes=bmx.bm_workspace_bytes(d))) == BAD
    assert "work_bytes" in bmx.bm_last_error()
    assert resume(fake(d), 200, 300) == BAD               # more entries than slots
    assert resume(fake(d), 10, 5) == BAD                  # more entries than positions
    assert status_of(bmx.bm_kv4_resume, dims(n_heads=16), fake(d), 0, 0) == UNSUP
    assert status_of(bmx.bm_kv4_init, dims(b=0), fake(d), 0) == BAD


def test_null_arguments_of_the_c_calls():
    import ctypes

    d, out = dims(), ctypes.c_void_p()
    c = fake(d)
    p, lib = ctypes.byref, bmx._lib
    assert lib.bm_kv4_init(p(d), None, None, p(out)) == BAD
    assert lib.bm_kv4_init(p(d), p(c), None, None) == BAD
    assert lib.bm_kv4_init(None, p(c), None, p(out)) == BAD
    assert lib.bm_kv4_resume(p(d), p(c), 0, 0, None) == BAD
    assert lib.bm_kv4_write(p(d), None, 0, 1, FAKE, FAKE, 1, None) == BAD
    assert lib.bm_kv4_read(None, p(c), 0, 1, FAKE, FAKE, 1, None) == BAD
    assert lib.bm_kv4_workspace_bytes(None) == 0
    assert out.value is None


@pytest.mark.parametrize("call", [bmx.bm_kv4_write, bmx.bm_kv4_read])
def test_row_calls_refuse(call):
    d = dims()                                            # 192 slots
    go = lambda slot0, n, k=FAKE, v=FAKE, ld=192, **kw: status_of(                # noqa: E731
        call, d, fake(d, **kw), slot0, n, k, v, ld, 0)
    assert go(-1, 1) == BAD and go(0, -1) == BAD
    assert go(192, 1) == CAP and go(1, 192) == CAP and go(0, 193) == CAP
    assert go(2**31 - 1, 2**31 - 1) == CAP
    assert go(0, 4, k=0) == BAD and go(0, 4, v=0) == BAD
    assert go(0, 4, k=FAKE + 8) == BAD and go(0, 4, v=FAKE + 4) == BAD
    assert go(0, 4, ld=3) == BAD
    for name in ("k", "v", "k_scale", "v_scale"):
        assert go(0, 4, **{name: 0}) == BAD
    assert go(0, 4, k_scale=FAKE + 4) == BAD and go(0, 4, v=FAKE + 8) == BAD
    # nothing to do: no device work; score, pos, len and work do not matter
    assert go(0, 0, k=0, v=0, score=0, pos=0, len=0, work=0) == bmx.BM_OK
    assert go(192, 0) == bmx.BM_OK
    assert status_of(call, dims(head_dim=32), fake(d), 0, 1, FAKE, FAKE, 1, 0) == UNSUP


def test_context_keeps_the_checks_of_every_call():
    d, P = dims(), FAKE
    ctx = bmx.bm_kv4_resume(d, fake(d), 128, 192)
    try:
        pre, cut = bmx.bm_prefill_block, bmx.bm_prefill_block_cut
        for f in (pre, cut):
            assert status_of(f, ctx, 100, 64, P, P, P, P, 64, 0) == ORDER
            assert status_of(f, ctx, 192, 65, P, P, P, P, 65, 0) == BAD
            assert status_of(f, ctx, 192, 64, P, P, P, P, 32, 0) == BAD
            assert status_of(f, ctx, 192, 64, P + 2, P, P, P, 64, 0) == BAD
        assert status_of(bmx.bm_decode_step, ctx, 192, P, P, P, P, 1, 0) == ORDER
        assert status_of(bmx.bm_evict_compact, ctx, 190, 0) == ORDER
        bmx.bm_evict_compact(ctx, 191, 0)                 # within the bound: no device work
        assert status_of(bmx.bm_set_rank_rule, ctx, 9) == BAD
        assert bmx.bm_ctx_len(ctx) == 128 and bmx.bm_ctx_next_pos(ctx) == 192
    finally:
        bmx.bm_destroy(ctx)
    # a scoring step takes at most 4097 entries, as over a cache of the element type
    big = dims(s=8192, kv_max=6000)
    ctx = bmx.bm_kv4_resume(big, fake(big), 5000, 8192)
    try:
        assert status_of(bmx.bm_decode_step, ctx, 8192, P, P, P, P, 1, 0) == UNSUP
    finally:
        bmx.bm_destroy(ctx)


def att(**kw):
    base = dict(b=2, s=64, kv_max=32, block=16, max_gen=8, n_heads=4, n_kv_heads=2, head_dim=64,
                device="cpu", init=False)
    return bmx.PDAttentionKV4(**{**base, **kw})


def test_python_object_checks_its_tensors():
    a = att()
    assert a.k.shape == (2, 2, 64, 32) and a.k_scale.shape == (2, 2, 64, 2) and a.k.dtype == torch.uint8
    x = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16)
    for bad in (x.float(), x[:, :, :, :32].contiguous(), x[:1], x.transpose(2, 3), x[0]):
        with pytest.raises(ValueError):
            a.write_rows(0, bad, x)
        with pytest.raises(ValueError):
            a.read_rows(0, 3, x, bad)
    with pytest.raises(ValueError):
        a.write_rows(0, x, torch.zeros(2, 2, 4, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        a.read_rows(0, 2, x, x.clone())
    with pytest.raises(ValueError):
        att(static_workspace=True)
    parts = [getattr(a, n) for n in ("k", "v", "k_scale", "v_scale", "score", "pos", "len", "work")]
    att(buffers=parts)
    with pytest.raises(ValueError):
        att(buffers=[parts[0][:, :, :40], *parts[1:]])
    with pytest.raises(ValueError):
        att(buffers=parts[:-1])
    with pytest.raises(ValueError):
        att(buffers=[*parts[:-1], parts[-1][:100]])


@pytest.mark.parametrize("cls", [bmx.PDAttentionKV4, bmx.PDAttention])
def test_buffers_of_another_element_size_are_refused(cls):
    a = cls(b=2, s=64, kv_max=32, block=8, max_gen=16, n_heads=4, n_kv_heads=2, head_dim=64, device="cpu",
            init=False)
    names = [*a._buffers(), "work"]
    parts = [getattr(a, n) for n in names]
    args = dict(b=2, s=64, kv_max=32, block=8, max_gen=16, n_heads=4, n_kv_heads=2, head_dim=64, device="cpu",
                init=False)
    cls(**args, buffers=parts)
    small = {1: None, 2: torch.uint8, 4: torch.float16}
    for i, x in enumerate(parts[:-1]):
        if (dt := small[x.element_size()]) is not None:
            with pytest.raises(ValueError, match=names[i]):
                cls(**args, buffers=[*parts[:i], x.to(dt), *parts[i + 1:]])
    wide = torch.empty(2 * parts[-1].numel(), dtype=torch.uint8)[::2]
    for work in (wide, parts[-1].to("meta")):
        with pytest.raises(ValueError, match="work"):
            cls(**args, buffers=[*parts[:-1], work])


def test_stack_bytes_at_four_bits():
    shape = dict(b=3, kv_max=512, block=256, n_kv_heads=8, head_dim=128, dtype="bf16")
    full, four = bmx.stack_layer_bytes(**shape), bmx.stack_layer_bytes(**shape, kv_bits=4)
    rows = 3 * 8 * 768
    assert full == rows * (512 + 8) + 256              # (the lengths: 96 bytes, padded)
    assert four == rows * (2 * (64 + 4) + 8) + 256
    shape.update(kv_max=500, block=250)                # 750 slots, 768 in the planes
    rows, entries = 24 * 768, 24 * 750 * 4             # (an array of 4 bytes an entry: padded to 256)
    assert bmx.stack_layer_bytes(**shape, kv_bits=4) == \
        rows * 2 * (64 + 4) + 2 * (-entries % 256 + entries) + 256
    with pytest.raises(ValueError):
        bmx.stack_layer_bytes(**shape, kv_bits=8)
    plan = dict(n_layers=32, s=8192, kv_max=512, block=256, max_gen=256, n_heads=32, n_kv_heads=8,
                head_dim=128, dtype="bf16")
    b16, b4 = (bmx.plan_stack_batch(280 << 30, kv_bits=n, **plan) for n in (16, 4))
    assert 2.5 * b16 < b4 < 3.76 * b16


def test_reference_format_by_hand():
    x = torch.zeros(1, 32)
    x[0, :6] = torch.tensor([7.0, 0.5, -1.5, 3.0, 5.0, 0.49])
    # 7 > 6 2^0, so E = 1: steps of 1 up to 4, of 2 up to 8, of 4 beyond (on a scale of 2)
    assert stored(x)[0, :6].tolist() == [8.0, 0.0, -2.0, 3.0, 4.0, 0.0]
    x[0, 0] = 6.0                                          # E = 0
    assert stored(x)[0, :6].tolist() == [6.0, 0.5, -1.5, 3.0, 4.0, 0.5]

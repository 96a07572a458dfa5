"""Window caches and drafted tokens without a GPU: every refusal comes before any device
work (placeholder addresses are never followed)."""
import ctypes

import pytest
import torch

from paper_2412_05693_amd import batchmax as bmx
from test_abi_cpu import FAKE, dims, fake_cache, status_of
from test_kv4_cpu import fake as fake_kv4

BAD, UNSUP, CAP, ORDER = (bmx.BM_ERR_INVALID_ARG, bmx.BM_ERR_UNSUPPORTED, bmx.BM_ERR_CAPACITY,
                          bmx.BM_ERR_ORDER)


def fake_win(d, **kw):
    c = bmx.bm_win_cache(FAKE, FAKE + 0x1000000, FAKE + 0x2000000, bmx.bm_win_workspace_bytes(d))
    for name, x in kw.items():
        setattr(c, name, x)
    return c


def win(next_pos=0, sinks=4, **kw):
    d = dims(**kw)
    return bmx.bm_win_resume(d, sinks, fake_win(d), next_pos)


def test_window_dims():
    ok = lambda sinks=0, **kw: status_of(bmx.bm_win_validate, dims(**kw), sinks)     # noqa: E731
    assert ok() == bmx.BM_OK and ok(4) == bmx.BM_OK and ok(127) == bmx.BM_OK
    assert ok(128) == BAD and ok(-1) == BAD                     # no window left
    assert ok(block=1 << 20) == bmx.BM_OK and ok(block=0) == BAD
    assert ok(kv_max=65535) == bmx.BM_OK and ok(kv_max=65536) == UNSUP
    assert ok(head_dim=96) == UNSUP and ok(n_heads=16) == UNSUP and ok(b=0) == BAD
    assert bmx.bm_win_workspace_bytes(dims(b=0)) == 0
    assert bmx.bm_win_workspace_bytes(dims(block=1 << 20)) > 0
    for b in (1, 3, 40, 1000):                                  # longer calls never need less
        need = [bmx.bm_win_workspace_bytes(dims(b=b, block=n)) for n in (*range(1, 700), 1 << 14, 1 << 20)]
        assert need == sorted(need)
    assert status_of(bmx.bm_win_validate, dims(dtype=3), 0) == UNSUP


def test_window_context_checks():
    d = dims()
    go = lambda c=None, sinks=4, pos=0, dd=d: status_of(                             # noqa: E731
        bmx.bm_win_resume, dd, sinks, fake_win(d) if c is None else c, pos)
    assert go() == bmx.BM_OK and go(pos=544) == bmx.BM_OK
    for name in ("k", "v", "work"):
        assert go(fake_win(d, **{name: 0})) == BAD, name
        assert go(fake_win(d, **{name: FAKE + 8})) == BAD, name
    assert go(fake_win(d, work_bytes=0)) == BAD and "work_bytes" in bmx.bm_last_error()
    assert go(pos=-1) == BAD and go(pos=545) == BAD and go(sinks=128) == BAD
    out, lib, p = ctypes.c_void_p(), bmx._lib, ctypes.byref
    c = fake_win(d)
    assert lib.bm_win_init(p(d), 4, None, p(out)) == BAD and lib.bm_win_init(None, 4, p(c), p(out)) == BAD
    assert lib.bm_win_init(p(d), 4, p(c), None) == BAD and lib.bm_win_resume(p(d), 4, p(c), 0, None) == BAD
    assert out.value is None
    ctx = win(100)
    assert (bmx.bm_ctx_len(ctx), bmx.bm_ctx_next_pos(ctx)) == (100, 100)
    bmx.bm_destroy(ctx)
    ctx = win(300)
    assert bmx.bm_ctx_len(ctx) == 128
    bmx.bm_destroy(ctx)


def test_window_settings_of_scores_and_cuts_are_refused():
    ctx = win(100)
    assert status_of(bmx.bm_set_rank_rule, ctx, bmx.BM_RANK_SUM) == UNSUP
    assert status_of(bmx.bm_set_decode_bound, ctx, 10) == UNSUP
    assert status_of(bmx.bm_set_decode_removal, ctx, 0) == UNSUP
    assert status_of(bmx.bm_set_score_accumulation, ctx, 1) == UNSUP
    assert status_of(bmx.bm_set_left_padding, ctx, FAKE) == bmx.BM_OK
    assert status_of(bmx.bm_set_left_padding, ctx, FAKE + 2) == BAD
    assert status_of(bmx.bm_evict_compact, ctx, 99, 0) == bmx.BM_OK       # nothing to cut
    assert status_of(bmx.bm_evict_compact, ctx, 98, 0) == ORDER
    assert bmx.bm_prefill_tile_workgroups(ctx, 1, FAKE, FAKE, 1) == -1
    bmx.bm_destroy(ctx)


@pytest.mark.parametrize("call", [bmx.bm_prefill_block, bmx.bm_prefill_block_cut])
def test_window_prompt_refuses(call):
    ctx = win(100)
    go = lambda t0=100, n=64, q=FAKE, k=FAKE, v=FAKE, o=FAKE, ld=512: status_of(     # noqa: E731
        call, ctx, t0, n, q, k, v, o, ld, 0)
    assert go(n=0) == BAD and go(n=65) == BAD and go(ld=63) == BAD
    for name in "qkvo":
        assert go(**{name: 0}) == BAD and go(**{name: FAKE + 8}) == BAD
    assert go(t0=99) == ORDER and go(t0=101) == ORDER
    bmx.bm_destroy(ctx)
    ctx = win(500)
    assert go(t0=500) == ORDER                                         # past the prompt
    bmx.bm_destroy(ctx)
    # more rows than one launch has workgroups
    ctx = win(0, b=1 << 20, n_kv_heads=8, n_heads=32, s=1 << 28, block=1 << 28)
    assert go(t0=0, n=1 << 28, ld=1 << 28) == UNSUP
    bmx.bm_destroy(ctx)


def test_window_step_refuses():
    ctx = win(512)
    go = lambda pos=512, q=FAKE, k=FAKE, v=FAKE, o=FAKE, ld=1: status_of(            # noqa: E731
        bmx.bm_decode_step, ctx, pos, q, k, v, o, ld, 0)
    assert go(ld=0) == BAD and go(pos=511) == ORDER and go(pos=513) == ORDER
    for name in "qkvo":
        assert go(**{name: 0}) == BAD and go(**{name: FAKE + 4}) == BAD
    bmx.bm_destroy(ctx)
    for pos in (511, 544):
        ctx = win(pos)
        assert go(pos=pos) == ORDER
        bmx.bm_destroy(ctx)


def contexts(next_pos=512, length=100, **kw):
    """A bounded and a window context at the same place."""
    d = dims(**kw)
    return (bmx.bm_resume(d, fake_cache(d), length, next_pos),
            bmx.bm_win_resume(d, 4, fake_win(d), next_pos))


def attend(ctx, n=5, parent=FAKE, q=FAKE, k=FAKE, v=FAKE, o=FAKE, ld=64, lse=0, work=FAKE, size=1 << 30):
    return status_of(bmx.bm_draft_attend, ctx, n, parent, q, k, v, o, ld, lse, work, size, 0)


def accept(ctx, n=5, m=3, path=FAKE, count=0, q=FAKE, k=FAKE, v=FAKE, ld=64, lse=FAKE):
    return status_of(bmx.bm_draft_accept, ctx, n, m, path, count, q, k, v, ld, lse, 0)


def test_draft_attend_refuses():
    for ctx in contexts():
        assert attend(ctx, n=0) == BAD and attend(ctx, n=65) == UNSUP and attend(ctx, ld=4) == BAD
        for name in ("parent", "q", "k", "v", "o", "work"):
            assert attend(ctx, **{name: 0}) == BAD, name
        for name in ("q", "k", "v", "o", "work"):
            assert attend(ctx, **{name: FAKE + 8}) == BAD, name
        for name in ("parent", "lse"):
            assert attend(ctx, **{name: FAKE + 2}) == BAD, name
        assert attend(ctx, size=bmx.bm_draft_workspace_bytes(dims(), 5) - 1) == BAD
        bmx.bm_destroy(ctx)
    for pos in (511, 544):
        for ctx in contexts(pos):
            assert attend(ctx) == ORDER
            bmx.bm_destroy(ctx)
    for ctx in contexts(length=129)[:1]:
        assert attend(ctx) == CAP
        bmx.bm_destroy(ctx)
    assert attend(None) == BAD


def test_draft_accept_refuses():
    for i, ctx in enumerate(contexts()):
        assert accept(ctx, n=0) == BAD and accept(ctx, n=65, m=1) == UNSUP and accept(ctx, ld=4) == BAD
        assert accept(ctx, m=0) == BAD and accept(ctx, m=6) == BAD
        for name in ("path", "k", "v"):
            assert accept(ctx, **{name: 0}) == BAD, name
        for name in ("path", "count", "lse"):
            assert accept(ctx, **{name: FAKE + 2}) == BAD, name
        for name in "qkv":
            assert accept(ctx, **{name: FAKE + 8}) == BAD, name
        assert accept(ctx, count=FAKE) == ORDER                       # no left padding to grow
        if i == 0:
            assert accept(ctx, q=0) == BAD and accept(ctx, lse=0) == BAD
        bmx.bm_destroy(ctx)
    for ctx in contexts(542):
        assert accept(ctx) == ORDER and "s + max_gen" in bmx.bm_last_error()
        bmx.bm_destroy(ctx)
    for ctx in contexts(511):
        assert accept(ctx) == ORDER
        bmx.bm_destroy(ctx)
    assert accept(None) == BAD


def test_draft_accept_of_a_bounded_cache():
    # free slots: cap = 128 + 2
    ctx = contexts(block=2, length=128)[0]
    assert accept(ctx) == CAP
    # above the decode bound: the attention cuts first
    bmx.bm_set_decode_bound(ctx, 100)
    assert accept(ctx, m=2) == ORDER and "decode bound" in bmx.bm_last_error()
    bmx.bm_destroy(ctx)
    # removals of more than one
    ctx = contexts()[0]
    bmx.bm_set_decode_removal(ctx, 2)
    assert attend(ctx) == UNSUP and accept(ctx) == UNSUP
    bmx.bm_destroy(ctx)
    # a cut by scores that this call does not add to
    ctx = contexts(length=127)[0]
    bmx.bm_set_score_accumulation(ctx, 0)
    assert accept(ctx, lse=0) == ORDER
    bmx.bm_destroy(ctx)


def test_four_bit_caches_are_refused():
    d = dims()
    ctx = bmx.bm_kv4_resume(d, fake_kv4(d), 100, 512)
    assert attend(ctx) == UNSUP and accept(ctx) == UNSUP
    bmx.bm_destroy(ctx)


def test_draft_workspace():
    assert bmx.bm_draft_workspace_bytes(dims(), 0) == 0
    assert bmx.bm_draft_workspace_bytes(dims(), 65) == 0
    assert bmx.bm_draft_workspace_bytes(dims(b=0), 5) == 0
    assert bmx.bm_draft_workspace_bytes(dims(block=1 << 20), 5) > 0       # a window context's
    for b in (1, 7, 4096):
        need = [bmx.bm_draft_workspace_bytes(dims(b=b), n) for n in range(1, 65)]
        assert need[0] > 0 and need == sorted(need)               # larger trees never need less


def test_window_attention_object_refuses():
    kw = dict(b=2, s=64, max_gen=8, n_heads=8, n_kv_heads=2, head_dim=64, device="cpu", init=False)
    for bad in (dict(window=0), dict(window=-3), dict(window=2**40), dict(window=8, sinks=-1)):
        with pytest.raises(ValueError):
            bmx.WindowAttention(**bad, **kw)
    with pytest.raises(ValueError):
        bmx.WindowAttention(window=8, static_workspace=True, **kw)
    with pytest.raises(bmx.BatchMaxError):
        bmx.WindowAttention(window=65535, sinks=1, **kw)
    att = bmx.WindowAttention(window=8, sinks=2, **kw)
    assert tuple(att.k.shape) == (2, 2, 10, 64) and att.k.dtype == torch.bfloat16 and att.dims.block == 64
    with pytest.raises(ValueError):
        att.resume(2**40)
    work = torch.empty(att.work_bytes, dtype=torch.uint8)
    good = [att.k, att.v, work]
    bmx.WindowAttention(window=8, sinks=2, buffers=good, **kw)
    for i, x in ((0, att.k.float()), (1, att.v[:, :, :9]), (2, work[:-1]), (0, att.k.transpose(0, 1))):
        with pytest.raises(ValueError):
            bmx.WindowAttention(window=8, sinks=2, buffers=good[:i] + [x] + good[i + 1:], **kw)


def test_draft_tensors_are_checked():
    kw = dict(b=2, s=64, kv_max=32, block=16, max_gen=8, n_heads=8, n_kv_heads=2, head_dim=64, device="cpu",
              init=False)
    att = bmx.PDAttention(**kw)
    q, k = torch.zeros((2, 8, 5, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 5, 64), dtype=torch.bfloat16)
    tree, path = torch.zeros((2, 5), dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32)
    for bad in (tree.long(), tree[:1], tree.t().contiguous().t(), torch.zeros(5, dtype=torch.int32)):
        with pytest.raises(ValueError):
            att.draft_attend(bad, q, k, k, q)
    with pytest.raises(ValueError):
        att.draft_attend(torch.zeros((2, 6), dtype=torch.int32), q, k, k, q)      # more nodes than rows
    with pytest.raises(ValueError):
        att.draft_attend(tree, q.float(), k, k, q)
    with pytest.raises(ValueError):
        att.draft_attend(tree, q, k, k[:, :, :4], q)
    with pytest.raises(ValueError):
        att.draft_attend(tree, q, k, k, q, row=-1)
    for lse in (torch.zeros((2, 8, 5), dtype=torch.float64), torch.zeros((2, 8, 4)), torch.zeros((2, 5, 8)).mT):
        with pytest.raises(ValueError):
            att.draft_attend(tree, q, k, k, q, lse=lse)
    for kw2 in (dict(count=torch.zeros(2)), dict(count=torch.zeros(3, dtype=torch.int32)), dict(n=6)):
        with pytest.raises(ValueError):
            att.draft_accept(path, q, k, k, **kw2)
    with pytest.raises(ValueError):
        att.draft_accept(path.long(), q, k, k)


def test_scratch_of_trees_is_counted():
    kw = dict(b=2, s=64, kv_max=32, block=16, max_gen=8, n_heads=8, n_kv_heads=2, head_dim=64, dtype="bf16")
    stack = bmx.PDStack(n_layers=3, device="cpu", **kw)
    need = stack.layers[0].draft_work_bytes()
    assert need == bmx.bm_draft_workspace_bytes(stack.layers[0].dims, bmx.BM_DRAFT_MAX)
    assert stack.layers[0].draft_work_bytes(5) == bmx.bm_draft_workspace_bytes(stack.layers[0].dims, 5) < need
    one = [layer._draft_scratch(None) for layer in stack.layers]
    assert one[0] == one[1] == one[2] and one[0][1] == need
    extra = bmx.stack_bytes(n_layers=3, drafts=True, **kw) - bmx.stack_bytes(n_layers=3, **kw)
    assert need <= extra < need + 256
    own = torch.empty(need // 4, dtype=torch.float32)
    assert stack.layers[1]._draft_scratch(own) == (own.data_ptr(), own.numel() * 4)
    with pytest.raises(ValueError):
        stack.layers[0]._draft_scratch(own[::2])
    with pytest.raises(ValueError):
        stack.layers[0]._draft_scratch(own.to("meta"))


def test_a_refused_resume_keeps_the_prompt_length():
    att = bmx.WindowAttention(window=8, sinks=2, b=2, s=64, max_gen=8, n_heads=8, n_kv_heads=2, head_dim=64,
                              device="cpu")
    att.resume(70, s=90)
    assert (att.dims.s, att.next_pos, att.length) == (90, 70, 10)
    for bad in (dict(next_pos=70, s=0), dict(next_pos=70, s=61), dict(next_pos=-1, s=80), dict(next_pos=70, s=2 ** 30)):
        with pytest.raises(bmx.BatchMaxError):
            att.resume(**bad)
        assert (att.dims.s, att.next_pos) == (90, 70)
    with pytest.raises(ValueError):
        att.resume(70, s=2 ** 40)
    assert (att.dims.s, att.next_pos) == (90, 70)
    att.resume(64)
    assert (att.dims.s, att.next_pos) == (90, 64)

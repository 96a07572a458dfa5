"""The bounded cache held in 4 bits on the GPU against a 64-bit reference."""
import math

import pytest
import torch

from kv4_reference import Reference, check, stored
from paper_2412_05693_amd import batchmax as bmx

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(*, b=2, s=64, kv_max=32, block=16, max_gen=64, heads=4, kv_heads=2, d=128, dtype="bf16", **kw):
    return bmx.PDAttentionKV4(b=b, s=s, kv_max=kv_max, block=block, max_gen=max_gen, n_heads=heads,
                              n_kv_heads=kv_heads, head_dim=d, dtype=dtype, **kw)


def rows(g, shape, dtype, spread=0.7):
    """N(0, 1) rows, each times a lognormal factor."""
    x = torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(shape[:-1] + (1,), generator=g))
    return x.to(DT[dtype]).cuda()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def junk(att):
    """Every byte of the cache's rows as a NaN group's (scale 255) before anything is stored."""
    for x in (att.k, att.v, att.k_scale, att.v_scale):
        x.fill_(255)


def live(att):
    n = att.length
    k, v = att.read_rows(0, n)
    return k.cpu().double(), v.cpu().double(), att.pos[:, :, :n].cpu().long(), att.score[:, :, :n]


def same_cache(att, ref, seen, steps, scores=True):
    """Live entries slot by slot: positions and rows exactly, scores within rounding."""
    k, v, pos, score = live(att)
    assert torch.equal(pos, ref.pos)
    assert torch.equal(torch.isnan(k), torch.isnan(ref.k)) and torch.equal(k.nan_to_num(), ref.k.nan_to_num())
    assert torch.equal(torch.isnan(v), torch.isnan(ref.v)) and torch.equal(v.nan_to_num(), ref.v.nan_to_num())
    assert (att.len == ref.n).all()
    if scores:
        check(score, ref.score, ref.score_tol(seen, steps), "scores")


# --------------------------------------------------------------------------
# rows in and out
# --------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("b,kv_heads,n,slot0", [(1, 1, 1, 0), (2, 3, 1, 47), (3, 2, 17, 5), (1, 5, 48, 0),
                                                (7, 4, 33, 15)])
def test_rows_store_and_read_back(dtype, d, b, kv_heads, n, slot0):
    att = make(b=b, heads=kv_heads, kv_heads=kv_heads, d=d, dtype=dtype, s=64)
    junk(att)
    att.score.fill_(3.0), att.pos.fill_(7), att.len.fill_(9)
    g = gen(d + n)
    other = [rows(g, (b, kv_heads, att.cap, d), dtype) for _ in range(2)]
    att.write_rows(0, *other)
    k, v = rows(g, (b, kv_heads, n, d), dtype, 2.0), rows(g, (b, kv_heads, n, d), dtype, 2.0)
    att.write_rows(slot0, k, v)
    # other slots, scores, positions and lengths are left alone
    for x, y in zip(att.read_rows(0, att.cap), other):
        x, y = x.cpu().double(), stored(y)
        assert torch.equal(x[:, :, :slot0], y[:, :, :slot0])
        assert torch.equal(x[:, :, slot0 + n:], y[:, :, slot0 + n:])
    assert (att.score == 3).all() and (att.pos == 7).all() and (att.len == 9).all()
    ko, vo = att.read_rows(slot0, n)
    assert ko.dtype == DT[dtype]
    assert torch.equal(ko.cpu().double(), stored(k)) and torch.equal(vo.cpu().double(), stored(v))
    # a row that was read back and is written again keeps its values
    att.write_rows(slot0, ko, vo)
    k2, v2 = att.read_rows(slot0, n)
    assert torch.equal(ko, k2) and torch.equal(vo, v2)
    # a group whose scale byte is 255 reads as NaN
    junk(att)
    assert torch.isnan(att.read_rows(0, att.cap)[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_format_at_its_edges(dtype):
    """Ties, group maxima at 6 and 1.5 times a power of two and just past them, zeros of both
    signs, values below and above the scales' range, infinities and NaN."""
    top = 3.3895313892515355e38 if dtype == "bf16" else 3.4028234663852886e38
    step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
    groups = [
        [6.0] + [i * 0.25 for i in range(24)] + [-i * 0.25 for i in range(7)],
        [1.5 * (1 + step)] + [0.1] * 31,
        [1.5] + [0.0, -0.0] * 15 + [-1.5],
        [3.0 * (1 - step / 2), 0.74, 0.76] + [1.26] * 29,
        [0.0] * 32,
        [-0.0] * 32,
        [1e-40, -3e-39] + [0.0] * 30,
        [2.0 ** -121, 2.0 ** -120, 3 * 2.0 ** -121, 2.0 ** -119] + [2.0 ** -126] * 28,
        [top, -top, 2.0 ** 127, 1.5 * 2.0 ** 127, 2.0 ** 125, -(2.0 ** 126)] + [1.0] * 26,
        [math.inf] + [1.0] * 31,
        [1.0] * 31 + [-math.inf],
        [0.5] * 16 + [math.nan] + [0.5] * 15,
    ]
    x = torch.tensor(groups, dtype=torch.float64).to(DT[dtype])
    x = x.view(1, 1, 3, 128).cuda()
    att = make(b=1, heads=1, kv_heads=1, kv_max=4, block=1, dtype=dtype)
    att.write_rows(1, x, x.flip(2).contiguous())
    k, v = att.read_rows(1, 3)
    want = stored(x)
    assert torch.equal(torch.isnan(k.cpu()), torch.isnan(want))
    assert torch.equal(k.cpu().double().nan_to_num(), want.nan_to_num())
    assert torch.equal(v.cpu().double().nan_to_num(), want.flip(2).nan_to_num())
    assert torch.equal(torch.isnan(want).sum(), torch.tensor(96))


def test_rows_by_their_stride():
    """The C calls take rows out of longer planes and leave the planes' other rows alone."""
    b, hk, d, ld, n = 2, 3, 64, 11, 4
    att = make(b=b, heads=hk, kv_heads=hk, d=d)
    g = gen(5)
    k, v = rows(g, (b, hk, ld, d), "bf16"), rows(g, (b, hk, ld, d), "bf16")
    stream = torch.cuda.current_stream().cuda_stream
    at = 3 * d * 2                      # rows 3..6 of every plane
    bmx.bm_kv4_write(att.dims, att.cache, 2, n, k.data_ptr() + at, v.data_ptr() + at, ld, stream)
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    bmx.bm_kv4_read(att.dims, att.cache, 2, n, ko.data_ptr() + at, vo.data_ptr() + at, ld, stream)
    for x, y in ((k, ko), (v, vo)):
        assert torch.equal(y[:, :, 3:3 + n].cpu().double(), stored(x[:, :, 3:3 + n]))
        assert (y[:, :, :3] == 7).all() and (y[:, :, 3 + n:] == 7).all()


# --------------------------------------------------------------------------
# decode
# --------------------------------------------------------------------------
def filled(att, ref, n, seed, dtype, first, ave=True):
    """The same n entries on both sides: random rows, positions below `first`, scores of
    distinct averages; junk behind them."""
    g = gen(seed)
    b, hk, d = ref.b, ref.hk, ref.d
    junk(att)
    k, v = rows(g, (b, hk, n, d), dtype), rows(g, (b, hk, n, d), dtype, 0.0)
    pos = torch.stack([torch.randperm(first, generator=g)[:n] for _ in range(b * hk)]).view(b, hk, n)
    score = torch.rand((b, hk, n), generator=g) * 0.3 + 0.01
    score = (score * (first - pos) if ave else score) * (pos >= ref.pads[:, None, None])
    att.score.fill_(math.nan), att.pos.fill_(1 << 29)
    if n:
        att.write_rows(0, k, v)
        att.pos[:, :, :n], att.score[:, :, :n] = pos.int().cuda(), score.cuda()
    att.len.fill_(n)
    ref.k, ref.v, ref.pos, ref.score = stored(k), stored(v), pos, score.float().double()
    ref.last = torch.zeros_like(ref.score)
    att.resume(n, first)


def step_rows(g, b, heads, hk, d, dtype, r=1):
    return (rows(g, (b, heads, r, d), dtype, 0.2), rows(g, (b, hk, r, d), dtype),
            rows(g, (b, hk, r, d), dtype, 0.0))


def decode(att, ref, pos, q, k, v, dtype, bound, rule="ave", scores=True):
    o = torch.full_like(q, 9.0)
    n = ref.n
    att.decode_step(pos, q, k, v, o)
    want = ref.attend(pos, q, k, v, scores)
    check(o, want, ref.out_tol(want, dtype, n + 1), "outputs")
    if ref.n > bound:
        ref.cut(bound, pos, rule, att.pos[:, :, :bound])
    assert att.length == ref.n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 4])
@pytest.mark.parametrize("n", [0, 1, 15, 63, 64, 65, 130, 257, 601])
def test_decode_step(dtype, d, group, n):
    """Steps over a cache that grows, over one at its bound, with every boundary of tiles."""
    b, hk, first = 2, 3, max(2 * n, 8)
    bound = n + 2                       # two steps append, the next two remove
    att = make(b=b, s=first, kv_max=bound, block=1, heads=hk * group, kv_heads=hk, d=d, dtype=dtype)
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d)
    filled(att, ref, n, 7 * n + d, dtype, first)
    g = gen(n)
    for i in range(4):
        decode(att, ref, first + i, *step_rows(g, b, hk * group, hk, d, dtype), dtype, bound)
        same_cache(att, ref, n + 4, i + 1)


@pytest.mark.parametrize("dtype,d,group", [("bf16", 128, 4), ("bf16", 64, 2), ("f32", 128, 1), ("f32", 64, 4)])
@pytest.mark.parametrize("n,padded", [(127, False), (300, True), (1023, False)])
def test_decode_step_of_many_units(dtype, d, group, n, padded):
    """More units than every compute unit's three, which take one wave each up to 1023
    entries: a step that appends and one that removes."""
    b, hk, first = 771, 1, 2 * n
    pads = torch.randint(0, first, (b,), generator=gen(n), dtype=torch.int32) if padded else None
    att = make(b=b, s=first, kv_max=n + 1, block=1, heads=hk * group, kv_heads=hk, d=d, dtype=dtype)
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d, pads=pads)
    if padded:
        att.set_left_padding(pads.cuda())
    filled(att, ref, n, n + d, dtype, first)
    g = gen(n)
    for i in range(2):
        decode(att, ref, first + i, *step_rows(g, b, hk * group, hk, d, dtype), dtype, n + 1)
        same_cache(att, ref, n + 2, i + 1)


@pytest.mark.parametrize("rule", ["sum", "recent", "tova"])
@pytest.mark.parametrize("group", [1, 4])
def test_decode_rules_and_removal_schedules(rule, group):
    b, hk, d, n, first, dtype = 2, 2, 64, 70, 150, "bf16"
    att = make(b=b, s=first, kv_max=n, block=1, heads=hk * group, kv_heads=hk, d=d, dtype=dtype)
    att.set_rank_rule(rule)
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d)
    filled(att, ref, n, 11, dtype, first, ave=False)
    g = gen(3)
    for i in range(5):
        decode(att, ref, first + i, *step_rows(g, b, hk * group, hk, d, dtype), dtype, n, rule)
        same_cache(att, ref, n + 5, i + 1)
    # Algorithm 1's loop: a full cache first loses p entries (rows moved in 4 bits)
    att.set_decode_removal(9)
    q, k, v = step_rows(g, b, hk * group, hk, d, dtype)
    o = torch.empty_like(q)
    att.decode_step(first + 5, q, k, v, o)
    ref.cut(n - 9, first + 4, rule, att.pos[:, :, :n - 9])
    want = ref.attend(first + 5, q, k, v)
    check(o, want, ref.out_tol(want, dtype, n), "outputs")
    same_cache(att, ref, n + 5, 6)
    # a lower decode bound: a cut, then one removal a step
    att.set_decode_removal(0)
    att.set_decode_bound(20)
    q, k, v = step_rows(g, b, hk * group, hk, d, dtype)
    before = ref.n
    att.decode_step(first + 6, q, k, v, o)
    assert before > 20 and att.length == 20


@pytest.mark.parametrize("n", [4095, 4096])
def test_longest_scoring_step(n):
    """The largest cache that a scoring step takes: 4096 entries and the step's own."""
    b, hk, group, d, dtype, first = 1, 2, 4, 128, "bf16", 9000
    att = make(b=b, s=first, kv_max=4096, block=1, heads=hk * group, kv_heads=hk, d=d, dtype=dtype)
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d)
    filled(att, ref, n, 1, dtype, first)
    g = gen(2)
    for i in range(2):
        decode(att, ref, first + i, *step_rows(g, b, hk * group, hk, d, dtype), dtype, 4096)
    same_cache(att, ref, n, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [5, 64, 100, 300])
def test_hidden_entries_weigh_nothing(dtype, n):
    """Left padding: pad rows that read back as NaN or as the largest values, a sample
    whose every cached entry is a pad, one with none."""
    b, hk, group, d = 3, 2, 2, 128
    first = n
    pads = torch.tensor([0, n // 2, n], dtype=torch.int32)
    att = make(b=b, s=first, kv_max=n + 4, block=1, heads=hk * group, kv_heads=hk, d=d, dtype=dtype)
    att.set_left_padding(pads.cuda())
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d, pads=pads)
    filled(att, ref, n, 4, dtype, first)
    bad = ref.pos < pads[:, None, None]
    assert bad.any()
    for i, x in enumerate(att.read_rows(0, n)):
        x[(bad & (ref.pos % 2 == i)).cuda()] = math.nan
        x[(bad & (ref.pos % 2 != i)).cuda()] = 2.5e38
        y = att.read_rows(0, n)
        att.write_rows(0, *((x, y[1]) if i == 0 else (y[0], x)))
    k, v, _, _ = live(att)
    ref.k, ref.v = k, v
    assert not torch.isfinite(ref.k).all()
    g = gen(6)
    for i in range(3):
        decode(att, ref, first + i, *step_rows(g, b, hk * group, hk, d, dtype), dtype, n + 4)
    same_cache(att, ref, n + 3, 3)


def test_visible_nan_reaches_its_unit_alone():
    b, hk, group, d, n, first, dtype = 2, 2, 2, 64, 90, 200, "bf16"
    att = make(b=b, s=first, kv_max=n + 1, block=1, heads=hk * group, kv_heads=hk, d=d, dtype=dtype)
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d)
    filled(att, ref, n, 4, dtype, first)
    k, v = att.read_rows(0, n)
    k[0, 0, 3, 40] = math.nan           # a key: all of unit (0, 0)
    v[1, 1, 89, 5] = math.inf           # a value: 32 elements of unit (1, 1)'s outputs
    att.write_rows(0, k, v)
    q, k, v = step_rows(gen(1), b, hk * group, hk, d, dtype)
    o = torch.zeros_like(q)
    att.decode_step(first, q, k, v, o)
    want = torch.zeros_like(q, dtype=torch.bool)
    want[0, :group] = True
    want[1, group:, :, :32] = True
    assert torch.equal(torch.isnan(o), want)


@pytest.mark.parametrize("dtype,d,group", [("bf16", 128, 4), ("bf16", 64, 1), ("f32", 128, 2), ("f32", 64, 4)])
@pytest.mark.parametrize("n", [4097, 5000, 8192])
def test_long_decode(dtype, d, group, n):
    b, hk = 2, 2
    pads = torch.tensor([0, 1500], dtype=torch.int32)
    att = make(b=b, s=n, kv_max=n + 2, block=1, heads=hk * group, kv_heads=hk, d=d, dtype=dtype)
    att.set_score_accumulation(False)
    att.set_left_padding(pads.cuda())
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d, pads=pads)
    filled(att, ref, n, n + d, dtype, n)
    k, v = att.read_rows(0, n)
    for x in (k, v):
        x[(ref.pos < pads[:, None, None]).cuda()] = math.nan
    att.write_rows(0, k, v)
    ref.k, ref.v = live(att)[:2]
    g = gen(9)
    for i in range(2):
        q, k, v = step_rows(g, b, hk * group, hk, d, dtype)
        o = torch.empty_like(q)
        att.decode_step(n + i, q, k, v, o)
        want = ref.attend(n + i, q, k, v, scores=False)
        check(o, want, ref.out_tol(want, dtype, n), "outputs")
    same_cache(att, ref, n, 2, scores=False)
    assert (att.score[:, :, n:n + 2] == 0).all()


# --------------------------------------------------------------------------
# prefill and cuts
# --------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,group", [(64, 1), (64, 4), (128, 2)])
@pytest.mark.parametrize("n,r", [(0, 1), (0, 33), (1, 64), (50, 7), (130, 65), (257, 100)])
def test_prefill_block(dtype, d, group, n, r):
    b, hk = 2, 2
    att = make(b=b, s=n + r, kv_max=max(n, 1), block=r, heads=hk * group, kv_heads=hk, d=d, dtype=dtype)
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d)
    filled(att, ref, n, n + r, dtype, n)
    q, k, v = step_rows(gen(r), b, hk * group, hk, d, dtype, r)
    o = torch.empty_like(q)
    att.prefill_block(n, r, q, k, v, o, row=0)
    want = ref.attend(n, q, k, v)
    # (a block's probabilities are one bfloat16 each)
    check(o, want, ref.out_tol(want, dtype, n + r, 2.0 ** -8), "outputs")
    same_cache(att, ref, n + r, r)


@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("rule", ["ave", "tova"])
@pytest.mark.parametrize("dtype,d,group,padded", [("bf16", 128, 4, False), ("bf16", 64, 2, True),
                                                  ("f32", 64, 1, False), ("f32", 128, 2, True)])
def test_prompt_and_generation(fused, rule, dtype, d, group, padded):
    """The whole schedule: blocks (the last one partial), cuts that move 4-bit rows,
    decode steps with one removal each."""
    b, hk, s, kv_max, block, gen_steps = 3, 2, 203, 56, 40, 6
    pads = torch.tensor([0, 30, 75], dtype=torch.int32) if padded else None
    att = make(b=b, s=s, kv_max=kv_max, block=block, max_gen=gen_steps, heads=hk * group, kv_heads=hk,
               d=d, dtype=dtype)
    junk(att)
    att.set_rank_rule(rule)
    if padded:
        att.set_left_padding(pads.cuda())
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d, pads=pads)
    q, k, v = step_rows(gen(d + group), b, hk * group, hk, d, dtype, s + gen_steps)
    o = torch.empty_like(q)
    for t0 in range(0, s, block):
        r = min(block, s - t0)
        at = slice(t0, t0 + r)
        if fused:
            att.prefill_block_cut(t0, r, q, k, v, o)
        else:
            att.prefill_block(t0, r, q, k, v, o)
            att.evict_compact(t0 + r - 1)
        want = ref.attend(t0, q[:, :, at], k[:, :, at], v[:, :, at])
        check(o[:, :, at], want, ref.out_tol(want, dtype, 96, 2.0 ** -8), f"block {t0}")
        if ref.n > kv_max:
            ref.cut(kv_max, t0 + r - 1, rule, att.pos[:, :, :kv_max])
        same_cache(att, ref, 96, t0 + r)
    for i in range(gen_steps):
        at = slice(s + i, s + i + 1)
        att.decode_step(s + i, q, k, v, o, row=s + i)
        want = ref.attend(s + i, q[:, :, at], k[:, :, at], v[:, :, at])
        check(o[:, :, at], want, ref.out_tol(want, dtype, 57), f"step {i}")
        ref.cut(kv_max, s + i, rule, att.pos[:, :, :kv_max])
        same_cache(att, ref, 96, s + i + 1)


@pytest.mark.parametrize("dtype,d,group,padded", [("bf16", 128, 4, False), ("bf16", 64, 2, True),
                                                  ("f32", 64, 1, True)])
def test_rows_left_in_the_workspace_change_nothing(dtype, d, group, padded):
    """The space for rows read back holds NaN, or zeros, before every call: the same bits."""
    b, hk, s, kv_max, block = 2, 2, 203, 57, 39
    q, k, v = step_rows(gen(7), b, hk * group, hk, d, dtype, s + 2)
    got = []
    for fill in (0, 255):
        att = make(b=b, s=s, kv_max=kv_max, block=block, max_gen=2, heads=hk * group, kv_heads=hk, d=d,
                   dtype=dtype)
        junk(att)
        if padded:
            att.set_left_padding(torch.tensor([0, 75], dtype=torch.int32).cuda())
        rows_at = -(-bmx.bm_workspace_bytes(att.dims) // 256) * 256
        o = torch.zeros_like(q)
        for t0 in range(0, s, block):
            att.work[rows_at:].fill_(fill)
            att.prefill_block_cut(t0, min(block, s - t0), q, k, v, o)
        for i in range(2):
            att.work[rows_at:].fill_(fill)
            att.decode_step(s + i, q, k, v, o, row=s + i)
        got.append((o, *live(att)))
    assert all(torch.equal(x, y) for x, y in zip(*got, strict=True))
    assert torch.isfinite(got[0][0]).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,keep", [(700, 400), (1000, 999), (2500, 1500), (4600, 4000)])
def test_cut_moves_codes_and_scales(d, n, keep):
    """Cuts of every kind (one launch, select and compaction, streamed keys): kept rows come
    along bit for bit, kept slots below the bound stay where they are."""
    b, hk = 2, 2
    att = make(b=b, s=n + 5, kv_max=keep, block=n - keep, heads=hk, kv_heads=hk, d=d)
    att.set_rank_rule("sum")
    ref = Reference(b=b, heads=hk, kv_heads=hk, d=d)
    filled(att, ref, n, n, "bf16", n + 5, ave=False)
    before = att.pos.clone()
    att.evict_compact(n + 4)
    ref.cut(keep, n + 4, "sum", att.pos[:, :, :keep])
    same_cache(att, ref, 1, 0)
    gone = ~(before[:, :, :keep, None] == att.pos[:, :, None, :keep]).any(dim=3)
    assert torch.equal(before[:, :, :keep][~gone], att.pos[:, :, :keep][~gone])


# --------------------------------------------------------------------------
# streams, graphs, batches, memory
# --------------------------------------------------------------------------
def state_of(att, n):
    """Every live entry, bit for bit (slots past them are scratch)."""
    return [*att.read_rows(0, n), att.score[:, :, :n].clone(), att.pos[:, :, :n].clone(), att.len.clone()]


def same_state(att, other, n):
    for x, y in zip(state_of(att, n), other):
        assert torch.equal(x, y)


def test_graph_of_steps_replays():
    b, hk, group, d, n, first, steps, dtype = 4, 2, 4, 128, 200, 400, 5, "bf16"
    att = make(b=b, s=first, kv_max=n, block=1, max_gen=steps, heads=hk * group, kv_heads=hk, d=d)
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d)
    q, k, v = step_rows(gen(3), b, hk * group, hk, d, dtype, steps)
    names = ("k", "v", "k_scale", "v_scale", "score", "pos", "len")
    filled(att, ref, n, 8, dtype, first)
    start = {x: getattr(att, x).clone() for x in names}
    o = torch.zeros_like(q)
    att.run_decode(q, k, v, o, steps, 0)
    eager, want = state_of(att, n), o.clone()
    att.resume(n, first)
    graph = att.capture_decode(q, k, v, o, steps, 0)
    for _ in range(4):
        for x in names:
            getattr(att, x).copy_(start[x])
        o.zero_()
        att.read_rows(0, 3)                       # eager work between the replays
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)
        same_state(att, eager, n)


def test_long_step_in_a_graph():
    b, hk, group, d, n, dtype = 2, 2, 4, 64, 6000, "bf16"
    att = make(b=b, s=n, kv_max=n + 1, block=1, heads=hk * group, kv_heads=hk, d=d)
    att.set_score_accumulation(False)
    filled(att, Reference(b=b, heads=hk * group, kv_heads=hk, d=d), n, 8, dtype, n)
    q, k, v = step_rows(gen(3), b, hk * group, hk, d, dtype)
    o, want = torch.zeros_like(q), torch.zeros_like(q)
    att.decode_step(n, q, k, v, want)
    att.resume(n, n)
    graph = att.capture_decode(q, k, v, o, 1, 0)
    for _ in range(3):
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)


def test_prefill_block_in_a_graph():
    b, hk, group, d, n, r, dtype = 2, 2, 2, 128, 100, 48, "bf16"
    att = make(b=b, s=n + r, kv_max=n, block=r, heads=hk * group, kv_heads=hk, d=d)
    filled(att, Reference(b=b, heads=hk * group, kv_heads=hk, d=d), n, 8, dtype, n)
    names = ("k", "v", "k_scale", "v_scale", "score", "pos", "len")
    start = {x: getattr(att, x).clone() for x in names}
    q, k, v = step_rows(gen(3), b, hk * group, hk, d, dtype, r)
    o = torch.zeros_like(q)
    att.prefill_block_cut(n, r, q, k, v, o, row=0)
    want, eager = o.clone(), state_of(att, n)
    att.resume(n, n)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        att.prefill_block_cut(n, r, q, k, v, o, row=0)
    for _ in range(3):
        for x in names:
            getattr(att, x).copy_(start[x])
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)
        same_state(att, eager, n)


def test_calls_run_on_the_current_stream():
    b, hk, d, n, dtype = 2, 2, 128, 100, "bf16"
    att = make(b=b, s=n, kv_max=n, block=1, heads=hk, kv_heads=hk, d=d)
    ref = Reference(b=b, heads=hk, kv_heads=hk, d=d)
    filled(att, ref, n, 8, dtype, n)
    q, k, v = step_rows(gen(3), b, hk, hk, d, dtype)
    o = torch.zeros_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device="cuda")
        late = torch.zeros_like(q)
        for _ in range(20):
            big = big @ big * 1e-3
        late.copy_(q)                              # behind the products on this stream
        att.decode_step(n, late, k, v, o)
    side.synchronize()
    want = ref.attend(n, q, k, v)
    check(o, want, ref.out_tol(want, dtype, n + 1), "outputs")


def test_another_current_device_is_refused(monkeypatch):
    att = make()
    x = torch.zeros(2, 2, 3, 128, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(2, 4, 64, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 2, 64, 128, dtype=torch.bfloat16, device="cuda")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: att.device.index + 1)
    for call in (lambda: att.write_rows(0, x, x), lambda: att.read_rows(0, 3, x, x.clone()),
                 lambda: att.prefill_block(0, 16, q, k, k, q), lambda: att.evict_compact(-1),
                 lambda: att.decode_step(64, q, k, k, q)):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert att.length == 0 and att.next_pos == 0


def test_whole_prompt_kept_then_a_long_step():
    """Blocks without score sums, nothing removed, then steps over more entries than a
    scoring one takes (the full-cache comparator on a 4-bit cache)."""
    b, hk, group, d, s, block, steps, dtype = 1, 2, 2, 64, 4200, 1024, 2, "bf16"
    att = make(b=b, s=s, kv_max=s + steps, block=block, max_gen=steps, heads=hk * group, kv_heads=hk, d=d)
    att.set_score_accumulation(False)
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d)
    q, k, v = step_rows(gen(4), b, hk * group, hk, d, dtype, s + steps)
    o = torch.empty_like(q)
    att.run_prefill(q, k, v, o, fused_cut=True)
    att.run_decode(q, k, v, o)
    for t0 in (*range(0, s, block), *range(s, s + steps)):
        r = min(block, s - t0) if t0 < s else 1
        at = slice(t0, t0 + r)
        want = ref.attend(t0, q[:, :, at], k[:, :, at], v[:, :, at], scores=False)
        check(o[:, :, at], want, ref.out_tol(want, dtype, s, 2.0 ** -8), f"position {t0}")
    same_cache(att, ref, s, 1, scores=False)


@pytest.mark.parametrize("n", [100, 300, 1500])
def test_a_sample_has_the_same_bits_in_any_batch(n):
    hk, group, d, dtype, first = 2, 4, 128, "bf16", 4000
    g = gen(n)
    k, v = rows(g, (1, hk, n, d), dtype), rows(g, (1, hk, n, d), dtype)
    pos = torch.randperm(first, generator=g)[:n].int().cuda()
    score = torch.rand((1, hk, n), generator=g).cuda()
    q1, k1, v1 = step_rows(g, 1, hk * group, hk, d, dtype)
    got = []
    for b in (1, 3, 400):               # 2 to 800 units: one wave per unit and four
        att = make(b=b, s=first, kv_max=n, block=1, heads=hk * group, kv_heads=hk, d=d)
        rep = lambda x: x.expand(b, *x.shape[1:]).contiguous()    # noqa: E731
        att.write_rows(0, rep(k), rep(v))
        att.pos[:, :, :n], att.score[:, :, :n] = pos, rep(score)
        att.len.fill_(n)
        att.resume(n, first)
        o = torch.zeros(b, hk * group, 1, d, dtype=DT[dtype], device="cuda")
        att.decode_step(first, rep(q1), rep(k1), rep(v1), o)
        got.append((o, att.score[:, :, :n].clone(), att.pos[:, :, :n].clone()))
    for x in got:
        for y, z in zip(x, got[0]):
            assert (y == z[:1]).all()


def test_layers_share_one_workspace():
    """A stack of 4-bit layers in one arena: each layer's results are its own."""
    shape = dict(b=2, s=100, kv_max=40, block=30, max_gen=4, n_heads=8, n_kv_heads=2, head_dim=64)
    stack = bmx.PDStack(n_layers=3, kv_bits=4, **shape)
    one = [bmx.PDAttentionKV4(**shape) for _ in range(3)]
    stack.reset()
    ins = [step_rows(gen(i), 2, 8, 2, 64, "bf16", 104) for i in range(3)]
    outs = [[torch.zeros_like(x[0]) for x in ins] for _ in range(2)]
    for t0 in range(0, 100, 30):
        r = min(30, 100 - t0)
        for which, atts in enumerate((stack.layers, one)):
            for att, (q, k, v), o in zip(atts, ins, outs[which]):
                att.prefill_block_cut(t0, r, q, k, v, o)
    for i in range(4):
        for which, atts in enumerate((stack.layers, one)):
            for att, (q, k, v), o in zip(atts, ins, outs[which]):
                att.decode_step(100 + i, q, k, v, o, row=100 + i)
    for i in range(3):
        assert torch.equal(outs[0][i], outs[1][i])
        for x, y in zip(live(stack.layers[i]), live(one[i])):
            assert torch.equal(x, y)
    per = bmx.stack_layer_bytes(b=2, kv_max=40, block=30, n_kv_heads=2, head_dim=64, dtype="bf16", kv_bits=4)
    assert stack.arena_bytes >= 3 * per


def test_offsets_past_32_bits():
    """Codes of more than 2^32 bytes, rows and outputs of the last unit."""
    b, hk, d, n, cap, dtype = 70, 16, 128, 6000, 65000, "bf16"
    assert b * hk * cap * (d // 2) > 1 << 32         # bytes of each code plane
    att = make(b=b, s=n, kv_max=cap - 1, block=1, heads=hk, kv_heads=hk, d=d)
    att.set_score_accumulation(False)
    for x in (att.k, att.v, att.k_scale, att.v_scale):
        x.zero_()
    g = gen(1)
    k, v = rows(g, (1, 1, n, d), dtype), rows(g, (1, 1, n, d), dtype)
    zero = torch.zeros((b, hk, n, d), dtype=DT[dtype], device="cuda")
    kk, vv = zero.clone(), zero.clone()
    kk[-1, -1], vv[-1, -1] = k[0, 0], v[0, 0]
    att.write_rows(0, kk, vv)
    att.read_rows(0, n, kk, vv)
    assert torch.equal(kk[-1, -1].cpu().double(), stored(k)[0, 0]) and (kk[:-1] == 0).all()
    assert torch.equal(vv[-1, -1].cpu().double(), stored(v)[0, 0]) and (vv[:, :-1] == 0).all()
    att.resume(n, n)
    q1, k1, v1 = step_rows(g, b, hk, hk, d, dtype)
    o = torch.zeros_like(q1)
    att.decode_step(n, q1, k1, v1, o)
    ref = Reference(b=1, heads=1, kv_heads=1, d=d)
    ref.k, ref.v = stored(k), stored(v)
    ref.pos = torch.zeros((1, 1, n), dtype=torch.long)
    ref.score = torch.zeros((1, 1, n), dtype=torch.float64)
    last = lambda x: x[-1:, -1:]                               # noqa: E731
    want = ref.attend(n, last(q1), last(k1), last(v1), scores=False)
    check(last(o), want, ref.out_tol(want, dtype, n), "outputs")

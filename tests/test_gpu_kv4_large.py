"""The 4-bit cache at sizes that take launches of their own: caches past the last-level
cache (non-temporal loads), row launches of many pairs in both directions, prefill blocks
of a large batch, and a decode bound lowered below the cache's entries."""
import math

import pytest
import torch

from kv4_reference import Reference, check
from test_gpu_kv4 import decode, filled, gen, make, same_cache, step_rows

pytestmark = pytest.mark.gpu

LAST_LEVEL = 256 << 20       # bytes of cached entries from which loads are non-temporal


def tiled(x, b):
    return x.repeat(b // x.shape[0], *[1] * (x.dim() - 1))


def same_tiles(big, small, what):
    """Every sample of `big` is the one of `small` that it repeats, bit for bit."""
    m = small.shape[0]
    kind = {2: torch.int16, 4: torch.int32}[small.element_size()]
    x, y = big.contiguous().view(kind).view(-1, *small.shape), small.contiguous().view(kind)
    for i in range(m):
        assert torch.equal(x[:, i], y[i].expand_as(x[:, i])), f"{what}: samples like {i}"


def repeated(att, small, b, n, first):
    """att's cache: sample i holds what sample i % m of `small` does."""
    k, v = (tiled(x, b) for x in small.read_rows(0, n))
    att.write_rows(0, k, v)
    att.pos[:, :, :n], att.score[:, :, :n] = tiled(small.pos[:, :, :n], b), tiled(small.score[:, :, :n], b)
    att.len.fill_(n)
    att.resume(n, first)


def both_steps(small, big, ref, pos, ins, dtype, scores=True):
    """One decode step of the small launch, as the reference's, and of the big one, as the small's."""
    q, b = ins[0], big.dims.b
    o, o_big = torch.full_like(q, 9.0), torch.full_like(tiled(q, b), 9.0)
    n = ref.n
    small.decode_step(pos, *ins, o)
    big.decode_step(pos, *(tiled(x, b) for x in ins), o_big)
    want = ref.attend(pos, *ins, scores)
    check(o, want, ref.out_tol(want, dtype, n + 1), "outputs")
    same_tiles(o_big, o, "outputs")


def same_entries(big, small):
    n = small.length
    assert big.length == n and (big.len == n).all()
    same_tiles(big.score[:, :, :n], small.score[:, :, :n], "scores")
    same_tiles(big.pos[:, :, :n], small.pos[:, :, :n], "positions")
    for x, y in zip(big.read_rows(0, n), small.read_rows(0, n)):
        same_tiles(x, y, "rows")


def past_last_level(m, n, entry):
    """The fewest whole repetitions of m samples whose entries exceed the last-level cache."""
    b = m * (LAST_LEVEL // (m * n * entry) + 1)
    assert b * n * entry > LAST_LEVEL
    return b


@pytest.mark.parametrize("dtype,d,group", [("bf16", 128, 4), ("bf16", 64, 2), ("f32", 128, 1), ("f32", 64, 4)])
@pytest.mark.parametrize("n", [509, 1301])      # one wave a unit, and four
@pytest.mark.parametrize("padded", [False, True])
def test_decode_over_a_cache_past_the_last_level(dtype, d, group, n, padded):
    """A step that appends and one that removes: each sample as in a batch of five (four
    waves, loads through the caches), and those five as the reference."""
    m, first = 5, 2 * n
    b = past_last_level(m, n, d + d // 16 + 8)
    pads = torch.randint(0, first, (m,), generator=gen(n), dtype=torch.int32) if padded else None
    small, big = (make(b=x, s=first, kv_max=n + 1, block=1, heads=group, kv_heads=1, d=d, dtype=dtype)
                  for x in (m, b))
    ref = Reference(b=m, heads=group, kv_heads=1, d=d, pads=pads)
    if padded:
        small.set_left_padding(pads.cuda())
        big.set_left_padding(tiled(pads, b).cuda())
    filled(small, ref, n, n + d, dtype, first)
    repeated(big, small, b, n, first)
    g = gen(n)
    for i in range(2):
        both_steps(small, big, ref, first + i, step_rows(g, m, group, 1, d, dtype), dtype)
        if ref.n > n + 1:
            ref.cut(n + 1, first + i, "ave", small.pos[:, :, :n + 1])
        same_cache(small, ref, n + 2, i + 1)
        same_entries(big, small)


@pytest.mark.parametrize("dtype,d,group", [("bf16", 128, 4), ("bf16", 64, 2), ("f32", 128, 2), ("f32", 64, 1)])
def test_long_decode_past_the_last_level(dtype, d, group):
    m, n = 3, 4501
    b = past_last_level(m, n, d + d // 16)
    pads = torch.tensor([0, 700, 4501], dtype=torch.int32)
    small, big = (make(b=x, s=n, kv_max=n + 2, block=1, heads=group, kv_heads=1, d=d, dtype=dtype) for x in (m, b))
    ref = Reference(b=m, heads=group, kv_heads=1, d=d, pads=pads)
    for att, x in ((small, pads), (big, tiled(pads, b))):
        att.set_score_accumulation(False)
        att.set_left_padding(x.cuda())
    filled(small, ref, n, n + d, dtype, n)
    k, v = small.read_rows(0, n)
    for x in (k, v):
        x[(ref.pos < pads[:, None, None]).cuda()] = math.nan
    small.write_rows(0, k, v)
    ref.k, ref.v = (x.cpu().double() for x in small.read_rows(0, n))
    repeated(big, small, b, n, n)
    g = gen(9)
    for i in range(2):
        both_steps(small, big, ref, n + i, step_rows(g, m, group, 1, d, dtype), dtype, scores=False)
        same_cache(small, ref, n, 1, scores=False)
        same_entries(big, small)


@pytest.mark.parametrize("dtype,d,group,padded", [("bf16", 128, 2, False), ("bf16", 64, 4, True),
                                                  ("f32", 128, 1, True), ("f32", 64, 2, False)])
def test_prefill_block_of_many_rows(dtype, d, group, padded):
    """More than 2^16 row pairs read back and stored by one launch, both directions ending
    inside a workgroup (of 64 pairs, or 128); then the cut of every unit."""
    b, hk, n, r = 37, 5, 301, 77
    units = b * hk
    assert units * (n + r) >= 1 << 16 and units * n % 64 and units * r % 64
    pads = torch.randint(0, n + r, (b,), generator=gen(d), dtype=torch.int32) if padded else None
    att = make(b=b, s=n + r, kv_max=n, block=r, heads=hk * group, kv_heads=hk, d=d, dtype=dtype)
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d, pads=pads)
    if padded:
        att.set_left_padding(pads.cuda())
    filled(att, ref, n, n + r, dtype, n)
    q, k, v = step_rows(gen(r), b, hk * group, hk, d, dtype, r)
    o = torch.empty_like(q)
    att.prefill_block(n, r, q, k, v, o, row=0)
    want = ref.attend(n, q, k, v)
    check(o, want, ref.out_tol(want, dtype, n + r, 2.0 ** -8), "outputs")
    same_cache(att, ref, n + r, r)
    att.evict_compact(n + r - 1)
    ref.cut(n, n + r - 1, "ave", att.pos[:, :, :n])
    same_cache(att, ref, n + r, r)


def ranked_cut(ref, keep, curr, rule):
    """The reference's own cut: the smallest (key, position) leave, and the survivors behind
    slot keep - 1 take the holes in front of it, both in slot order."""
    age = (curr + 1 - ref.pos).double()
    key = {"ave": ref.score / age, "sum": ref.score, "recent": ref.pos.double(), "tova": ref.last}[rule]
    rank = key.sort(dim=2).values
    leaves, stays = rank[:, :, ref.n - keep - 1], rank[:, :, ref.n - keep]
    assert (stays > leaves * (1 + 1e-4)).all()         # (rounding decides nothing)
    gone = key <= leaves[:, :, None]
    idx = torch.arange(keep).repeat(ref.b, ref.hk, 1)
    for u in range(ref.b):
        for h in range(ref.hk):
            holes = gone[u, h, :keep].nonzero()[:, 0]
            idx[u, h, holes] = keep + (~gone[u, h, keep:]).nonzero()[:, 0]
    for name in ("pos", "score", "last"):
        setattr(ref, name, getattr(ref, name).gather(2, idx))
    for name in ("k", "v"):
        x = getattr(ref, name)
        setattr(ref, name, x.gather(2, idx[..., None].expand(-1, -1, -1, ref.d)))


@pytest.mark.parametrize("rule", ["ave", "sum", "recent", "tova"])
@pytest.mark.parametrize("dtype,d,group,n,bound", [("bf16", 64, 1, 70, 20), ("bf16", 128, 4, 1300, 700),
                                                   ("f32", 128, 2, 90, 64)])
def test_a_lowered_bound_cuts_and_then_removes(rule, dtype, d, group, n, bound):
    """A step over more entries than the bound: a cut to it, ranked at the last position,
    then the step's own removal; and one more step, which only removes."""
    b, hk, first = 2, 2, 2 * n
    att = make(b=b, s=first, kv_max=n + 2, block=1, heads=hk * group, kv_heads=hk, d=d, dtype=dtype)
    att.set_rank_rule(rule)
    ref = Reference(b=b, heads=hk * group, kv_heads=hk, d=d)
    filled(att, ref, n, 13, dtype, first, ave=rule == "ave")
    g = gen(8)
    decode(att, ref, first, *step_rows(g, b, hk * group, hk, d, dtype), dtype, n + 2, rule)
    att.set_decode_bound(bound)
    ranked_cut(ref, bound, first, rule)
    for i in (1, 2):
        decode(att, ref, first + i, *step_rows(g, b, hk * group, hk, d, dtype), dtype, bound, rule)
        same_cache(att, ref, n + 3, i + 1)

"""Attention with a sliding window and sinks against a 64-bit reference that keeps every
token (tests/window_reference.py)."""
import pytest
import torch

from paper_2412_05693_amd import batchmax as bmx
from window_reference import WindowReference, check_rows

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN = float("nan")


def rows(seed, b, heads, t, d, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((b, heads, t, d), generator=g) * scale).to(DT[dtype])


class Run:
    """A window cache and its reference, driven side by side."""

    def __init__(self, *, dtype="bf16", b=2, heads=4, kv_heads=1, d=128, window=37, sinks=4, s=64,
                 max_gen=1 << 20, pads=None, sm_scale=0.0, seed=1, block=None):
        self.dtype, self.b, self.h, self.hk, self.d, self.seed = dtype, b, heads, kv_heads, d, seed
        self.att = bmx.WindowAttention(b=b, s=s, max_gen=max_gen, window=window, sinks=sinks, n_heads=heads,
                                       n_kv_heads=kv_heads, head_dim=d, dtype=dtype, sm_scale=sm_scale, block=block)
        # slots without a token hold what a fresh allocation might
        self.att.k.fill_(NAN)
        self.att.v.fill_(NAN)
        self.att.work.fill_(255)
        self.ref = WindowReference(b=b, heads=heads, kv_heads=kv_heads, d=d, window=window, sinks=sinks,
                                   dtype=DT[dtype], pads=pads, scale=sm_scale or None)
        self.pads = pads
        if pads is not None:
            self.att.set_left_padding(torch.tensor(pads, dtype=torch.int32, device="cuda"))

    def qkv(self, t):
        self.seed += 1
        x = [rows(100 * self.seed + i, self.b, hh, t, self.d, self.dtype) for i, hh in enumerate((self.h, self.hk, self.hk))]
        if self.pads is not None:          # pad tokens' rows are never read
            for j in range(self.b):
                n = min(self.ref.skip[j], t)
                for y in x:
                    y[j, :, :n] = NAN
        return x

    def go(self, t, heads=None, samples=None, step=False, ld=None, row=0):
        """t tokens through both; buffers of ld rows, the call's from `row` on."""
        q, k, v = self.qkv(t)
        ld = row + t if ld is None else ld
        big = []
        for y in (q, k, v):
            z = torch.full((self.b, y.shape[1], ld, self.d), NAN, dtype=y.dtype)
            z[:, :, row:row + t] = y
            big.append(z.cuda())
        o = torch.full_like(big[0], 77.0)
        if step:
            self.att.decode_step(self.att.next_pos, *big, o, row=row)
        else:
            self.att.prefill_block(self.att.next_pos, t, *big, o, row=row)
        want = self.ref.tokens(q, k, v, packed=self.dtype == "bf16" and not step, heads=heads, samples=samples)
        o = o.cpu()
        for (j, head), exact in want.items():
            check_rows(o[j, head, row:row + t], exact, f"sample {j} head {head}")
        assert (o[:, :, :row] == 77).all() and (o[:, :, row + t:] == 77).all()

    def check_slots(self):
        """Every kept token in its slot, bit for bit, and the other slots as they were."""
        for name, own in (("k", self.ref.k), ("v", self.ref.v)):
            x = getattr(self.att, name).cpu().double()
            for j in range(self.b):
                slots = self.ref.slots(j)
                for slot in range(x.shape[2]):
                    if slot in slots:
                        assert torch.equal(x[j, :, slot], own[j][:, slots[slot]]), (name, j, slot)
                    else:
                        assert torch.isnan(x[j, :, slot]).all(), (name, j, slot)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,heads,kv_heads", [(128, 4, 1), (64, 4, 2), (128, 2, 2), (64, 4, 1), (64, 3, 3), (128, 4, 2)])
@pytest.mark.parametrize("window,sinks", [(37, 4), (1, 0), (200, 0), (64, 16)])
def test_prompts_turns_and_tokens(dtype, d, heads, kv_heads, window, sinks):
    r = Run(dtype=dtype, d=d, heads=heads, kv_heads=kv_heads, window=window, sinks=sinks, s=300)
    for t in (1, 5, 150, 63, 2, 79):
        r.go(t)
    r.check_slots()
    for _ in range(3):
        r.go(1, step=True)
    r.check_slots()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads", [(4, 1), (2, 1), (2, 2)])
@pytest.mark.parametrize("pads", [(0, 3, 70), (150, 151, 149), (40, 1000, 200), (-5, 64, 128)])
def test_left_padding(dtype, heads, kv_heads, pads):
    """Pads that end inside a call, at its border, and beyond the prompt."""
    r = Run(dtype=dtype, b=3, heads=heads, kv_heads=kv_heads, window=50, sinks=3, s=200, pads=list(pads), d=64)
    for t in (40, 110, 50):
        r.go(t)
    r.check_slots()
    for _ in range(2):
        r.go(1, step=True)
    r.check_slots()


@pytest.mark.parametrize("t", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129])
@pytest.mark.parametrize("group", [1, 2, 4])
def test_lengths_at_tile_borders(t, group):
    r = Run(heads=group, kv_heads=1, window=64, sinks=2, s=2 * t + 1, b=1)
    r.go(t)
    r.go(1)
    r.go(t)
    r.check_slots()


@pytest.mark.parametrize("window,sinks", [(31, 1), (32, 0), (33, 4), (63, 1), (64, 64), (65, 63), (128, 5), (1, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_windows_at_tile_borders(window, sinks, dtype):
    r = Run(window=window, sinks=sinks, s=400, b=1, heads=2, kv_heads=1, d=64, dtype=dtype)
    r.go(170)
    r.go(230)
    r.check_slots()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_long_prompt(dtype):
    r = Run(window=700, sinks=4, s=2500, b=1, heads=4, kv_heads=1, dtype=dtype)
    r.go(1800, heads=(1,))
    r.go(700, heads=(3,))
    for _ in range(2):
        r.go(1, step=True)
    r.check_slots()


@pytest.mark.parametrize("window,sinks", [(2048, 4), (5000, 0), (300, 16)])
@pytest.mark.parametrize("dtype,d,heads,kv_heads", [("bf16", 128, 4, 1), ("f32", 64, 2, 2), ("bf16", 64, 4, 2)])
def test_tokens_over_long_caches(window, sinks, dtype, d, heads, kv_heads):
    """Caches that several workgroups share, before they are full and after."""
    r = Run(window=window, sinks=sinks, s=1500, b=2, heads=heads, kv_heads=kv_heads, d=d, dtype=dtype)
    r.go(1500, heads=(), samples=())
    r.go(1, step=True)
    r.go(1, step=True)
    r = Run(window=window, sinks=sinks, s=6001, b=2, heads=heads, kv_heads=kv_heads, d=d, dtype=dtype, pads=(0, 4500))
    r.go(6001, heads=(), samples=())
    for _ in range(3):
        r.go(1, step=True)


@pytest.mark.parametrize("window,sinks", [(1500, 4), (777, 0), (3000, 64)])
@pytest.mark.parametrize("dtype,d,heads,kv_heads", [("bf16", 128, 4, 1), ("f32", 64, 2, 2), ("bf16", 64, 4, 2),
                                                    ("bf16", 128, 1, 1), ("f32", 128, 4, 1)])
def test_turns_over_long_caches(window, sinks, dtype, d, heads, kv_heads):
    """Few rows over many keys, which several workgroups share: before the window is full,
    and after; a sample that begins within a turn, one that has not begun."""
    r = Run(window=window, sinks=sinks, s=3756, b=3, heads=heads, kv_heads=kv_heads, d=d, dtype=dtype,
            pads=(0, 1490, 5000))
    r.go(1400, heads=(heads - 1,))
    r.go(133, heads=(0,))
    r.go(1900, heads=(), samples=())
    r.go(66, heads=(0,))
    r.go(257, heads=(heads - 1,), ld=300, row=11)
    r.go(1, step=True)
    r.check_slots()


def test_rows_inside_larger_buffers():
    """Rows before and behind the call's are neither read nor written."""
    r = Run(window=20, sinks=2, s=100)
    r.go(50, ld=70, row=9)
    r.go(50, ld=61, row=11)
    r.go(1, step=True, ld=3, row=1)


def test_attention_in_place():
    r = Run(window=40, sinks=2, s=150, b=2)
    q, k, v = (x.cuda() for x in r.qkv(150))
    want = r.ref.tokens(q, k, v, packed=True)
    r.att.prefill_block(0, 150, q, k, v, q)
    for (j, head), exact in want.items():
        check_rows(q[j, head], exact)
    q, k, v = (x.cuda() for x in r.qkv(1))
    want = r.ref.tokens(q, k, v, packed=False)
    r.att.decode_step(150, q, k, v, q)
    for (j, head), exact in want.items():
        check_rows(q[j, head], exact)


def test_softmax_scale_and_large_logits():
    r = Run(window=90, sinks=2, s=300, sm_scale=0.7)     # logits of tens: one key takes it all
    r.go(300)
    r.go(1, step=True)
    r = Run(window=90, sinks=2, s=300, sm_scale=0.7, dtype="f32", d=64)
    r.go(300)
    r.go(1, step=True)


def test_logits_far_below_zero():
    """A row whose visible keys all have logits near -1000 is still a softmax."""
    att = bmx.WindowAttention(b=1, s=80, max_gen=4, window=30, sinks=2, n_heads=1, n_kv_heads=1, head_dim=64, dtype="f32")
    ref = WindowReference(b=1, heads=1, kv_heads=1, d=64, window=30, sinks=2, dtype=torch.float32)
    q, k, v = (rows(i, 1, 1, 81, 64, "f32") for i in range(3))
    k = -q.mean(dim=2, keepdim=True).sign() * 20 + 0.01 * k
    q = q.mean(dim=2, keepdim=True).sign() * 6 + 0.01 * q
    want = ref.tokens(q, k, v, packed=False)[0, 0]
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    o = torch.zeros_like(q)
    att.prefill_block(0, 80, q, k, v, o)
    att.decode_step(80, q, k, v, o, row=80)
    check_rows(o[0, 0], want)


def test_block_cut_is_the_same_call_and_nothing_is_evicted():
    a, b = (Run(window=30, sinks=3, s=200, b=1) for _ in range(2))
    q, k, v = (x.cuda() for x in a.qkv(200))
    outs = []
    for r, fused in ((a, False), (b, True)):
        o = torch.zeros_like(q)
        r.att.dims.block = 70                   # (run_prefill's own loop)
        r.att.run_prefill(q, k, v, o, fused_cut=fused)
        outs.append(o)
        assert r.att.length == 33 and r.att.next_pos == 200
    assert torch.equal(outs[0], outs[1]) and torch.equal(a.att.k, b.att.k)


def test_a_prompt_does_not_depend_on_its_cuts_into_calls():
    """Outputs of one long call and of many short ones agree within their bounds, and the
    caches bit for bit."""
    a, b = (Run(window=130, sinks=4, s=500, b=1) for _ in range(2))
    q, k, v = (x.cuda() for x in a.qkv(500))
    o = torch.zeros_like(q)
    for r, step in ((a, 500), (b, 37)):
        for t0 in range(0, 500, step):
            r.att.prefill_block(t0, min(step, 500 - t0), q, k, v, o)
        want = r.ref.tokens(q, k, v, packed=True, heads=(2,))
        check_rows(o[0, 2], want[0, 2])
        r.check_slots()


def test_resume_goes_on_where_the_rows_left():
    a = Run(window=30, sinks=3, s=90, b=2)
    a.go(90)
    b = Run(window=30, sinks=3, s=90, b=2)
    b.att.k.copy_(a.att.k)
    b.att.v.copy_(a.att.v)
    b.att.resume(90)
    q, k, v = (x.cuda() for x in a.qkv(1))
    oa, ob = torch.zeros_like(q), torch.zeros_like(q)
    a.att.decode_step(90, q, k, v, oa)
    b.att.decode_step(90, q, k, v, ob)
    assert torch.equal(oa, ob) and torch.equal(a.att.k.nan_to_num(), b.att.k.nan_to_num())
    a.att.reset()
    assert a.att.next_pos == 0 and a.att.length == 0


def test_captured_steps_replay():
    """A captured run of steps, replayed from the same state with other work between."""
    r = Run(window=40, sinks=2, s=100, b=3, pads=[0, 10, 99])
    r.go(100, heads=(0,), samples=(0,))
    q, k, v = (x.cuda() for x in r.qkv(6))
    k0, v0 = r.att.k.clone(), r.att.v.clone()
    eager = torch.zeros_like(q)
    r.att.run_decode(q, k, v, eager, steps=6, first_row=0)
    k1 = r.att.k.clone()
    want = r.ref.tokens(q, k, v, packed=False)
    for (j, head), exact in want.items():
        check_rows(eager[j, head], exact)
    r.att.k.copy_(k0)
    r.att.v.copy_(v0)
    r.att.resume(100)
    o = torch.zeros_like(q)
    g = r.att.capture_decode(q, k, v, o, steps=6, first_row=0)
    other = Run(window=16, sinks=0, s=50, b=1)
    for i in range(3):
        r.att.k.copy_(k0)
        r.att.v.copy_(v0)
        o.zero_()
        g.replay()
        if i == 0:
            other.go(20)
        torch.cuda.synchronize()
        assert torch.equal(o, eager) and torch.equal(r.att.k.nan_to_num(), k1.nan_to_num())


@pytest.mark.parametrize("dtype,t", [("bf16", 200), ("bf16", 20), ("f32", 150)])
def test_a_captured_turn_replays(dtype, t):
    """Turns whose keys several workgroups share, replayed from the same state; another cache
    uses the same workspace in between."""
    r, other = (Run(window=2000, sinks=4, s=3000, b=2, dtype=dtype, seed=x) for x in (1, 50))
    for x in (r, other):
        x.go(2600, heads=(), samples=())
    other.att.work = r.att.work
    other.att.cache = other.att._cache()
    other.att.resume(2600)
    q, k, v = (x.cuda() for x in r.qkv(t))
    oq, ok, ov = (x.cuda() for x in other.qkv(t))
    k0, v0 = r.att.k.clone(), r.att.v.clone()
    eager = torch.zeros_like(q)
    r.att.prefill_block(2600, t, q, k, v, eager, row=0)
    k1, v1 = r.att.k.clone(), r.att.v.clone()
    r.att.resume(2600)
    o, g = torch.zeros_like(q), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.att.prefill_block(2600, t, q, k, v, o, row=0)
    for i in range(3):
        r.att.k.copy_(k0)
        r.att.v.copy_(v0)
        o.zero_()
        g.replay()
        if i < 2:
            other.att.prefill_block(2600 + i * t, t, oq, ok, ov, torch.zeros_like(oq), row=0)
        torch.cuda.synchronize()
        assert torch.equal(o, eager) and torch.equal(r.att.k, k1) and torch.equal(r.att.v, v1)


def test_streams_and_two_caches_at_once():
    a, b = Run(window=300, sinks=4, s=900, b=2, seed=3), Run(window=300, sinks=4, s=900, b=2, seed=40)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    data = [[x.cuda() for x in r.qkv(900)] for r in (a, b)]
    outs = [torch.zeros_like(x[0]) for x in data]
    torch.cuda.synchronize()
    for r, st, x, o in zip((a, b), streams, data, outs):
        with torch.cuda.stream(st):
            r.att.prefill_block(0, 900, *x, o)
            # the same rows again as a generated token
            r.att.decode_step(900, *(y[:, :, :1].contiguous() for y in x), torch.empty_like(o[:, :, :1]))
    torch.cuda.synchronize()
    for r, x, o in zip((a, b), data, outs):
        want = r.ref.tokens(*x, packed=True, heads=(1,), samples=(1,))
        check_rows(o[1, 1], want[1, 1])


def test_results_are_the_same_every_time():
    r = Run(window=500, sinks=4, s=1200, b=2)
    q, k, v = (x.cuda() for x in r.qkv(1200))
    outs = []
    for _ in range(3):
        r.att.reset()
        o = torch.zeros_like(q)
        r.att.prefill_block(0, 1200, q, k, v, o)
        r.att.decode_step(1200, q, k, v, o, row=7)
        outs.append(o)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_offsets_past_32_bits():
    """A cache and rows of more than 2^31 elements each: the last units are right."""
    b, hk, d, slots = 40, 8, 128, 60000            # 2.46e9 elements a plane
    r = bmx.WindowAttention(b=b, s=70000, max_gen=8, window=slots - 4, sinks=4, n_heads=hk, n_kv_heads=hk,
                            head_dim=d, dtype="bf16", block=64)
    r.k.normal_()
    r.v.normal_()
    r.resume(69999)
    q, k, v = (torch.randn((b, hk, 1, d), device="cuda").bfloat16() for _ in range(3))
    last = (b - 1, hk - 1)
    # the history of the last unit, in order
    index = torch.tensor(list(range(4)) + list(range(69999 - (slots - 4), 69999)))
    slot = torch.where(index < 4, index, 4 + (index - 4) % (slots - 4)).cuda()
    kk, vv = r.k[last][slot].cpu().double(), r.v[last][slot].cpu().double()
    o = torch.zeros_like(q)
    r.prefill_block(69999, 1, q, k, v, o, row=0)
    r.decode_step(70000, q, k, v, o.clone())

    from window_reference import Row
    seen = (index < 4) | (69999 - index < slots - 4)
    row = Row(q[last][0].cpu().double(), torch.cat([kk, k[last].cpu().double()]), torch.cat([vv, v[last].cpu().double()]),
              torch.cat([seen, torch.ones(1, dtype=torch.bool)]), d ** -0.5, torch.bfloat16, True)
    check_rows(o[last], [row])
    at = 4 + (69999 - 4) % (slots - 4)
    assert torch.equal(r.k[last][at], k[last][0]) and torch.equal(r.v[last][at], v[last][0])


@pytest.mark.parametrize("dtype,d,heads", [("bf16", 64, 8), ("bf16", 128, 32), ("f32", 64, 16), ("f32", 128, 8)])
def test_tokens_over_caches_beyond_the_last_level_one(dtype, d, heads):
    """Launches that stream their rows: the first and the last unit, one sample with padding."""
    from window_reference import Row
    b, hk, window, sinks, end, group = 128, 8, 2100, 4, 5000, heads // 8       # 0.55 GB and more
    r = bmx.WindowAttention(b=b, s=end, max_gen=8, window=window, sinks=sinks, n_heads=heads, n_kv_heads=hk,
                            head_dim=d, dtype=dtype, block=4)
    pads = torch.zeros(b, dtype=torch.int32)
    pads[-1] = 1001
    r.set_left_padding(pads.cuda())
    g = torch.Generator(device="cuda").manual_seed(5)
    r.k.normal_(generator=g)
    r.v.normal_(generator=g)
    r.resume(end)
    q, k, v = (torch.randn((b, h, 1, d), device="cuda", generator=g).to(DT[dtype]) for h in (heads, hk, hk))
    old_k, old_v = {}, {}
    for j, u in ((0, 0), (b - 1, hk - 1)):
        old_k[j, u], old_v[j, u] = r.k[j, u].cpu().double(), r.v[j, u].cpu().double()
    o = torch.zeros_like(q)
    r.decode_step(end, q, k, v, o)
    for (j, u), kk in old_k.items():
        now = end - int(pads[j])                                                # the token's index
        index = torch.tensor([*range(sinks), *range(now - window, now)])
        slot = torch.where(index < sinks, index, sinks + (index - sinks) % window)
        keys = torch.cat([kk[slot], k[j, u].cpu().double()])
        values = torch.cat([old_v[j, u][slot], v[j, u].cpu().double()])
        seen = torch.cat([(index < sinks) | (now - index < window), torch.ones(1, dtype=torch.bool)])
        for head in range(group * u, group * (u + 1)):
            check_rows(o[j, head], [Row(q[j, head, 0].cpu().double(), keys, values, seen, d ** -0.5, DT[dtype], False)])
        at = sinks + (now - sinks) % window
        assert torch.equal(r.k[j, u, at], k[j, u, 0]) and torch.equal(r.v[j, u, at], v[j, u, 0])


def test_another_current_device_is_refused():
    r = Run(window=8, sinks=0, s=10, b=1)
    q, k, v = (x.cuda() for x in r.qkv(10))
    with pytest.MonkeyPatch.context() as mp:
        mp.setattr(torch.cuda, "current_device", lambda: 1)
        with pytest.raises(ValueError):
            r.att.prefill_block(0, 10, q, k, v, torch.zeros_like(q))
    assert r.att.next_pos == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks,calls", [(50, 4, (200, 70, 1)), (8, 4, (12, 13, 1)), (700, 6, (900, 90, 3))])
def test_samples_that_never_begin(dtype, window, sinks, calls):
    """The largest pads, in calls longer than the window: those samples see nothing, give zeros
    and store nothing, whichever kernel takes the call (a prompt, the nodes of a chain, keys
    over several workgroups), while the others go on."""
    top = 2 ** 31 - 1
    r = Run(dtype=dtype, window=window, sinks=sinks, s=sum(calls), b=5, d=64, pads=[0, top, top - 1, 2 ** 30, 3])
    for t in calls:
        r.go(t, heads=(3,) if t > 500 else None)
        r.check_slots()
    r.go(1, step=True)
    r.check_slots()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_turns_behind_generated_tokens(dtype):
    """A conversation: a prompt, tokens, a turn of several calls, tokens, a short turn, a token."""
    r = Run(dtype=dtype, window=50, sinks=3, s=70, b=3, d=64, pads=[0, 60, 73])
    r.go(70)
    for turn in ((40, 21), (5,), (1,)):
        for _ in range(3):
            r.go(1, step=True)
        p = r.att.next_pos
        r.att.resume(p, s=p + sum(turn))
        for t in turn:
            r.go(t)
        assert r.att.next_pos == r.att.dims.s
        r.check_slots()
    r.go(1, step=True)
    r.check_slots()

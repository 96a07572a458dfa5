"""Performance cases of attention with a sliding window and of drafted tokens.

Window: a query at index i of its sequence (its position less the sample's left pad)
sees the last ``window`` tokens, its own included, and the first ``sinks``:

    key j is visible  <=>  0 <= j <= i  and  (j < sinks  or  i - j < window)
    o_i = sum_j exp(s q_i.k_j) v_j / sum_j exp(s q_i.k_j),  s = 1 / sqrt(d)

The cache holds window + sinks rows a unit: token j < sinks in slot j, the others in
slot sinks + (j - sinks) mod window.

Draft: the nodes of a tree of drafted tokens behind a cache.  Node a at depth t (0 for a
root) stands at position next + t; it sees the cache, its ancestors and itself (over a
window cache, those of them that the window shows).

Accepting a path of m nodes appends them to the cache.  A bounded cache adds their
probabilities to its entries' scores and is cut back by the smallest average
(score / age, the older first on a tie); survivors behind the bound fill the holes in
slot order.  A sample that accepts c < m tokens of the call's m stays m - c positions
behind: its left pad and its entries' positions grow by that, and hidden entries of
score 0 stand for the tokens it did not take (a window cache has none).

Four operators:

* ``prompt``: a prompt or a turn through a window cache;
* ``token``: generated tokens through a window cache;
* ``draft``: a tree's outputs and log-sum-exps over a bounded or a window cache;
* ``round``: those, and the acceptance of a path: a round of speculation.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_FOREVER = 1 << 28      # tokens go on for as long as the program runs


def _case(op, *, name=None, dtype="bf16", b, heads, kv_heads, d=128, n, window=0, sinks=0, rows=1,
          steps=1, accept=0, ragged=False, pad_max=0):
    """n: tokens before the call (window > 0) or entries in the bounded cache (window 0);
    rows: the prompt's tokens or the tree's nodes; steps: generated tokens; accept: the
    path's nodes (ragged: each sample takes 1 to that many)."""
    c = dict(op=op, dtype=dtype, b=b, heads=heads, kv_heads=kv_heads, d=d, n=n, window=window,
             sinks=sinks, rows=rows, steps=steps, accept=accept, ragged=ragged, pad_max=pad_max)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's short turn in a running conversation: latency is what it costs
        _case("prompt", name="prompt-b1-t64-w1024", b=1, heads=32, kv_heads=8, n=8000, window=1024,
              sinks=4, rows=64),
        # an ordinary batch of whole prompts
        _case("prompt", name="prompt-b8-t4096-w1024", b=8, heads=32, kv_heads=8, n=0, window=1024,
              sinks=4, rows=4096),
        # two long documents under a wide window
        _case("prompt", name="prompt-b2-t32768-w4096", b=2, heads=32, kv_heads=8, n=0, window=4096,
              sinks=4, rows=32768),
        # float32, multi-head, small heads, odd sizes, padded on the left, behind an earlier turn
        _case("prompt", name="prompt-f32-mha-padded-t777-w200", dtype="f32", b=3, heads=12, kv_heads=12,
              d=64, n=333, window=200, sinks=3, rows=777, pad_max=500),
        # one user's next tokens
        _case("token", name="token-b1-w1024", b=1, heads=32, kv_heads=8, n=9001, window=1024, sinks=4,
              steps=8),
        # an ordinary batch, some samples with less behind them than the window holds
        _case("token", name="token-b64-w1024", b=64, heads=32, kv_heads=8, n=1500, window=1024, sinks=4,
              steps=4, pad_max=1200),
        # throughput serving under a wide window
        _case("token", name="token-b64-w4096", b=64, heads=32, kv_heads=8, n=20000, window=4096, sinks=4,
              steps=2),
        # one user's drafted tokens over a cache at its bound
        _case("draft", name="draft-b1-n512-t16", b=1, heads=32, kv_heads=8, n=512, rows=16),
        # a batch's wide trees over window caches
        _case("draft", name="draft-b16-w4096-t64", b=16, heads=32, kv_heads=8, n=9999, window=4096,
              sinks=4, rows=64),
        # float32, multi-head, small heads, an odd tree over an odd cache, padded on the left
        _case("draft", name="draft-f32-mha-padded-n333-t13", dtype="f32", b=6, heads=12, kv_heads=12,
              d=64, n=333, rows=13, pad_max=100),
        # one user's whole round: draft, and three tokens taken
        _case("round", name="round-b1-n512-t16", b=1, heads=32, kv_heads=8, n=512, rows=16, accept=3),
        # an ordinary batch's round: each sample takes one to four tokens
        _case("round", name="round-b64-n512-t32-ragged", b=64, heads=32, kv_heads=8, n=512, rows=32,
              accept=4, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("prompt", "prompt", "prompt", "token", "token", "draft", "draft", "round", "round"))
    while True:
        group, kv = rng.choice((1, 2, 4, 4)), rng.choice((1, 2, 4, 5, 8, 8))
        shape = dict(dtype=rng.choice(("bf16",) * 4 + ("f32",)), heads=kv * group, kv_heads=kv,
                     d=rng.choice((64, 128, 128)))
        windowed = dict(window=_log_int(rng, 16, 8192), sinks=rng.choice((0, 1, 4, 4, 16)))
        nodes = _log_int(rng, 2, 64)
        if op == "prompt":
            n = rng.choice((0, 0, _log_int(rng, 1, 20000)))
            rows = _log_int(rng, 2, 32768)
            case = _case(op, b=_log_int(rng, 1, 16), n=n, rows=rows,
                         pad_max=rng.choice((0, 0, (n + rows) // 2)), **windowed, **shape)
        elif op == "token":
            n = _log_int(rng, 1, 40000)
            case = _case(op, b=_log_int(rng, 1, 256), n=n, steps=rng.randint(2, 8),
                         pad_max=rng.choice((0, 0, n // 2)), **windowed, **shape)
        elif op == "draft" and rng.random() < 0.5:
            n = _log_int(rng, 1, 40000)
            case = _case(op, b=_log_int(rng, 1, 128), n=n, rows=nodes,
                         pad_max=rng.choice((0, 0, n // 2)), **windowed, **shape)
        elif op == "draft":
            n = _log_int(rng, 1, 16384)
            case = _case(op, b=_log_int(rng, 1, 128), n=n, rows=nodes,
                         pad_max=rng.choice((0, 0, n // 2)), **shape)
        else:
            accept, ragged = rng.randint(1, min(nodes, 8)), rng.random() < 0.5
            if rng.random() < 0.3:
                case = _case(op, b=_log_int(rng, 1, 64), n=_log_int(rng, 1, 20000), rows=nodes,
                             accept=accept, ragged=ragged, **windowed, **shape)
            else:
                case = _case(op, b=_log_int(rng, 1, 64), n=_log_int(rng, 40, 4000), rows=nodes,
                             accept=accept, ragged=ragged, **shape)
        w = work(case)
        slow = 16 if case["dtype"] == "f32" else 1          # float32 matrix instructions' rate
        if w["bytes"] < 2.1e9 and w["flops"] * slow < 4e12 and _plain_bytes(case) < 6e9:
            return case


def _entries(case):
    """Cached entries that a call of the case sees."""
    return min(case["n"], case["window"] + case["sinks"]) if case["window"] else case["n"]


def _slots(case):
    return case["window"] + case["sinks"] if case["window"] else case["n"] + case["accept"]


def _plain_bytes(case):
    """The plain form's largest intermediate results (a prompt's logits are made in parts)."""
    if case["op"] == "prompt":
        return 0
    keys = _slots(case) + case["rows"]
    es = 4 if case["dtype"] == "f32" else 2
    rows = 2 * (4 + es) * case["b"] * case["kv_heads"] * keys * case["d"]
    return rows + 8 * case["b"] * case["heads"] * case["rows"] * keys


def _visible(case):
    """(query, key) pairs of one query head of a prompt, padding aside."""
    n, t, w, s = case["n"], case["rows"], case["window"], case["sinks"]

    def below(x):               # the pairs of queries 0 .. x - 1
        full = max(0, x - (w + s))
        x -= full
        return x * (x + 1) // 2 + full * (w + s)
    return below(n + t) - below(n)


def work(case):
    """Every input read once, every output written once (a cache that is updated: its
    changed rows, scores and positions); 4 d flops per visible (query, key) pair.  Padded
    batches count as unpadded, a tree's nodes without their ancestors."""
    d, es = case["d"], 2 if case["dtype"] == "bf16" else 4
    units, heads, t, live = case["b"] * case["kv_heads"], case["b"] * case["heads"], case["rows"], _entries(case)
    row = 2 * d * es                    # a key's and a value's row
    if case["op"] == "prompt":
        kept = min(t, _slots(case))
        return {"bytes": (units * (min(live, case["window"]) + t + kept) + heads * t) * row,
                "flops": 4 * d * heads * _visible(case)}
    if case["op"] == "token":
        return {"bytes": case["steps"] * (units * (live + 2) + heads) * row,
                "flops": case["steps"] * 4 * d * heads * (live + 1)}
    nbytes = (units * (live + t) + heads * t) * row + 4 * case["b"] * t + 4 * heads * t
    if case["op"] == "round":
        m = case["accept"]
        nbytes += units * m * row + 4 * case["b"] * m
        if not case["window"]:
            nbytes += units * live * 12             # scores read and written, positions read
    return {"bytes": nbytes, "flops": 4 * d * heads * t * (live + 1)}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dt):
    return torch.randn(shape, generator=g, device="cuda", dtype=dt)


def _keys(g, shape, dt):
    """N(0, 1) rows times a lognormal factor per (sample, head, position)."""
    k = _normal(g, shape, dt)
    return k.mul_(torch.exp(0.5 * torch.randn(shape[:3] + (1,), generator=g, device="cuda")).to(dt))


def _first(case):
    """The position of the call's first token: a bounded cache at its bound has long lost
    entries, one that is padded has not."""
    full = not case["window"] and not case["pad_max"]
    return 200 * case["n"] + 100000 if full else case["n"]


def _inputs(case, seed):
    """The call's rows, the cache before it, and for drafts the tree and the path."""
    g, dt = _generator(seed), _DTYPES[case["dtype"]]
    b, h, hk, d, n = case["b"], case["heads"], case["kv_heads"], case["d"], case["n"]
    t, slots = max(case["rows"], case["steps"]), _slots(case)
    x = {"q": _normal(g, (b, h, t, d), dt), "kin": _keys(g, (b, hk, t, d), dt),
         "vin": _normal(g, (b, hk, t, d), dt), "k": _keys(g, (b, hk, slots, d), dt),
         "v": _normal(g, (b, hk, slots, d), dt), "pads": None}
    if case["pad_max"] or case["ragged"]:
        x["pads"] = torch.randint(0, case["pad_max"] + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
    if case["op"] in ("draft", "round"):
        # each node hangs from one of the eight before it; the first two of a sample and one
        # in sixteen are roots, and the path's nodes follow each other
        i, m = torch.arange(t, device="cuda"), case["accept"]
        back = torch.randint(1, 9, (b, t), generator=g, device="cuda")
        alone = torch.rand((b, t), generator=g, device="cuda") < 1 / 16
        parent = torch.where(alone | (i < 2), -1, (i - back).clamp_min(0))
        if m:
            path = torch.rand((b, t), generator=g, device="cuda").topk(m).indices.sort(dim=1).values
            before = torch.cat([torch.full_like(path[:, :1], -1), path[:, :-1]], dim=1)
            parent.scatter_(1, path, before)
            x["path"] = path.int()
            x["count"] = torch.randint(1, m + 1, (b,), generator=g, device="cuda", dtype=torch.int32) \
                if case["ragged"] else None
        x["parent"] = parent.int()
    if not case["window"]:
        # a full cache: increasing positions, one in each of n equal segments, and a few
        # entries that get next to nothing, which leave in turn
        first, group = _first(case), h // hk
        i = torch.arange(n, device="cuda")
        if first > n:
            seg = first / n
            lo, hi = torch.floor(i * seg), torch.floor((i + 1) * seg)
            pos = torch.minimum(lo + torch.floor(torch.rand((b, hk, n), generator=g, device="cuda") * (hi - lo)), hi - 1)
        else:
            pos = i.expand(b, hk, n).float()
        ave = torch.exp(0.5 * torch.randn((b, hk, n), generator=g, device="cuda"))
        if case["accept"]:
            idle = 2 * case["accept"] + 1
            at = torch.rand((b, hk, n // 2), generator=g, device="cuda").topk(idle).indices
            ave.scatter_(2, at, 0.005 * (1.25 ** torch.arange(idle, device="cuda")).expand(b, hk, -1))
        x["pos"] = torch.zeros((b, hk, slots), device="cuda", dtype=torch.int32)
        x["score"] = torch.zeros((b, hk, slots), device="cuda")
        x["pos"][:, :, :n] = pos.int()
        x["score"][:, :, :n] = ave * group / (n + 1) * (first - pos)
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    b, h, hk, d, n = case["b"], case["heads"], case["kv_heads"], case["d"], case["n"]
    state = {"case": case, "o": torch.zeros_like(x["q"]), "next": _first(case), **x}
    if case["op"] in ("draft", "round"):
        state["lse"] = torch.zeros((b, h, case["rows"]), device="cuda")
    if own:
        # the layer's cache as the tokens before left it, and its context
        from paper_2412_05693_amd import batchmax

        layer = dict(b=b, max_gen=_FOREVER, n_heads=h, n_kv_heads=hk, head_dim=d, dtype=case["dtype"])
        if case["window"]:
            prompt = case["op"] == "prompt"
            att = batchmax.WindowAttention(window=case["window"], sinks=case["sinks"], block=case["rows"],
                                           s=_FOREVER if prompt else n, **layer)
            att.k.copy_(x["k"])
            att.v.copy_(x["v"])
            att.resume(n)
        else:
            att = batchmax.PDAttention(kv_max=n, block=max(1, case["accept"]), s=_first(case), **layer)
            for name in ("k", "v", "score", "pos"):
                getattr(att, name)[:, :, :n] = x[name][:, :, :n]
            att.len.fill_(n)
            att.resume(n, _first(case))
        if x["pads"] is not None:
            att.set_left_padding(x["pads"])
        state["att"] = att
    return state


# --------------------------------------------------------------------------
# one pass: the package's calls
# --------------------------------------------------------------------------
def _run_own(state):
    case, att = state["case"], state["att"]
    q, kin, vin, o, n = state["q"], state["kin"], state["vin"], state["o"], case["n"]
    if case["op"] == "prompt":
        if n == 0:
            att.reset()
        att.prefill_block(att.next_pos, case["rows"], q, kin, vin, o, row=0)
        return {"o": o, "k": att.k, "v": att.v}
    if case["op"] == "token":
        for i in range(case["steps"]):
            att.decode_step(att.next_pos, q, kin, vin, o, row=i)
        return {"o": o, "k": att.k, "v": att.v}
    att.draft_attend(state["parent"], q, kin, vin, o, lse=state["lse"])
    out = {"o": o, "lse": state["lse"]}
    if case["op"] == "round":
        att.draft_accept(state["path"], q, kin, vin, lse=state["lse"], count=state["count"])
        live = slice(0, case["window"] + case["sinks"] if case["window"] else n)
        out |= {"k": att.k[:, :, live], "v": att.v[:, :, live]}
        if not case["window"]:
            out |= {"score": att.score[:, :, live], "pos": att.pos[:, :, live]}
        if state["pads"] is not None:
            out["pads"] = state["pads"]
    return out


# --------------------------------------------------------------------------
# one pass: the plain form
# --------------------------------------------------------------------------
def _indices(state):
    """The sequence index of every cached entry, [b, 1 or kv heads, slots]; below 0 where
    there is none."""
    case, now = state["case"], state["next"]
    pad = state["pads"][:, None, None] if state["pads"] is not None else 0
    if not case["window"]:
        return state["pos"][:, :, :case["n"]] - pad
    w, s, end = case["window"], case["sinks"], now - pad        # the next token's index
    slot = torch.arange(_slots(case), device="cuda")[None, None]
    # the largest index below `end` that falls into the slot
    ring = end - 1 - torch.remainder(end - 1 - slot, w)
    index = torch.where(slot < s, slot, torch.where(ring >= s, ring, -1))
    return torch.where(index < end, index, -1).expand(case["b"], 1, -1)


def _shown(case, i, j):
    """Whether the query at index i sees the key at index j (the tree aside)."""
    seen = (j >= 0) & (j <= i)
    if case["window"]:
        seen = seen & ((j < case["sinks"]) | (i - j < case["window"]))
    return seen


def _attend(q, kk, vv, seen):
    """q [b, h, r, d] over kk, vv [b, hk, l, d] under seen [b, 1 or hk, r, l] -> outputs,
    log-sum-exps [b, h, r], probabilities [b, hk, group, r, l]."""
    (b, h, r, d), (hk, l) = q.shape, kk.shape[1:3]
    group = h // hk
    z = torch.matmul(q.float().reshape(b, hk, group * r, d), kk.float().transpose(2, 3).contiguous())
    z = z.view(b, hk, group, r, l).mul_(1 / math.sqrt(d)).masked_fill_(~seen[:, :, None], float("-inf"))
    m = z.amax(dim=-1, keepdim=True)
    p = torch.exp_(z.sub_(torch.where(torch.isinf(m), 0.0, m)))
    total = p.sum(dim=-1, keepdim=True)
    p = p.div_(total.clamp_min(1e-30))
    o = torch.matmul(p.view(b, hk, group * r, l), vv.float()).view(b, h, r, d)
    return o.to(q.dtype), (m + torch.log(total)).view(b, h, r), p


def _store(state, index, k, v):
    """Rows of the tokens at `index` [b, t] into a window cache's slots (below 0: none)."""
    case, s, w = state["case"], state["case"]["sinks"], state["case"]["window"]
    last = index.amax(dim=1, keepdim=True)
    keep = (index >= 0) & ((index < s) | (index > last - w))
    sample, row = keep.nonzero(as_tuple=True)
    at = index[sample, row]
    slot = torch.where(at < s, at, s + torch.remainder(at - s, w))
    for name, x in (("k", k), ("v", v)):
        state[name][sample, :, slot] = x[sample, :, row]


def _prompt(state):
    case, now, t = state["case"], state["next"], state["case"]["rows"]
    q, kin, vin, w = state["q"], state["kin"], state["vin"], case["window"]
    pad = state["pads"][:, None].long() if state["pads"] is not None else torch.zeros((case["b"], 1), device="cuda", dtype=torch.long)
    old = _indices(state)[:, 0]
    new = now + torch.arange(t, device="cuda") - pad                # [b, t]
    head = max(0, min(t, case["pad_max"] + case["sinks"] - now))    # rows that hold sinks
    span = min(case["n"] + t, 2 * w) + case["sinks"] + w
    part = max(64, int(6e8 / (case["b"] * case["heads"] * span)))
    for c0 in range(0, t, part):
        c1, lo = min(t, c0 + part), max(0, c0 - w + 1)
        kept = case["sinks"] if c0 - w + 1 > 0 else _slots(case)    # cached entries still shown
        lead = slice(0, min(head, lo))
        j = torch.cat([old[:, :kept], new[:, lead], new[:, lo:c1]], dim=1)
        kk, vv = (torch.cat([c[:, :, :kept], x[:, :, lead], x[:, :, lo:c1]], dim=2)
                  for c, x in ((state["k"], kin), (state["v"], vin)))
        # (what a slot without an entry holds is not part of the sum)
        vv = vv.masked_fill((j < 0)[:, None, :, None], 0.0)
        seen = _shown(case, new[:, c0:c1, None], j[:, None])[:, None]
        state["o"][:, :, c0:c1] = _attend(q[:, :, c0:c1], kk, vv, seen)[0]
    _store(state, new, kin, vin)
    state["next"] = now + t
    return {"o": state["o"], "k": state["k"], "v": state["v"]}


def _nodes(state, q, kin, vin, reach):
    """Tree nodes over the cache and their ancestors (reach [b, r, r]: a sees b)."""
    case, r = state["case"], reach.shape[1]
    pad = state["pads"][:, None] if state["pads"] is not None else 0
    at = state["next"] - pad + reach.sum(dim=2) - 1                 # the nodes' indices [b, r]
    old = _indices(state)
    entries = old.shape[2]
    kk, vv = (torch.cat([c[:, :, :entries], x], dim=2) for c, x in ((state["k"], kin), (state["v"], vin)))
    seen_old = _shown(case, at[:, None, :, None], old[:, :, None])
    seen_new = (reach & _shown(case, at[:, :, None], at[:, None]))[:, None].expand(-1, seen_old.shape[1], -1, -1)
    return _attend(q, kk, vv, torch.cat([seen_old, seen_new], dim=3))


def _token(state):
    case = state["case"]
    b, steps = case["b"], case["steps"]
    alone = torch.ones((b, 1, 1), device="cuda", dtype=torch.bool)
    pad = state["pads"][:, None].long() if state["pads"] is not None else torch.zeros((b, 1), device="cuda", dtype=torch.long)
    for i in range(steps):
        row = (slice(None), slice(None), slice(i, i + 1))
        state["o"][row] = _nodes(state, state["q"][row], state["kin"][row], state["vin"][row], alone)[0]
        _store(state, state["next"] - pad, state["kin"][row], state["vin"][row])
        state["next"] += 1
    return {"o": state["o"], "k": state["k"], "v": state["v"]}


def _reach(parent):
    """parent [b, n] -> [b, n, n]: whether the node of a row sees that of a column."""
    n = parent.shape[1]
    up = torch.arange(n, device="cuda") == parent[:, :, None]
    steps = torch.eye(n, device="cuda") + up.float()        # (powers count paths: at most 2^64)
    return torch.linalg.matrix_power(steps, n) > 0


def _accept(state, p):
    """Append the path and, in a bounded cache, add its probabilities and cut back."""
    case, now, m, n = state["case"], state["next"], state["case"]["accept"], state["case"]["n"]
    path = state["path"].long()
    taken = state["count"][:, None] if state["count"] is not None else torch.full_like(path[:, :1], m)
    i = torch.arange(m, device="cuda")
    mine = i < taken                                                # [b, m]
    behind = m - taken
    state["next"] = now + m
    rows = [x.gather(2, path[:, None, :, None].expand(-1, x.shape[1], -1, x.shape[3])) for x in (state["kin"], state["vin"])]
    pad = state["pads"][:, None].long() if state["pads"] is not None else torch.zeros_like(behind)
    if case["window"]:
        _store(state, torch.where(mine, now - pad + i, -1), *rows)
    else:
        score, pos = state["score"], state["pos"]
        p = p.sum(dim=2)                                            # [b, hk, r, n + r]
        p = p.gather(2, path[:, None, :, None].expand(-1, p.shape[1], -1, p.shape[3]))
        p = p.masked_fill(~mine[:, None, :, None], 0.0)
        total = p.sum(dim=2)
        score[:, :, :n] += total[:, :, :n]
        gain = total[:, :, n:].gather(2, path[:, None].expand(-1, p.shape[1], -1))
        score[:, :, n:] = gain.masked_fill(~mine[:, None], 0.0)
        pos[:, :, :n] += behind[:, :, None].int()
        pos[:, :, n:] = torch.where(mine, now + i + behind, i - taken)[:, None].int()
        for name, x in zip("kv", rows):
            state[name][:, :, n:] = x.masked_fill(~mine[:, None, :, None], 0.0)
        # the m smallest (average, position) leave
        order = pos.argsort(dim=2)
        ave = (score / (now + m - pos).float()).gather(2, order)
        gone = order.gather(2, ave.argsort(dim=2, stable=True))[:, :, :m]
        out = torch.zeros_like(pos, dtype=torch.bool).scatter_(2, gone, True)
        holes = (~out[:, :, :n]).byte().argsort(dim=2, stable=True)[:, :, :m]
        left = n + out[:, :, n:].byte().argsort(dim=2, stable=True)
        moves = i < out[:, :, :n].sum(dim=2, keepdim=True)
        left = torch.where(moves, left, holes)
        for y in (score, pos):
            y.scatter_(2, holes, y.gather(2, left))
        for name in ("k", "v"):
            y = state[name]
            wide = (-1, -1, -1, y.shape[3])
            y.scatter_(2, holes[..., None].expand(wide), y.gather(2, left[..., None].expand(wide)))
    if state["pads"] is not None:
        state["pads"] += behind[:, 0].int()


def _run_plain(state):
    case, n = state["case"], state["case"]["n"]
    if case["op"] == "prompt":
        if n == 0:
            state["next"] = 0
        return _prompt(state)
    if case["op"] == "token":
        return _token(state)
    o, lse, p = _nodes(state, state["q"], state["kin"], state["vin"], _reach(state["parent"]))
    state["o"].copy_(o)
    state["lse"].copy_(lse)
    out = {"o": state["o"], "lse": state["lse"]}
    if case["op"] == "round":
        _accept(state, p)
        live = slice(0, _slots(case) if case["window"] else n)
        out |= {"k": state["k"][:, :, live], "v": state["v"][:, :, live]}
        if not case["window"]:
            out |= {"score": state["score"][:, :, live], "pos": state["pos"][:, :, live]}
        if state["pads"] is not None:
            out["pads"] = state["pads"]
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# --------------------------------------------------------------------------
# the same in 64 bits, sample by sample
# --------------------------------------------------------------------------
def _softmax_over(q, kk, vv, seen):
    """q [hk, g, r, d], kk and vv [hk, l, d], seen [1 or hk, r, l] -> o, log-sum-exps,
    probabilities, all in 64 bits."""
    hk, g, r, d = q.shape
    z = torch.bmm(q.reshape(hk, g * r, d).double(), kk.double().transpose(1, 2).contiguous()).view(hk, g, r, -1)
    z = torch.where(seen[:, None], z / math.sqrt(d), -math.inf)
    m = z.amax(dim=-1, keepdim=True).clamp_min(-1e300)
    e = torch.where(seen[:, None], torch.exp(z - m), 0.0)
    total = e.sum(dim=-1, keepdim=True)
    p = e / total.clamp_min(1e-300)
    o = torch.bmm(p.view(hk, g * r, -1), vv.double()).view(hk, g, r, d)
    return o, (m + torch.log(total))[..., 0], p


def _sample(case, x, j):
    """Sample j: its rows, its cached entries in order of index, and their indices."""
    group = case["heads"] // case["kv_heads"]
    q = x["q"][j].unflatten(0, (-1, group))
    pad = int(x["pads"][j]) if x["pads"] is not None else 0
    end = _first(case) - pad                                # the index of the next token
    w, s = case["window"], case["sinks"]
    index = [i for i in range(min(s, max(end, 0)))] + list(range(max(s, end - w), end))
    slot = torch.tensor([i if i < s else s + (i - s) % w for i in index], device="cuda", dtype=torch.long)
    return q, x["k"][j][:, slot], x["v"][j][:, slot], torch.tensor(index, device="cuda", dtype=torch.long), end


def _seen(case, i, j):
    near = (i[:, None] - j[None] < case["window"]) | (j[None] < case["sinks"])
    return (near & (j[None] <= i[:, None]) & (j[None] >= 0))[None]


def _exact_prompt(case, x):
    t, out = case["rows"], []
    for j in range(case["b"]):
        q, ck, cv, index, end = _sample(case, x, j)
        new = end + torch.arange(t, device="cuda")
        kk, vv = torch.cat([ck, x["kin"][j]], dim=1), torch.cat([cv, x["vin"][j]], dim=1)
        index = torch.cat([index, new])
        parts = []
        for c0 in range(0, t, 512):
            i = new[c0:c0 + 512]
            wanted = ((index <= i[-1]) & (index > i[0] - case["window"])) | ((index >= 0) & (index < case["sinks"]))
            pick = wanted.nonzero()[:, 0]
            parts.append(_softmax_over(q[:, :, c0:c0 + 512], kk[:, pick], vv[:, pick], _seen(case, i, index[pick]))[0])
        out.append(torch.cat(parts, dim=2).flatten(0, 1))
        x["last"] = x.get("last", []) + [(index, kk, vv, end + t)]
    return torch.stack(out)


def _exact_ring(case, x, rows):
    """The window cache of every sample once the tokens `rows` (index, k, v per sample) are in."""
    out = {"k": x["k"].double(), "v": x["v"].double()}
    w, s = case["window"], case["sinks"]
    for j, (index, k, v) in enumerate(rows):
        newest = int(index[-1]) if len(index) else -1
        for name, src in (("k", k), ("v", v)):
            keep = ((index >= 0) & ((index < s) | (index > newest - w))).nonzero()[:, 0]
            at = index[keep]
            out[name][j][:, torch.where(at < s, at, s + (at - s) % w)] = src[:, keep].double()
    return out


def _lineage(parent):
    """parent (a list) -> for each node the list of its ancestors and itself."""
    seen = []
    for a, up in enumerate(parent):
        seen.append((seen[up] if up >= 0 else []) + [a])
    return seen


def _exact_nodes(case, x, j):
    """Sample j's tree -> o, log-sum-exps, probabilities over its entries and the nodes."""
    parent, r = x["parent"][j].tolist(), case["rows"]
    lines = _lineage(parent)
    reach = torch.zeros((r, r), dtype=torch.bool)
    for a, line in enumerate(lines):
        reach[a, line] = True
    reach = reach.cuda()
    depth = torch.tensor([len(line) - 1 for line in lines], device="cuda")
    if case["window"]:
        q, ck, cv, index, end = _sample(case, x, j)
        at = end + depth
        seen = torch.cat([_seen(case, at, index), _seen(case, at, at) & reach], dim=2)
    else:
        n, pad = case["n"], int(x["pads"][j]) if x["pads"] is not None else 0
        q = x["q"][j].unflatten(0, (-1, case["heads"] // case["kv_heads"]))
        ck, cv, pos = x["k"][j][:, :n], x["v"][j][:, :n], x["pos"][j][:, :n]
        seen = torch.cat([(pos >= pad)[:, None].expand(-1, r, -1), reach.expand(pos.shape[0], -1, -1)], dim=2)
        seen = seen & (_first(case) + depth >= pad)[None, :, None]
    return _softmax_over(q, torch.cat([ck, x["kin"][j]], dim=1), torch.cat([cv, x["vin"][j]], dim=1), seen)


def _exact_cut(case, x, j, p):
    """Sample j's bounded cache behind the round: k, v, scores."""
    n, m, now = case["n"], case["accept"], _first(case)
    path = x["path"][j].tolist()
    c = int(x["count"][j]) if x["count"] is not None else m
    path, late = path[:c], m - c
    p = p[:, :, path].sum(dim=(1, 2))                       # [hk, n + r]
    zero = torch.zeros((p.shape[0], late), device="cuda", dtype=torch.float64)
    score = torch.cat([x["score"][j][:, :n].double() + p[:, :n], p[:, [n + a for a in path]], zero], dim=1)
    added = [now + late + i for i in range(c)] + list(range(late))
    pos = torch.cat([x["pos"][j][:, :n].long() + late,
                     torch.tensor(added, device="cuda").expand(p.shape[0], -1)], dim=1)
    rows = {}
    for y, z in (("k", "kin"), ("v", "vin")):
        new = x[z][j][:, path].double()
        rows[y] = torch.cat([x[y][j][:, :n].double(), new, torch.zeros_like(new[:, :1]).expand(-1, late, -1)], dim=1)
    value = (score / (now + m - pos)).cpu().tolist()
    where = pos.cpu().tolist()
    source = []
    for keys, at in zip(value, where):
        gone = set(sorted(range(n + m), key=lambda e: (keys[e], at[e]))[:m])
        spare = iter(e for e in range(n, n + m) if e not in gone)
        source.append([next(spare) if e in gone else e for e in range(n)])
    pick = torch.tensor(source, device="cuda")
    take = lambda y: y.gather(1, pick[..., None].expand(-1, -1, y.shape[2]))        # noqa: E731
    return take(rows["k"]), take(rows["v"]), score.gather(1, pick)


def exact(case, seed):
    if 2 * case["d"] * case["b"] * case["heads"] * case["rows"] * _slots(case) > 1.5e13:
        return None                                         # (64-bit products take too long)
    x = _inputs(case, seed)
    b, n = case["b"], case["n"]
    if case["op"] == "prompt":
        o = _exact_prompt(case, x)
        first = [_first(case) - (int(x["pads"][j]) if x["pads"] is not None else 0) for j in range(b)]
        rows = [(i0 + torch.arange(case["rows"], device="cuda"), x["kin"][j], x["vin"][j]) for j, i0 in enumerate(first)]
        return {"o": o, **_exact_ring(case, x, rows)}
    if case["op"] == "token":
        outs, rows = [], []
        for j in range(b):
            q, kk, vv, index, end = _sample(case, x, j)
            i = end + torch.arange(case["steps"], device="cuda")
            index = torch.cat([index, i])
            kk, vv = torch.cat([kk, x["kin"][j]], dim=1), torch.cat([vv, x["vin"][j]], dim=1)
            outs.append(_softmax_over(q, kk, vv, _seen(case, i, index))[0].flatten(0, 1))
            rows.append((i, x["kin"][j], x["vin"][j]))
        return {"o": torch.stack(outs), **_exact_ring(case, x, rows)}
    got, cut, rows = [], [], []
    for j in range(b):
        o, lse, p = _exact_nodes(case, x, j)
        got.append((o.flatten(0, 1), lse.flatten(0, 1)))
        if case["op"] == "round" and not case["window"]:
            cut.append(_exact_cut(case, x, j, p))
        elif case["op"] == "round":
            c = int(x["count"][j]) if x["count"] is not None else case["accept"]
            path = x["path"][j][:c].long()
            end = n - (int(x["pads"][j]) if x["pads"] is not None else 0)
            rows.append((end + torch.arange(c, device="cuda"), x["kin"][j][:, path], x["vin"][j][:, path]))
    out = {"o": torch.stack([y[0] for y in got]), "lse": torch.stack([y[1] for y in got])}
    if case["op"] == "round":
        if case["window"]:
            out |= _exact_ring(case, x, rows)
        else:
            out |= {name: torch.stack([y[i] for y in cut]) for i, name in enumerate(("k", "v", "score"))}
            out["pos"] = None
        if x["pads"] is not None:
            out["pads"] = None
    return out

"""64-bit references of attention over a window cache and of drafted tokens over any cache
(test infrastructure, written from include/bm_window.h and include/bm_draft.h).

Nothing here knows slots: a reference keeps every token of every sample.  Each result comes
with the error that the arithmetic may have (see ``bounds``)."""
import math

import torch

NEG = -math.inf


def bounds(dtype, z_off, p, vv, *, packed):
    """How far a row's outputs may be off: before their rounding, and that one's share.

    z_off: the logits' error, p: weights [L], vv: |v| rows [L, d] (all 64 bits).  A logit is a float32 sum of d products that are each off by 2^-24 (a float32 product; a
    bfloat16 one is exact), times the scale (2^-24), in log2 units (2^-24): with the sum of
    the absolute products at most A, off by (d + 3) 2^-24 A; exp2 and its argument add 2 ulp
    (2^-22).  A weight p = e / l has that error twice (its own and the sum's), sums of L terms
    add L 2^-24 each way, and rescaling by the running maximum one rounding a tile of 32 keys.
    Packed weights are one bfloat16 each (half a step: 2^-8 relative).  Others of a bfloat16
    product are two, the nearest bfloat16, off by at most 2^-8 p, and the nearest one to
    that rest, off by at most 2^-8 of it: 2^-16 p.  Outputs are rounded once to their type
    (half a step of their size).
    """
    length = p.shape[-1]
    rel_p = 2 * (z_off + 2.0 ** -22) + (2 * length + length / 16 + 8) * 2.0 ** -24
    if dtype == torch.bfloat16:
        rel_p = rel_p + (2.0 ** -8 if packed else 2.0 ** -16)
    return rel_p * (p @ vv), torch.finfo(dtype).eps / 2


class Row:
    """One query row's exact result and its bounds."""

    def __init__(self, q, kk, vv, seen, scale, dtype, packed):
        d = q.shape[-1]
        z = (kk @ q) * scale
        z = torch.where(seen, z, torch.full_like(z, NEG))
        if not seen.any():
            self.o, self.lse, self.p = torch.zeros(d, dtype=torch.float64), NEG, torch.zeros_like(z)
            self.tol, self.lse_tol = torch.zeros(d, dtype=torch.float64), 0.0
            self.p_rel = 0.0
            return
        m = z.max()
        e = torch.exp(z - m)
        self.lse = float(m + torch.log(e.sum()))
        self.p = e / e.sum()
        kept = vv[seen]
        self.o = self.p[seen] @ kept
        size = (kk[seen].abs() @ q.abs()).max() * scale
        z_off = (d + 3) * 2.0 ** -24 * size
        tol, half = bounds(dtype, z_off, self.p[seen], kept.abs(), packed=packed)
        self.tol = tol + half * (self.o.abs() + tol) + 1e-30
        n = int(seen.sum())
        self.lse_tol = float(z_off + (n + n / 32 + 8) * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -22 * abs(self.lse))
        self.p_rel = float(2 * (z_off + 2.0 ** -22) + (2 * n + n / 16 + 8) * 2.0 ** -24 + 2.0 ** -22 * abs(self.lse))


def check_rows(o, rows, what=""):
    """o [r, d] against a list of Row."""
    o = o.detach().cpu().double()
    for i, row in enumerate(rows):
        off = (o[i] - row.o).abs()
        assert torch.isfinite(o[i]).all(), f"{what} row {i}: not finite"
        worst = (off / row.tol.clamp_min(1e-300)).max()
        assert (off <= row.tol).all(), f"{what} row {i}: off by {off.max():.3g}, {worst:.3g} times the bound"


class WindowReference:
    """All tokens of every sample; the window as bm_window.h defines it."""

    def __init__(self, *, b, heads, kv_heads, d, window, sinks, dtype, pads=None, scale=None):
        self.b, self.h, self.hk, self.group, self.d = b, heads, kv_heads, heads // kv_heads, d
        self.window, self.sinks, self.dtype = window, sinks, dtype
        self.scale = 1.0 / math.sqrt(d) if scale is None else scale
        pads = [0] * b if pads is None else [int(x) for x in pads]
        self.skip = [max(0, x) for x in pads]                     # pad tokens still to come
        self.k = [torch.zeros((kv_heads, 0, d), dtype=torch.float64) for _ in range(b)]
        self.v = [x.clone() for x in self.k]

    def _sees(self, i, j):
        return (j <= i) & ((j < self.sinks) | (i - j < self.window))

    def _row(self, j, head, q, kk, vv, index, i, extra=None):
        seen = self._sees(i, index)
        if extra is not None:
            seen = seen & extra
        return Row(q, kk, vv, seen, self.scale, self.dtype, self.packed)

    packed = False

    def tokens(self, q, k, v, *, packed, heads=None, samples=None, store=True):
        """T tokens [b, heads, T, d] -> {(sample, head): [Row, ...]} for the asked ones."""
        q, k, v = (x.detach().cpu().double() for x in (q, k, v))
        self.packed = packed
        out, t = {}, q.shape[2]
        for j in range(self.b):
            skip = min(self.skip[j], t)
            base = self.k[j].shape[1]
            kk, vv = torch.cat([self.k[j], k[j][:, skip:]], dim=1), torch.cat([self.v[j], v[j][:, skip:]], dim=1)
            if samples is None or j in samples:
                for head in range(self.h) if heads is None else heads:
                    rows, u = [], head // self.group
                    for r in range(t):
                        if r < skip:
                            rows.append(Row(q[j, head, r], kk[u][:0], vv[u][:0], torch.zeros(0, dtype=torch.bool),
                                            self.scale, self.dtype, packed))
                            continue
                        i = base + r - skip
                        lo = max(0, i - self.window + 1)
                        index = torch.cat([torch.arange(min(self.sinks, lo)), torch.arange(lo, i + 1)])
                        rows.append(self._row(j, head, q[j, head, r], kk[u][index], vv[u][index], index, i))
                    out[j, head] = rows
            if store:
                self.k[j], self.v[j], self.skip[j] = kk, vv, self.skip[j] - skip
        return out

    def tree(self, parent, q, k, v, heads=None, samples=None):
        q, k, v = (x.detach().cpu().double() for x in (q, k, v))
        self.packed = False
        out = {}
        for j in range(self.b) if samples is None else samples:
            lines = lineage(parent[j].tolist())
            base = self.k[j].shape[1] - self.skip[j]               # (below 0: more pads than positions)
            for head in range(self.h) if heads is None else heads:
                u, rows = head // self.group, []
                for a, line in enumerate(lines):
                    i = base + len(line) - 1
                    index = torch.cat([torch.arange(self.k[j].shape[1]), base + torch.arange(len(line))])
                    kk, vv = torch.cat([self.k[j][u], k[j, u][line]]), torch.cat([self.v[j][u], v[j, u][line]])
                    ok = (index >= 0) & torch.tensor(i >= 0)
                    rows.append(Row(q[j, head, a], kk, vv, self._sees(i, index) & ok, self.scale, self.dtype, False))
                out[j, head] = rows
        return out

    def accept(self, path, count, k, v):
        k, v = (x.detach().cpu().double() for x in (k, v))
        for j in range(self.b):
            line = path[j].tolist()[:path.shape[1] if count is None else int(count[j])]
            skip = min(self.skip[j], len(line))
            self.skip[j] -= skip
            self.k[j] = torch.cat([self.k[j], k[j][:, line[skip:]]], dim=1)
            self.v[j] = torch.cat([self.v[j], v[j][:, line[skip:]]], dim=1)

    def slots(self, j):
        """{slot: index} of what a window cache keeps of sample j."""
        n = self.k[j].shape[1]
        keep = list(range(min(self.sinks, n))) + list(range(max(self.sinks, n - self.window), n))
        return {i if i < self.sinks else self.sinks + (i - self.sinks) % self.window: i for i in keep}


def lineage(parent):
    """For each node its ancestors, root first, and itself (a parent that does not come
    before its node makes a root)."""
    out = []
    for a, up in enumerate(parent):
        out.append((out[up] if 0 <= up < a else []) + [a])
    return out


def tree_over(kk, vv, visible, parent, q, k, v, scale, dtype):
    """One sample and head: nodes over entries kk, vv [L, d] of which `visible` [L] are seen."""
    kk, vv, q, k, v = (x.detach().cpu().double() for x in (kk, vv, q, k, v))
    visible = visible.cpu()
    rows = []
    for a, line in enumerate(lineage(parent)):
        rows.append(Row(q[a], torch.cat([kk, k[line]]), torch.cat([vv, v[line]]),
                        torch.cat([visible, torch.ones(len(line), dtype=torch.bool)]), scale, dtype, False))
    return rows


def random_tree(b, n, seed, roots=0.1, span=6):
    g = torch.Generator().manual_seed(seed)
    i = torch.arange(n)
    parent = (i - torch.randint(1, span + 1, (b, n), generator=g)).clamp_min(-1)
    parent[torch.rand((b, n), generator=g) < roots] = -1
    return parent.int()

"""64-bit reference of the bounded cache held in 4 bits (test infrastructure,
written from the definitions in include/bm_kv4.h and Sec. 3.1/3.2)."""
import math

import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def stored(x):
    """float64 values that rows x [..., d] stand for once held in 4 bits."""
    g = x.detach().cpu().double().unflatten(-1, (-1, 32))
    out = torch.empty_like(g)
    top = g.abs().amax(dim=-1)
    ok = torch.isfinite(g).all(dim=-1)
    # the smallest E with top <= 6 2^E: top / 6 = f 2^x with f in [.5, 1), in float64, where no
    # quotient of a float32 rounds to a power of two that it is not
    f, x = torch.frexp(top.nan_to_num(nan=1.0, posinf=1.0) / 6.0)
    e = torch.where(f > 0.5, x, x - 1).clamp(-119, 125)
    s = torch.ldexp(torch.ones_like(top), e)[..., None]
    a = (g / s).abs()
    # distance to every grid value; the even code wins a tie (it is tried first)
    order = [0, 2, 4, 6, 1, 3, 5, 7]
    best = (a[..., None] - GRID[order]).abs().nan_to_num(nan=math.inf).argmin(dim=-1)
    out = torch.copysign(GRID[torch.tensor(order)[best]] * s, g)
    out[~ok] = math.nan
    return out.flatten(-2)


class Reference:
    """Every unit's entries in the device's slot order, float64."""

    def __init__(self, *, b, heads, kv_heads, d, pads=None, scale=None):
        self.b, self.hk, self.group, self.d = b, kv_heads, heads // kv_heads, d
        self.scale = 1.0 / math.sqrt(d) if scale is None else scale
        self.pads = torch.zeros(b, dtype=torch.long) if pads is None else pads.cpu().long()
        row = (b, kv_heads, 0)
        self.k = torch.zeros(row + (d,), dtype=torch.float64)
        self.v = self.k.clone()
        self.pos = torch.zeros(row, dtype=torch.long)
        self.score = torch.zeros(row, dtype=torch.float64)
        self.last = torch.zeros(row, dtype=torch.float64)
        self.zmax = 0.0     # largest logit seen (log2 units), for tolerances
        self.vmax = 0.0

    @property
    def n(self):
        return self.pos.shape[2]

    def attend(self, t0, q, k, v, scores=True):
        """Rows q, k, v [b, heads, r, d] at positions t0..: over the entries as stored and
        the rows as given; then they are entries themselves."""
        q, k, v = (x.detach().cpu().double() for x in (q, k, v))
        r = q.shape[2]
        at = torch.arange(t0, t0 + r)
        pos = torch.cat([self.pos, at.expand(self.b, self.hk, r)], dim=2)
        seen = pos[:, :, None] <= at[:, None]
        seen = seen & (pos[:, :, None] >= self.pads[:, None, None, None])
        seen = seen & (at[:, None] >= self.pads[:, None, None, None])
        kk, vv = torch.cat([self.k, k], dim=2), torch.cat([self.v, v], dim=2)
        # what a hidden entry holds counts nowhere, infinities and NaN included
        hidden = pos < self.pads[:, None, None]
        kk = torch.where(hidden[..., None], 0.0, kk)
        vv = torch.where(hidden[..., None], 0.0, vv)
        qq = q.view(self.b, self.hk, self.group * r, self.d)
        z = (qq @ kk.transpose(2, 3)).view(self.b, self.hk, self.group, r, -1) * self.scale
        z = torch.where(seen[:, :, None], z, -math.inf)
        m = z.amax(dim=-1, keepdim=True)
        p = torch.exp(z - torch.where(torch.isinf(m) & (m < 0), 0.0, m))
        p = p / torch.where(seen.any(dim=-1)[:, :, None, :, None], p.sum(dim=-1, keepdim=True), 1.0)
        o = (p.view(self.b, self.hk, self.group * r, -1) @ vv).view(self.b, -1, r, self.d)
        fine = z[torch.isfinite(z)]
        if fine.numel():
            self.zmax = max(self.zmax, float(fine.abs().max()) / math.log(2.0))
        if vv.numel() and torch.isfinite(vv).all():
            self.vmax = max(self.vmax, float(vv.abs().max()))
        zero = torch.zeros((self.b, self.hk, r), dtype=torch.float64)
        self.score = torch.cat([self.score, zero], dim=2)
        if scores:
            self.score = self.score + p.sum(dim=(2, 3))
        self.last = p[:, :, :, r - 1].sum(dim=2)
        self.k = torch.cat([self.k, stored(k)], dim=2)
        self.v = torch.cat([self.v, stored(v)], dim=2)
        self.pos = pos
        return o

    def cut(self, keep, curr, rule, device_pos):
        """Entries from n down to `keep`; of two sets that rounding cannot tell apart the
        device's is taken.  Entries are then in its slot order."""
        dev = device_pos.cpu().long()
        assert dev.shape[2] == keep
        age = (curr + 1 - self.pos).double()
        key = {"ave": self.score / age, "sum": self.score, "recent": self.pos.double(),
               "tova": self.last}[rule]
        match = dev[:, :, :, None] == self.pos[:, :, None, :]
        assert (match.sum(dim=3) == 1).all(), "the device holds an entry that was not there"
        kept = match.any(dim=2)
        assert (kept.sum(dim=2) == keep).all()
        out_key = torch.where(kept, -math.inf, key).amax(dim=2)
        in_key = torch.where(kept, key, math.inf).amin(dim=2)
        band = 1e-5 * out_key.abs() + (0 if rule == "recent" else 1e-12)
        assert (out_key <= in_key + band).all(), "an entry left that ranks above one that stayed"
        # exact ties (entries no query has seen): the older one leaves
        ties = (out_key == in_key) & (out_key == 0)
        old = torch.where(kept | (key != 0), -1, self.pos).amax(dim=2)
        young = torch.where(kept & (key == 0), self.pos, 1 << 40).amin(dim=2)
        assert (~ties | (old < young)).all(), "of two equal entries the younger one left"
        idx = match.long().argmax(dim=3)
        for name in ("pos", "score", "last"):
            setattr(self, name, getattr(self, name).gather(2, idx))
        for name in ("k", "v"):
            x = getattr(self, name)
            setattr(self, name, x.gather(2, idx[..., None].expand(-1, -1, -1, self.d)))

    # -- tolerances ------------------------------------------------------------
    # Both products add float32 terms whose partial sums are at most zmax (logits, in log2
    # units) and 1 (weights): about sqrt(terms) half-steps of 2^-24 each, to which 16
    # zmax + 2 sqrt(n) + 8 leaves a margin of four and more.  A relative error of a
    # weight moves an output by at most that much of the largest value.
    def weight_err(self, seen):
        return 2.0 ** -24 * (16 * self.zmax + 2 * math.sqrt(seen) + 8)

    def out_tol(self, o, dtype, seen, parts=2.0 ** -16):
        """bfloat16: the result's rounding (half a step, eps / 2 = 2^-8), and `parts`: what
        the weights lose in bfloat16 (two parts: 2^-8 of 2^-8; a block's queries: 2^-8)."""
        tol = self.vmax * self.weight_err(seen)
        if dtype == "bf16":
            tol = tol + self.vmax * parts + o.abs() * 2.0 ** -8
        return tol + 1e-30

    def score_tol(self, seen, steps=1):
        return (self.weight_err(seen) + 2.0 ** -23) * steps * self.group + 2.0 ** -23 * steps * self.score.abs()


def check(got, want, tol, what):
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    err = (got - want).abs().nan_to_num(nan=0.0)
    bad = err > tol
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(err.max()):.3g}"

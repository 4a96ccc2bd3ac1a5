"""A paged cache on the GPU and its copy for the float64 oracle, and the comparison of the two."""
from __future__ import annotations

import numpy as np
import torch

from oracle import cache_oracle as O

D = 128
STEP32, STEP16 = 2.0 ** -24, 2.0 ** -8          # half a step of fp32 and of bf16, relative


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


class Paged:
    """counts: [B][L][H] nested.  layout: how the pool lies in memory.  fill: what slots that no token is in hold."""

    def __init__(self, C, dev, counts, page=16, room=0, layout="token", seed=0, state=True, spare=3, gain=1.0, fill=None):
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        self.C, self.dev, self.page = C, dev, page
        c = torch.tensor(counts, dtype=torch.int32)
        self.B, self.L, self.H = B, L, H = c.shape
        self.per = max(1, -(-(int(c.max()) + room) // page))
        self.pages = B * self.per + spare
        self.capacity = self.per * page
        shape = {"token": (self.pages, L, page, H, D), "head": (self.pages, L, H, page, D),
                 "layer": (L, self.pages, page, H, D)}[layout]
        order = {"token": (0, 1, 2, 3, 4), "head": (0, 1, 3, 2, 4), "layer": (1, 0, 2, 3, 4)}[layout]
        self.k, self.v = (torch.randn(shape, generator=g, device=dev).to(torch.bfloat16).permute(order) for _ in range(2))
        if gain != 1.0:
            self.k[..., 5] *= gain
        self.tables = torch.randperm(self.pages, generator=g, device=dev)[:B * self.per].to(torch.int32).view(B, self.per)
        self.counts = c.to(dev)
        self.seen = self.counts * 2 + 7
        self.mass = torch.rand(self.pages, L, H, page, generator=g, device=dev)
        self.positions = torch.zeros(self.pages, L, H, page, dtype=torch.int32, device=dev)
        if fill is not None:
            for b in range(B):
                for l in range(L):
                    for h in range(H):
                        for s in range(counts[b][l][h], self.capacity):
                            p, a = int(self.tables[b, s // page]), s % page
                            self.k[p, l, a, h] = fill
                            self.v[p, l, a, h] = fill
                            self.mass[p, l, h, a] = fill
        self.state = state
        self.cache = self.handle()

    def handle(self):
        s = (self.seen, self.mass, self.positions) if self.state else (None, None, None)
        return self.C.Cache(self.k, self.v, self.tables, self.counts, *s)

    def fill_positions(self, g=None):
        """Distinct positions below seen, in a random order of slots."""
        pos = torch.zeros_like(self.positions)
        rng = np.random.default_rng(11)
        for b in range(self.B):
            for l in range(self.L):
                for h in range(self.H):
                    n = int(self.counts[b, l, h])
                    p = rng.permutation(int(self.seen[b, l, h]))[:n]
                    for s in range(n):
                        pos[int(self.tables[b, s // self.page]), l, h, s % self.page] = int(p[s])
        self.positions.copy_(pos)

    # -- the same in host arrays, by logical slot
    def there(self, b):
        t = self.tables[b].cpu().numpy()
        ok = (t >= 0) & (t < self.pages)
        return np.repeat(ok, self.page), np.where(ok, t, 0)

    def head(self, b, l, h):
        """-> (K, V [capacity, d] f64, mass f32, positions, there)"""
        there, t = self.there(b)
        idx = torch.from_numpy(t.astype(np.int64)).to(self.dev)
        k, v = (f64(p[idx, l, :, h].reshape(-1, D)) for p in (self.k, self.v))
        return k, v, self.mass[idx, l, h].reshape(-1).cpu().numpy(), self.positions[idx, l, h].reshape(-1).cpu().numpy(), there

    def snapshot(self):
        return {n: getattr(self, n).clone() for n in ("k", "v", "mass", "positions", "counts", "seen")}


def bits(t):
    return t.contiguous().view(torch.int16)


def same_pool(P, want, what=""):
    """Everything the cache consists of, bit by bit."""
    for n in ("counts", "seen", "positions"):
        assert torch.equal(getattr(P, n), want[n]), "%s: %s" % (what, n)
    for n in ("k", "v"):
        assert torch.equal(bits(getattr(P, n)), bits(want[n])), "%s: %s" % (what, n)
    assert torch.equal(P.mass.contiguous().view(torch.int32), want["mass"].contiguous().view(torch.int32)), what + ": mass"


def attention_bounds(q, k, v, see, there, scale, cap, out, p):
    """How far one row's outputs may be off.  With u = 2^-24: a logit is a sum of d exact products, in any order
    off by (d - 1) u scale sum |q_c k_c|, its scaling and its way into the exponent's argument (two multiplications and a
    subtraction of numbers up to the largest |x|) by 6 u max |x|; a cap has slope <= 1 and is itself off by 2^-21 cap (its tanh
    is 1 - 2 / (e + 1) with e off by a few u relative), and by no more than 2^-19 |x| where x is small beside it (that form is taken from
    tanh = 0.245 on, where 2^-21 is 2^-19 of the value; below it stands y (1 - y^2/3 + .. ), off by some 10 u).  A weight e^(x - m) / sum is then off by 2 dx relative, by 2^-21 for the
    exponentials, reciprocals and products, and by (n + 16) u for the sum; a weight that underflows is off by 2^-120.  The product with
    V takes it with 16 mantissa bits (2^-16 for the two roundings), and sums n terms (n + 16) u.  The output is rounded to bf16 once.
    -> (bound of out [d], of lse, relative bound of the weights)"""
    u = STEP32
    at = np.flatnonzero(there[:see])
    n = len(at)
    if n == 0:
        return np.zeros(D), 0.0, 0.0
    x = scale * (k[at] @ q)
    dx = (D - 1) * u * scale * float(np.max(np.abs(k[at]) @ np.abs(q))) + 6 * u * float(np.max(np.abs(x)))
    if cap > 0:
        dx += min(2.0 ** -21 * cap, 2.0 ** -19 * float(np.max(np.abs(x))))
    rel = 2 * dx + 2.0 ** -21 + (n + 16) * u
    size = p[at] @ np.abs(v[at])
    b_out = size * (rel + 2.0 ** -16 + (n + 16) * u) + 2.0 ** -120 * np.abs(v[at]).sum(0)
    b_out = b_out + STEP16 * (np.abs(out) + b_out) + 2.0 ** -133
    return b_out, dx + rel + 4 * u * (abs(float(np.max(x))) + np.log(n) + 1), rel


def check_attention(P, q, new, scale, cap, got, got_lse, before, accumulate, most=0, what=""):
    """got, got_lse and the cache's mass against the oracle; `before`: P.snapshot() of before the call."""
    B, L, T, Hq, _ = q.shape
    G = Hq // P.H
    qd, od = f64(q), f64(got)
    ld = got_lse.double().cpu().numpy() if got_lse is not None else None
    counts = P.counts.cpu().numpy()
    worst = 0.0
    touched = torch.zeros_like(P.mass, dtype=torch.bool)
    for b in range(B):
        n_new = T if new is None else min(max(int(new[b]), 0), T)
        for l in range(L):
            for h in range(P.H):
                k, v, mass, _, there = P.head(b, l, h)
                c = min(max(int(counts[b, l, h]), 0), P.capacity)
                see = O.sees(c, n_new, T)
                weight, slack = np.zeros(P.capacity), np.zeros(P.capacity)
                for t in range(T):
                    for g in range(G):
                        row = (b, l, t, h * G + g)
                        out, lse, p = O.attend(qd[row], k, v, see[t], there, scale, cap)
                        b_out, b_lse, rel = attention_bounds(qd[row], k, v, see[t], there, scale, cap, out, p)
                        err = np.abs(od[row] - out)
                        assert np.all(err <= b_out), "%s %s: out off by %.3g of %.3g allowed" % (what, row, err.max(), b_out[np.argmax(err - b_out)])
                        worst = max(worst, float(np.max(err / np.maximum(b_out, 1e-300))) if see[t] else 0.0)
                        if ld is not None:
                            if np.isinf(lse):
                                assert ld[row] == -np.inf, "%s %s: lse of a row that sees nothing" % (what, row)
                            else:
                                assert abs(ld[row] - lse) <= b_lse, "%s %s: lse off by %.3g of %.3g" % (what, row, abs(ld[row] - lse), b_lse)
                        weight += p / G
                        slack += p / G * (rel + 2 * STEP32)
                if accumulate:
                    old = before["mass"]
                    there_at, t_np = P.there(b)
                    idx = torch.from_numpy(t_np.astype(np.int64)).to(P.dev)
                    was = old[idx, l, h].reshape(-1).double().cpu().numpy()
                    fits = most == 0 or c <= most
                    seen_any = np.zeros(P.capacity, bool)
                    if fits:
                        seen_any[:max(see)] = True
                        seen_any &= there_at
                    want = np.where(seen_any, was + weight, was)
                    bound = np.where(seen_any, slack + (T * G + 2) * STEP32 * (weight + np.abs(was)) + 2.0 ** -120, 0.0)
                    with np.errstate(invalid="ignore"):
                        ok = np.where(np.isnan(want), np.isnan(mass), (mass == want) | (np.abs(mass - want) <= bound))
                    ok |= ~there_at
                    assert np.all(ok), "%s %s: mass of slots %s" % (what, (b, l, h), np.flatnonzero(~ok)[:8])
    return worst

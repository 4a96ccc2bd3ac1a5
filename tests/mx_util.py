"""A paged cache in 4 bits beside one of 16 that holds the same values: what checks the second checks the first."""
from __future__ import annotations

import math

import numpy as np
import torch

from oracle import mx_oracle as M
from tests import cache_util as U


def pack(codes):
    """Codes [..., 128] -> bytes [..., 64]"""
    codes = np.asarray(codes, np.uint8)
    return codes[..., 0::2] | codes[..., 1::2] << 4


def unpack(rows):
    rows = np.asarray(rows)
    return np.stack((rows & 15, rows >> 4), -1).reshape(*rows.shape[:-1], 128)


class Paged(U.Paged):
    """U.Paged, whose k and v are the values of k4, k_scales, v4 and v_scales.  fill: bytes of codes and scales in slots that no token is in."""

    def __init__(self, C, dev, counts, page=16, layout="token", fill=None, gain=1.0, **kw):
        super().__init__(C, dev, counts, page=page, layout=layout, **kw)
        order = {"token": (0, 1, 2, 3, 4), "head": (0, 1, 3, 2, 4), "layer": (1, 0, 2, 3, 4)}[layout]
        g = torch.Generator(device=dev)
        g.manual_seed(kw.get("seed", 0) + 1)
        shape = [self.k.shape[order.index(i)] for i in range(4)]
        self.k4, self.v4 = (torch.randint(0, 256, (*shape, 64), generator=g, device=dev, dtype=torch.uint8).permute(order) for _ in range(2))
        self.k_scales, self.v_scales = (torch.randint(122, 128, (self.pages, self.L, self.H, page, 4), generator=g, device=dev,
                                                      dtype=torch.uint8) for _ in range(2))
        self.k_scales[..., 0] += int(math.log2(gain))
        if fill is not None:
            held = torch.zeros(self.pages, self.L, page, self.H, dtype=torch.bool, device=dev)
            for b in range(self.B):
                for l in range(self.L):
                    for h in range(self.H):
                        for s in range(counts[b][l][h]):
                            held[int(self.tables[b, s // page]), l, s % page, h] = True
            for rows, scales in ((self.k4, self.k_scales), (self.v4, self.v_scales)):
                rows[~held] = fill
                scales.transpose(2, 3)[~held] = fill
            self.mass.transpose(2, 3)[~held] = float("nan")
        self.values()
        self.mx = self.mx_handle()

    def values(self):
        """k and v from the rows of 4 bits."""
        numbers = torch.tensor(list(M.NUMBERS) + list(-M.NUMBERS), device=self.dev)
        for t, rows, scales in ((self.k, self.k4, self.k_scales), (self.v, self.v4, self.v_scales)):
            codes = torch.stack((rows & 15, rows >> 4), -1).reshape(*rows.shape[:4], 4, 32)
            size = torch.ldexp(torch.ones((), dtype=torch.float64, device=self.dev), scales.transpose(2, 3).to(torch.int32) - 127)
            size = torch.where(scales.transpose(2, 3) == M.NAN, float("nan"), size)
            t.copy_((numbers[codes.int()] * size.unsqueeze(-1)).reshape(t.shape).to(torch.bfloat16))

    def mx_handle(self):
        s = (self.seen, self.mass, self.positions) if self.state else (None, None, None)
        return self.C.MxCache(self.k4, self.v4, self.k_scales, self.v_scales, self.tables, self.counts, *s)

    def snapshot(self):
        return {**super().snapshot(), **{n: getattr(self, n).clone() for n in ("k4", "v4", "k_scales", "v_scales")}}


ROWS = ("k4", "v4", "k_scales", "v_scales")


def same(P, want, names=ROWS + ("counts", "seen", "positions"), what=""):
    for n in names:
        assert torch.equal(getattr(P, n), want[n]), "%s: %s" % (what, n)
    assert torch.equal(P.mass.contiguous().view(torch.int32), want["mass"].contiguous().view(torch.int32)), what + ": mass"

"""The 4-bit form of a row and the generation step on such rows, plainly, in 64 bits.  Not collected by pytest itself.

The format's roundings (to bf16, to 32 bits) are steps of its definition; they are taken one by one here.
"""
from __future__ import annotations

import math

import torch

GROUP = 32


def _f32(x):
    return x.float().double()


def _next_bf16(x, way):
    """The bf16 value beside x (a bf16 tensor), downwards (-1) or upwards (1)."""
    i = x.view(torch.int16)
    step = torch.where(x < 0, -torch.ones_like(i), torch.ones_like(i)) * way
    zero = torch.full_like(i, 1 if way > 0 else -32767)
    return torch.where(x == 0, zero, i + step).view(torch.bfloat16)


def _rounded(x, way):
    """x (64 bits) to bf16 as 64 bits, never past x in the direction `way`."""
    y = x.float().bfloat16()
    past = y.double() < x if way > 0 else y.double() > x
    return torch.where(past, _next_bf16(y, way), y).double()


def quantise(rows):
    """[.., d] to codes (int, [.., d]), scales and low ends ([.., d / 32], 64 bits)."""
    x = rows.double().unflatten(-1, (-1, GROUP))
    least, most = x.amin(-1), x.amax(-1)
    lo = _rounded(least, -1)
    sc = _rounded(_f32(_f32(most - lo) / torch.full_like(lo, 15.0)), 1)
    sc = torch.where(sc < 2.0 ** -100, torch.zeros_like(sc), sc)
    inv = torch.where(sc > 0, _f32(1.0 / torch.where(sc > 0, sc, torch.ones_like(sc))), torch.zeros_like(sc))
    codes = _f32(_f32(x - lo[..., None]) * inv[..., None]).round().clamp(max=15.0)
    return codes.flatten(-2).long(), sc, lo


def values(codes, sc, lo):
    return (codes.double().unflatten(-1, (-1, GROUP)) * sc[..., None] + lo[..., None]).flatten(-2)


def stored(rows):
    return values(*quantise(rows))


def to_bytes(codes):
    """Codes [.., d] to a row's bytes, one nibble after the other from the written rule."""
    d = codes.shape[-1]
    out = torch.zeros(*codes.shape[:-1], d // 2, dtype=torch.long, device=codes.device)
    for c in range(d):
        g, j, e = c // 32, c % 32 // 4, c % 4
        out[..., j * (d // 16) + 2 * g + e // 2] |= codes[..., c] << (4 * (e % 2))
    return out.to(torch.uint8)


def params(sc, lo):
    return torch.stack((sc, lo), dim=-1).to(torch.bfloat16)


def norm_of(v, kind):
    v = v.double()
    return v.abs().sum(-1) if kind == "l1" else v.pow(2).sum(-1).sqrt() if kind == "l2" else v.abs().amax(-1)


class State:
    """All units of a decode state in 64 bits, by slot: [units, cap]."""

    def __init__(self, cache, d, B, F, R, scale, window=0, norm="l1"):
        """cache: a CacheQ4 whose rows were written by `fill`."""
        n, cap = cache.pos.shape[0] * cache.pos.shape[1], cache.pos.shape[2]
        self.n, self.cap, self.d, self.B, self.F, self.R, self.scale, self.w, self.norm = n, cap, d, B, F, R, scale, window, norm
        self.pos = cache.pos.view(n, cap).long().clone()
        self.S = cache.acc.view(n, cap).double().clone()
        self.vnorm = cache.vnorm.view(n, cap).double().clone()
        self.len, self.free, self.t = (x.view(n).long().clone() for x in (cache.len, cache.free_slot, cache.next_pos))
        self.last = cache.last_slot.view(n).long().clone()
        if window:
            self.hist = cache.ring.view(n, window, cap).double().clone()
        self.k, self.v = self._rows(cache.k_codes, cache.k_params), self._rows(cache.v_codes, cache.v_params)

    def _rows(self, codes, par):
        b, d = codes.view(self.n, self.cap, -1).long(), self.d
        c = torch.arange(d, device=codes.device)
        byte = (c % 32 // 4) * (d // 16) + 2 * (c // 32) + c % 4 // 2
        code = b[..., byte] >> (4 * (c % 2)) & 15
        p = par.view(self.n, self.cap, d // 32, 2).double()
        # (magnitude: what the two parts of a product may amount to, for the bounds on rounding)
        self.mag = getattr(self, "mag", []) + [p[..., 1].abs() + 15 * p[..., 0]]
        return values(code, p[..., 0], p[..., 1])

    def step(self, q, k, v):
        """q [units, G, d], k and v [units, d] as given.  Returns out, p, importances, which slots may go, and a bound on the
        relative error that the logits' rounding to 32 bits gives a probability."""
        u = torch.arange(self.n, device=self.pos.device)
        for x, new, m in ((self.k, k, 0), (self.v, v, 1)):
            codes, sc, lo = quantise(new)
            x[u, self.free] = values(codes, sc, lo)
            self.mag[m][u, self.free] = lo.abs() + 15 * sc
        self.pos[u, self.free], self.vnorm[u, self.free] = self.t, norm_of(v, self.norm)
        live = self.pos >= 0
        q = q.double()
        s = torch.einsum("ngd,ncd->ngc", q, self.k) * self.scale
        p = torch.softmax(s.masked_fill(~live[:, None], -math.inf), -1)
        out = torch.einsum("ngc,ncd->ngd", p, self.v)
        # d products and as many sums of 32 bits a logit (2^-23 a step: the tensor cores cut off), exponential and normaliser
        most = torch.einsum("ngk,nck->ngc", q.abs().unflatten(-1, (-1, GROUP)).sum(-1), self.mag[0]).masked_fill(~live[:, None], 0.0)
        rel = 2 * (self.d + 8) * 2.0 ** -23 * self.scale * most.amax(-1) + 64 * 2.0 ** -24         # [n, G]
        v_mag = torch.einsum("ngc,nck->ngk", p, self.mag[1]).repeat_interleave(GROUP, -1)          # [n, G, d]
        pm = p.mean(1)
        if self.w:
            at = self.t % self.w
            self.hist[u, :, self.free] = 0.0
            self.hist[u, at] = torch.where(live, pm, self.hist[u, at])
            self.S = torch.where(live, self.hist.sum(1), self.S)
        else:
            self.S[u, self.free] = 0.0
            self.S = torch.where(live, self.S + pm, self.S)
        I = self.S * self.vnorm
        may_go = live & (self.pos >= self.F) & (self.pos <= self.t[:, None] - self.R)
        return out, pm, I, may_go, rel, v_mag

    def finish(self, evicted):
        """evicted [units]: the positions that went, -1 where the cache grows."""
        u = torch.arange(self.n, device=self.pos.device)
        went = evicted.long()
        full = self.len + 1 > self.B
        assert torch.equal(went >= 0, full)
        slot = (self.pos == went[:, None]).long().argmax(-1)
        self.last = self.free
        self.free = torch.where(full, slot, self.len + 1)
        self.pos[u[full], slot[full]] = -1
        self.len = torch.where(full, self.len, self.len + 1)
        self.t = self.t + 1

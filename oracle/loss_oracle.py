"""The head's losses in 64 bits, from their definition, with the bounds that an implementation with half-precision operands
and float32 sums can be held to.  torch on any device; products, exponentials and sums only."""
from __future__ import annotations

import math

import torch

F64 = torch.float64
H16, F32 = 2.0 ** -11, 2.0 ** -24          # half a step of half precision and of float32, relative
OUT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def target(V, labels=None, top_logits=None, top_ids=None, tau=1.0):
    """[T, V] target distribution; a row without target is zeros."""
    if labels is not None:
        r = torch.zeros(len(labels), V, dtype=F64, device=labels.device)
        for t, y in enumerate(labels.tolist()):
            if 0 <= y < V:
                r[t, y] = 1.0
        return r
    T, k = top_ids.shape
    ids, logits = top_ids.tolist(), top_logits.double().tolist()
    r = torch.zeros(T, V, dtype=F64)
    for t in range(T):
        there = [(i, l / tau) for i, l in zip(ids[t], logits[t]) if 0 <= i < V and l != -math.inf]
        if not there:
            continue
        m = max(l for _, l in there)
        e = [math.exp(l - m) for _, l in there]
        for (i, _), x in zip(there, e):
            r[t, i] += x / sum(e)
    return r.to(top_ids.device)


class Loss:
    """h [T, d], W [V, d] as given to the implementation; r [T, V] from target()."""

    def __init__(self, h, W, r, tau=1.0):
        self.dtype, self.tau, self.r = h.dtype, tau, r
        self.live = r.sum(1) > 0
        self.h = h.double().masked_fill(~self.live[:, None], 0.0)
        self.W = W.double()
        self.z = self.h @ self.W.T / tau
        m = self.z.max(1).values
        self.lse = m + torch.log(torch.exp(self.z - m[:, None]).sum(1))
        self.q = torch.exp(self.z - self.lse[:, None])
        logr = torch.log(torch.where(r > 0, r, 1.0))
        self.loss = torch.where(self.live, (r * (logr - self.z + self.lse[:, None])).sum(1), 0.0)
        # probabilities of the target: a float32 softmax (2^-17), of one id 1 but for a few roundings
        self.e_r = torch.where((r.max(1).values == 1.0) | ~self.live, 2.0 ** -22, 2.0 ** -17)[:, None] * r
        # |error of z|: a float32 sum of d products in some order, at most d / 4 + 8 additions behind one another, W in steps of
        # 2^-33; as two terms also 2^-22 for either factor and for the product of the low terms, and h in steps of 2^-38 of its row
        d, V = h.shape[1], W.shape[0]
        two = self.dtype == torch.float32
        ah, aW = self.h.abs(), self.W.abs()
        err = (ah @ aW.T) * ((d / 4 + 8) * F32 + (3 * H16 * H16 if two else 0.0)) + 2.0 ** -33 * ah.sum(1)[:, None]
        if two:
            err = err + 2.0 ** -38 * ah.max(1).values[:, None] * aW.sum(1)[None, :]
        # its scale, the difference to a maximum or to lse and log2(e), six roundings, and the hardware's exp2 (2^-21 in all)
        self.e_z = err / tau + 6 * F32 * self.z.abs() + 2.0 ** -21
        self.e_lse = self.e_z.max(1).values + 6 * F32 * (self.z.abs().max(1).values + self.lse.abs()) + (V / 16 + 32) * F32

    def loss_bounds(self):
        """(loss, lse, bound of loss, bound of lse)"""
        logr = torch.log(torch.where(self.r > 0, self.r, 1.0)).abs()
        b = self.e_lse + (self.r * self.e_z + (self.e_r + 2.0 ** -21 * self.r) * (logr + self.z.abs() + self.lse.abs()[:, None] + 1.0)).sum(1)
        lse = torch.where(self.live, self.lse, 0.0)
        return self.loss, lse, torch.where(self.live, b, 0.0), torch.where(self.live, self.e_lse, 0.0)

    def grad_bounds(self, g):
        """((grad_hidden, bound), (grad_head, bound)) for the rows' coefficients g."""
        c = torch.where(self.live, g.double(), 0.0) / self.tau
        dz = torch.where(self.live[:, None], self.q - self.r, 0.0)
        two = self.dtype == torch.float32
        step = H16 * H16 if two else H16
        # dz: the error of the exponent and of the target, a rounding of the difference, and its own in steps of 2^-40 or more
        e = self.q * (self.e_z + self.e_lse[:, None]) + self.e_r + 2 * F32 * (self.r > 0) + step * dz.abs() + 2.0 ** -40
        e = torch.where(self.live[:, None], e, 0.0)
        aW, ah, adz = self.W.abs(), self.h.abs(), dz.abs()
        T, V = dz.shape
        more = 2 * step if two else 0.0                                # the other factor, the product of the low terms
        gh = (dz @ self.W) * c[:, None]
        bh = ((e + adz * (more + (V / 4 + 16) * F32)) @ aW + (adz + e).sum(1)[:, None] * 2.0 ** -33) * c.abs()[:, None]
        hc = self.h * c[:, None]
        gw, ahc = dz.T @ hc, hc.abs()                                  # h g: its own rounding, in steps of 2^-38 of its maximum
        bw = (e + adz * (more + step + (T / 4 + 16) * F32)).T @ ahc + (adz + e).sum(0)[:, None] * 2.0 ** -37 * ahc.max()
        # dz g as the first factor of grad_head has one scale for all rows, that of the largest c |h|: row t carries
        # x = dz 2^15 c_t 2^-e_t f, f a power of two that brings the largest c 2^-e into [1/2, 1), against h_t 2^e_t, at most 2^14,
        # whose largest in the row is at least 2^13.  Below half precision's normal numbers x is off by up to half a step of
        # 2^-24 (two terms: the low one by that), so that row t is off by 2^-25 2^14 / (2^15 f), and 1 / f is at most
        # 2 max |c| 2^-e <= 2 max |c h| 2^-13: 2^-38 max |c h| a row, however small its own c and dz are.
        bw = bw + float(self.live.sum()) * 2.0 ** -38 * ahc.max()
        out = OUT[self.dtype] * 1.01 + 6 * F32                         # (and of g / tau and the products with it)
        return (gh, bh + gh.abs() * out + 1e-40), (gw, bw + gw.abs() * out + 1e-40)

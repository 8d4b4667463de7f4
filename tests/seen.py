"""Attention over the keys that a mask names, in 64 bits, with sequences.py's element-wise tolerances."""
import torch

from sequences import U, Head


class Seen(Head):
    """One head: q [n, d] against k, v [m, d], row i over the keys with sees[i, j]; and its gradient for g.  A row that sees nothing is zero, its LSE
    minus infinity."""

    def __init__(self, q, k, v, scale, sees, g=None):
        q, k, v = q.double(), k.double(), v.double()
        x = (scale * q @ k.t()).masked_fill(~sees, -torch.inf)
        some = sees.any(1)
        self.lse = torch.logsumexp(x, 1)
        self.p = torch.exp(x - torch.where(some, self.lse, torch.zeros_like(self.lse))[:, None])
        self.out = self.p @ v
        size = (scale * q.abs() @ k.abs().t()).masked_fill(~sees, 0)
        d, m = q.shape[1], k.shape[0]
        self.weight = 2 * (d + 8) * U * size.amax(1, keepdim=True) + 4 * U * (1 + x.masked_fill(~sees, 0).abs().amax(1, keepdim=True)) + (m + 16) * U
        self.lse_off = self.weight[:, 0] + 4 * U * torch.where(some, self.lse, torch.zeros_like(self.lse)).abs()
        self.spread = self.p @ v.abs()
        if g is None:
            return
        g = g.double()
        dp = g @ v.t()
        delta = (g * self.out).sum(1, keepdim=True)
        ds = self.p * (dp - delta)
        self.dv, self.dq, self.dk = self.p.t() @ g, scale * ds @ k, scale * ds.t() @ q
        self.parts = (q, k, v, g, dp, delta, ds, scale)


def window_mask(n, window, sinks):
    """[n, n]: row a sees key b."""
    a, b = torch.arange(n)[:, None], torch.arange(n)[None, :]
    return (b <= a) & ((a - b < window) | (b < sinks))

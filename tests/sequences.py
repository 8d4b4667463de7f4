"""Attention over sequences in 64 bits, element by element what a result may be off by, and the inputs of its tests.

Where the tolerances come from: u = 2^-24 is half a step of fp32, r half a step of the storage type (bf16 2^-8, fp32 2^-24).
 * A score is a sum of d products in fp32: off by e_ij = (d + 2) u scale sum |q||k|, and a weight exp(S - reference) by a factor
   1 + e_ij, a few u of the exponential, and u times the size of the exponent's argument.
 * Weights are rounded to w before they meet V or dO (packed, bf16: w = 2^-8; decode, bf16: two terms, 2^-17; fp32: 0).
 * A sum of n terms in fp32 is off by n u times the sum of their magnitudes, in whatever order.
 * A result is rounded once, by r.
 * What is below fp32's normal numbers may be taken as zero, 2^-126 a term: of fewer than 2^20 terms with factors below 2^6 no more
   than 2^-100.
"""
import torch

U = 2.0 ** -24
TINY = 2.0 ** -100
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


def lengths_to_offsets(lens, first=0):
    return torch.tensor([first] + lens, dtype=torch.int64).cumsum(0).to(torch.int32)


def normal(shape, seed, dtype, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale).to(dtype)


class Head:
    """One head of one sequence: q [n, d] against k, v [m, d] in 64 bits, causal (n == m) or not; and its gradient for g."""

    def __init__(self, q, k, v, scale, causal, g=None):
        q, k, v = q.double(), k.double(), v.double()
        x = scale * q @ k.t()
        if causal:
            x = x.masked_fill(torch.ones(x.shape, dtype=torch.bool).triu(1), -torch.inf)
        self.lse = torch.logsumexp(x, 1)
        self.p = torch.exp(x - self.lse[:, None])
        self.out = self.p @ v
        size = scale * q.abs() @ k.abs().t()
        if causal:
            size = size.tril()
        d, m = q.shape[1], k.shape[0]
        # a weight's relative error: its score's and its row sum's, both exponents' rounding, the sum of the row
        self.weight = 2 * (d + 8) * U * size.amax(1, keepdim=True) + 4 * U * (1 + x.masked_fill(x == -torch.inf, 0).abs().amax(1, keepdim=True)) + (m + 16) * U
        self.lse_off = self.weight[:, 0] + 4 * U * self.lse.abs()
        self.spread = self.p @ v.abs()
        if g is None:
            return
        g = g.double()
        dp = g @ v.t()
        delta = (g * self.out).sum(1, keepdim=True)
        ds = self.p * (dp - delta)
        self.dv, self.dq, self.dk = self.p.t() @ g, scale * ds @ k, scale * ds.t() @ q
        self.parts = (q, k, v, g, dp, delta, ds, scale)

    def out_off(self, dtype, w):
        r = HALF_STEP[dtype]
        return r * self.out.abs() + (1 + r) * self.spread * (w + self.weight)

    def grad_off(self, dtype, w):
        """(dq, dk, dv): how far off.  delta is formed from the rounded result."""
        q, k, v, g, dp, delta, ds, scale = self.parts
        r = HALF_STEP[dtype]
        d, n, m = q.shape[1], q.shape[0], k.shape[0]
        delta_off = (g.abs() * self.out_off(dtype, w)).sum(1, keepdim=True) + (d + 2) * U * (g * self.out).abs().sum(1, keepdim=True)
        dp_off = (d + 2) * U * g.abs() @ v.abs().t()
        # P from the stored LSE, and the three roundings of dS = P (dP - delta) in fp32
        p_off = self.weight + 2 * self.lse_off[:, None]
        ds_off = ds.abs() * (w + p_off + 4 * U) + self.p * (dp_off + delta_off) * (1 + w)
        dq = r * self.dq.abs() + scale * (ds_off @ k.abs() + (m + 2) * U * ds.abs() @ k.abs())
        dk = r * self.dk.abs() + scale * (ds_off.t() @ q.abs() + (n + 2) * U * ds.abs().t() @ q.abs())
        dv = r * self.dv.abs() + ((w + p_off) * self.p).t() @ g.abs() + (n + 2) * U * self.p.t() @ g.abs()
        return dq, dk, dv


def check(name, got, want, off):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), name
    worst = ((got - want).abs() - off - TINY).max().item() if got.numel() else 0.0
    assert worst <= 0, (name, "beyond its tolerance by", worst)

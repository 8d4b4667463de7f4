"""Packed sequences that do not lie one behind the other: any order, gaps, and offsets that give a row to two of them."""
import pytest
import torch

from paper_2311_09431_amd import binding as sa
from sequences import check, Head
from test_packed_gpu import BF16, F32, ROUNDED, rows

pytestmark = pytest.mark.gpu


def both(offsets, T, H, H_kv, d, dtype, max_len):
    q, g = (rows((T, H, d), s, dtype) for s in (1, 2))
    k, v = (rows((T, H_kv, d), s, dtype) for s in (3, 4))
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 7), torch.full((H, T), 7.0, device="cuda")
    grads = [torch.full_like(x, 7) for x in (q, k, v)]
    sa.sa_attn_packed_fwd(q, k, v, off, out, lse, max_len)
    sa.sa_attn_packed_bwd(q, k, v, out, g, lse, off, torch.empty_like(lse), *grads, max_len)
    return [x.cpu() for x in (q, k, v, g)], out, lse, grads


def spans(offsets, T, max_len):
    for a, b in zip(offsets, offsets[1:]):
        a = min(max(a, 0), T)
        yield a, min(min(max(b, a), T), a + max_len)


def stays(offsets, T, max_len, out, lse, grads):
    held = torch.zeros(T, dtype=torch.bool)
    for a, b in spans(offsets, T, max_len):
        held[a:b] = True
    for x in (out, lse.t(), *grads):
        assert (x.cpu()[~held] == 7).all() and torch.isfinite(x).all()


# (an end before a beginning is an empty sequence: by those the others come in any order); d 100 of 40 heads: 128-row workgroups
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,H_kv,d", [(2, 1, 64), (40, 40, 100), (2, 2, 132)])
@pytest.mark.parametrize("offsets,T", [([200, 256, 0, 150], 256), ([90, 90, 10, 70, 71], 120), ([5000, 2 ** 31 - 1, 600, 601, 300, 431, 0, 290, -7], 640),
                                       ([99, 100, 98, 99, 97, 98, 0, 97], 100)])
def test_sequences_in_any_order(offsets, T, H, H_kv, d, dtype):
    (q, k, v, g), out, lse, grads = both(offsets, T, H, H_kv, d, dtype, T)
    taken = [(a, b) for a, b in spans(offsets, T, T) if b > a]
    assert sum(b - a for a, b in taken) == len({r for a, b in taken for r in range(a, b)})          # no row in two of them
    stays(offsets, T, T, out, lse, grads)
    G, w = H // H_kv, ROUNDED[dtype]
    for a, b in taken:
        r = slice(a, b)
        for kvh in {0, H_kv - 1}:
            dk = dv = dk_off = dv_off = 0
            for h in range(kvh * G, (kvh + 1) * G):
                x = Head(q[r, h], k[r, kvh], v[r, kvh], d ** -0.5, True, g[r, h])
                check(("out", a, h), out[r, h], x.out, x.out_off(dtype, w))
                check(("lse", a, h), lse[h, r], x.lse, x.lse_off)
                dq_off, i, j = x.grad_off(dtype, w)
                check(("dq", a, h), grads[0][r, h], x.dq, dq_off)
                dk, dv, dk_off, dv_off = dk + x.dk, dv + x.dv, dk_off + i, dv_off + j
            check(("dk", a, kvh), grads[1][r, kvh], dk, dk_off)
            check(("dv", a, kvh), grads[2][r, kvh], dv, dv_off)


# more tiles than a launch has workgroups for: 13 of 32 rows for 9, and many times as many
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offsets,T,max_len", [([0, 100, 0, 100, 0, 100, 120], 125, 100), ([300, 600, 0] * 40 + [640], 700, 650),
                                               ([600, 601, 300, 431, 0, 290, 5000, 2 ** 31 - 1, -7, 0], 640, 640)])
def test_rows_in_two_sequences_leave_the_others_tensors_and_gaps_alone(offsets, T, max_len, dtype):
    _, out, lse, grads = both(offsets, T, 2, 2, 64, dtype, max_len)
    stays(offsets, T, max_len, out, lse, grads)

"""Every kind of kernel that packed sequences are played by (the cases and the rules that lead there: packed_routes.py, asked on the host in
test_packed_rules.py), against 64 bits: odd lengths, groups of heads, columns that are no whole 16 bytes, neighbours that are no numbers."""
import pytest
import torch

from sequences import Head, check
from tests.packed_routes import CASES, ROWS_AROUND
from test_packed_gpu import BF16, F32, ROUNDED, compare, run, untouched

pytestmark = pytest.mark.gpu

TYPES = {"bf16": BF16, "fp32": F32}
NAMES = ["%s-%d-%d-%d-%d" % (c[0], i, *c[2:5]) for i, c in enumerate(CASES)]


def play(case, mutate=None):
    kind, lens, H, H_kv, d, max_len, _, _ = case
    first, behind = ROWS_AROUND
    return run(list(lens), H, H_kv, d, TYPES[kind], first=first, behind=behind, max_len=max_len or None, mutate=mutate)


@pytest.mark.parametrize("case", CASES, ids=NAMES)
def test_results(case):
    kind, lens, H, H_kv, d, _, _, _ = case
    ins, out, lse, grads = play(case)
    compare(list(lens), H, H_kv, d, TYPES[kind], ROWS_AROUND[0], ins, out, lse, grads, heads={0, H_kv - 1})
    untouched(list(lens), ROWS_AROUND[0], (out, 0), (lse, 1), *((x, 0) for x in grads))
    again = play(case)
    for x, y in zip((out, lse, *grads), (again[1], again[2], *again[3])):
        assert torch.equal(x, y)


@pytest.mark.parametrize("case", CASES, ids=NAMES)
def test_neighbours_that_are_no_numbers(case):
    """The second sequence, the rows around all of them and the last key/value head with its queries hold NaN and infinities: the
    sequences and heads beside them do not see it."""
    kind, lens, H, H_kv, d, _, _, _ = case
    dtype, first, G = TYPES[kind], ROWS_AROUND[0], H // H_kv
    bad = slice(first + lens[0], first + lens[0] + lens[1])

    def mutate(q, k, v, g):
        for x, group in ((q, G), (k, 1), (v, 1), (g, G)):
            if H_kv > 1:
                x[:, -group:] = float("nan")
            x[bad] = float("nan")
            x[:first], x[first + sum(lens):] = float("inf"), float("nan")
    ins, out, lse, grads = play(case, mutate)
    assert out[bad].isnan().all() and lse[:, bad].isnan().all() and all(x[bad].isnan().all() for x in grads)
    q, k, v, g = (x.cpu() for x in ins)
    at = first
    for s, n in enumerate(lens):
        r = slice(at, at + n)
        at += n
        if s == 1:
            continue
        # (the head beside the one that is no number, and another)
        for kvh in {max(0, H_kv - 2), 0}:
            dk = dv = dk_off = dv_off = 0
            for h in range(kvh * G, (kvh + 1) * G):
                x = Head(q[r, h], k[r, kvh], v[r, kvh], d ** -0.5, True, g[r, h])
                check(("out", s, h), out[r, h], x.out, x.out_off(dtype, ROUNDED[dtype]))
                check(("lse", s, h), lse[h, r], x.lse, x.lse_off)
                dq_off, a, b = x.grad_off(dtype, ROUNDED[dtype])
                check(("dq", s, h), grads[0][r, h], x.dq, dq_off)
                dk, dv, dk_off, dv_off = dk + x.dk, dv + x.dv, dk_off + a, dv_off + b
            check(("dk", s, kvh), grads[1][r, kvh], dk, dk_off)
            check(("dv", s, kvh), grads[2][r, kvh], dv, dv_off)


@pytest.mark.parametrize("what", ["first query", "last value"])
@pytest.mark.parametrize("case", [c for c in CASES if c[0] == "fp32"], ids=[n for n in NAMES if n.startswith("fp32")])
def test_masked_pairs_are_not_looked_at(case, what):
    """fp32: a query that is no number reaches the first key alone, an infinite last value the last row alone; rows that share a tile with
    them are done over and right."""
    _, lens, H, H_kv, d, _, _, _ = case
    first, G = ROWS_AROUND[0], H // H_kv
    begins = [first + sum(lens[:s]) for s in range(len(lens))]

    def mutate(q, k, v, g):
        for a, n in zip(begins, lens):
            if what == "first query":
                q[a] = g[a] = float("nan")
            else:
                v[a + n - 1] = float("inf")
    ins, out, lse, grads = play(case, mutate)
    q, k, v, g = (x.cpu().nan_to_num(0., 0.) for x in ins)
    for a, n in zip(begins, lens):
        r, keep = slice(a, a + n), slice(1, n) if what == "first query" else slice(0, n - 1)
        if n == 1:
            continue
        for kvh in {0, H_kv - 1}:
            dk = dv = dk_off = dv_off = 0
            for h in range(kvh * G, (kvh + 1) * G):
                x = Head(q[r, h], k[r, kvh], v[r, kvh], d ** -0.5, True, g[r, h])
                check(("out", a, h), out[r, h][keep], x.out[keep], x.out_off(F32, 0.)[keep])
                check(("lse", a, h), lse[h, r][keep], x.lse[keep], x.lse_off[keep])
                dq_off, i, j = x.grad_off(F32, 0.)
                check(("dq", a, h), grads[0][r, h][keep], x.dq[keep], dq_off[keep])
                dk, dv, dk_off, dv_off = dk + x.dk, dv + x.dv, dk_off + i, dv_off + j
            if what == "first query":
                check(("dk", a, kvh), grads[1][r, kvh][keep], dk[keep], dk_off[keep])
                check(("dv", a, kvh), grads[2][r, kvh][keep], dv[keep], dv_off[keep])

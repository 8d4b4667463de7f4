"""Packed attention with a sliding window and first tokens that stay visible, and its gradient, against 64 bits."""
import random

import pytest
import torch

import sequences
from paper_2311_09431_amd import binding as sa
from seen import Seen, window_mask
from sequences import check, normal

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
ROUNDED = {BF16: 2.0 ** -8, F32: 0.0}           # how far a weight is rounded before it meets V
NAN, INF = float("nan"), float("inf")
EMPTY = [0]


@pytest.fixture(autouse=True, params=[0, 300])
def empty_ones(request):
    """How many sequences without a row follow those of a test: with many a launch has as many tiles as the large ones."""
    EMPTY[0] = request.param
    yield
    EMPTY[0] = 0


def lengths_to_offsets(lens, first=0):
    return sequences.lengths_to_offsets(list(lens) + [0] * EMPTY[0], first)


def rows(shape, seed, dtype, order="shd"):
    x = normal(shape, seed, dtype).cuda()
    return x if order == "shd" else x.permute(1, 0, 2).contiguous().permute(1, 0, 2)


def backward(ins, out, lse, off, grads, top, window, sinks, scale=None):
    q, k, v, g = ins
    work = torch.full((sa.sa_attn_window_bwd_workspace(q, k, off, top, window, sinks),), 255, dtype=torch.uint8, device="cuda")
    sa.sa_attn_window_bwd(q, k, v, out, g, lse, off, torch.empty_like(lse), *grads, work, top, window, sinks, scale)


def run(lens, H, H_kv, d, dtype, window, sinks, order="shd", first=0, behind=0, max_len=None, scale=None, mutate=None):
    T = first + sum(lens) + behind
    q, g = (rows((T, H, d), s, dtype, order) for s in (1, 2))
    k, v = (rows((T, H_kv, d), s, dtype, order) for s in (3, 4))
    if mutate:
        mutate(q, k, v, g)
    off = lengths_to_offsets(lens, first).cuda()
    out, lse = torch.full_like(q, 7), torch.full((H, T), 7.0, device="cuda")
    top = max(lens + [1]) if max_len is None else max_len
    sa.sa_attn_window_fwd(q, k, v, off, out, lse, top, window, sinks, scale)
    grads = [torch.full_like(x, 7) for x in (q, k, v)]
    backward((q, k, v, g), out, lse, off, grads, top, window, sinks, scale)
    return (q, k, v, g), out, lse, grads


def compare(lens, H, H_kv, d, dtype, window, sinks, ins, out, lse, grads, first=0, scale=None, heads=None):
    q, k, v, g = (x.cpu() for x in ins)
    out, lse, grads = out.cpu(), lse.cpu(), [x.cpu() for x in grads]
    scale, w, G, at = scale or d ** -0.5, ROUNDED[dtype], H // H_kv, first
    for s, n in enumerate(lens):
        r = slice(at, at + n)
        at += n
        sees = window_mask(n, window, sinks)
        for kvh in range(H_kv):
            if n == 0 or (heads is not None and kvh not in heads):
                continue
            dk = dv = dk_off = dv_off = 0
            for h in range(kvh * G, (kvh + 1) * G):
                x = Seen(q[r, h], k[r, kvh], v[r, kvh], scale, sees, g[r, h])
                check(("out", s, h), out[r, h], x.out, x.out_off(dtype, w))
                check(("lse", s, h), lse[h, r], x.lse, x.lse_off)
                dq_off, a, b = x.grad_off(dtype, w)
                check(("dq", s, h), grads[0][r, h], x.dq, dq_off)
                dk, dv, dk_off, dv_off = dk + x.dk, dv + x.dv, dk_off + a, dv_off + b
            check(("dk", s, kvh), grads[1][r, kvh], dk, dk_off)
            check(("dv", s, kvh), grads[2][r, kvh], dv, dv_off)


LENS = [1, 127, 0, 128, 129, 33, 300, 2]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [4, 32, 36, 64, 68, 96, 100, 112, 128, 132, 192, 256])
def test_head_dimensions(d, dtype):
    compare(LENS, 2, 1, d, dtype, 40, 3, *run(LENS, 2, 1, d, dtype, 40, 3))


# around the tiles' 32, 64 and 128 rows; the row's own key alone; more first tokens than the window, than rows
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 0), (1, 200), (31, 0), (32, 5), (33, 0), (64, 1), (127, 0), (128, 4), (129, 0), (200, 129), (500, 0),
                                          (7, 1000), (1 << 30, 1 << 30), (255, 128), (256, 33)])
def test_windows_and_first_tokens(window, sinks, dtype):
    lens = [520, 1, 130, 64]
    compare(lens, 2, 1, 64, dtype, window, sinks, *run(lens, 2, 1, 64, dtype, window, sinks))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (3, 3), (6, 2), (8, 1), (16, 8)])
@pytest.mark.parametrize("order", ["shd", "hsd"])
def test_heads_and_orders(H, H_kv, order, dtype):
    lens = [70, 1, 300]
    compare(lens, H, H_kv, 64, dtype, 50, 2, *run(lens, H, H_kv, 64, dtype, 50, 2, order))


@pytest.mark.parametrize("dtype,n,window,sinks", [(BF16, 2500, 600, 4), (F32, 900, 130, 40), (BF16, 3001, 100, 0), (BF16, 2049, 1, 2)])
def test_longer(dtype, n, window, sinks):
    lens = [n, 17, n // 2]
    compare(lens, 2, 1, 128, dtype, window, sinks, *run(lens, 2, 1, 128, dtype, window, sinks))


# first keys that are seen from far: workgroups of their own, more than one part of the rows, more than one block of first keys, groups of heads, and
# sequences with and without such rows
@pytest.mark.parametrize("dtype,d", [(BF16, 4), (BF16, 32), (BF16, 60), (BF16, 64), (BF16, 100), (BF16, 128), (BF16, 132), (BF16, 256), (F32, 20), (F32, 64), (F32, 100),
                                     (F32, 128), (F32, 256)])
@pytest.mark.parametrize("H,H_kv,lens,window,sinks", [(2, 1, [1300, 40, 0, 700, 100], 70, 4), (8, 1, [33, 400], 5, 37), (2, 2, [1900], 800, 130), (16, 4, [700, 300, 128, 2], 100, 20)])
def test_first_keys_seen_from_far(H, H_kv, lens, window, sinks, d, dtype):
    r = run(lens, H, H_kv, d, dtype, window, sinks)
    assert sa.sa_attn_window_bwd_workspace(r[0][0], r[0][1], lengths_to_offsets(lens), max(lens), window, sinks) > 0
    compare(lens, H, H_kv, d, dtype, window, sinks, *r)
    again = run(lens, H, H_kv, d, dtype, window, sinks)
    for x, y in zip(r[3], again[3]):
        assert torch.equal(x, y)


# so many of them that all walk on
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("H,H_kv,lens,window,sinks", [(8, 8, [1500, 20], 40, 600), (16, 8, [500] * 6, 100, 330)])
def test_many_first_keys(H, H_kv, lens, window, sinks, d, dtype):
    r = run(lens, H, H_kv, d, dtype, window, sinks)
    assert sa.sa_attn_window_bwd_workspace(r[0][0], r[0][1], lengths_to_offsets(lens), max(lens), window, sinks) == 0
    compare(lens, H, H_kv, d, dtype, window, sinks, *r, heads=[0, H_kv - 1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_infinities_and_first_keys_seen_from_far(dtype):
    """A query and its gradient that are no numbers, far behind a window: they reach dK and dV of the first keys and of its window, no other."""
    lens, window, sinks, d, at = [1500], 60, 5, 64, 1200
    (q, k, v, g), out, lse, clean = run(lens, 2, 1, d, dtype, window, sinks)
    off, n = lengths_to_offsets(lens).cuda(), torch.arange(1500)
    reached = (n < sinks) | ((n <= at) & (n > at - window))
    for which in (0, 3):
        ins = [x.clone() for x in (q, k, v, g)]
        ins[which][at, 1, 3] = NAN
        grads = [torch.full_like(x, 7) for x in (q, k, v)]
        backward(ins, out, lse, off, grads, 1500, window, sinks)
        for x, y in zip(grads[1:], clean[1:]):
            x, y = x.cpu().float(), y.cpu().float()
            assert torch.isfinite(x[~reached]).all() and (x[~reached] - y[~reached]).abs().max() <= 2.0 ** -6 * y.abs().max()
        assert not torch.isfinite(grads[1].cpu()[reached]).all(2).any()
    # another key's value: the first keys' own gradients know nothing of it
    ins = [x.clone() for x in (q, k, v, g)]
    ins[2][30] = NAN
    grads = [torch.full_like(x, 7) for x in (q, k, v)]
    backward(ins, out, lse, off, grads, 1500, window, sinks)
    assert torch.isfinite(grads[1].cpu()[n != 30]).all() and torch.isfinite(grads[2].cpu()).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 64, 100, 128, 256])
def test_many_workgroups(d, dtype):
    lens = [700, 300, 1, 1100 if dtype is BF16 else 500]
    compare(lens, 24, 12, d, dtype, 150, 7, *run(lens, 24, 12, d, dtype, 150, 7), heads=[0, 5, 11])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n_seq", [64, 65, 200])
def test_many_sequences(n_seq, dtype):
    lens = [(7 * i) % 40 + (250 if i % 50 == 3 else 0) for i in range(n_seq)]
    compare(lens, 2, 1, 32, dtype, 20, 2, *run(lens, 2, 1, 32, dtype, 20, 2))


def test_random_sizes():
    rng = random.Random(3)
    for i in range(24):
        dtype, H_kv, d = rng.choice([BF16, BF16, F32]), rng.choice([1, 2]), rng.choice([4, 20, 32, 64, 80, 100, 128, 160, 256])
        H, lens = H_kv * rng.choice([1, 2, 3]), [rng.randint(0, 400) for _ in range(rng.randint(1, 5))]
        window, sinks, order = rng.choice([1, 17, 64, 100, 128, 300]), rng.choice([0, 1, 4, 40, 128, 150]), rng.choice(["shd", "hsd"])
        print(i, lens, H, H_kv, d, dtype, window, sinks, order, flush=True)
        compare(lens, H, H_kv, d, dtype, window, sinks, *run(lens, H, H_kv, d, dtype, window, sinks, order, first=3, behind=2), first=3)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 100])
def test_rows_of_no_sequence_stay(d, dtype):
    lens, first = [5, 0, 200], 37
    ins, out, lse, grads = run(lens, 4, 2, d, dtype, 30, 2, first=first, behind=61)
    compare(lens, 4, 2, d, dtype, 30, 2, ins, out, lse, grads, first)
    for x in (out, lse.t(), *grads):
        assert (x[:first] == 7).all() and (x[first + sum(lens):] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_longest_length_cuts_off(dtype):
    """Of a sequence beyond max_len the rows from there on are left alone, and no row or key of theirs is seen."""
    lens, cut, d = [300, 90], 210, 64
    ins, out, lse, grads = run(lens, 2, 2, d, dtype, 50, 3, max_len=cut)
    keep = torch.cat([torch.arange(cut), torch.arange(300, 390)])
    compare([cut, 90], 2, 2, d, dtype, 50, 3, [x[keep.cuda()] for x in ins], out[keep.cuda()], lse[:, keep.cuda()], [x[keep.cuda()] for x in grads])
    for x in (out, lse.t(), *grads):
        assert (x[cut:300] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offsets", [[0, 300, 100, 400], [-50, 60, 1000, 20], [90, 90, 10, 120], [2 ** 30, -2 ** 30, 2 ** 31 - 1, 40], [0, 256, 0, 256, 0, 256]])
@pytest.mark.parametrize("window,sinks", [(20, 3), (1, 130)])
def test_any_offsets_stay_within_the_tensors(offsets, window, sinks, dtype):
    T = 256
    q, k, v, g = (rows((T, 2, 64), s, dtype) for s in (1, 2, 3, 4))
    out, lse = torch.full_like(q, 7), torch.full((2, T), 7.0, device="cuda")
    off = torch.tensor(offsets + offsets[-1:] * EMPTY[0], dtype=torch.int32, device="cuda")
    sa.sa_attn_window_fwd(q, k, v, off, out, lse, 256, window, sinks)
    grads = [torch.full_like(x, 7) for x in (q, k, v)]
    backward((q, k, v, g), out, lse, off, grads, 256, window, sinks)
    covered = torch.zeros(T, dtype=torch.bool)
    for a, b in zip(offsets, offsets[1:]):
        a = min(max(a, 0), T)
        covered[a:min(max(b, a), T)] = True
    for x in (out, lse.t(), *grads):
        assert (x.cpu()[~covered] == 7).all()


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 100), (BF16, 128), (BF16, 132), (BF16, 256), (F32, 64), (F32, 100), (F32, 256)])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_what_a_row_does_not_see_does_not_reach_it(bad, d, dtype):
    """A key and value, a query and gradient that are no numbers: rows and keys that see nothing of them have what they have without."""
    lens, window, sinks, at = [300, 40], 50, 2, 150
    clean = run(lens, 2, 2, d, dtype, window, sinks)

    def poison(*which):
        def mutate(*tensors):
            for i in which:
                tensors[i][at] = bad
        return mutate
    n = torch.arange(340)
    sees = (n >= at) & (n < at + window)        # rows that see the key
    for which in ((1,), (2,), (1, 2)):
        _, out, lse, _ = run(lens, 2, 2, d, dtype, window, sinks, mutate=poison(*which))
        # (rows done over have the other rows' tolerance: two roundings, of values below 4)
        assert (out.cpu()[~sees].float() - clean[1].cpu()[~sees].float()).abs().max() <= {BF16: 2.0 ** -7, F32: 2.0 ** -16}[dtype] * 4
        assert torch.isfinite(out.cpu()[~sees]).all() and torch.isfinite(lse.cpu()[:, ~sees]).all()
        assert not torch.isfinite(out.cpu()[sees]).all(1).any()
    # the gradient, with the statistics of the clean call
    (q, k, v, g), out, lse, _ = clean
    off = lengths_to_offsets(lens).cuda()
    for which in range(4):
        ins = [x.clone() for x in (q, k, v, g)]
        ins[which][at] = bad
        grads = [torch.full_like(x, 7) for x in (q, k, v)]
        backward(ins, out, lse, off, grads, 300, window, sinks)
        dq, dk, dv = (x.cpu() for x in grads)
        seen_by = ((n <= at) & (n > at - window)) | (n < sinks)       # keys that row `at` sees
        if which in (1, 2):         # of a key: its rows' dq, its own dk and dv, and delta knows nothing of it
            assert torch.isfinite(dq[~sees]).all()
            others = n != at
            assert torch.isfinite(dk[others]).all() and torch.isfinite(dv[others]).all()
        else:
            others = n != at
            assert torch.isfinite(dq[others]).all()
            assert torch.isfinite(dk[~seen_by]).all() and torch.isfinite(dv[~seen_by]).all()
        for got, want, ok in zip((dq, dk, dv), clean[3], ((~sees if which in (1, 2) else others), *[(others if which in (1, 2) else ~seen_by)] * 2)):
            assert (got[ok].float() - want.cpu()[ok].float()).abs().max() <= 2.0 ** -6 * want.float().abs().max()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_that_are_no_numbers(dtype):
    """A NaN or +inf score makes its row NaN, -inf has no weight, a row of nothing else is NaN."""
    lens, window, d = [200], 30, 64
    first = lambda q: q[:, :, 0].copy_(q[:, :, 0].abs() + 0.25)      # noqa: E731

    def keys(value, r):
        def mutate(q, k, v, g):
            first(q)
            k[r, :, 0] = value
        return mutate
    n = torch.arange(200)
    sees = (n >= 100) & (n < 130)
    for value in (NAN, INF):
        _, out, lse, _ = run(lens, 2, 2, d, dtype, window, 0, mutate=keys(value, slice(100, 101)))
        assert out.cpu()[sees].isnan().all() and lse.cpu()[:, sees].isnan().all()
        assert torch.isfinite(out.cpu()[~sees]).all() and torch.isfinite(lse.cpu()[:, ~sees]).all()
    (q, k, v, g), out, lse, _ = run(lens, 2, 2, d, dtype, window, 0, mutate=keys(-INF, slice(60, 120)))
    weightless = (n >= 60 + window - 1) & (n < 120)
    assert out.cpu()[weightless].isnan().all() and lse.cpu()[:, weightless].isnan().all()
    q, k, v = (x.cpu() for x in (q, k, v))
    sees = window_mask(200, window, 0) & ~((n >= 60) & (n < 120))[None, :]
    k[60:120, :, 0] = 0
    x = Seen(q[:, 1], k[:, 1], v[:, 1], d ** -0.5, sees)
    ok = sees.any(1)
    check("out", out[ok.cuda(), 1], x.out[ok], x.out_off(dtype, ROUNDED[dtype])[ok])
    check("lse", lse[1, ok.cuda()], x.lse[ok], x.lse_off[ok])


@pytest.mark.parametrize("d", [68, 100, 132])
def test_anything_between_the_rows(d):
    """Rows at a larger pitch, NaN in the gap; parts of larger tensors, what lies beside them stays."""
    lens, H, H_kv, dtype = [200, 1, 60], 4, 2, BF16
    T = sum(lens)
    (q, k, v, g), out, lse, grads = run(lens, H, H_kv, d, dtype, 40, 3)

    def part(x, heads):
        whole = torch.full((T + 3, heads + 3, d + 12), NAN, dtype=dtype, device="cuda")
        inside = whole[1:T + 1, 2:2 + heads, :d]
        if x is not None:
            inside.copy_(x)
        return whole, inside
    off = lengths_to_offsets(lens).cuda()
    Q, G, O, DQ = (part(x, H) for x in (q, g, None, None))
    K, V, DK, DV = (part(x, H_kv) for x in (k, v, None, None))
    L = torch.full((H + 1, T + 5), 9.0, device="cuda")
    sa.sa_attn_window_fwd(Q[1], K[1], V[1], off, O[1], L[:H, :T], 200, 40, 3)
    work = torch.empty(sa.sa_attn_window_bwd_workspace(Q[1], K[1], off, 200, 40, 3), dtype=torch.uint8, device="cuda")
    delta = torch.empty_like(L)
    sa.sa_attn_window_bwd(Q[1], K[1], V[1], O[1], G[1], L[:H, :T], off, delta[:H, :T], DQ[1], DK[1], DV[1], work, 200, 40, 3)
    for (whole, got), want in ((O, out), (DQ, grads[0]), (DK, grads[1]), (DV, grads[2])):
        assert torch.equal(got, want)
        got.fill_(NAN)
        assert whole.isnan().all()
    assert torch.equal(L[:H, :T], lse) and (L[H:] == 9).all() and (L[:, T:] == 9).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_a_window_beyond_the_sequences_is_none(d, dtype):
    """As the packed entry points, to the roundings of both."""
    lens = [300, 1, 129]
    ins, out, lse, grads = run(lens, 4, 2, d, dtype, 300, 0)
    off = lengths_to_offsets(lens).cuda()
    o, l = torch.empty_like(out), torch.empty_like(lse)
    sa.sa_attn_packed_fwd(*ins[:3], off, o, l, 300)
    other = [torch.empty_like(x) for x in grads]
    sa.sa_attn_packed_bwd(*ins[:3], o, ins[3], l, off, torch.empty_like(l), *other, 300)
    for x, y in zip((out, *grads), (o, *other)):
        assert (x.float() - y.float()).norm() <= {BF16: 2.0 ** -7, F32: 1e-5}[dtype] * y.float().norm()
    assert (lse - l).abs().max() <= 1e-5


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_scores(dtype):
    lens = [260, 31]
    compare(lens, 2, 2, 64, dtype, 60, 3, *run(lens, 2, 2, 64, dtype, 60, 3, mutate=lambda q, k, v, g: q.mul_(40)))


def test_scale_is_taken():
    lens = [100, 60]
    compare(lens, 2, 2, 64, BF16, 33, 1, *run(lens, 2, 2, 64, BF16, 33, 1, scale=0.5), scale=0.5)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradient_against_differences(dtype):
    """<dQ, e> and its like against (f(x + t e) - f(x - t e)) / 2t of f = <out, g> in 64 bits."""
    lens, H, H_kv, d, window, sinks = [37, 90], 2, 1, 32, 12, 2
    ins, out, lse, grads = run(lens, H, H_kv, d, dtype, window, sinks)
    q, k, v, g = (x.cpu().double() for x in ins)

    def f(q, k, v):
        total, at = 0.0, 0
        for n in lens:
            r = slice(at, at + n)
            at += n
            total += sum((Seen(q[r, h], k[r, 0], v[r, 0], d ** -0.5, window_mask(n, window, sinks)).out * g[r, h]).sum() for h in range(H))
        return total
    for i, got in enumerate(grads):
        e = normal(got.shape, 50 + i, torch.float64)
        t = 1e-5
        up, down = ([x + sign * t * e if j == i else x for j, x in enumerate((q, k, v))] for sign in (1, -1))
        want = (f(*up) - f(*down)) / (2 * t)
        # what a gradient of this size may be off in such a direction: r of each element, its parts' likewise (three roundings)
        off = 4 * {BF16: 2.0 ** -8, F32: 1e-5}[dtype] * got.cpu().double().norm() * e.norm() / got.numel() ** 0.5 * 3 + 1e-5
        assert abs((got.cpu().double() * e).sum() - want) <= off


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_captured_and_replayed(dtype, d):
    """Forward and backward in one graph, replayed beside eager work; the offsets are read when it is played."""
    H, H_kv, T, window, sinks = 4, 2, 900, 100, 3
    q, g = (rows((T, H, d), s, dtype) for s in (1, 2))
    k, v = (rows((T, H_kv, d), s, dtype) for s in (3, 4))
    off = lengths_to_offsets([250, 0, 650]).cuda()
    out, lse = torch.empty_like(q), torch.empty(H, T, device="cuda")
    delta, grads = torch.empty_like(lse), [torch.empty_like(x) for x in (q, k, v)]
    work = torch.empty(sa.sa_attn_window_bwd_workspace(q, k, off, T, window, sinks), dtype=torch.uint8, device="cuda")

    def both():
        sa.sa_attn_window_fwd(q, k, v, off, out, lse, T, window, sinks)
        sa.sa_attn_window_bwd(q, k, v, out, g, lse, off, delta, *grads, work, T, window, sinks)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for lens in ([250, 0, 650], [1, 898, 1], [900, 0, 0], [300, 300, 300]):
        off.copy_(lengths_to_offsets(lens))
        both()
        torch.cuda.synchronize()
        want = [x.clone() for x in (out, lse, *grads)]
        for x in (out, lse, delta, *grads):
            x.fill_(3)
        work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((out, lse, *grads), want):
            assert torch.equal(x, y)


def test_two_streams_at_once():
    lens, args = [700, 50, 333], [(8, 2, 64, BF16, 100, 4), (8, 2, 128, BF16, 200, 2)]
    want = [run(lens, *a) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in want]
    for _ in range(4):
        got = []
        for stream, a in zip(streams, args):
            with torch.cuda.stream(stream):
                got.append(run(lens, *a))
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            for u, w in zip((x[1], x[2], *x[3]), (y[1], y[2], *y[3])):
                assert torch.equal(u, w)


def test_empty_calls():
    q = torch.empty(0, 2, 64, dtype=BF16, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    sa.sa_attn_window_fwd(q, q, q, off, q, torch.empty(2, 0, device="cuda"), 5, 3)
    ins, out, lse, grads = run([0, 0], 2, 2, 64, BF16, 5, 1, behind=10)
    for x in (out, lse, *grads):
        assert (x == 7).all()


def test_more_heads_than_a_launch_takes():
    H, lens = 65535, [2, 1] * 100
    compare(lens, H, H, 4, BF16, 1, 0, *run(lens, H, H, 4, BF16, 1, 0), heads=[0, 20970, 20971, 41942, 62912, 62913, 65534])


# launches of few tiles, by workgroups of 32 rows, and others
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [8, 32, 52, 64, 100, 104, 128, 132])
@pytest.mark.parametrize("H,H_kv,lens,window,sinks", [(2, 1, [300, 33, 0, 1, 95], 1, 0), (2, 2, [500, 64], 33, 40), (16, 4, [200, 190, 180, 170, 160], 64, 4),
                                                      (48, 8, [31, 1, 17, 0, 32, 30], 7, 2), (48, 8, [700, 300], 130, 0)])
def test_launches_of_few_tiles(H, H_kv, lens, window, sinks, d, dtype):
    compare(lens, H, H_kv, d, dtype, window, sinks, *run(lens, H, H_kv, d, dtype, window, sinks))


@pytest.mark.parametrize("d", [64, 100])
@pytest.mark.parametrize("H", [2, 40])
def test_infinities_in_launches_of_few_tiles(H, d):
    """A value that is no number reaches the rows that see its key, of the heads that share it, and no others, whichever workgroups a launch has."""
    lens, window, sinks, at = [300, 200], 50, 3, 260
    (q, k, v, g), out, lse, clean = run(lens, H, H // 2, d, BF16, window, sinks)
    off, n = lengths_to_offsets(lens).cuda(), torch.arange(500)
    # rows beside them may be formed anew without rounding their probabilities: 2^-8 of the values, and both results' own rounding; lse, sums of up to
    # 64 terms of either order
    off_out, off_lse = 2.0 ** -8 * (v.float().abs().max() + 2 * out.float().abs().max()), 64 * 2.0 ** -24 * (1 + lse.abs().max())
    for key, rows in ((at, (n >= at) & (n < 300)), (301, n >= 301)):
        seen, other = rows.cuda(), ~rows.cuda()
        for which in (1, 2):
            ins = [q, k.clone(), v.clone()]
            ins[which][key, 0, 5] = NAN
            o2, lse2 = torch.full_like(out, 7), torch.full_like(lse, 7)
            sa.sa_attn_window_fwd(*ins, off, o2, lse2, max(lens), window, sinks)
            assert torch.isnan(o2[seen][:, :2, slice(None) if which == 1 else 5]).all()
            assert torch.equal(torch.isnan(lse2[:2, seen]), torch.full_like(lse2[:2, seen], which == 1, dtype=torch.bool))
            assert torch.equal(o2[:, 2:], out[:, 2:]) and torch.equal(lse2[2:], lse[2:])
            assert (o2[other].float() - out[other].float()).abs().max() <= off_out and (lse2[:, other] - lse[:, other]).abs().max() <= off_lse

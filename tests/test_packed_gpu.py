"""Causal attention of packed sequences and its gradient, against 64 bits."""
import pytest
import torch

from paper_2311_09431_amd import binding as sa
from sequences import Head, check, lengths_to_offsets, normal

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
# how far a weight is rounded before it meets V
ROUNDED = {BF16: 2.0 ** -8, F32: 0.0}


def rows(shape, seed, dtype, order="shd"):
    """[rows, heads, d] on the GPU: heads inside a row, or apart"""
    x = normal(shape, seed, dtype).cuda()
    return x if order == "shd" else x.permute(1, 0, 2).contiguous().permute(1, 0, 2)


def run(lens, H, H_kv, d, dtype, order="shd", first=0, behind=0, max_len=None, scale=None, backward=True, mutate=None):
    T = first + sum(lens) + behind
    q, g = (rows((T, H, d), s, dtype, order) for s in (1, 2))
    k, v = (rows((T, H_kv, d), s, dtype, order) for s in (3, 4))
    if mutate:
        mutate(q, k, v, g)
    off = lengths_to_offsets(lens, first).cuda()
    out, lse = torch.full_like(q, 7), torch.full((H, T), 7.0, device="cuda")
    top = max(lens + [1]) if max_len is None else max_len
    sa.sa_attn_packed_fwd(q, k, v, off, out, lse, top, scale)
    if not backward:
        return (q, k, v, g), out, lse, None
    delta, grads = torch.empty_like(lse), [torch.full_like(x, 7) for x in (q, k, v)]
    sa.sa_attn_packed_bwd(q, k, v, out, g, lse, off, delta, *grads, top, scale)
    return (q, k, v, g), out, lse, grads


def compare(lens, H, H_kv, d, dtype, first, ins, out, lse, grads, scale=None, heads=None):
    q, k, v, g = (x.cpu() for x in ins)
    scale = scale or d ** -0.5
    w, G = ROUNDED[dtype], H // H_kv
    at = first
    for s, n in enumerate(lens):
        r = slice(at, at + n)
        at += n
        for kvh in range(H_kv):
            if n == 0 or (heads is not None and kvh not in heads):
                continue
            dk = dv = dk_off = dv_off = 0
            for h in range(kvh * G, (kvh + 1) * G):
                x = Head(q[r, h], k[r, kvh], v[r, kvh], scale, True, g[r, h] if grads else None)
                check(("out", s, h), out[r, h], x.out, x.out_off(dtype, w))
                check(("lse", s, h), lse[h, r], x.lse, x.lse_off)
                if grads:
                    dq_off, a, b = x.grad_off(dtype, w)
                    check(("dq", s, h), grads[0][r, h], x.dq, dq_off)
                    dk, dv, dk_off, dv_off = dk + x.dk, dv + x.dv, dk_off + a, dv_off + b
            if grads:
                check(("dk", s, kvh), grads[1][r, kvh], dk, dk_off)
                check(("dv", s, kvh), grads[2][r, kvh], dv, dv_off)


def untouched(lens, first, *tensors):
    """Rows in front of the first and behind the last sequence hold what was there."""
    for x, axis in tensors:
        n = x.shape[axis]
        for r in (slice(0, first), slice(first + sum(lens), n)):
            assert (x.movedim(axis, 0)[r] == 7).all()


LENS = [1, 127, 0, 128, 129, 33, 300, 2]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [4, 32, 36, 64, 68, 96, 100, 112, 128, 132, 192, 256])
def test_head_dimensions(d, dtype):
    r = run(LENS, 2, 1, d, dtype)
    compare(LENS, 2, 1, d, dtype, 0, *r)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (3, 3), (6, 2), (8, 1), (16, 8)])
@pytest.mark.parametrize("order", ["shd", "hsd"])
def test_heads_and_orders(H, H_kv, order, dtype):
    lens = [70, 1, 200]
    r = run(lens, H, H_kv, 64, dtype, order)
    compare(lens, H, H_kv, 64, dtype, 0, *r)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 100])
def test_rows_of_no_sequence_stay(d, dtype):
    lens, first = [5, 0, 140], 37
    ins, out, lse, grads = run(lens, 4, 2, d, dtype, first=first, behind=61)
    compare(lens, 4, 2, d, dtype, first, ins, out, lse, grads)
    untouched(lens, first, (out, 0), (lse, 1), *((x, 0) for x in grads))


@pytest.mark.parametrize("dtype,n", [(BF16, 1500), (F32, 700), (BF16, 2049)])
def test_longer(dtype, n):
    lens = [n, 17, n // 2]
    r = run(lens, 2, 2, 128, dtype)
    compare(lens, 2, 2, 128, dtype, 0, *r)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n_seq", [64, 65, 200])
def test_many_sequences(n_seq, dtype):
    lens = [(7 * i) % 40 + (130 if i % 50 == 3 else 0) for i in range(n_seq)]
    r = run(lens, 2, 1, 32, dtype)
    compare(lens, 2, 1, 32, dtype, 0, *r)


# workgroups by ranks over all heads, and in groups of them; several rounds of the chip
@pytest.mark.parametrize("H,lens", [(40, [513, 900, 30, 700]), (72, [900] * 6), (9, [2500, 1])])
def test_many_workgroups(H, lens):
    r = run(lens, H, H, 64, BF16)
    compare(lens, H, H, 64, BF16, 0, *r, heads={0, H // 2, H - 1})


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_longest_length_cuts_off(dtype):
    """Of a sequence beyond max_len the rows from there on are left alone, and no key of theirs is seen."""
    lens, cut = [200, 90], 150
    ins, out, lse, grads = run(lens, 2, 2, 64, dtype, max_len=cut)
    q, k, v, g = (x.cpu() for x in ins)
    for r in (slice(0, cut), slice(200, 290)):
        x = Head(q[r, 1], k[r, 1], v[r, 1], 0.125, True, g[r, 1])
        check("out", out[r, 1], x.out, x.out_off(dtype, ROUNDED[dtype]))
        for got, want, off in zip(grads, (x.dq, x.dk, x.dv), x.grad_off(dtype, ROUNDED[dtype])):
            check("gradient", got[r, 1], want, off)
    for x in (out, lse.t(), *grads):
        assert (x[cut:200] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offsets", [[0, 300, 100, 400], [-50, 60, 1000, 20], [90, 90, 10, 120], [2 ** 30, -2 ** 30, 2 ** 31 - 1, 40]])
def test_any_offsets_stay_within_the_tensors(offsets, dtype):
    """Offsets are read as documented: clamped to the rows, an end before a beginning is empty.  Sequences that overlap
    write the same rows, so only that everything is a number and what no sequence covers stays is looked at."""
    T = 256
    q, k, v, g = (rows((T, 2, 64), s, dtype) for s in (1, 2, 3, 4))
    out, lse = torch.full_like(q, 7), torch.full((2, T), 7.0, device="cuda")
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    sa.sa_attn_packed_fwd(q, k, v, off, out, lse, 128)
    grads = [torch.full_like(x, 7) for x in (q, k, v)]
    sa.sa_attn_packed_bwd(q, k, v, out, g, lse, off, torch.empty_like(lse), *grads, 128)
    covered = torch.zeros(T, dtype=torch.bool)
    for a, b in zip(offsets, offsets[1:]):
        a = min(max(a, 0), T)
        covered[a:min(max(b, a), T, a + 128)] = True
    for x in (out, lse.t(), *grads):
        assert torch.isfinite(x).all() and (x.cpu()[~covered] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_nothing_of_one_sequence_reaches_another(dtype):
    """Infinities and NaN in the neighbours and in rows of no sequence."""
    lens, first = [150, 40, 131], 9

    def mutate(q, k, v, g):
        for x in (q, k, v, g):
            x[first + 150:first + 190] = float("nan")
            x[:first], x[first + 321:] = float("inf"), float("nan")
    ins, out, lse, grads = run(lens, 2, 1, 100, dtype, first=first, behind=30, mutate=mutate)
    q, k, v, g = (x.cpu() for x in ins)
    for r in (slice(first, first + 150), slice(first + 190, first + 321)):
        dk = dv = a = b = 0
        for h in range(2):
            x = Head(q[r, h], k[r, 0], v[r, 0], 0.1, True, g[r, h])
            check("out", out[r, h], x.out, x.out_off(dtype, ROUNDED[dtype]))
            offs = x.grad_off(dtype, ROUNDED[dtype])
            check("dq", grads[0][r, h], x.dq, offs[0])
            dk, dv, a, b = dk + x.dk, dv + x.dv, a + offs[1], b + offs[2]
        check("dk", grads[1][r, 0], dk, a)
        check("dv", grads[2][r, 0], dv, b)
    assert out[first + 150:first + 190].isnan().all() and lse[:, first + 150:first + 190].isnan().all()
    assert (out[:first] == 7).all() and (out[first + 321:] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_scores(dtype):
    """Softmax rows of one key: scores of hundreds."""
    def mutate(q, k, v, g):
        q.mul_(40)
    lens = [260, 31]
    r = run(lens, 2, 2, 64, dtype, mutate=mutate)
    compare(lens, 2, 2, 64, dtype, 0, *r)


def test_scale_is_taken():
    lens = [100, 60]
    r = run(lens, 2, 2, 64, BF16, scale=0.5)
    compare(lens, 2, 2, 64, BF16, 0, *r, scale=0.5)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradient_against_differences(dtype):
    """<dQ, e> and its like against (f(x + t e) - f(x - t e)) / 2t of f = <out, g> in 64 bits."""
    lens, H, d = [37, 90], 2, 32
    (q, k, v, g), out, lse, grads = run(lens, H, H, d, dtype)
    ins = [x.cpu().double() for x in (q, k, v)]
    g = g.cpu().double()

    def f(q, k, v):
        total, at = 0.0, 0
        for n in lens:
            r = slice(at, at + n)
            at += n
            total += sum((Head(q[r, h], k[r, h], v[r, h], d ** -0.5, True).out * g[r, h]).sum() for h in range(H))
        return total
    for i, got in enumerate(grads):
        e = normal(ins[i].shape, 50 + i, torch.float64)
        t = 1e-5
        up, down = ([x + sign * t * e if j == i else x for j, x in enumerate(ins)] for sign in (1, -1))
        want = (f(*up) - f(*down)) / (2 * t)
        # what a gradient of this size may be off in such a direction: r of each element, its parts' likewise (three roundings)
        off = 4 * {BF16: 2.0 ** -8, F32: 1e-5}[dtype] * got.cpu().double().norm() * e.norm() / got.numel() ** 0.5 * 3 + 1e-5
        assert abs((got.cpu().double() * e).sum() - want) <= off


def test_same_bits_again():
    lens = [700, 3, 1100]
    a = run(lens, 4, 2, 128, BF16)
    b = run(lens, 4, 2, 128, BF16)
    for x, y in zip((a[1], a[2], *a[3]), (b[1], b[2], *b[3])):
        assert torch.equal(x, y)


def test_empty_calls():
    q = torch.empty(0, 2, 64, dtype=BF16, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    sa.sa_attn_packed_fwd(q, q, q, off, q, torch.empty(2, 0, device="cuda"), 5)
    ins, out, lse, grads = run([0, 0], 2, 2, 64, BF16, behind=10)
    untouched([0], 0, (out, 0), (lse, 1), *((x, 0) for x in grads))
    # no sequence at all
    out.fill_(7)
    sa.sa_attn_packed_fwd(*ins[:3], off[:1], out, lse, 5)
    assert (out == 7).all()


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_captured_and_replayed(dtype, d):
    """Forward and backward in one graph; the offsets are read when it is played."""
    H, H_kv, T = 4, 2, 400
    q, g = (rows((T, H, d), s, dtype) for s in (1, 2))
    k, v = (rows((T, H_kv, d), s, dtype) for s in (3, 4))
    off = lengths_to_offsets([250, 0, 150]).cuda()
    out, lse = torch.empty_like(q), torch.empty(H, T, device="cuda")
    delta, grads = torch.empty_like(lse), [torch.empty_like(x) for x in (q, k, v)]

    def both():
        sa.sa_attn_packed_fwd(q, k, v, off, out, lse, T)
        sa.sa_attn_packed_bwd(q, k, v, out, g, lse, off, delta, *grads, T)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for lens in ([250, 0, 150], [1, 398, 1], [400, 0, 0]):
        off.copy_(lengths_to_offsets(lens))
        both()
        torch.cuda.synchronize()
        want = [x.clone() for x in (out, lse, *grads)]
        for x in (out, lse, delta, *grads):
            x.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((out, lse, *grads), want):
            assert torch.equal(x, y)


def test_other_stream():
    lens = [600, 50]
    want = run(lens, 4, 4, 64, BF16)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = run(lens, 4, 4, 64, BF16)
    stream.synchronize()
    for x, y in zip((got[1], got[2], *got[3]), (want[1], want[2], *want[3])):
        assert torch.equal(x, y)


def test_as_the_ring_step():
    """A sequence of whole tiles by itself is one triangular block of the ring step: the same products in the same order."""
    n, H, d = 512, 2, 128
    (q, k, v, _), out, lse, _ = run([n], H, H, d, BF16, backward=False)
    x = [t.permute(1, 0, 2)[None] for t in (q, k, v)]
    O, L = torch.empty(1, H, n, d, device="cuda"), torch.empty(1, H, n, device="cuda")
    Q, K, V = (t.contiguous() for t in x)
    shape = sa.shard_shape(Q, n, L)
    sa.sa_state_init(O, L, shape)
    sa.sa_attn_step_fwd(Q, K, V, O, L, 0, 0, 1, sa.CONTIGUOUS, shape)
    done = torch.empty_like(Q)
    sa.sa_finalize(O, done, shape)
    # the step's state passes through fp32 once more before it is rounded
    assert (out.permute(1, 0, 2).float() - done[0].float()).abs().max() <= 2.0 ** -8 * done.float().abs().max()
    assert (lse - L[0]).abs().max() <= 1e-5


# 32-row and 128-row workgroups, forward and backward each (launches of few and of many tiles), at every number of columns computed
# (above 128 columns: halves of dK and dV, and all columns, in a workgroup)
@pytest.mark.parametrize("d", [32, 64, 100, 128, 256])
@pytest.mark.parametrize("H,H_kv,lens", [(4, 1, [200, 31, 1, 65]), (24, 24, [500, 33, 257]), (32, 4, [900, 129, 64]), (48, 2, [257, 31])])
def test_few_and_many_tiles(H, H_kv, lens, d):
    r = run(lens, H, H_kv, d, BF16)
    compare(lens, H, H_kv, d, BF16, 0, *r, heads={0, H_kv - 1})


def test_more_heads_than_a_launch_takes():
    """Launches of whole key/value heads, 20971 of them in the first three."""
    H, lens = 65535, [2, 1] * 100
    r = run(lens, H, H, 4, BF16)
    compare(lens, H, H, 4, BF16, 0, *r, heads=[0, 1, 20970, 20971, 41941, 41942, 50000, 62912, 62913, 65534])


def test_two_streams_at_once():
    lens = [700, 50, 333]
    want = [run(lens, 8, 2, d, BF16) for d in (64, 128)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in want]
    for _ in range(4):
        got = []
        for stream, d in zip(streams, (64, 128)):
            with torch.cuda.stream(stream):
                got.append(run(lens, 8, 2, d, BF16))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for x, y in zip((g[1], g[2], *g[3]), (w[1], w[2], *w[3])):
                assert torch.equal(x, y)


@pytest.mark.parametrize("d", [68, 100, 112, 128, 132, 256])
@pytest.mark.parametrize("H,H_kv,lens", [(24, 12, [700, 300, 129, 1]), (14, 14, [1500, 0, 64]), (9, 9, [100, 3, 128, 77]), (36, 12, [2500])])
def test_both_kinds_of_backward_workgroups_in_a_launch(H, H_kv, lens, d):
    """108 to 252 tiles: one launch, or two by the head dimension and the groups."""
    r = run(lens, H, H_kv, d, BF16)
    compare(lens, H, H_kv, d, BF16, 0, *r, heads=[0, H_kv // 2, H_kv - 1])
    again = run(lens, H, H_kv, d, BF16)
    for x, y in zip(r[3], again[3]):
        assert torch.equal(x, y)


@pytest.mark.parametrize("d", [100, 128, 256])
def test_tiles_in_groups_of_heads(d):
    """Over 180 MB of keys and values, as many as 100 tiles a head: the order of the workgroups is another."""
    lens = [1900, 20, 700] + [20] * 58 + [2600]
    assert 4 * sum(lens) * 80 * d > 180e6
    r = run(lens, 80, 80, d, BF16)
    compare(lens, 80, 80, d, BF16, 0, *r, heads=[0, 39, 79])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_parts_of_larger_tensors(dtype):
    """Rows, heads and sums that are parts of larger tensors; what lies beside them stays."""
    lens, H, H_kv, d = [200, 1, 60], 4, 2, 64
    T = sum(lens)
    (q, k, v, g), out, lse, grads = run(lens, H, H_kv, d, dtype)

    def part(x, heads):
        whole = torch.full((T + 3, heads + 3, d + 8), 9, dtype=dtype, device="cuda")
        inside = whole[1:T + 1, 2:2 + heads, :d]
        if x is not None:
            inside.copy_(x)
        return whole, inside

    sums = [torch.full((H + 1, T + 5), 9.0, device="cuda") for _ in range(2)]
    L, D = (x[:H, :T] for x in sums)
    off = lengths_to_offsets(lens).cuda()
    Q, G, O, DQ = (part(x, H) for x in (q, g, None, None))
    K, V, DK, DV = (part(x, H_kv) for x in (k, v, None, None))
    sa.sa_attn_packed_fwd(Q[1], K[1], V[1], off, O[1], L, 200)
    sa.sa_attn_packed_bwd(Q[1], K[1], V[1], O[1], G[1], L, off, D, DQ[1], DK[1], DV[1], 200)
    for (whole, got), want in ((O, out), (DQ, grads[0]), (DK, grads[1]), (DV, grads[2])):
        assert torch.equal(got, want)
        got.fill_(9)
        assert (whole == 9).all()
    assert torch.equal(L, lse) and (sums[0][H:] == 9).all() and (sums[0][:, T:] == 9).all()

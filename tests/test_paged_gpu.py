"""The paged key/value cache: appending rotated rows, attention of one new token, and both with the packed prompt, against 64 bits."""
import pytest
import torch

from paper_2311_09431_amd import binding as sa
from sequences import HALF_STEP, U, Head, check, lengths_to_offsets, normal

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
ROUNDED = {BF16: 2.0 ** -17, F32: 0.0}          # a weight as two bf16 terms, or as it is


def cache(pages, page, heads, d, dtype, order, fill=float("nan")):
    """[pages, page, heads, d] on the GPU; order of the memory: heads inside a token's step, or apart.  What nobody wrote is NaN."""
    if order == "shd":
        return torch.full((pages, page, heads, d), fill, dtype=dtype, device="cuda")
    return torch.full((pages, heads, page, d), fill, dtype=dtype, device="cuda").permute(0, 2, 1, 3)


def tables(lens, page, seed, spare=2, width=None):
    """Pages of a pool in no order; entries behind a sequence's last page are no page."""
    n = [-(-x // page) for x in lens]
    ids = torch.randperm(sum(n) + spare, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(lens), width or max(n + [1])), -1, dtype=torch.int32)
    at = 0
    for s, x in enumerate(n):
        table[s, :x] = ids[at:at + x]
        at += x
    return table, len(ids)


def fill(k_cache, v_cache, table, lens, seed):
    """Gaussians in the slots that the sequences use; returns them, [tokens, heads, d] a sequence."""
    page, (heads, d) = k_cache.shape[1], k_cache.shape[2:]
    rows = []
    for s, n in enumerate(lens):
        kv = [normal((n, heads, d), seed + 2 * s + i, k_cache.dtype) for i in (0, 1)]
        rows.append(kv)
        t = torch.arange(n)
        for c, x in zip((k_cache, v_cache), kv):
            c[table[s][t // page].long().cuda(), (t % page).cuda()] = x.cuda()
    return rows


def decode(lens, H, H_kv, d, dtype, page=16, order="shd", seed=1, scale=None, mutate=None, width=None, with_lse=True):
    table, pool = tables(lens, page, seed, width=width)
    k_cache, v_cache = (cache(pool, page, H_kv, d, dtype, order) for _ in range(2))
    rows = fill(k_cache, v_cache, table, lens, 10 * seed)
    q = normal((len(lens), H, d), seed + 5, dtype)
    if mutate:
        mutate(q, rows, k_cache, v_cache, table)
    out, lse = torch.full((len(lens), H, d), 7, dtype=dtype, device="cuda"), torch.full((len(lens), H), 7.0, device="cuda")
    work = torch.full((sa.sa_attn_decode_workspace(q, k_cache),), 255, dtype=torch.uint8, device="cuda")       # NaN
    sa.sa_attn_decode(q.cuda(), k_cache, v_cache, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse if with_lse else None,
                      work, scale)
    return q, rows, out.cpu(), lse.cpu()


def compare(q, rows, out, lse, dtype, scale=None, heads=None):
    B, H, d = q.shape
    scale = scale or d ** -0.5
    for b in range(B):
        k, v = rows[b]
        if k.shape[0] == 0:
            assert (out[b] == 0).all() and (lse[b] == -torch.inf).all()
            continue
        G = H // k.shape[1]
        for kvh in range(k.shape[1]):
            if heads is not None and kvh not in heads:
                continue
            h = slice(kvh * G, (kvh + 1) * G)
            x = Head(q[b, h], k[:, kvh], v[:, kvh], scale, False)
            check(("out", b, kvh), out[b, h], x.out, x.out_off(dtype, ROUNDED[dtype]))
            check(("lse", b, kvh), lse[b, h], x.lse, x.lse_off)


LENS = [1, 15, 16, 0, 17, 31, 33, 128, 129, 500]


# Tables of so few pages that a workgroup takes a unit, and of so many that the tokens are dealt out in shares.
WIDTHS = [None, 200]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [4, 20, 32, 64, 68, 100, 128, 132, 200, 256])
@pytest.mark.parametrize("width", WIDTHS)
def test_decode_head_dimensions(width, d, dtype):
    compare(*decode(LENS, 4, 2, d, dtype, width=width), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (5, 5), (12, 3), (16, 1), (17, 1), (32, 8), (40, 1), (66, 2)])
@pytest.mark.parametrize("order", ["shd", "hsd"])
@pytest.mark.parametrize("width", WIDTHS)
def test_decode_heads_and_orders(width, H, H_kv, order, dtype):
    compare(*decode([90, 1, 300], H, H_kv, 64, dtype, order=order, width=width), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [16, 48, 64, 80, 256, 1024])
def test_decode_page_sizes(page, dtype):
    compare(*decode([1, 47, 200, 1100, 256], 8, 2, 128, dtype, page=page), dtype)


# one sequence over many workgroups, many sequences in one workgroup, and both beside each other
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens", [[20000], [1] * 700, [0] * 70 + [9000] + [3] * 90, [130] * 65, list(range(1, 300, 7))])
def test_decode_shares(lens, dtype):
    compare(*decode(lens, 4, 2, 64, dtype, page=64), dtype)


def test_decode_long():
    lens = [70001, 5, 33333]
    compare(*decode(lens, 8, 2, 128, BF16, page=128), BF16)


def test_decode_offsets_beyond_32_bits():
    """A cache of 6 GB: the pages used lie at its end."""
    page, heads, d, pages = 256, 8, 128, 6000
    lens = [700, 300]
    k_cache, v_cache = (cache(pages, page, heads, d, BF16, "shd", 0) for _ in range(2))
    assert k_cache.numel() > 2 ** 30 and k_cache.numel() * 2 > 2 ** 31
    table = torch.tensor([[pages - 1, pages - 5, pages - 3], [pages - 2, 0, 0]], dtype=torch.int32)
    table[1, 1] = pages - 4
    rows = fill(k_cache, v_cache, table, lens, 3)
    q = normal((2, 16, d), 9, BF16)
    out, lse = torch.empty(2, 16, d, dtype=BF16, device="cuda"), torch.empty(2, 16, device="cuda")
    work = torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    sa.sa_attn_decode(q.cuda(), k_cache, v_cache, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse, work)
    compare(q, rows, out.cpu(), lse.cpu(), BF16)
    # and appending there
    slot = torch.tensor([(pages - 1) * page + 255, pages * page - 2, -1], dtype=torch.int32, device="cuda")
    k, v = (normal((3, heads, d), s, BF16).cuda() for s in (20, 21))
    sa.sa_cache_append(k, v, slot, k_cache, v_cache)
    for c, x in ((k_cache, k), (v_cache, v)):
        assert torch.equal(c[pages - 1, 255], x[0]) and torch.equal(c[pages - 1, 254], x[1])


@pytest.mark.parametrize("width", WIDTHS)
def test_decode_scale_and_no_lse(width):
    q, rows, out, lse = decode([77, 200], 4, 2, 64, BF16, scale=0.5, width=width)
    compare(q, rows, out, lse, BF16, scale=0.5)
    again = decode([77, 200], 4, 2, 64, BF16, scale=0.5, with_lse=False, width=width)
    assert torch.equal(again[2], out) and (again[3] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_decode_large_scores(dtype):
    def mutate(q, rows, *_):
        q.mul_(50)
    compare(*decode([1, 300, 2000], 4, 2, 64, dtype, mutate=mutate), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [7, 200])
def test_decode_pages_that_are_none(width, dtype):
    """Tokens of a page number that is none of the cache's are left out, all of them: no token."""
    page, lens = 32, [100, 200, 64]
    table, pool = tables(lens, page, 4, width=width)
    k_cache, v_cache = (cache(pool, page, 2, 64, dtype, "shd") for _ in range(2))
    rows = fill(k_cache, v_cache, table, lens, 40)
    table[0, 1], table[1, 0], table[1, 6] = pool, -2 ** 31, 2 ** 31 - 1
    table[2, :2] = -1
    gone = [torch.ones(n, dtype=torch.bool) for n in lens]
    gone[0][32:64] = gone[1][0:32] = gone[1][192:] = gone[2][:] = False
    rows = [[x[keep] for x in kv] for kv, keep in zip(rows, gone)]
    q = normal((3, 4, 64), 6, dtype)
    out, lse = torch.full_like(q, 7).cuda(), torch.full((3, 4), 7.0, device="cuda")
    work = torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    sa.sa_attn_decode(q.cuda(), k_cache, v_cache, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse, work)
    compare(q, rows, out.cpu(), lse.cpu(), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_decode_any_length_stays_within_the_table(dtype):
    page = 16
    table, pool = tables([40, 40, 40], page, 2)
    k_cache, v_cache = (cache(pool, page, 1, 64, dtype, "shd") for _ in range(2))
    rows = fill(k_cache, v_cache, table, [48, 48, 48], 4)
    q = normal((3, 2, 64), 6, dtype)
    out, lse = torch.empty_like(q).cuda(), torch.empty(3, 2, device="cuda")
    work = torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    lens = torch.tensor([2 ** 31 - 1, -5, 49], dtype=torch.int32, device="cuda")
    sa.sa_attn_decode(q.cuda(), k_cache, v_cache, table.cuda(), lens, out, lse, work)
    rows[1] = [x[:0] for x in rows[1]]
    compare(q, rows, out.cpu(), lse.cpu(), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,width", [(20, None), (20, 200), (3000, None)])
def test_decode_infinities_and_nan(n, width, dtype):
    """A key at -inf has no weight; alone, or beside NaN or +inf, the row is no number.  Other sequences do not notice."""
    d, inf = 64, float("inf")
    def mutate(q, rows, k_cache, v_cache, table):
        q[:] = q.abs() + 0.1                    # a key of infinities has that score
        page = k_cache.shape[1]
        def put(s, t, value):
            rows[s][0][t] = value
            k_cache[int(table[s, t // page]), t % page] = value
        for t in range(0, n, 2):
            put(0, t, -inf)
        for t in range(n):
            put(1, t, -inf)
        put(2, n - 1, inf)
        put(3, n // 2, float("nan"))
    q, rows, out, lse = decode([n] * 5, 2, 1, d, dtype, mutate=mutate, width=width)
    keep = torch.arange(n) % 2 == 1
    rows[0] = [x[keep] for x in rows[0]]
    for s in (0, 4):
        compare(q[s:s + 1], [rows[s]], out[s:s + 1], lse[s:s + 1], dtype)
    assert out[1:4].isnan().all() and lse[1:4].isnan().all()


@pytest.mark.parametrize("width", [20, 200])
def test_decode_captured_and_replayed(width):
    """Lengths and tables are read when the graph is played."""
    page, most = 32, 640
    table, pool = tables([most] * 3, page, 8, width=width)
    k_cache, v_cache = (cache(pool, page, 2, 128, BF16, "shd") for _ in range(2))
    fill(k_cache, v_cache, table, [most] * 3, 5)
    q = normal((3, 8, 128), 6, BF16).cuda()
    table, lens = table.cuda(), torch.tensor([640, 5, 0], dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(3, 8, device="cuda")
    work = torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    call = lambda: sa.sa_attn_decode(q, k_cache, v_cache, table, lens, out, lse, work)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for now in ([640, 5, 0], [0, 0, 640], [33, 640, 1]):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        call()
        torch.cuda.synchronize()
        want = out.clone(), lse.clone()
        out.fill_(3), lse.fill_(3), work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("width", WIDTHS)
def test_decode_shared_pages(width):
    """Sequences with the same beginning share its pages; a page may also stand twice in one sequence."""
    page, lens = 16, [100, 90, 33]
    table, pool = tables(lens, page, 3, width=width)
    k_cache, v_cache = (cache(pool, page, 2, 64, BF16, "shd") for _ in range(2))
    rows = fill(k_cache, v_cache, table, lens, 7)
    table[1, :4], table[2, 1] = table[0, :4], table[2, 0]
    rows[1] = [torch.cat([a[:64], b[64:]]) for a, b in zip(rows[0], rows[1])]
    rows[2] = [torch.cat([x[:16], x[:16], x[32:]]) for x in rows[2]]
    q = normal((3, 4, 64), 2, BF16)
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(3, 4, device="cuda")
    work = torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    sa.sa_attn_decode(q.cuda(), k_cache, v_cache, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse, work)
    compare(q, rows, out.cpu(), lse.cpu(), BF16)


def test_decode_two_streams_at_once():
    """A workspace each."""
    lens = [3000, 4, 900]
    want = [decode(lens, 8, 2, d, BF16) for d in (64, 128)]
    streams = [torch.cuda.Stream() for _ in want]
    for _ in range(4):
        got = []
        for stream, d in zip(streams, (64, 128)):
            with torch.cuda.stream(stream):
                got.append(decode(lens, 8, 2, d, BF16))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g[2], w[2]) and torch.equal(g[3], w[3])


def test_two_captured_calls_with_a_workspace_each():
    lens = torch.tensor([3000, 70], dtype=torch.int32)
    table, pool = tables(lens.tolist(), 16, 8)
    k_cache, v_cache = (cache(pool, 16, 2, 128, BF16, "shd") for _ in range(2))
    fill(k_cache, v_cache, table, lens.tolist(), 5)
    table, lens = table.cuda(), lens.cuda()
    qs = [normal((2, 8, 128), seed, BF16).cuda() for seed in (6, 7)]
    outs, lses = [torch.empty_like(q) for q in qs], [torch.empty(2, 8, device="cuda") for _ in qs]
    works = [torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda") for q in qs]
    calls = [lambda i=i: sa.sa_attn_decode(qs[i], k_cache, v_cache, table, lens, outs[i], lses[i], works[i]) for i in (0, 1)]
    for call in calls:
        call()
    torch.cuda.synchronize()
    want = [x.clone() for x in outs + lses]
    graphs = [torch.cuda.CUDAGraph() for _ in calls]
    for graph, call in zip(graphs, calls):
        with torch.cuda.graph(graph):
            call()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        for x in outs + lses:
            x.fill_(3)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(outs + lses, want):
            assert torch.equal(x, y)


def test_a_single_page_of_any_page_stride():
    """(nothing is a step of it away)"""
    k, v = (normal((1, 48, 2, 64), s, BF16).cuda() for s in (1, 2))
    odd = [x.as_strided(x.shape, (1, *x.stride()[1:])) for x in (k, v)]
    q = normal((1, 4, 64), 3, BF16)
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(1, 4, device="cuda")
    work = torch.empty(sa.sa_attn_decode_workspace(q, odd[0]), dtype=torch.uint8, device="cuda")
    one = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    sa.sa_attn_decode(q.cuda(), *odd, one, torch.full((1,), 41, dtype=torch.int32, device="cuda"), out, lse, work)
    compare(q, [[x[0, :41].cpu() for x in (k, v)]], out.cpu(), lse.cpu(), BF16)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", WIDTHS)
def test_decode_strided(width, dtype):
    """Queries and results side by side with other heads, a table and sums that are parts of larger ones; nothing beside them changes."""
    lens, H, H_kv, d, page = [77, 1, 0, 300], 4, 2, 68, 16
    q, rows, out, lse = decode(lens, H, H_kv, d, dtype, page, width=width)
    table, pool = tables(lens, page, 1, width=width)
    k_cache, v_cache = (cache(pool, page, H_kv, d, dtype, "shd") for _ in range(2))
    fill(k_cache, v_cache, table, lens, 10)
    wide = torch.full((len(lens), H + 5, d + 4), 9, dtype=dtype, device="cuda")
    q_wide = wide.clone()
    q_wide[:, 1:1 + H, :d] = q.cuda()
    pages = torch.full((len(lens), table.shape[1] + 3), 2 ** 30, dtype=torch.int32)
    pages[:, 2:-1] = table
    sums = torch.full((len(lens), H + 2), 9.0, device="cuda")
    q_part, out_part = q_wide[:, :, :d][:, 1:1 + H], wide[:, :, :d][:, 1:1 + H]
    work = torch.empty(sa.sa_attn_decode_workspace(q_part, k_cache), dtype=torch.uint8, device="cuda")
    sa.sa_attn_decode(q_part, k_cache, v_cache, pages.cuda()[:, 2:-1], torch.tensor(lens, dtype=torch.int32, device="cuda"), out_part, sums[:, :H],
                      work)
    assert torch.equal(out_part.cpu(), out) and torch.equal(sums[:, :H].cpu(), lse)
    assert (wide[:, 0] == 9).all() and (wide[:, 1 + H:] == 9).all() and (wide[..., d:] == 9).all() and (sums[:, H:] == 9).all()


# ---------------------------------------------------------------- append


def rotated(x, pos, base):
    half = x.shape[-1] // 2
    a = pos.double()[:, None] * base ** (-torch.arange(half, dtype=torch.float64) * 2 / x.shape[-1])
    c, s = a.cos()[:, None], a.sin()[:, None]
    lo, hi = x.double().split(half, -1)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def off_of(x, want, dtype):
    """One rounding of the result; a sine or cosine in fp32 from an angle off by 2^-24 of half a turn (4 u in all), times both elements
    of the pair; the two products and their sum in fp32."""
    half = x.shape[-1] // 2
    size = x.double().abs()
    pair = size + torch.cat([size[..., half:], size[..., :half]], -1)
    return HALF_STEP[dtype] * want.abs() + 8 * U * pair


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [4, 12, 32, 64, 100, 112, 128, 256])
@pytest.mark.parametrize("rows,order", [(1, "shd"), (37, "hsd"), (1500, "shd")])
def test_append(rows, order, d, dtype):
    H, H_kv, page = 6, 2, 32
    pages = rows // page + 3
    k_cache, v_cache = (cache(pages, page, H_kv, d, dtype, order, 7) for _ in range(2))
    q, k, v = normal((rows, H, d), 1, dtype), normal((rows, H_kv, d), 2, dtype), normal((rows, H_kv, d), 3, dtype)
    gen = torch.Generator().manual_seed(rows)
    slot = torch.randperm(pages * page, generator=gen)[:rows].to(torch.int32)
    pos = torch.randint(0, 1 << 20, (rows,), generator=gen).to(torch.int32)
    padding = torch.arange(rows) % 5 == 4
    slot[padding] = torch.tensor([-1, -2 ** 31, pages * page, 2 ** 31 - 1], dtype=torch.int32)[torch.arange(int(padding.sum())) % 4]
    q_out, k_out = torch.empty_like(q).cuda(), torch.empty_like(k).cuda()
    gq, gk, gv = q.cuda(), k.cuda(), v.cuda()
    sa.sa_cache_append(gk, gv, slot.cuda(), k_cache, v_cache, pos=pos.cuda(), k_out=k_out, q=gq, q_out=q_out, base=5000.0)
    assert torch.equal(gq.cpu(), q) and torch.equal(gk.cpu(), k)
    for got, x in ((q_out, q), (k_out, k)):
        want = rotated(x, pos, 5000.0)
        check("rotated", got, want, off_of(x, want, dtype))
    kept = slot[~padding].long()
    for c, x in ((k_cache, k_out.cpu()), (v_cache, v)):
        want = torch.full((pages * page, H_kv, d), 7, dtype=dtype)
        want[kept] = x[~padding]
        assert torch.equal(c.cpu().reshape(-1, H_kv, d), want)
    # in place, and without what is not wanted
    again = [cache(pages, page, H_kv, d, dtype, order, 7) for _ in range(2)]
    sa.sa_cache_append(gk, gv, slot.cuda(), *again, pos=pos.cuda(), k_out=gk, q=gq, q_out=gq, base=5000.0)
    assert torch.equal(gq, q_out) and torch.equal(gk, k_out) and torch.equal(again[0], k_cache) and torch.equal(again[1], v_cache)
    again = [cache(pages, page, H_kv, d, dtype, order, 7) for _ in range(2)]
    sa.sa_cache_append(k.cuda(), gv, slot.cuda(), *again, pos=pos.cuda(), base=5000.0)
    assert torch.equal(again[0], k_cache) and torch.equal(again[1], v_cache)
    # not rotated
    sa.sa_cache_append(k.cuda(), gv, slot.cuda(), *again)
    want = torch.full((pages * page, H_kv, d), 7, dtype=dtype)
    want[kept] = k[~padding]
    assert torch.equal(again[0].cpu().reshape(-1, H_kv, d), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_strided_rows(dtype):
    """Rows as one projection writes them, q, k and v side by side; and with the heads apart."""
    rows, H, H_kv, d, page = 21, 4, 2, 64, 16
    for apart in (False, True):
        x = normal((rows, H + 2 * H_kv, d), 4, dtype).cuda()
        if apart:
            x = x.permute(1, 0, 2).contiguous().permute(1, 0, 2)
        q, k, v = x.split([H, H_kv, H_kv], 1)
        kept = x.clone()
        pos = torch.arange(rows, dtype=torch.int32, device="cuda") + 1000
        slot = torch.arange(rows, dtype=torch.int32, device="cuda") + 5
        got = [cache(3, page, H_kv, d, dtype, "shd", 0) for _ in range(2)]
        sa.sa_cache_append(k, v, slot, *got, pos=pos, k_out=k, q=q, q_out=q)
        plain = [t.contiguous() for t in kept.split([H, H_kv, H_kv], 1)]
        want = [cache(3, page, H_kv, d, dtype, "shd", 0) for _ in range(2)]
        sa.sa_cache_append(plain[1], plain[2], slot, *want, pos=pos, k_out=plain[1], q=plain[0], q_out=plain[0])
        assert torch.equal(q, plain[0]) and torch.equal(k, plain[1]) and torch.equal(v, plain[2])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("base", [1.5, 500000.0])
def test_append_positions_of_any_sign(base):
    x, v = normal((4, 2, 64), 1, F32), normal((4, 2, 64), 2, F32)
    pos = torch.tensor([-3, 0, -100000, 7], dtype=torch.int32)
    k_cache, v_cache = (cache(1, 16, 2, 64, F32, "shd", 0) for _ in range(2))
    sa.sa_cache_append(x.cuda(), v.cuda(), torch.arange(4, dtype=torch.int32, device="cuda"), k_cache, v_cache, pos=pos.cuda(), base=base)
    want = rotated(x, pos, base)
    check("rotated", k_cache[0, :4], want, off_of(x, want, F32))


def test_append_more_rows_than_a_launch_takes():
    """(2^24 - 1) * 8 rows go in the first one."""
    n, page = (2 ** 24 - 1) * 8 + 21, 16
    pages = -(-n // page)
    k = torch.arange(4 * n, device="cuda").remainder_(251).to(BF16).view(n, 1, 4)
    v = torch.arange(4 * n, device="cuda").remainder_(247).to(BF16).view(n, 1, 4)
    k_cache, v_cache = (torch.zeros(pages, page, 1, 4, dtype=BF16, device="cuda") for _ in range(2))
    slot = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda")
    sa.sa_cache_append(k, v, slot, k_cache, v_cache)
    for x, c in ((k, k_cache), (v, v_cache)):
        assert torch.equal(c.view(-1, 1, 4)[:n], x.flip(0)) and (c.view(-1, 4)[n:] == 0).all()


def test_append_rotates_as_rope_does():
    rows, H, d = 200, 3, 128
    k = normal((rows, H, d), 3, F32).cuda()
    pos = torch.arange(rows, dtype=torch.int32, device="cuda") * 999
    k_out, c = torch.empty_like(k), [cache(13, 16, H, d, F32, "shd", 0) for _ in range(2)]
    sa.sa_cache_append(k, k, pos * 0 - 1, *c, pos=pos, k_out=k_out)
    x = k.permute(1, 0, 2)[None]
    y = torch.empty_like(x)
    sa.sa_rope(x, y, pos, sa.shard_shape(x, rows))
    # both: a sine in fp32, two products and a sum; 8 u of the pair each
    assert (y[0].permute(1, 0, 2) - k_out).abs().max() <= 16 * U * 2 * k.abs().max()


# ---------------------------------------------------------------- together


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,H_kv,d,page", [(4, 2, 64, 16), (8, 8, 100, 48), (8, 1, 128, 64)])
def test_prompt_then_tokens(H, H_kv, d, page, dtype):
    """Prompts of different lengths into the cache and through packed attention, then new tokens one at a time: each token's
    attention is that of the whole sequence's last row."""
    prompts, steps, n = [33, 1, 150], 3, 3
    most = max(prompts) + steps
    table, pool = tables([most] * n, page, 6)
    k_cache, v_cache = (cache(pool, page, H_kv, d, dtype, "shd") for _ in range(2))
    seqs = [[normal((x + steps, h, d), 7 * s + i, dtype) for i, h in enumerate((H, H_kv, H_kv))] for s, x in enumerate(prompts)]
    slot_of = lambda s, t: (table[s][t // page].long() * page + t % page).to(torch.int32)
    pos = torch.cat([torch.arange(x) for x in prompts])
    slot = torch.cat([slot_of(s, torch.arange(x)) for s, x in enumerate(prompts)])
    q, k, v = (torch.cat([x[i][:p] for x, p in zip(seqs, prompts)]).cuda() for i in range(3))
    sa.sa_cache_append(k, v, slot.cuda(), k_cache, v_cache, pos=pos.to(torch.int32).cuda(), k_out=k, q=q, q_out=q)
    off = lengths_to_offsets(prompts).cuda()
    out, lse = torch.empty_like(q), torch.empty(H, q.shape[0], device="cuda")
    sa.sa_attn_packed_fwd(q, k, v, off, out, lse, max(prompts))
    at, keys = 0, []
    for s, x in enumerate(prompts):
        r = slice(at, at + x)
        at += x
        keys.append([k[r].cpu(), v[r].cpu()])
        for h in range(H):
            y = Head(q[r, h].cpu(), k[r, h // (H // H_kv)].cpu(), v[r, h // (H // H_kv)].cpu(), d ** -0.5, True)
            check(("prompt", s, h), out[r, h], y.out, y.out_off(dtype, HALF_STEP[dtype] if dtype == BF16 else 0))
    work = torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    for step in range(steps):
        now = torch.tensor([x + step for x in prompts])
        q, k, v = (torch.stack([x[i][p + step] for x, p in zip(seqs, prompts)]).cuda() for i in range(3))
        slot = torch.cat([slot_of(s, now[s:s + 1]) for s in range(n)])
        sa.sa_cache_append(k, v, slot.cuda(), k_cache, v_cache, pos=now.to(torch.int32).cuda(), k_out=k, q=q, q_out=q)
        out, lse = torch.empty_like(q), torch.empty(n, H, device="cuda")
        sa.sa_attn_decode(q, k_cache, v_cache, table.cuda(), (now + 1).to(torch.int32).cuda(), out, lse, work)
        for s in range(n):
            keys[s] = [torch.cat([old, x[s:s + 1].cpu()]) for old, x in zip(keys[s], (k, v))]
        compare(q.cpu(), keys, out.cpu(), lse.cpu(), dtype)
        # the rotated query and key are those of the token's place
        for s in range(n):
            x = seqs[s][0][prompts[s] + step][None]
            want = rotated(x, now[s:s + 1], 10000.0)
            check("query", q[s:s + 1], want, off_of(x, want, dtype))


def test_other_stream():
    want = decode([300, 4], 4, 2, 64, BF16)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = decode([300, 4], 4, 2, 64, BF16)
    assert torch.equal(got[2], want[2]) and torch.equal(got[3], want[3])


def test_empty_calls():
    k_cache = cache(2, 16, 2, 64, BF16, "shd", 0)
    q = torch.empty(0, 2, 64, dtype=BF16, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    sa.sa_cache_append(q, q, none, k_cache, k_cache.clone())
    work = torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    sa.sa_attn_decode(q, k_cache, k_cache, none.view(0, 0), none, q, torch.empty(0, 2, device="cuda"), work)
    assert (k_cache == 0).all()
    # a table without pages: no token
    q = normal((2, 2, 64), 1, BF16).cuda()
    out, lse = torch.empty_like(q), torch.empty(2, 2, device="cuda")
    sa.sa_attn_decode(q, k_cache, k_cache, torch.empty(2, 0, dtype=torch.int32, device="cuda"), torch.full((2,), 9, dtype=torch.int32, device="cuda"), out,
                      lse, work)
    assert (out == 0).all() and (lse == -torch.inf).all()

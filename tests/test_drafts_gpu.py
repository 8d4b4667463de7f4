"""Attention over the paged cache under a window and of drafted tokens, what is accepted of drafts moved up, pages copied; against 64 bits and against plain
indexing, and together as a step of drafting uses them."""
import random

import pytest
import torch

from paper_2311_09431_amd import binding as sa
from seen import Seen
from sequences import HALF_STEP, check, normal
from test_paged_gpu import ROUNDED, cache, fill, tables

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")
# tables of so few pages that a workgroup takes a unit, and of so many that the tokens are dealt out in shares
WIDTHS = [None, 200]


def ints(x):
    return torch.as_tensor(x).to(torch.int32).cuda()


# ---------------------------------------------------------------- one new token under a window


def visible(n, window, sinks):
    t = torch.arange(n)
    return (t >= n - window) | (t < sinks)


def hide(lens, window, sinks, page, k_cache, v_cache, table):
    """NaN in every token that is not seen, and no page number for pages without one that is."""
    for s, n in enumerate(lens):
        gone = (~visible(n, window, sinks)).nonzero()[:, 0]
        for c in (k_cache, v_cache):
            c[table[s][gone // page].long().cuda(), (gone % page).cuda()] = NAN
        for p in range(-(-n // page)):
            if not visible(n, window, sinks)[p * page:(p + 1) * page].any():
                table[s, p] = -5 if p % 2 else 2 ** 30


def window_decode(lens, H, H_kv, d, dtype, window, sinks, page=16, order="shd", seed=1, scale=None, width=None, with_lse=True, hidden=True):
    table, pool = tables(lens, page, seed, width=width)
    k_cache, v_cache = (cache(pool, page, H_kv, d, dtype, order) for _ in range(2))
    rows = fill(k_cache, v_cache, table, lens, 10 * seed)
    if hidden:
        hide(lens, window, sinks, page, k_cache, v_cache, table)
    q = normal((len(lens), H, d), seed + 5, dtype)
    out, lse = torch.full((len(lens), H, d), 7, dtype=dtype, device="cuda"), torch.full((len(lens), H), 7.0, device="cuda")
    work = torch.full((sa.sa_attn_decode_workspace(q, k_cache),), 255, dtype=torch.uint8, device="cuda")       # NaN
    sa.sa_attn_window_decode(q.cuda(), k_cache, v_cache, table.cuda(), ints(lens), out, lse if with_lse else None, work, window, sinks, scale)
    return q, rows, out.cpu(), lse.cpu()


def compare_window(q, rows, out, lse, dtype, window, sinks, scale=None):
    B, H, d = q.shape
    for b in range(B):
        k, v = rows[b]
        n = k.shape[0]
        if n == 0:
            assert (out[b] == 0).all() and (lse[b] == -INF).all()
            continue
        G = H // k.shape[1]
        for kvh in range(k.shape[1]):
            h = slice(kvh * G, (kvh + 1) * G)
            x = Seen(q[b, h], k[:, kvh], v[:, kvh], scale or d ** -0.5, visible(n, window, sinks).expand(G, n))
            check(("out", b, kvh), out[b, h], x.out, x.out_off(dtype, ROUNDED[dtype]))
            check(("lse", b, kvh), lse[b, h], x.lse, x.lse_off)


LENS = [1, 15, 16, 0, 17, 31, 33, 128, 129, 500]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [4, 20, 32, 64, 68, 100, 128, 132, 200, 256])
@pytest.mark.parametrize("width", WIDTHS)
def test_window_decode_head_dimensions(width, d, dtype):
    compare_window(*window_decode(LENS, 4, 2, d, dtype, 40, 3, width=width), dtype, 40, 3)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (15, 0), (16, 16), (17, 5), (64, 0), (100, 130), (128, 1), (130, 64), (500, 3), (5, 1000), (1 << 30, 1 << 30)])
@pytest.mark.parametrize("width", WIDTHS)
def test_windows(width, window, sinks, dtype):
    lens = [700, 1, 129, 0, 1500, 257]
    compare_window(*window_decode(lens, 4, 1, 64, dtype, window, sinks, width=width), dtype, window, sinks)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (6, 2), (32, 1), (40, 2), (16, 16)])
@pytest.mark.parametrize("order", ["shd", "hsd"])
def test_window_decode_heads_and_orders(H, H_kv, order, dtype):
    compare_window(*window_decode([300, 1, 77], H, H_kv, 64, dtype, 50, 2, order=order), dtype, 50, 2)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [16, 32, 48, 64, 256])
def test_window_decode_page_sizes(page, dtype):
    for width in WIDTHS:
        compare_window(*window_decode([700, 1, 129, 0, 64], 4, 2, 64, dtype, 150, 33, page=page, width=width), dtype, 150, 33)


@pytest.mark.parametrize("lens,window,sinks", [([70001, 5, 33333], 20000, 700), ([9000] * 40, 1000, 4), ([3000, 1] * 70, 129, 1), ([100000], 30000, 0)])
def test_window_decode_shares(lens, window, sinks):
    compare_window(*window_decode(lens, 8, 2, 128, BF16, window, sinks, page=128), BF16, window, sinks)


def test_window_decode_random():
    rng = random.Random(5)
    for i in range(20):
        dtype, d, H_kv = rng.choice([BF16, F32]), rng.choice([32, 64, 100, 128, 256]), rng.choice([1, 2, 3])
        lens, window, sinks = [rng.randint(0, 2000) for _ in range(rng.randint(1, 9))], rng.randint(1, 900), rng.choice([0, 1, 4, 100, 300])
        page, width = rng.choice([16, 48, 128]), rng.choice([None, 200])
        print(i, dtype, d, H_kv, lens, window, sinks, page, width, flush=True)
        compare_window(*window_decode(lens, 2 * H_kv, H_kv, d, dtype, window, sinks, page=page, width=width), dtype, window, sinks)


def test_a_window_beyond_the_cache_is_none():
    """The same products in the same order as sa_attn_decode."""
    lens, page = [300, 17, 1000], 32
    table, pool = tables(lens, page, 2)
    k_cache, v_cache = (cache(pool, page, 2, 128, BF16, "shd") for _ in range(2))
    fill(k_cache, v_cache, table, lens, 4)
    q = normal((3, 8, 128), 6, BF16).cuda()
    work = torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    outs = []
    for call in (lambda o, l: sa.sa_attn_decode(q, k_cache, v_cache, table.cuda(), ints(lens), o, l, work),
                 lambda o, l: sa.sa_attn_window_decode(q, k_cache, v_cache, table.cuda(), ints(lens), o, l, work, 5000, 7)):
        outs.append((torch.empty_like(q), torch.empty(3, 8, device="cuda")))
        call(*outs[-1])
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_window_decode_scale_and_no_lse():
    q, rows, out, lse = window_decode([300, 20], 4, 2, 64, BF16, 70, 2, scale=0.4, with_lse=False)
    assert (lse == 7).all()
    for b, n in enumerate((300, 20)):
        x = Seen(q[b, :2], rows[b][0][:, 0], rows[b][1][:, 0], 0.4, visible(n, 70, 2).expand(2, n))
        check("out", out[b, :2], x.out, x.out_off(BF16, ROUNDED[BF16]))


@pytest.mark.parametrize("width", WIDTHS)
def test_window_decode_captured_and_replayed(width):
    page, most, window, sinks = 32, 640, 150, 4
    table, pool = tables([most] * 3, page, 8, width=width)
    k_cache, v_cache = (cache(pool, page, 2, 128, BF16, "shd") for _ in range(2))
    fill(k_cache, v_cache, table, [most] * 3, 5)
    q = normal((3, 8, 128), 6, BF16).cuda()
    table, lens = table.cuda(), ints([640, 5, 0])
    out, lse = torch.empty_like(q), torch.empty(3, 8, device="cuda")
    work = torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    call = lambda: sa.sa_attn_window_decode(q, k_cache, v_cache, table, lens, out, lse, work, window, sinks)     # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for now in ([640, 5, 0], [0, 0, 640], [33, 640, 1]):
        lens.copy_(ints(now))
        call()
        torch.cuda.synchronize()
        want = out.clone(), lse.clone()
        out.fill_(3), lse.fill_(3), work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_window_decode_any_length_stays_within_the_table(dtype, width):
    lens, page = [64, 64], 16
    table, pool = tables(lens, page, 3, width=width)
    k_cache, v_cache = (cache(pool, page, 1, 64, dtype, "shd", 0.5) for _ in range(2))
    q = normal((2, 2, 64), 1, dtype).cuda()
    work = torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    for n in (-3, 2 ** 31 - 1, 5000):
        out, lse = torch.empty_like(q), torch.empty(2, 2, device="cuda")
        sa.sa_attn_window_decode(q, k_cache, v_cache, table.cuda(), ints([n, 64]), out, lse, work, 2 ** 31 - 1, 2 ** 31 - 1)
        # (pages that the table does not have are none: of those sequences that say more, the tokens that there are)
        assert (out[1] == 0.5).all()
        assert (out[0] == (0 if n < 0 else 0.5)).all()


# ---------------------------------------------------------------- drafted tokens

# tables of few pages and of many, in small launches and beside so many sequences without a draft that the launch is a large one
WAYS = WIDTHS + [(None, 260), (200, 260)]


def trees(drafts, T, seed, empty=False):
    """int64 [B, T] masks of random trees, whose tokens see whom they descend from and themselves (empty: some see nothing), and as booleans."""
    rng = random.Random(seed)
    masks, sees = torch.zeros(len(drafts), T, dtype=torch.int64), torch.zeros(len(drafts), T, T, dtype=torch.bool)
    for b, n in enumerate(drafts):
        for i in range(T):
            up = rng.randint(-1, i - 1)
            bits = (masks_of(masks[b, up]) if up >= 0 else 0) | 1 << i
            if empty and rng.random() < 0.3:
                bits = 0
            sees[b, i] = torch.tensor([bool(bits >> j & 1) and j < n for j in range(T)])
            bits |= rng.getrandbits(T) & ~((1 << n) - 1)        # of tokens that there are not: not looked at
            masks[b, i] = bits - (1 << 64) if bits >> 63 else bits
    return masks, sees


def masks_of(x):
    return int(x) & ((1 << 64) - 1)


class Tree:
    """A call of sa_attn_tree: lens tokens in front, drafts tokens drafted."""

    def __init__(self, lens, drafts, T, H, H_kv, d, dtype, page=16, order="shd", seed=1, width=None, empty=False, scale=None, mutate=None, with_lse=True,
                 with_drafts=True):
        width, others = width if isinstance(width, tuple) else (width, 0)
        lens, drafts = list(lens) + [0] * others, list(drafts) + [0] * others
        self.lens, self.drafts, self.dtype, self.scale, self.shape = lens, drafts, dtype, scale, (len(lens), T, H, H_kv, d)
        total = [a + b for a, b in zip(lens, drafts)]
        self.table, pool = tables(total, page, seed, width=width)
        self.k_cache, self.v_cache = (cache(pool, page, H_kv, d, dtype, order) for _ in range(2))
        self.rows = fill(self.k_cache, self.v_cache, self.table, total, 10 * seed)
        self.q = normal((len(lens), T, H, d), seed + 5, dtype)
        self.masks, self.sees = trees(drafts, T, seed, empty)
        if mutate:
            mutate(self)
        self.out = torch.full(self.q.shape, 7, dtype=dtype, device="cuda")
        self.lse = torch.full(self.q.shape[:3], 7.0, device="cuda")
        self.work = torch.full((sa.sa_attn_tree_workspace(self.q, self.k_cache),), 255, dtype=torch.uint8, device="cuda")
        sa.sa_attn_tree(self.q.cuda(), self.k_cache, self.v_cache, self.table.cuda(), ints(lens), self.masks.cuda(), self.out, self.lse if with_lse else None,
                        self.work, ints(drafts) if with_drafts else None, scale)

    def compare(self, heads=None, sequences=None):
        B, T, H, H_kv, d = self.shape
        out, lse, G = self.out.cpu(), self.lse.cpu(), H // H_kv
        for b in range(B) if sequences is None else sequences:
            n, m = self.lens[b], self.drafts[b]
            assert (out[b, m:] == 7).all() and (lse[b, m:] == 7).all()
            if m == 0:
                continue
            sees = torch.cat([torch.ones(m, n, dtype=torch.bool), self.sees[b, :m, :m]], 1).repeat_interleave(G, 0)
            for kvh in range(H_kv) if heads is None else heads:
                h = slice(kvh * G, (kvh + 1) * G)
                x = Seen(self.q[b, :m, h].reshape(m * G, d), self.rows[b][0][:, kvh], self.rows[b][1][:, kvh], self.scale or d ** -0.5, sees)
                some = sees.any(1)
                got, sums = out[b, :m, h].reshape(m * G, d), lse[b, :m, h].reshape(m * G)
                check(("out", b, kvh), got, x.out, x.out_off(self.dtype, ROUNDED[self.dtype]))
                check(("lse", b, kvh), sums[some], x.lse[some], x.lse_off[some])
                assert (got[~some] == 0).all() and (sums[~some] == -INF).all()
        return self


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [4, 20, 32, 64, 68, 100, 128, 132, 200, 256])
@pytest.mark.parametrize("width", WAYS)
def test_tree_head_dimensions(width, d, dtype):
    Tree([1, 0, 17, 300, 129, 14], [5, 3, 1, 0, 4, 5], 5, 4, 2, d, dtype, width=width).compare()


# from one row a unit to more than a unit holds
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,H,H_kv", [(1, 1, 1), (1, 16, 1), (1, 17, 1), (3, 15, 3), (8, 4, 2), (11, 6, 2), (16, 8, 2), (13, 40, 8), (33, 2, 1),
                                      (64, 1, 1), (64, 4, 1), (63, 12, 2), (5, 64, 1)])
@pytest.mark.parametrize("order", ["shd", "hsd"])
def test_tree_rows(order, T, H, H_kv, dtype):
    for width in WAYS:
        drafts = [T, max(1, T // 2), 0, 1]
        Tree([250, 33, 5, 0], drafts, T, H, H_kv, 64, dtype, order=order, width=width, seed=T + H).compare()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [32, 128, 256])
@pytest.mark.parametrize("T,H", [(4, 4), (9, 4), (30, 4)])
def test_tree_rows_and_dimensions(T, H, d, dtype):
    for width in WAYS:
        Tree([300, 129], [T, T - 1], T, H, 1, d, dtype, width=width, seed=T).compare()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [16, 32, 48, 64, 256])
def test_tree_page_sizes(page, dtype):
    for width in WAYS:
        Tree([500, 1, 129, 0, 64], [7, 20, 3, 20, 16], 20, 4, 2, 64, dtype, page=page, width=width).compare()


@pytest.mark.parametrize("lens,drafts,T,d", [([5000, 7, 3000], [12, 1, 16], 16, 128), ([2000, 1] * 40, [8, 64] * 40, 64, 64), ([700] * 65, [3] * 65, 4, 32),
                                             ([40000], [24], 24, 128)])
def test_tree_shares(lens, drafts, T, d):
    Tree(lens, drafts, T, 8, 2, d, BF16, page=128).compare(heads=[0, 1], sequences=[0, 1, len(lens) - 1] if len(lens) > 1 else [0])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", WAYS)
def test_tree_rows_that_see_nothing(width, dtype):
    """Masks that leave a row empty, in front of which no token lies: zero and -inf; with tokens in front these are what it sees."""
    Tree([0, 40, 0], [6, 6, 1], 6, 4, 2, 64, dtype, width=width, empty=True, seed=4).compare()


def test_tree_every_draft_is_whole():
    Tree([100, 3], [9, 9], 9, 4, 2, 64, BF16, with_drafts=False).compare()


def test_tree_without_lse_and_with_a_scale():
    x = Tree([100, 3], [9, 5], 9, 4, 2, 64, BF16, scale=0.3, with_lse=False)
    assert (x.lse == 7).all()
    x.lse = Tree([100, 3], [9, 5], 9, 4, 2, 64, BF16, scale=0.3).compare().lse
    x.compare()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tree_large_scores(dtype):
    Tree([300, 3], [9, 5], 9, 4, 2, 64, dtype, mutate=lambda x: x.q.mul_(40)).compare()


def test_tree_random():
    rng = random.Random(8)
    for i in range(24):
        dtype, d, H_kv, T = rng.choice([BF16, BF16, F32]), rng.choice([32, 64, 96, 100, 128, 256]), rng.choice([1, 2, 3]), rng.randint(1, 64)
        n = rng.randint(1, 9)
        lens, drafts = [rng.randint(0, 900) for _ in range(n)], [rng.randint(0, T) for _ in range(n)]
        H, page, width, order = H_kv * rng.choice([1, 2, 4, 8]), rng.choice([16, 48, 128]), rng.choice([None, 200]), rng.choice(["shd", "hsd"])
        print(i, dtype, d, H, H_kv, T, lens, drafts, page, width, order, flush=True)
        Tree(lens, drafts, T, H, H_kv, d, dtype, page, order, seed=i, width=(width, 0 if i % 2 else 260 // H_kv), empty=rng.random() < 0.3).compare()


def test_tree_offsets_beyond_32_bits():
    page, heads, d, pages = 256, 8, 128, 6000
    k_cache, v_cache = (cache(pages, page, heads, d, BF16, "shd", 0) for _ in range(2))
    table = torch.tensor([[pages - 1, pages - 5, pages - 3], [pages - 2, pages - 4, 0]], dtype=torch.int32)

    def there(x):
        x.k_cache, x.v_cache, x.table = k_cache, v_cache, table
        x.rows = fill(k_cache, v_cache, table, [708, 305], 10)
    Tree([700, 300], [8, 5], 8, 16, 8, d, BF16, page=256, mutate=there).compare()
    # and the moves there
    src, dst = ints([pages - 1]), ints([pages - 7])
    sa.sa_cache_copy(k_cache, v_cache, src, dst)
    assert torch.equal(k_cache[pages - 7], k_cache[pages - 1]) and torch.equal(v_cache[pages - 7], v_cache[pages - 1]) and (k_cache[pages - 6] == 0).all()
    want = v_cache[pages - 3, 190].clone()
    sa.sa_cache_accept(k_cache, v_cache, table.cuda(), ints([700, 300]), ints([[2, 5, 0, 0, 0, 0], [0] * 6]), ints([1, 0]))
    assert torch.equal(v_cache[pages - 3, 188], want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", WAYS)
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("d", [64, 100, 256])
def test_drafted_tokens_that_are_no_numbers(d, bad, width, dtype):
    """They reach the rows that see them, and no others."""
    lens, drafts, T, H, H_kv, nth = [50, 0], [6, 6], 6, 4, 2, 2
    for part in (0, 1):
        def poison(x):
            for b, n in enumerate(lens):
                page, at = int(x.table[b, (n + nth) // 16]), (n + nth) % 16
                (x.k_cache, x.v_cache)[part][page, at, :, 1] = bad
                x.rows[b][part][n + nth] = 0
        x = Tree(lens, drafts, T, H, H_kv, d, dtype, width=width, seed=3, mutate=poison)
        sees = x.sees[:, :, nth].clone()
        x.sees[:, :, nth] = False
        out, lse = x.out.cpu(), x.lse.cpu()
        assert sees.any() and not sees.all()
        if part == 1:
            assert not torch.isfinite(out[sees][..., 1]).any() and torch.isfinite(out[sees][..., 2:]).all() and torch.isfinite(lse).all()
            value = out[sees][..., 1]
            assert value.isnan().all() if bad != bad else (value == bad).all()
        elif bad != bad:
            assert out[sees].isnan().all() and lse[sees].isnan().all()
        # the others are as without the token
        for b in range(2):
            for kvh in range(H_kv):
                h, ok = slice(2 * kvh, 2 * kvh + 2), ~sees[b]
                mask = torch.cat([torch.ones(6, lens[b], dtype=torch.bool), x.sees[b, :6, :6]], 1)[ok].repeat_interleave(2, 0)
                y = Seen(x.q[b, ok][:, h].reshape(-1, d), x.rows[b][0][:, kvh], x.rows[b][1][:, kvh], d ** -0.5, mask)
                check("out", out[b, ok][:, h].reshape(-1, d), y.out, y.out_off(dtype, ROUNDED[dtype]))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", WAYS)
def test_tree_pages_that_are_none(width, dtype):
    """Tokens of a page that is none of the cache's are left out, drafted ones too."""
    lens, drafts, page = [100, 20], [10, 10], 16

    def cut(x):
        x.table[0, 2], x.table[0, 6], x.table[1, 1] = -1, 2 ** 30, 10 ** 6      # tokens 32 .. 47, 96 .. 111 (draft 0 .. 9 among them); 16 .. 31
        x.gone = [torch.tensor([32 <= t < 48 or t >= 96 for t in range(110)]), torch.tensor([t >= 16 for t in range(30)])]
    x = Tree(lens, drafts, 10, 4, 2, 64, dtype, page, width=width, mutate=cut)
    for b in range(2):
        sees = torch.cat([torch.ones(10, lens[b], dtype=torch.bool), x.sees[b, :, :10]], 1) & ~x.gone[b]
        y = Seen(x.q[b, :, 0], x.rows[b][0][:, 0], x.rows[b][1][:, 0], 0.125, sees)
        check("out", x.out[b, :, 0], y.out, y.out_off(dtype, ROUNDED[dtype]))


@pytest.mark.parametrize("width", [4, 200])
@pytest.mark.parametrize("H,B", [(2, 4), (8, 4), (8, 300), (20, 300)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tree_any_numbers_stay_within_the_table(dtype, H, B, width):
    """Lengths and drafts of any size; a table of 64 tokens (or whose other pages are none)."""
    page, T, none = 16, 6, [0] * (B - 4)
    table = torch.full((B, width), -1, dtype=torch.int32)
    table[:4, :4] = torch.arange(16).view(4, 4)
    k_cache, v_cache = (cache(16, page, 1, 64, dtype, "shd", 0.5) for _ in range(2))
    q = normal((B, T, H, 64), 1, dtype).cuda()
    out, lse = torch.full_like(q, 7), torch.full((B, T, H), 7.0, device="cuda")
    work = torch.empty(sa.sa_attn_tree_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    seen = torch.full((B, T), -1, dtype=torch.int64, device="cuda")
    sa.sa_attn_tree(q, k_cache, v_cache, table.cuda(), ints([-5, 2 ** 31 - 1, 62, 2 ** 31 - 3] + none), seen, out, lse, work, ints([3, 100, 5, -2] + none))
    # (a length below zero is none: the draft itself is cached from token 0 on)
    assert (out[0, :3] == 0.5).all() and (out[1] == 0.5).all() and (out[2, :5] == 0.5).all()
    assert (out[0, 3:] == 7).all() and (out[2, 5:] == 7).all() and (out[3] == 7).all() and (lse[3] == 7).all()
    assert torch.isfinite(lse).all()


def test_tree_without_pages():
    q = normal((2, 3, 2, 64), 1, BF16).cuda()
    k_cache = cache(2, 16, 2, 64, BF16, "shd", 0)
    out, lse = torch.full_like(q, 7), torch.full((2, 3, 2), 7.0, device="cuda")
    work = torch.empty(sa.sa_attn_tree_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    seen = torch.full((2, 3), 7, dtype=torch.int64, device="cuda")
    sa.sa_attn_tree(q, k_cache, k_cache, torch.empty(2, 0, dtype=torch.int32, device="cuda"), ints([9, 0]), seen, out, lse, work, ints([3, 2]))
    assert (out[0] == 0).all() and (out[1, :2] == 0).all() and (out[1, 2] == 7).all() and (lse[0] == -INF).all() and (lse[1, 2] == 7).all()
    sa.sa_attn_tree(q[:0], k_cache, k_cache, torch.empty(0, 0, dtype=torch.int32, device="cuda"), ints([]), seen[:0], out[:0], None, work)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", WAYS)
def test_tree_strided(width, dtype):
    """Everything a part of something larger; nothing beside it changes."""
    lens, drafts, T, H, H_kv, d = [77, 1, 0, 300], [5, 2, 4, 0], 5, 4, 2, 68
    x = Tree(lens, drafts, T, H, H_kv, d, dtype, width=width).compare()
    B = len(x.lens)
    wide = torch.full((B, T + 2, H + 3, d + 4), 9, dtype=dtype, device="cuda")
    q_wide = torch.full_like(wide, NAN)
    part = lambda y: y[:, 1:1 + T, 2:2 + H, :d]      # noqa: E731
    part(q_wide).copy_(x.q)
    part(wide).fill_(7)
    pages = torch.full((B, x.table.shape[1] + 3), 2 ** 30, dtype=torch.int32)
    pages[:, 2:-1] = x.table
    seen = torch.full((B, T + 4), -1, dtype=torch.int64, device="cuda")
    seen[:, 3:-1] = x.masks.cuda()
    sums = torch.full((B, T + 1, H + 2), 9.0, device="cuda")
    sums[:, :T, :H] = 7
    sa.sa_attn_tree(part(q_wide), x.k_cache, x.v_cache, pages.cuda()[:, 2:-1], ints(x.lens), seen[:, 3:-1], part(wide), sums[:, :T, :H], x.work, ints(x.drafts))
    assert torch.equal(part(wide), x.out) and torch.equal(sums[:, :T, :H], x.lse)
    part(wide).fill_(9)
    sums[:, :T, :H] = 9
    assert (wide == 9).all() and (sums == 9).all()


@pytest.mark.parametrize("width", WAYS)
def test_tree_captured_and_replayed(width):
    """Lengths, drafts and masks are read when the graph is played."""
    page, T = 32, 20
    x = Tree([600, 600, 600], [T] * 3, T, 8, 2, 128, BF16, page, width=width)
    q, table, lens, drafts, seen = x.q.cuda(), x.table.cuda(), ints(x.lens), ints(x.drafts), x.masks.cuda()
    call = lambda: sa.sa_attn_tree(q, x.k_cache, x.v_cache, table, lens, seen, x.out, x.lse, x.work, drafts)      # noqa: E731
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i, (a, b) in enumerate([([600, 600, 600], [20, 20, 20]), ([0, 5, 600], [3, 0, 20]), ([33, 590, 1], [20, 1, 9])]):
        lens[:3].copy_(ints(a)), drafts[:3].copy_(ints(b)), seen[:3].copy_(trees(b, T, 50 + i)[0])
        x.out.fill_(7), x.lse.fill_(7)
        call()
        torch.cuda.synchronize()
        want = x.out.clone(), x.lse.clone()
        x.out.fill_(7), x.lse.fill_(7), x.work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x.out, want[0]) and torch.equal(x.lse, want[1])


def test_tree_two_streams_at_once():
    """A workspace each, eager and as graphs."""
    make = lambda: [Tree([3000, 4, 900], [9, 16, 2], 16, 8, 2, d, BF16) for d in (64, 128)]      # noqa: E731
    want = make()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in want]
    for _ in range(3):
        got = []
        for stream, d in zip(streams, (64, 128)):
            with torch.cuda.stream(stream):
                got.append(Tree([3000, 4, 900], [9, 16, 2], 16, 8, 2, d, BF16))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g.out, w.out) and torch.equal(g.lse, w.lse)
    calls = []
    for x in want:
        a = (x.q.cuda(), x.k_cache, x.v_cache, x.table.cuda(), ints(x.lens), x.masks.cuda(), x.out.clone(), x.lse.clone(), x.work, ints(x.drafts))
        calls.append((a, lambda a=a: sa.sa_attn_tree(*a)))
    graphs = [torch.cuda.CUDAGraph() for _ in calls]
    torch.cuda.synchronize()
    for graph, (_, call) in zip(graphs, calls):
        with torch.cuda.graph(graph):
            call()
    for _ in range(3):
        for a, _ in calls:
            a[6].fill_(7), a[7].fill_(7)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for (a, _), w in zip(calls, want):
            assert torch.equal(a[6], w.out) and torch.equal(a[7], w.lse)


# ---------------------------------------------------------------- moves


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("order", ["shd", "hsd"])
@pytest.mark.parametrize("H_kv,d,page", [(1, 4, 16), (2, 64, 16), (3, 68, 48), (8, 128, 64), (2, 100, 32), (1, 256, 128)])
def test_copy(H_kv, d, page, order, dtype):
    """Whole pages and their first tokens; numbers that are none of the cache's and pairs of the same are left out."""
    k, v = (cache(20, page, H_kv, d, dtype, order, 0).copy_(normal((20, page, H_kv, d), s, dtype)) for s in (1, 2))
    src, dst = [3, 7, 3, -1, 5, 20, 9, 2, 4], [0, 19, 1, 6, 5, 8, 10, -7, 2 ** 30]
    for tokens in (None, [page, 1, 0, 5, page - 1, 3, page // 2 + 1, 4, 2], [page + 9, -4, 7] * 3):
        want = [x.cpu() for x in (k, v)]
        for x in want:
            for i, (a, b) in enumerate(zip(src, dst)):
                if 0 <= a < 20 and 0 <= b < 20:
                    n = page if tokens is None else min(max(tokens[i], 0), page)
                    x[b, :n] = x[a, :n].clone()
        got = [x.clone() for x in (k, v)]
        sa.sa_cache_copy(*got, ints(src), ints(dst), None if tokens is None else ints(tokens))
        for x, y in zip(got, want):
            assert x.stride() == k.stride() and torch.equal(x.cpu(), y)


@pytest.mark.parametrize("d", [60, 64])
def test_copy_strided(d):
    """Pages, tokens and heads with gaps between them, which stay."""
    whole = [normal((9, 18, 5, d + 4), s, BF16).cuda() for s in (1, 2)]
    want = [x.cpu() for x in whole]
    part = lambda x: x[1:, 1:17, 1:4, :d]       # noqa: E731
    sa.sa_cache_copy(*(part(x) for x in whole), ints([0, 6]), ints([3, 7]), ints([16, 9]))
    for x in want:
        part(x)[3], part(x)[7, :9] = part(x)[0].clone(), part(x)[6, :9].clone()
    for x, y in zip(whole, want):
        assert torch.equal(x.cpu(), y)


def test_copy_many_pages():
    """More than the workgroups of a slice each; a captured call follows its numbers."""
    n, page = 3000, 16
    k, v = (normal((2 * n, page, 1, 32), s, F32).cuda() for s in (1, 2))
    order = torch.randperm(2 * n, generator=torch.Generator().manual_seed(1))
    src, dst = ints(order[:n]), ints(order[n:])
    graph = torch.cuda.CUDAGraph()
    sa.sa_cache_copy(k.clone(), v.clone(), src, dst)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sa.sa_cache_copy(k, v, src, dst)
    for _ in range(3):
        want = [x.clone() for x in (k, v)]
        for x in want:
            x[dst.long()] = x[src.long()]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
        src.copy_(src.flip(0)), dst.copy_(dst.roll(1))
    sa.sa_cache_copy(k, v, src[:0], dst[:0])


def accept_plainly(k, v, table, lens, chosen, accepted, pages):
    page, room = k.shape[1], table.shape[1] * k.shape[1]
    for b in range(len(lens)):
        n = max(lens[b], 0)
        for i in range(min(max(accepted[b], 0), chosen.shape[1])):
            a, c = n + int(chosen[b, i]), n + i
            if not 0 <= chosen[b, i] < chosen.shape[1] or a >= room or c >= room:
                continue
            p, r = int(table[b, a // page]), int(table[b, c // page])
            if 0 <= p < pages and 0 <= r < pages:
                for x in (k, v):
                    x[r, c % page] = x[p, a % page].clone()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("order", ["shd", "hsd"])
@pytest.mark.parametrize("H_kv,d,page,T", [(1, 4, 16, 1), (2, 64, 16, 40), (3, 68, 48, 64), (8, 128, 64, 17), (16, 256, 32, 9)])
def test_accept(H_kv, d, page, T, order, dtype):
    rng = random.Random(T)
    lens = [30, 0, 100, 15, -4, 7]
    drafts = [rng.randint(1, T) for _ in lens]
    table, pool = tables([max(n, 0) + m for n, m in zip(lens, drafts)], page, 3, spare=0)
    chosen, accepted = torch.zeros(len(lens), T, dtype=torch.int32), []
    for b, m in enumerate(drafts):
        n = rng.randint(0, m)
        chosen[b, :n] = torch.tensor(sorted(rng.sample(range(m), n)), dtype=torch.int32)
        chosen[b, n:] = -1
        accepted.append(n)
    accepted[3] = 0
    table[2, 1] = -1            # a page that is none
    k, v = (cache(pool, page, H_kv, d, dtype, order, 0).copy_(normal((pool, page, H_kv, d), s, dtype)) for s in (1, 2))
    want = [x.cpu() for x in (k, v)]
    accept_plainly(*want, table, lens, chosen, accepted, pool)
    at, after = ints(lens), ints([9] * len(lens))
    for target in (after, at, None):        # (beside the lengths, in their place, nowhere)
        got = [x.clone() for x in (k, v)]
        sa.sa_cache_accept(*got, table.cuda(), at, chosen.cuda(), ints(accepted), target)
        for x, y in zip(got, want):
            assert torch.equal(x.cpu(), y)
        if target is not None:
            assert target.tolist() == [max(n, 0) + m for n, m in zip(lens, accepted)]
            at = ints(lens)


def test_accept_any_numbers_stay_within_the_table():
    """Numbers that do not ascend or are none, more accepted than there are, tokens behind the table: other tokens stay."""
    T, page, B = 6, 16, 5
    table = torch.tensor([[0, 1], [2, 3], [4, 5], [6, -1], [2 ** 30, 7]], dtype=torch.int32)
    lens, accepted = [3, 30, 2 ** 31 - 1, 14, 10], [99, 6, 6, 6, -3]
    chosen = torch.tensor([[5, 0, 3, 3, -9, 2 ** 30], [0, 1, 2, 3, 4, 5], [1, 2, 3, 4, 5, 5], [1, 2, 3, 4, 5, 5], [1, 2, 3, 4, 5, 5]], dtype=torch.int32)
    k, v = (normal((9, page, 2, 64), s, BF16).cuda() for s in (1, 2))
    before = [x.cpu() for x in (k, v)]
    after = ints([0] * B)
    sa.sa_cache_accept(k, v, table.cuda(), ints(lens), chosen.cuda(), ints(accepted), after)
    free = torch.ones(9, page, dtype=torch.bool)
    free[0, 3:9], free[3, 14:], free[6, 14:] = False, False, False
    for x, y in zip((k, v), before):
        assert torch.equal(x.cpu()[free], y[free])
    assert torch.isfinite(k).all() and after.tolist()[:2] == [9, 36] and after.tolist()[3:] == [20, 10]


def test_accept_strided_and_captured():
    whole = [normal((6, 18, 5, 68), s, BF16).cuda() for s in (1, 2)]
    part = lambda x: x[:, 1:17, 1:4, :64]       # noqa: E731
    tables_, numbers = torch.full((2, 5), 99, dtype=torch.int32), torch.full((2, 8), -3, dtype=torch.int32)
    tables_[:, 1:3], numbers[:, 2:6] = torch.tensor([[0, 2], [5, 1]]), torch.tensor([[1, 3, 0, 0], [0, 2, 3, 0]])
    lens, accepted = ints([13, 4]), ints([2, 3])
    a = (part(whole[0]), part(whole[1]), tables_.cuda()[:, 1:3], lens, numbers.cuda()[:, 2:6], accepted, lens)
    graph = torch.cuda.CUDAGraph()
    want = [x.cpu() for x in whole]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sa.sa_cache_accept(*a)
    at = [13, 4]
    for _ in range(3):          # the lengths go on by themselves
        accept_plainly(part(want[0]), part(want[1]), tables_[:, 1:3], at, numbers[:, 2:6], [2, 3], 6)
        graph.replay()
        torch.cuda.synchronize()
        at = [at[0] + 2, at[1] + 3]
        assert lens.tolist() == at
        for x, y in zip(whole, want):
            assert torch.equal(x.cpu(), y)


# ---------------------------------------------------------------- together


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,H_kv,d,page", [(4, 2, 64, 16), (8, 8, 100, 48), (8, 1, 128, 64)])
def test_drafts_verified_accepted_and_forked(H, H_kv, d, page, dtype):
    """Three rounds: a tree of tokens appended with the position ids of their depth, its attention, one branch accepted; then a fork of the first sequence
    by a copied last page and a token of each, plainly and under a window.  Every result is that of the whole sequence so far."""
    rng, prompts, T, B, most = random.Random(2), [33, 5, 70], 8, 3, 128
    table, pool = tables([most] * B, page, 6, spare=12)
    k_cache, v_cache = (cache(pool, page, H_kv, d, dtype, "shd") for _ in range(2))
    kept = fill(k_cache, v_cache, table, prompts, 70)       # keys as they are cached, [tokens, H_kv, d]
    kept = [[k, v] for k, v in kept]
    lens, table_gpu = ints(prompts), table.cuda()
    for step in range(3):
        parent = [[rng.randint(-1, i - 1) for i in range(T)] for _ in range(B)]
        line = [[[] for _ in range(T)] for _ in range(B)]
        for b in range(B):
            for i in range(T):
                line[b][i] = (line[b][parent[b][i]] if parent[b][i] >= 0 else []) + [i]
        seen = torch.tensor([[sum(1 << j for j in line[b][i]) for i in range(T)] for b in range(B)], dtype=torch.int64)
        now = [k.shape[0] for k, _ in kept]
        q, k, v = (normal((B, T, h, d), 100 * step + i, dtype).cuda() for i, h in enumerate((H, H_kv, H_kv)))
        pos = torch.tensor([[now[b] + len(line[b][i]) - 1 for i in range(T)] for b in range(B)])
        token = torch.tensor(now)[:, None] + torch.arange(T)
        slot = (table.gather(1, token // page).long() * page + token % page).to(torch.int32)
        flat = lambda x: x.view(B * T, *x.shape[2:])       # noqa: E731
        sa.sa_cache_append(flat(k), flat(v), slot.view(-1).cuda(), k_cache, v_cache, pos=ints(pos.view(-1)), k_out=flat(k), q=flat(q), q_out=flat(q))
        out, lse = torch.empty_like(q), torch.empty(B, T, H, device="cuda")
        work = torch.empty(sa.sa_attn_tree_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
        sa.sa_attn_tree(q, k_cache, v_cache, table_gpu, lens, seen.cuda(), out, lse, work)
        leaf = [max(range(T), key=lambda i: len(line[b][i])) for b in range(B)]
        for b in range(B):
            for i in range(T):
                keys, values = (torch.cat([kept[b][j], x[b, line[b][i]].cpu()]) for j, x in enumerate((k, v)))
                for h in range(H):
                    y = Seen(q[b, i, h].cpu()[None], keys[:, h * H_kv // H], values[:, h * H_kv // H], d ** -0.5, torch.ones(1, keys.shape[0], dtype=torch.bool))
                    check(("tree", b, i, h), out[b, i, h][None], y.out, y.out_off(dtype, ROUNDED[dtype]))
                    check(("lse", b, i, h), lse[b, i, h][None], y.lse, y.lse_off)
            kept[b] = [torch.cat([kept[b][j], x[b, line[b][leaf[b]]].cpu()]) for j, x in enumerate((k, v))]
        chosen = torch.full((B, T), -1, dtype=torch.int32)
        for b in range(B):
            chosen[b, :len(line[b][leaf[b]])] = torch.tensor(line[b][leaf[b]])
        sa.sa_cache_accept(k_cache, v_cache, table_gpu, lens, chosen.cuda(), ints([len(line[b][leaf[b]]) for b in range(B)]), lens)
        assert lens.tolist() == [x.shape[0] for x, _ in kept]
    # the fork shares the first sequence's whole pages and has a copy of its last one
    n = kept[0][0].shape[0]
    last, free = (n - 1) // page, sorted(set(range(pool)) - set(table.view(-1).tolist()))[0]
    fork = table[0].clone()
    fork[last] = free
    sa.sa_cache_copy(k_cache, v_cache, ints([int(table[0, last])]), ints([free]), ints([n - last * page]))
    both = torch.stack([table[0], fork])
    q, k, v = (normal((2, h, d), 900 + i, dtype).cuda() for i, h in enumerate((H, H_kv, H_kv)))
    at = torch.tensor([n, n])
    if n % page == 0:       # (the new tokens begin a page: one of the fork's own)
        both[1, last + 1] = sorted(set(range(pool)) - set(table.view(-1).tolist()))[1]
    slot = (both.gather(1, at[:, None] // page)[:, 0].long() * page + at % page).to(torch.int32)
    sa.sa_cache_append(k, v, slot.cuda(), k_cache, v_cache, pos=ints(at), k_out=k, q=q, q_out=q)
    work = torch.empty(sa.sa_attn_decode_workspace(q, k_cache), dtype=torch.uint8, device="cuda")
    for window, sinks in ((None, 0), (20, 3)):
        out, lse = torch.empty_like(q), torch.empty(2, H, device="cuda")
        if window is None:
            sa.sa_attn_decode(q, k_cache, v_cache, both.cuda(), ints([n + 1] * 2), out, lse, work)
        else:
            sa.sa_attn_window_decode(q, k_cache, v_cache, both.cuda(), ints([n + 1] * 2), out, lse, work, window, sinks)
        sees = torch.ones(n + 1, dtype=torch.bool) if window is None else visible(n + 1, window, sinks)
        for b in range(2):
            keys, values = (torch.cat([kept[0][j], x[b:b + 1].cpu()]) for j, x in enumerate((k, v)))
            for h in range(H):
                y = Seen(q[b, h].cpu()[None], keys[:, h * H_kv // H], values[:, h * H_kv // H], d ** -0.5, sees[None])
                check(("token", window, b, h), out[b, h][None], y.out, y.out_off(dtype, ROUNDED[dtype]))


def test_prompt_and_tokens_under_one_window():
    """A prompt through sa_attn_window_fwd and the cache, then a token at a time: each is the last row of the whole sequence under the window."""
    n, steps, H, H_kv, d, page, window, sinks, dtype = 150, 4, 4, 2, 64, 16, 40, 3, BF16
    table, pool = tables([n + steps], page, 6)
    k_cache, v_cache = (cache(pool, page, H_kv, d, dtype, "shd") for _ in range(2))
    q, k, v = (normal((n + steps, h, d), i, dtype).cuda() for i, h in enumerate((H, H_kv, H_kv)))
    t = torch.arange(n + steps)
    slot, pos = ints(table[0][t // page].long() * page + t % page), ints(t)
    sa.sa_cache_append(k[:n], v[:n], slot[:n], k_cache, v_cache, pos=pos[:n], k_out=k[:n], q=q[:n], q_out=q[:n])
    out, lse = torch.empty_like(q), torch.empty(H, n + steps, device="cuda")
    sa.sa_attn_window_fwd(q[:n], k[:n], v[:n], ints([0, n]), out[:n], lse[:, :n], n, window, sinks)
    work = torch.empty(sa.sa_attn_decode_workspace(q[:1], k_cache), dtype=torch.uint8, device="cuda")
    for i in range(n, n + steps):
        r = slice(i, i + 1)
        sa.sa_cache_append(k[r], v[r], slot[r], k_cache, v_cache, pos=pos[r], k_out=k[r], q=q[r], q_out=q[r])
        # pages that no later token sees again are given away
        for p in range(i // page):
            if p * page >= sinks and (p + 1) * page <= i + 1 - window and table[0, p] >= 0:
                k_cache[int(table[0, p])] = v_cache[int(table[0, p])] = NAN
                table[0, p] = -1
        sa.sa_attn_window_decode(q[r], k_cache, v_cache, table.cuda(), ints([i + 1]), out[r], None, work, window, sinks)
    a, b = t[:, None], t[None, :]
    sees = (b <= a) & ((a - b < window) | (b < sinks))
    for h in range(H):
        y = Seen(q[:, h].cpu(), k[:, h // 2].cpu(), v[:, h // 2].cpu(), d ** -0.5, sees)
        check(h, out[:, h], y.out, y.out_off(dtype, HALF_STEP[dtype]))

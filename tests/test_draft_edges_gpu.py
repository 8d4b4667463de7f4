"""Drafts and moves in the cache at the ends of their ranges: as many sequences as an entry point takes, drafted keys whose scores are no numbers."""
import pytest
import torch

from paper_2311_09431_amd import binding as sa
from seen import Seen
from sequences import check
from test_drafts_gpu import WAYS, Tree
from test_paged_gpu import ROUNDED

pytestmark = pytest.mark.gpu

BF16, F32, INF = torch.bfloat16, torch.float32, float("inf")


def ints(x):
    return torch.as_tensor(x).to(torch.int32).cuda()


@pytest.mark.parametrize("dtype,H_kv,d", [(F32, 8, 256), (BF16, 16, 256), (BF16, 1, 4)])
def test_accept_of_as_many_sequences_as_there_can_be(dtype, H_kv, d):
    """2^22 sequences, of which a token of 8192 bytes takes 1024 threads each: 2^32 of them.  The first and the last three move a token."""
    B, T, page = 1 << 22, 2, 16
    at = [0, B - 3, B - 2, B - 1]
    k, v = (torch.randn(2 + len(at), page, H_kv, d, generator=torch.Generator("cuda").manual_seed(i), device="cuda").to(dtype) for i in (1, 2))
    table, lens = torch.zeros(B, 1, dtype=torch.int32, device="cuda"), torch.full((B,), 3, dtype=torch.int32, device="cuda")
    chosen, accepted = torch.ones(B, T, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    accepted[at] = 1
    table[at, 0] = ints(range(2, 2 + len(at)))
    want = [x.clone() for x in (k, v)]
    for x in want:
        x[2:, 3] = x[2:, 4]
    after = torch.full_like(lens, 9)
    sa.sa_cache_accept(k, v, table, lens, chosen, accepted, after)
    for x, y in zip((k, v), want):
        assert torch.equal(x, y)
    assert torch.equal(after, lens + accepted)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", WAYS)
@pytest.mark.parametrize("d,T,H", [(64, 6, 4), (100, 20, 8), (128, 40, 8), (256, 6, 4)])
def test_scores_of_drafted_tokens_that_are_no_numbers(d, T, H, width, dtype):
    """+inf makes the rows that see it NaN, in out and LSE; -inf has no weight, and a row that sees nothing else is NaN; the others know nothing of it."""
    lens, H_kv, nth, page = [300, 0, 300, 200], 2, 2, 16
    for bad in (INF, -INF):
        bad_keys = [torch.zeros(n + T, dtype=torch.bool) for n in lens]
        for b, n in enumerate(lens):
            bad_keys[b][n + nth] = True
        if bad < 0:
            # of the third sequence every token but the draft's first, of the fourth all
            bad_keys[2][:], bad_keys[3][:] = True, True
            bad_keys[2][lens[2]] = False

        def poison(x):
            x.q[..., 1] = x.q[..., 1].abs() + 0.25
            # a row that sees that token alone, and one that sees another drafted one too
            x.masks[1, nth], x.masks[1, nth + 1] = 1 << nth, 1 << nth | 1 << nth + 1
            x.sees[1, nth:nth + 2] = False
            x.sees[1, nth, nth] = x.sees[1, nth + 1, nth] = x.sees[1, nth + 1, nth + 1] = True
            for b, which in enumerate(bad_keys):
                t = which.nonzero()[:, 0]
                x.k_cache[x.table[b][t // page].long().cuda(), (t % page).cuda(), :, 1] = bad
                x.rows[b][0][t, :, 1] = 0
        x = Tree(lens, [T] * 4, T, H, H_kv, d, dtype, page, width=width, seed=3, mutate=poison)
        out, lse, G = x.out.cpu(), x.lse.cpu(), H // H_kv
        kinds = set()
        for b, n in enumerate(lens):
            sees = torch.cat([torch.ones(T, n, dtype=torch.bool), x.sees[b, :T, :T]], 1)
            reached = (sees & bad_keys[b]).any(1)
            left = sees & ~bad_keys[b]
            gone = reached if bad > 0 else reached & ~left.any(1)
            kinds |= set(gone.tolist())
            assert out[b][gone].isnan().all() and lse[b][gone].isnan().all()
            ok = ~gone
            for kvh in range(H_kv):
                h = slice(G * kvh, G * kvh + G)
                y = Seen(x.q[b, ok][:, h].reshape(-1, d), x.rows[b][0][:, kvh], x.rows[b][1][:, kvh], d ** -0.5, left[ok].repeat_interleave(G, 0))
                check(("out", bad, b, kvh), out[b, ok][:, h].reshape(-1, d), y.out, y.out_off(dtype, ROUNDED[dtype]))
                check(("lse", bad, b, kvh), lse[b, ok][:, h].reshape(-1), y.lse, y.lse_off)
        assert kinds == {True, False}

"""Drafts and moves in the cache at the ends of their ranges: as many sequences as an entry point takes."""
import pytest
import torch

from paper_2311_09431_amd import binding as sa

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


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

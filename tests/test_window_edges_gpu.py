"""Packed attention with a window and first tokens that stay visible: the workspace of its gradient, whatever the offsets say, and rows that are no numbers."""
import pytest
import torch

from paper_2311_09431_amd import binding as sa
from sequences import lengths_to_offsets, normal
from test_window_gpu import compare

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
BESIDE = 1 << 16            # bytes on either side of a workspace


def gradient(q, k, v, g, off, top, window, sinks):
    """out, LSE, dQ, dK, dV, of tensors full of 7; the workspace, which there is, lies within a larger tensor, the rest of which stays."""
    out, lse = torch.full_like(q, 7), torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
    sa.sa_attn_window_fwd(q, k, v, off, out, lse, top, window, sinks)
    grads = [torch.full_like(x, 7) for x in (q, k, v)]
    size = sa.sa_attn_window_bwd_workspace(q, k, off, top, window, sinks)
    assert size > 0
    whole = torch.full((size + 2 * BESIDE,), 255, dtype=torch.uint8, device="cuda")
    delta = torch.empty(q.shape[1], q.shape[0], device="cuda")
    sa.sa_attn_window_bwd(q, k, v, out, g, lse, off, delta, *grads, whole[BESIDE:BESIDE + size], top, window, sinks)
    assert (whole[:BESIDE] == 255).all() and (whole[BESIDE + size:] == 255).all()
    return [out, lse, *grads]


def tensors(T, H, H_kv, d, dtype):
    return [normal((T, h, d), s, dtype).cuda() for s, h in ((1, H), (3, H_kv), (4, H_kv), (2, H))]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("empty", [0, 300])
@pytest.mark.parametrize("offsets", [[0, 1500, 0, 1500, 0, 1500], [0, 1500, 100, 1400, 0, 700, 650, 1500], [-7, 1500, -5, 1499, 3, 1500]])
def test_sequences_that_share_rows_stay_within_the_workspace(offsets, empty, d, dtype):
    """They need more of it than sequences of as many rows without a common one can; rows of none of them stay."""
    T, covered = 1600, 1500
    off = torch.tensor(offsets + [offsets[-1]] * empty, dtype=torch.int32, device="cuda")
    for x in gradient(*tensors(T, 8, 1, d, dtype), off, covered, 20, 37):
        rows = x if x.shape[0] == T else x.t()
        assert (rows[covered:] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("empty", [0, 300])
@pytest.mark.parametrize("lens", [[1500], [21] * 40, [400, 20, 21, 1000, 0, 22, 149]])
def test_workspace_is_as_large_as_it_says(lens, empty, d, dtype):
    """One long sequence, many that are hardly longer than the window, some of each; every byte beside it stays."""
    H, H_kv, window, sinks = 16, 1, 20, 5
    lens = [1100] + lens
    ins = tensors(sum(lens), H, H_kv, d, dtype)
    out, lse, *grads = gradient(*ins, lengths_to_offsets(lens + [0] * empty).cuda(), max(lens), window, sinks)
    q, k, v, g = ins
    compare(lens, H, H_kv, d, dtype, window, sinks, (q, k, v, g), out, lse, grads)

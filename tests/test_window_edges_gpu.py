"""Packed attention with a window and first tokens that stay visible: the workspace of its gradient, whatever the offsets say, and rows that are no numbers."""
import pytest
import torch

from paper_2311_09431_amd import binding as sa
from seen import window_mask
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


@pytest.mark.parametrize("small", ["q", "k", "v", "g"])
@pytest.mark.parametrize("d,H,H_kv,sinks", [(64, 2, 1, 4), (100, 2, 2, 40), (128, 16, 8, 33), (256, 2, 1, 5)])
def test_small_magnitudes_and_first_keys_seen_from_far(d, H, H_kv, sinks, small):
    # as the ring step has it: three bf16 terms hold fewer than 24 bits of a number below 2^-109, and every output's error in the 2-norm is as without
    n, window = 700, 100
    see = window_mask(n, window, sinks).cuda()
    for exponent in (-100, -105, -109, -112, -116, -120):
        x = dict(zip("qkvg", tensors(n, H, H_kv, d, F32)))
        x[small] = x[small] * 2.0 ** exponent
        out, _, *grads = gradient(*x.values(), lengths_to_offsets([n]).cuda(), n, window, sinks)
        q, k, v, g = (y.double().transpose(0, 1) for y in x.values())
        k, v = (y.repeat_interleave(H // H_kv, 0) for y in (k, v))
        t = lambda y: y.transpose(-1, -2).contiguous()      # noqa: E731
        p = (q @ t(k) * d ** -0.5).masked_fill(~see, -float("inf")).softmax(-1)
        ds = p * (g @ t(v) - (g * (p @ v)).sum(-1, keepdim=True)) * d ** -0.5
        shared = lambda y: y.view(H_kv, H // H_kv, n, d).sum(1)      # noqa: E731
        for name, got, want in (("O", out, p @ v), ("dQ", grads[0], ds @ k), ("dK", grads[1], shared(t(ds) @ q)), ("dV", grads[2], shared(t(p) @ g))):
            got = got.double().transpose(0, 1)
            # The first keys by themselves too.  (Not dQ of the first rows: dP - delta is a difference of two numbers that are alike, in row 0 the same, so
            # that what both are rounded by, about sqrt(d) 2^-24 of them each, 1e-6 at 256 columns, is not small beside what is left.)
            for rows in (slice(0, n), slice(0, sinks)) if name in ("dK", "dV") else (slice(0, n),):
                error = float((got - want)[:, rows].norm() / want[:, rows].norm())
                assert error <= 1e-6, (name, exponent, rows, error)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_peaked_scores_and_first_keys_take_no_longer(d):
    # scores of standard deviation 300 leave single first keys whose every probability is below 2^-105 beside others
    n, H, window, sinks, off = 700, 8, 128, 130, lengths_to_offsets([700]).cuda()
    times = []
    for spread in (1, 300):
        q, k, v, g = tensors(n, H, H, d, F32)
        q *= spread
        out, lse, *grads = gradient(q, k, v, g, off, n, window, sinks)
        delta, work = torch.empty_like(lse), torch.empty(sa.sa_attn_window_bwd_workspace(q, k, off, n, window, sinks), dtype=torch.uint8, device="cuda")
        taken = []
        for _ in range(5):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(4):
                sa.sa_attn_window_bwd(q, k, v, out, g, lse, off, delta, *grads, work, n, window, sinks)
            end.record()
            torch.cuda.synchronize()
            taken.append(start.elapsed_time(end))
        times.append(min(taken))
        faint = [int(((x[:sinks].abs().amax(-1) < 2.0 ** -105) & (x[:sinks] != 0).any(-1)).sum()) for x in grads[1:]]
    assert all(faint) and times[1] <= 2 * times[0], (faint, times)

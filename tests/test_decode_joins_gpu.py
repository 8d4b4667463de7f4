"""Attention of new tokens where pieces of many heads are joined by a wavefront each, and beside heads that are no numbers, against 64 bits."""
import pytest
import torch

from test_paged_gpu import BF16, F32, compare, decode

pytestmark = pytest.mark.gpu


# 133 sequences of four heads are more than the 512 that workgroups of eight wavefronts join
MANY = [0] * 20 + [4000, 1, 700] + [3] * 109 + [1300]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [4, 20, 32, 64, 100, 128, 132, 256])
def test_many_heads(d, dtype):
    assert len(MANY) * 4 > 512
    q, rows, out, lse = decode(MANY, 4, 2, d, dtype, page=64)
    compare(q, rows, out, lse, dtype)
    again = decode(MANY, 4, 2, d, dtype, page=64, with_lse=False)
    assert torch.equal(again[2], out) and (again[3] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_heads_with_scores_that_are_no_numbers(dtype):
    """Of four long sequences one has every other key at -inf, one all, one a key at +inf, one a NaN; the others notice nothing."""
    inf, n, at = float("inf"), 2000, 50

    def mutate(q, rows, k_cache, v_cache, table):
        q[:] = q.abs() + 0.1                    # a key of infinities has that score
        page = k_cache.shape[1]

        def put(s, t, value):
            rows[s][0][t] = value
            k_cache[int(table[s, t // page]), t % page] = value
        for t in range(n):
            put(at + 1, t, -inf)
            if t % 2 == 0:
                put(at, t, -inf)
        put(at + 2, n - 1, inf)
        put(at + 3, n // 2, float("nan"))
    lens = [3] * at + [n] * 4 + [5, 0, n] + [2] * 210
    q, rows, out, lse = decode(lens, 2, 1, 64, dtype, page=16, mutate=mutate)
    assert len(lens) * 2 > 512
    rows[at] = [x[1::2] for x in rows[at]]
    keep = [s for s in range(len(lens)) if not at < s < at + 4]
    compare(q[keep], [rows[s] for s in keep], out[keep], lse[keep], dtype)
    assert out[at + 1:at + 4].isnan().all() and lse[at + 1:at + 4].isnan().all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [36, 64, 100, 132, 252])
@pytest.mark.parametrize("order", ["shd", "hsd"])
@pytest.mark.parametrize("width", [None, 300])
def test_heads_beside_one_that_is_no_number(width, order, d, dtype):
    """The second of three key/value heads and its queries: what follows a row of the first in memory, and lies in front of the third's."""
    def mutate(q, rows, k_cache, v_cache, table):
        q[:, 2:4] = float("nan")
        k_cache[:, :, 1], v_cache[:, :, 1] = float("nan"), float("inf")
    q, rows, out, lse = decode([1, 77, 300, 16], 6, 3, d, dtype, order=order, width=width, mutate=mutate)
    assert out[:, 2:4].isnan().all() and lse[:, 2:4].isnan().all()
    heads = [0, 1, 4, 5]
    compare(q[:, heads], [[x[:, ::2] for x in kv] for kv in rows], out[:, heads], lse[:, heads], dtype)

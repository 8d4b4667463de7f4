"""Host-side rules of packed launches (no GPU needed)."""
import random

import pytest

from paper_2311_09431_amd import binding as sa
from tests import packed_routes as routes


def test_the_mirrored_struct_is_the_library_s():
    wanted = lambda *a: (routes.rows_of_32(routes.args(*a), False), routes.rows_of_32(routes.args(*a), True))      # noqa: E731
    assert wanted(5, 1000, 300, 4, 4, 128) == (True, True)
    assert wanted(5, 20000, 4096, 32, 8, 128) == (False, False)
    assert wanted(16, 2000, 128, 8, 8, 128) == (False, False)
    assert wanted(1, 8192, 8192, 4, 4, 128) == (True, False)


@pytest.mark.parametrize("backward", [False, True])
def test_a_launch_of_32_row_workgroups_holds_fewer_threads_than_hip_takes(backward):
    """The rule goes by the tiles of the key/value heads; the launch has workgroups for the query heads of each, 256 threads (512 forward)."""
    taken = []
    for d in (4, 32, 64, 100, 128):
        for H, H_kv in ((65535, 1), (65535, 3), (65535, 4369), (16383, 1), (8192, 1), (8191, 1), (4096, 2), (32, 8)):
            for n_seq, rows, max_len in ((1, 65408, 65408), (1, 8192, 8192), (1, 16384, 16384), (1, 4095, 4095), (7, 30000, 9000), (100, 3000, 64),
                                         (300, 9000, 33), (1, 128, 128)):
                p = routes.args(n_seq, rows, max_len, H, H_kv, d, apart=True)
                if routes.rows_of_32(p, backward):
                    workgroups = routes.most_tiles(p, 32) * (H + (H_kv if backward else 0))
                    assert workgroups * (256 if backward else 512) < 1 << 32, (H, H_kv, n_seq, rows, max_len, d)
                    taken.append(workgroups)
    assert taken and (not backward or max(taken) > 1 << 23)         # (it is not that large launches are never taken)


def test_128_row_workgroups_instead_of_too_many_of_32():
    # heads apart: both calls are within the limits of the entry points
    for rows, H in ((65408, 16383), (8192, 65535)):
        assert not routes.rows_of_32(routes.args(1, rows, rows, H, 1, 4, sa.BF16, apart=True), True)
    assert routes.rows_of_32(routes.args(1, 8192, 8192, 65534, 1, 4, sa.BF16, apart=True), True)


@pytest.mark.parametrize("kind,lens,H,H_kv,d,max_len,forward,backward", routes.CASES)
def test_cases_reach_the_kernels_that_they_name(kind, lens, H, H_kv, d, max_len, forward, backward):
    """What test_packed_routes_gpu.py runs: a rule that changes must not leave a kernel without a case."""
    rows = sum(lens) + sum(routes.ROWS_AROUND)
    p = routes.args(len(lens), rows, max_len or max(lens), H, H_kv, d, sa.BF16 if kind == "bf16" else sa.F32)
    if kind == "fp32":
        assert (routes.f32(p, False), routes.f32(p, True)) == (forward, backward)
    else:
        assert (("32 rows" if routes.rows_of_32(p, False) else "128 rows"), routes.backward(p)) == (forward, backward)


def test_every_kind_of_kernel_has_a_case():
    columns = lambda d: 32 if d <= 32 else 64 if d <= 64 else 128 if d <= 128 else 256       # noqa: E731
    have = {(kind, columns(d), route) for kind, _, _, _, d, _, forward, backward in routes.CASES for route in (forward, "backward: " + backward)}
    kinds = ("32 rows", "128 rows", "256 rows", "fp32 instruction")
    for c in (32, 64, 128):
        assert {("fp32", c, k) for k in kinds} <= have and {("fp32", c, "backward: " + k) for k in ("32 rows", "128 rows")} <= have
        assert {("bf16", c, k) for k in kinds[:2]} <= have and ("bf16", c, "backward: 32 rows") in have
    assert {("fp32", c, "backward: fp32 instruction") for c in (32, 128)} <= have
    assert {("fp32", 256, k + w) for k in ("", "backward: ") for w in ("few tiles", "many tiles")} <= have
    assert {("bf16", 32, "backward: two"), ("bf16", 64, "backward: two, one wavefront"), ("bf16", 64, "backward: two, two wavefronts"),
            ("bf16", 128, "backward: two"), ("bf16", 128, "backward: one launch")} <= have
    assert {("bf16", 256, "backward: " + k) for k in ("one launch", "two, halves", "two, all columns")} <= have


def test_no_fp32_instruction_in_the_backward_at_33_to_64_columns():
    """There is no such kernel: what is picked is one that there is, and short sequences go to those of 128 rows."""
    rng = random.Random(6)
    for _ in range(4000):
        n, longest = int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 15))
        H_kv = int(2 ** rng.uniform(0, 8))
        p = routes.args(n, max(longest, int(n * longest * rng.random())), longest, H_kv * int(2 ** rng.uniform(0, 7)), H_kv, rng.choice([36, 48, 60, 64]), sa.F32)
        assert routes.f32(p, True) in ("32 rows", "128 rows") and (longest > 32 or routes.f32(p, True) == "128 rows")

"""Host-side rules of packed launches (no GPU needed)."""
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

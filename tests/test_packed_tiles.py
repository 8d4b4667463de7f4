"""How a workgroup of a packed launch finds its tile (csrc/packed.h, compiled for the host): the sums that its search goes by."""
import ctypes

import numpy as np
import pytest

from tests import host_code

SOURCE = """
#include "packed.h"
// as a wavefront forms it: the sequences in turn to 64 lanes, then the lanes' sum
extern "C" int counted(const int* tiles, int n, int w) {
    int lane[64] = {};
    for (int s = 0; s < n; ++s) lane[s % 64] = sa::add_tiles(lane[s % 64], tiles[s], w);
    unsigned sum = 0;
    for (int x : lane) sum += (unsigned)x;
    return (int)sum;
}
extern "C" int64_t most(int n_seq, int rows, int max_len, int tile) {
    sa::PackedArgs p{};
    p.n_seq = n_seq; p.rows = rows; p.max_len = max_len;
    return sa::most_tiles(p, tile);
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    lib = host_code.library(tmp_path_factory.mktemp("tiles"), SOURCE)
    lib.counted.argtypes, lib.counted.restype = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int], ctypes.c_int
    lib.most.argtypes, lib.most.restype = [ctypes.c_int] * 4, ctypes.c_int64
    return lib


RANKS = 1 << 24         # more than a launch has


@pytest.mark.parametrize("n_seq,tiles", [(1, 3), (64, 7), (65, 1), (200, 40), (4096, 600), (1 << 17, 1 << 15), (1 << 20, 1 << 12), (33, 1 << 26), (1 << 16, 1 << 15),
                                         ((1 << 16) + 1, 1 << 15), (1 << 18, 1 << 14), (3 << 16, 1 << 15)])
def test_sums_are_right_up_to_any_rank_and_stay_above_behind_it(host, n_seq, tiles):
    """Offsets may give the same rows to many sequences: the sums then pass what 32 bits hold."""
    all_tiles = np.full(n_seq, tiles, np.int32)
    all_tiles[n_seq // 2:] //= 3
    for w in {1, 2, tiles // 3 + 1, tiles // 2 + 1, tiles, tiles + 1}:
        got = host.counted(all_tiles.ctypes.data, n_seq, w)
        want = int(np.maximum(0, all_tiles.astype(np.int64) - w + 1).sum())
        assert got == want if want < RANKS else RANKS <= got < 1 << 31, (w, got, want)


@pytest.mark.parametrize("seed", range(40))
def test_a_launch_has_a_rank_for_every_tile_of_sequences_that_share_no_row(host, seed):
    """In any order, with gaps, cut off at max_len."""
    rng = np.random.default_rng(seed)
    n, rows = int(rng.integers(1, 200)), int(rng.integers(1, 6000))
    cuts = np.sort(rng.integers(0, rows + 1, 2 * n))
    lens = np.diff(cuts)[::2] if seed % 2 else np.diff(np.concatenate([[0], cuts, [rows]]))
    lens = rng.permutation(lens)
    for max_len in {1, 31, 33, 128, 129, int(lens.max()) or 1, rows}:
        kept = np.minimum(lens, max_len)
        for tile in (32, 64, 128, 256):
            assert int((-(-kept // tile)).sum()) <= host.most(len(lens), rows, min(max_len, rows), tile)

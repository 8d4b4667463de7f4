"""The library's rules for packed sequences, asked on the host (they launch nothing), as routes.py asks the ring step's."""
import ctypes

from paper_2311_09431_amd import binding as sa
from tests.routes import StepArgs


class PackedArgs(StepArgs):                # csrc/packed.h
    _fields_ = ([("offsets", ctypes.c_void_p)] + [(n, ctypes.c_int) for n in ("n_seq", "rows", "max_len", "n_ranks", "es")]
                + [("by_rank", ctypes.c_bool)])


def args(n_seq, rows, max_len, H, H_kv, d, dtype=sa.BF16, apart=False):
    """As the entry points fill it in for tensors [rows, heads, d]; apart: their heads lie behind each other."""
    p = PackedArgs(B=1, H=H, H_kv=H_kv, d=d, c=0, scale=1.0, layout=sa.CONTIGUOUS, n_q=1, n_kv=1, fresh=True, n_seq=n_seq, rows=rows,
                   max_len=min(max_len, rows), es=2 if dtype == sa.BF16 else 4)
    p.stride_h, p.kv_stride_h = (rows * d, rows * d) if apart else (d, d)
    p.stride_s, p.kv_stride_s = (d, d) if apart else (H * d, H_kv * d)
    p.stat_stride_h = rows
    return p


def most_tiles(p, tile):
    """Tiles of `tile` rows a head has at most."""
    return min(-(-p.max_len // tile) * p.n_seq, p.rows // tile + p.n_seq)


def ask(name, p, *more):
    fn = getattr(sa.lib(), "_ZN2sa%d%sERKNS_10PackedArgsE%s" % (len(name), name, "b" * len(more)))
    fn.restype, fn.argtypes = ctypes.c_bool, [ctypes.c_void_p] + [ctypes.c_bool] * len(more)
    return fn(ctypes.byref(p), *more)


def rows_of_32(p, backward):
    """bf16: 32-row workgroups, not 128-row ones."""
    return ask("packed_split_wanted", p, backward)


def placed(p):
    p.n_ranks = most_tiles(p, 128)
    return p


def backward(p):
    """bf16: the launches of a backward call."""
    if rows_of_32(p, True):
        return "32 rows"
    placed(p)
    if p.d > 64 and ask("packed_one_launch", p):
        return "one launch"
    if p.d > 128:
        return "two, all columns" if p.d % 8 == 0 and ask("packed_all_columns", p) else "two, halves"
    if p.d <= 64 and not (p.d <= 32 and p.d % 8 == 0):
        return "two, two wavefronts" if ask("packed_two_wavefronts", p) else "two, one wavefront"
    return "two"


def f32(p, back):
    """fp32: the kind of kernels."""
    if p.d > 128:
        return "few tiles" if ask("packed_f32_few", p, back) else "many tiles"
    fn = getattr(sa.lib(), "_ZN2sa16packed_f32_routeERKNS_10PackedArgsEb")
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_bool]
    kind = ("fp32 instruction", "32 rows", "128 rows", "not for packed sequences")[fn(ctypes.byref(p), back)]
    return "256 rows" if kind == "128 rows" and not back and most_tiles(p, 128) * p.H >= 512 else kind


# Cases by the kernels that they reach: sequences, heads, key/value heads, columns, max_len (0: the longest); the routes forward and backward.
# Between them rows of no sequence in front and behind (ROWS_AROUND), odd lengths, groups, d % 8 == 4.
ROWS_AROUND = 3, 5
_FEW, _SOME, _SHORT = (130, 33, 1, 64), (700, 129, 1, 300, 257), (128, 77, 100, 1, 33, 128, 64, 2, 97, 31, 128, 60)
_LONG = (1700, 33, 900, 1, 1200, 129, 1500, 2930)
_ONES, _PAGES = tuple(32 - i % 20 for i in range(64)), tuple(200 - 7 * i for i in range(16))
BF16 = ([(_FEW, 2, 1, d, 0, "32 rows", "32 rows") for d in (32, 60, 64, 100, 104, 124, 128)]
        + [(_SOME, 40, 40, 32, 0, "128 rows", "two"), (_SOME, 64, 32, 24, 0, "128 rows", "two")]
        + [(_SOME, 40, 40, d, 0, "128 rows", "two, one wavefront") for d in (36, 60, 64)]
        + [(_LONG, 8, 8, d, 1 << 20, "128 rows", "two, two wavefronts") for d in (60, 64)]
        + [(_SOME, 12, 12, d, 0, "128 rows", "one launch") for d in (100, 104, 124, 128, 132, 252, 256)]
        + [(_SOME, 40, 40, d, 0, "128 rows", "two") for d in (68, 100, 104, 112)] + [(_SOME, 64, 32, d, 0, "128 rows", "two") for d in (124, 128)]
        + [(_SOME, 40, 40, d, 0, "128 rows", "two, halves") for d in (132, 252)] + [(_SOME, 64, 32, d, 0, "128 rows", "two, all columns") for d in (136, 256)]
        + [(_SHORT, 16, 8, d, 0, "128 rows", "two, halves") for d in (132, 192, 256)])
F32 = [(_PAGES, 2, 1, 32, 0, "32 rows", "32 rows"), (_ONES, 8, 4, 32, 0, "fp32 instruction", "fp32 instruction"), (_ONES, 8, 4, 28, 0, "fp32 instruction", "fp32 instruction"),
       (_PAGES, 48, 48, 20, 0, "256 rows", "128 rows"), ((31, 1, 17, 32, 9), 4, 4, 32, 0, "128 rows", "128 rows"),
       (_PAGES, 2, 1, 60, 0, "32 rows", "32 rows"), (_ONES, 8, 4, 60, 0, "fp32 instruction", "128 rows"), (_ONES, 12, 12, 64, 0, "fp32 instruction", "128 rows"),
       (_PAGES, 16, 8, 60, 0, "256 rows", "128 rows"), (_PAGES, 16, 8, 64, 0, "256 rows", "128 rows"), ((300, 129, 1, 257, 33), 32, 8, 60, 0, "128 rows", "32 rows"),
       (_PAGES, 2, 1, 100, 0, "32 rows", "32 rows"), (_PAGES, 2, 1, 128, 0, "32 rows", "32 rows"), (_PAGES, 16, 8, 100, 0, "256 rows", "128 rows"),
       (_PAGES, 16, 8, 124, 0, "256 rows", "128 rows"), (_ONES, 8, 4, 100, 0, "256 rows", "128 rows"), (_SOME, 32, 8, 100, 0, "128 rows", "32 rows"),
       ((300, 129, 1, 257, 33), 32, 8, 128, 0, "128 rows", "32 rows"), ((31, 1, 17, 32, 9), 48, 48, 124, 0, "128 rows", "fp32 instruction"),
       ((33, 5), 1, 1, 100, 0, "32 rows", "fp32 instruction"), ((300, 129, 1, 257, 33), 12, 12, 128, 0, "fp32 instruction", "128 rows"),
       ((300, 129, 1, 257, 33), 16, 8, 124, 0, "fp32 instruction", "32 rows"),
       (_FEW, 2, 1, 132, 0, "few tiles", "few tiles"), (_FEW, 2, 1, 256, 0, "few tiles", "few tiles"), (_ONES, 8, 4, 252, 0, "many tiles", "many tiles"),
       (_PAGES, 16, 8, 132, 0, "many tiles", "many tiles"), (_SOME, 32, 8, 256, 0, "many tiles", "few tiles")]
CASES = [("bf16", *x) for x in BF16] + [("fp32", *x) for x in F32]

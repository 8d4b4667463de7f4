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

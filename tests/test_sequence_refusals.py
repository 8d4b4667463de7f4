"""What the entry points for packed sequences and the paged cache refuse, before anything is launched: the C ABI with pointers that are
never followed, the binding with tensors."""
import ctypes

import pytest
import torch

from paper_2311_09431_amd import binding as sa

P, ODD, NULL = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004), ctypes.c_void_p(0)
OK, E_NULL, E_SHAPE, E_DTYPE, E_ALIGN = 0, -1, -2, -4, -6


class Packed(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_seq", "rows", "max_len", "H", "H_kv", "d")] + [
        (n, ctypes.c_int64) for n in ("stride_h", "stride_s", "kv_stride_h", "kv_stride_s", "stat_stride_h")] + [
        ("dtype", ctypes.c_int32), ("softmax_scale", ctypes.c_float)]


class Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "H_kv", "d")] + [
        (n, ctypes.c_int64) for n in ("stride_page", "stride_s", "stride_h")] + [("dtype", ctypes.c_int32)]


class Append(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("H", ctypes.c_int32)] + [
        (n, ctypes.c_int64) for n in ("stride_h", "stride_s", "kv_stride_h", "kv_stride_s")] + [("rope_base", ctypes.c_float)]


class Decode(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "H", "max_pages")] + [
        (n, ctypes.c_int64) for n in ("stride_b", "stride_h", "stat_stride_b", "table_stride")] + [("softmax_scale", ctypes.c_float)]


def packed(**kw):
    return Packed(**{**dict(n_seq=3, rows=300, max_len=200, H=4, H_kv=2, d=64, stride_h=64, stride_s=256, kv_stride_h=64, kv_stride_s=128,
                            stat_stride_h=300, dtype=sa.BF16), **kw})


def cache(**kw):
    return Cache(**{**dict(n_pages=10, page_size=32, H_kv=2, d=64, stride_page=32 * 128, stride_s=128, stride_h=64, dtype=sa.BF16), **kw})


def rows(**kw):
    return Append(**{**dict(rows=7, H=4, stride_h=64, stride_s=256, kv_stride_h=64, kv_stride_s=128, rope_base=10000.0), **kw})


def decode(**kw):
    return Decode(**{**dict(B=2, H=4, max_pages=5, stride_b=256, stride_h=64, stat_stride_b=4, table_stride=5), **kw})


BAD_PACKED = [(dict(n_seq=-1), E_SHAPE), (dict(rows=-1), E_SHAPE), (dict(max_len=-1), E_SHAPE), (dict(H=0), E_SHAPE), (dict(H_kv=0), E_SHAPE),
              (dict(H_kv=3), E_SHAPE), (dict(d=0), E_SHAPE), (dict(d=62), E_SHAPE), (dict(d=260), E_SHAPE), (dict(stat_stride_h=299), E_SHAPE),
              (dict(stride_s=255), E_SHAPE), (dict(kv_stride_s=60), E_SHAPE), (dict(stride_h=62), E_SHAPE), (dict(stride_s=258), E_ALIGN),
              (dict(kv_stride_s=130), E_ALIGN), (dict(dtype=2), E_DTYPE),
              # a sequence that reaches over 2^31 bytes; in fp32 there is no such limit, but a launch's
              (dict(rows=1 << 20, max_len=1 << 20, stat_stride_h=1 << 20, kv_stride_s=1024), E_SHAPE)]


@pytest.mark.parametrize("kw,status", BAD_PACKED)
def test_packed_shapes(kw, status):
    L, s = sa.lib(), packed(**kw)
    assert L.sa_attn_packed_fwd(P, P, P, P, P, P, ctypes.byref(s), None) == status
    assert L.sa_attn_packed_bwd(*[P] * 11, ctypes.byref(s), None) == status


def test_packed_rows_too_far_apart():
    """128 rows of queries beyond 2^31 bytes"""
    assert sa.lib().sa_attn_packed_fwd(*[P] * 6, ctypes.byref(packed(stride_s=1 << 23)), None) == E_SHAPE


def test_packed_pointers():
    L, s = sa.lib(), packed()
    assert L.sa_attn_packed_fwd(*[P] * 6, None, None) == E_NULL and L.sa_attn_packed_bwd(*[P] * 11, None, None) == E_NULL
    for i in range(6):
        at = [P] * 6
        at[i] = NULL
        assert L.sa_attn_packed_fwd(*at, ctypes.byref(s), None) == E_NULL
        at[i] = ctypes.c_void_p(0x1002)
        assert L.sa_attn_packed_fwd(*at, ctypes.byref(s), None) == E_ALIGN
        if i not in (3, 5):        # offsets and LSE are aligned to their elements
            at[i] = ODD
            assert L.sa_attn_packed_fwd(*at, ctypes.byref(s), None) == E_ALIGN
    for i in range(11):
        at = [P] * 11
        at[i] = NULL
        assert L.sa_attn_packed_bwd(*at, ctypes.byref(s), None) == E_NULL
        at[i] = ctypes.c_void_p(0x1002)
        assert L.sa_attn_packed_bwd(*at, ctypes.byref(s), None) == E_ALIGN
    # q's rows reach too far: the backward streams them
    far = packed(rows=1 << 20, max_len=1 << 20, stat_stride_h=1 << 20, stride_s=1024)
    assert L.sa_attn_packed_bwd(*[P] * 11, ctypes.byref(far), None) == E_SHAPE


@pytest.mark.parametrize("kw", [dict(n_seq=0), dict(rows=0), dict(max_len=0)])
def test_packed_nothing_to_do(kw):
    s = packed(**kw)
    assert sa.lib().sa_attn_packed_fwd(*[NULL] * 6, ctypes.byref(s), None) == OK
    assert sa.lib().sa_attn_packed_bwd(*[NULL] * 11, ctypes.byref(s), None) == OK


BAD_CACHE = [(dict(n_pages=0), E_SHAPE), (dict(page_size=0), E_SHAPE), (dict(page_size=8), E_SHAPE), (dict(page_size=40), E_SHAPE),
             (dict(H_kv=0), E_SHAPE), (dict(d=0), E_SHAPE), (dict(d=66), E_SHAPE), (dict(d=300), E_SHAPE), (dict(stride_s=120), E_SHAPE),
             (dict(stride_h=32), E_SHAPE), (dict(stride_page=32 * 128 - 4), E_SHAPE), (dict(stride_page=32 * 128 + 2), E_ALIGN),
             (dict(stride_s=130, stride_page=1 << 20), E_ALIGN), (dict(dtype=5), E_DTYPE), (dict(n_pages=1 << 26), E_SHAPE), (dict(H_kv=65536), E_SHAPE),
             (dict(stride_s=1 << 24, stride_page=1 << 30), E_SHAPE)]


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_cache_shapes(kw, status):
    L, c = sa.lib(), cache(**kw)
    assert L.sa_cache_append(*[P] * 9, ctypes.byref(rows()), ctypes.byref(c), None) == status
    assert L.sa_attn_decode(*[P] * 7, P, 1 << 30, ctypes.byref(decode()), ctypes.byref(c), None) == status
    assert L.sa_attn_decode_workspace(ctypes.byref(decode()), ctypes.byref(c)) == status


@pytest.mark.parametrize("kw,status", [(dict(rows=-1), E_SHAPE), (dict(H=0), E_SHAPE), (dict(stride_s=250), E_SHAPE), (dict(stride_h=66), E_SHAPE),
                                       (dict(stride_s=258), E_ALIGN), (dict(kv_stride_s=126), E_SHAPE), (dict(kv_stride_s=130), E_ALIGN),
                                       (dict(rope_base=1.0), E_SHAPE), (dict(rope_base=float("nan")), E_SHAPE)])
def test_append_shapes(kw, status):
    assert sa.lib().sa_cache_append(*[P] * 9, ctypes.byref(rows(**kw)), ctypes.byref(cache()), None) == status


def test_append_pointers():
    L, r, c = sa.lib(), rows(), cache()
    call = lambda *at: L.sa_cache_append(*at, ctypes.byref(r), ctypes.byref(c), None)
    # q, q_out, k, k_out, v, pos, slot, k_cache, v_cache
    for i in range(9):
        at = [P] * 9
        at[i] = NULL
        if i != 3:
            assert call(*at) == E_NULL
        at[i] = ctypes.c_void_p(0x1002)
        assert call(*at) == E_ALIGN
        if i not in (5, 6):
            at[i] = ODD
            assert call(*at) == E_ALIGN
    assert L.sa_cache_append(*[P] * 9, None, ctypes.byref(c), None) == E_NULL and L.sa_cache_append(*[P] * 9, ctypes.byref(r), None, None) == E_NULL
    assert L.sa_cache_append(*[NULL] * 9, ctypes.byref(rows(rows=0)), ctypes.byref(c), None) == OK


@pytest.mark.parametrize("kw,status", [(dict(B=-1), E_SHAPE), (dict(H=3), E_SHAPE), (dict(H=0), E_SHAPE), (dict(max_pages=-1), E_SHAPE),
                                       (dict(max_pages=1 << 26, table_stride=1 << 26), E_SHAPE), (dict(stride_h=60), E_SHAPE), (dict(stride_b=252), E_SHAPE),
                                       (dict(stride_b=258), E_ALIGN), (dict(table_stride=4), E_SHAPE), (dict(stat_stride_b=3), E_SHAPE),
                                       (dict(B=1 << 23), E_SHAPE)])
def test_decode_shapes(kw, status):
    assert sa.lib().sa_attn_decode(*[P] * 8, 1 << 30, ctypes.byref(decode(**kw)), ctypes.byref(cache()), None) == status


def test_decode_pointers():
    L, s, c = sa.lib(), decode(), cache()
    size = L.sa_attn_decode_workspace(ctypes.byref(s), ctypes.byref(c))
    assert size > 0 and size == L.sa_attn_decode_workspace(ctypes.byref(decode(B=100, stride_b=512)), ctypes.byref(c))
    # q, k_cache, v_cache, table, lens, out, lse, workspace
    for i in range(8):
        at = [P] * 8
        at[i] = NULL
        if i != 6:
            assert L.sa_attn_decode(*at, size, ctypes.byref(s), ctypes.byref(c), None) == E_NULL
        at[i] = ctypes.c_void_p(0x1002)
        assert L.sa_attn_decode(*at, size, ctypes.byref(s), ctypes.byref(c), None) == E_ALIGN
        if i not in (3, 4, 6):
            at[i] = ODD
            assert L.sa_attn_decode(*at, size, ctypes.byref(s), ctypes.byref(c), None) == E_ALIGN
    assert L.sa_attn_decode(*[P] * 8, size - 1, ctypes.byref(s), ctypes.byref(c), None) == E_SHAPE
    assert L.sa_attn_decode(*[P] * 8, size, None, ctypes.byref(c), None) == E_NULL
    assert L.sa_attn_decode(*[P] * 8, size, ctypes.byref(s), None, None) == E_NULL
    assert L.sa_attn_decode(*[NULL] * 8, 0, ctypes.byref(decode(B=0)), ctypes.byref(c), None) == OK


def test_the_binding_wants_gpu_tensors(monkeypatch):
    monkeypatch.setattr(sa, "_here", lambda: 0)
    monkeypatch.setattr(sa, "_stream", lambda: 0)
    x, i = torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.int32)
    c, lse = torch.zeros(2, 16, 2, 64), torch.zeros(2, 4)
    for call in (lambda: sa.sa_attn_packed_fwd(x, x, x, i, x, lse, 4), lambda: sa.sa_attn_packed_bwd(x, x, x, x, x, lse, i, lse, x, x, x, 4),
                 lambda: sa.sa_cache_append(x, x, i, c, c), lambda: sa.sa_attn_decode(x, c, c, i.view(4, 1), i, x, lse.t(), c)):
        with pytest.raises(TypeError, match="GPU tensor"):
            call()


@pytest.mark.gpu
def test_the_binding_looks_at_its_tensors():
    cuda = dict(device="cuda", dtype=torch.bfloat16)
    T, H, H_kv, d = 20, 4, 2, 64
    q, k = torch.zeros(T, H, d, **cuda), torch.zeros(T, H_kv, d, **cuda)
    off, lse = torch.tensor([0, 5, 20], dtype=torch.int32, device="cuda"), torch.zeros(H, T, device="cuda")

    def fwd(**kw):
        a = {**dict(q=q, k=k, v=k, offsets=off, out=q, lse=lse, max_len=15), **kw}
        return lambda: sa.sa_attn_packed_fwd(**a)

    def bwd(**kw):
        a = {**dict(q=q, k=k, v=k, out=q, dout=q, lse=lse, offsets=off, delta=lse, dq=q, dk=k, dv=k, max_len=15), **kw}
        return lambda: sa.sa_attn_packed_bwd(**a)
    c, slot = torch.zeros(3, 16, H_kv, d, **cuda), torch.zeros(T, dtype=torch.int32, device="cuda")

    def append(**kw):
        a = {**dict(k=k, v=k, slot=slot, k_cache=c, v_cache=c, pos=slot, k_out=k, q=q, q_out=q), **kw}
        return lambda: sa.sa_cache_append(**a)
    table, work = torch.zeros(T, 2, dtype=torch.int32, device="cuda"), torch.zeros(sa.sa_attn_decode_workspace(q, c), dtype=torch.uint8, device="cuda")

    def dec(**kw):
        a = {**dict(q=q, k_cache=c, v_cache=c, table=table, lens=slot, out=q, lse=lse.t().contiguous(), workspace=work), **kw}
        return lambda: sa.sa_attn_decode(**a)
    wrong = [fwd(q=q[:19]), fwd(k=k[..., :32]), fwd(k=k.float(), v=k.float()), fwd(v=k[:, :1]), fwd(q=q[0]), fwd(offsets=off.long()), fwd(offsets=off[::2]),
             fwd(offsets=off[:0]), fwd(out=q.permute(1, 0, 2).contiguous().permute(1, 0, 2)), fwd(out=q.float()), fwd(lse=lse.double()),
             fwd(lse=lse.t().contiguous().t()), fwd(lse=lse[:, :19]), fwd(q=q.half(), k=k.half(), v=k.half(), out=q.half()), fwd(q=q.cpu()),
             fwd(q=torch.zeros(T, H, 2 * d, **cuda)[..., ::2]), bwd(dq=k), bwd(dk=q), bwd(dv=k.float()), bwd(dout=q[:10]), bwd(delta=lse.double()),
             append(v=k.float()), append(slot=slot.long()), append(slot=slot[:5]), append(pos=slot[:5]), append(q_out=None), append(q=None),
             append(pos=None), append(k_out=q), append(k_cache=c[:, :, :1], v_cache=c[:, :, :1]), append(v_cache=c.float()), append(k_cache=c[0]),
             append(q=q[..., :32], q_out=q[..., :32]), append(q_out=q.float()), dec(q=q.float(), out=q.float()), dec(table=table.long()),
             dec(table=table[:5]), dec(lens=slot[:5]), dec(lens=slot.long()), dec(lse=lse), dec(workspace=work[::2]), dec(v_cache=c.float()),
             dec(out=q[:5]), dec(lens=slot.cpu())]
    for i, call in enumerate(wrong):
        with pytest.raises((ValueError, TypeError)):
            call()
            pytest.fail("case %d was taken" % i)
    for call in (fwd(q=q[:, :3], out=q[:, :3], lse=lse[:3]), append(base=1.0), dec(workspace=work[:-16]), dec(q=q[:, :3], out=q[:, :3], lse=None)):
        with pytest.raises(sa.StripedAttnError):
            call()
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_tensors_of_another_device_are_refused(monkeypatch):
    """The current device stands in for another one: the tensors' is 0."""
    monkeypatch.setattr(sa, "_here", lambda: 1)
    x, i = torch.zeros(4, 2, 64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    c, lse = torch.zeros(2, 16, 2, 64, device="cuda"), torch.zeros(2, 4, device="cuda")
    for call in (lambda: sa.sa_attn_packed_fwd(x, x, x, i, x, lse, 4), lambda: sa.sa_attn_packed_bwd(x, x, x, x, x, lse, i, lse, x, x, x, 4),
                 lambda: sa.sa_cache_append(x, x, i, c, c), lambda: sa.sa_attn_decode(x, c, c, i.view(4, 1), i, x, None, c)):
        with pytest.raises(ValueError, match="current device"):
            call()

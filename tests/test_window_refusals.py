"""What the entry points for attention with a window refuse, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2311_09431_amd import binding as sa
from tests.test_sequence_refusals import BAD_PACKED, E_ALIGN, E_NULL, E_SHAPE, NULL, ODD, OK, P, packed


class Window(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("sinks", ctypes.c_int32)]


def fwd(s, w=Window(10, 2), at=None):
    return sa.lib().sa_attn_window_fwd(*(at or [P] * 6), ctypes.byref(s), ctypes.byref(w), None)


def bwd(s, w=Window(10, 2), at=None, size=1 << 40):
    return sa.lib().sa_attn_window_bwd(*(at or [P] * 12), size, ctypes.byref(s), ctypes.byref(w), None)


def bytes_of(s, w):
    return sa.lib().sa_attn_window_bwd_workspace(ctypes.byref(s), ctypes.byref(w))


@pytest.mark.parametrize("kw,status", BAD_PACKED)
def test_shapes(kw, status):
    s = packed(**kw)
    assert fwd(s) == status and bwd(s) == status


@pytest.mark.parametrize("window,sinks", [(0, 0), (-1, 3), (5, -1), (-2 ** 31, 0), (1, -2 ** 31)])
def test_windows(window, sinks):
    w = Window(window, sinks)
    assert fwd(packed(), w) == E_SHAPE and bwd(packed(), w) == E_SHAPE and bytes_of(packed(), w) == E_SHAPE
    # said also where there is nothing to do
    assert fwd(packed(n_seq=0), w) == E_SHAPE and bwd(packed(rows=0), w) == E_SHAPE


def test_pointers():
    L, s, w = sa.lib(), packed(), Window(10, 2)
    assert L.sa_attn_window_fwd(*[P] * 6, None, ctypes.byref(w), None) == E_NULL and L.sa_attn_window_fwd(*[P] * 6, ctypes.byref(s), None, None) == E_NULL
    assert L.sa_attn_window_bwd(*[P] * 12, 0, None, ctypes.byref(w), None) == E_NULL
    assert L.sa_attn_window_bwd(*[P] * 12, 0, ctypes.byref(s), None, None) == E_NULL
    assert L.sa_attn_window_bwd_workspace(None, ctypes.byref(w)) == E_NULL and L.sa_attn_window_bwd_workspace(ctypes.byref(s), None) == E_NULL
    for call, n, loose in ((fwd, 6, (3, 5)), (bwd, 11, (5, 6, 7))):
        for i in range(n):
            at = [P] * (6 if call is fwd else 12)
            at[i] = NULL
            assert call(s, at=at) == E_NULL
            at[i] = ctypes.c_void_p(0x1002)
            assert call(s, at=at) == E_ALIGN
            if i not in loose:          # offsets, LSE and delta are aligned to their elements
                at[i] = ODD
                assert call(s, at=at) == E_ALIGN
    assert bwd(s, at=[P] * 11 + [ODD]) == E_ALIGN


def test_workspace():
    """Long sequences with first tokens take one; it is looked at."""
    s = packed(rows=20000, max_len=20000, stat_stride_h=20000)
    assert bytes_of(s, Window(10, 2)) > 0 and bytes_of(s, Window(10, 0)) == 0 and bytes_of(s, Window(20000, 2)) == 0 and bytes_of(packed(), Window(10, 2)) == 0
    for w in (Window(10, 2), Window(500, 4), Window(20000, 4), Window(1, 0), Window(7, 20000)):
        size = bytes_of(s, w)
        assert 0 <= size < 1 << 31
        if size:
            assert bwd(s, w, size=size - 1) == E_SHAPE and bwd(s, w, at=[P] * 11 + [NULL], size=size) == E_NULL


def test_longest_sequence():
    n, w = 2 ** 30 + 1, Window(10, 2 ** 31 - 1)
    for s in (packed(rows=n, max_len=n, stat_stride_h=n, dtype=1), packed(rows=2 ** 31 - 1, max_len=2 ** 31 - 1, stat_stride_h=2 ** 31, dtype=1)):
        assert fwd(s, w) == E_SHAPE and bwd(s, w) == E_SHAPE and bytes_of(s, w) == E_SHAPE
    for h, kv in ((1, 1), (64, 1), (65535, 65535)):
        for n_seq in (1, 2 ** 20):
            s = packed(rows=2 ** 30, max_len=2 ** 30, stat_stride_h=2 ** 30, dtype=1, H=h, H_kv=kv, n_seq=n_seq, stride_s=h * 64, kv_stride_s=kv * 64)
            for window in (Window(1, 1), Window(1, 2 ** 30), Window(2 ** 29, 5)):
                assert bytes_of(s, window) >= 0


@pytest.mark.parametrize("kw", [dict(n_seq=0), dict(rows=0), dict(max_len=0)])
def test_nothing_to_do(kw):
    s = packed(**kw)
    assert fwd(s, at=[NULL] * 6) == OK and bwd(s, at=[NULL] * 12, size=0) == OK and bytes_of(s, Window(3, 1)) == 0


def test_the_binding_wants_gpu_tensors(monkeypatch):
    monkeypatch.setattr(sa, "_here", lambda: 0)
    monkeypatch.setattr(sa, "_stream", lambda: 0)
    x, i, lse = torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.int32), torch.zeros(2, 4)
    for call in (lambda: sa.sa_attn_window_fwd(x, x, x, i, x, lse, 4, 2), lambda: sa.sa_attn_window_bwd(x, x, x, x, x, lse, i, lse, x, x, x, None, 4, 2)):
        with pytest.raises(TypeError, match="GPU tensor"):
            call()
    with pytest.raises(sa.StripedAttnError):
        sa.sa_attn_window_bwd_workspace(x, x, i, 4, 0)
    with pytest.raises(ValueError):
        sa.sa_attn_window_bwd_workspace(x, x[0], i, 4, 2)


@pytest.mark.gpu
def test_the_binding_looks_at_its_tensors():
    cuda = dict(device="cuda", dtype=torch.bfloat16)
    T, H, H_kv, d = 20, 4, 2, 64
    q, k = torch.zeros(T, H, d, **cuda), torch.zeros(T, H_kv, d, **cuda)
    off, lse = torch.tensor([0, 5, 20], dtype=torch.int32, device="cuda"), torch.zeros(H, T, device="cuda")
    work = torch.empty(64, 64, dtype=torch.uint8, device="cuda")

    def fwd(**kw):
        a = {**dict(q=q, k=k, v=k, offsets=off, out=q, lse=lse, max_len=15, window=3), **kw}
        return lambda: sa.sa_attn_window_fwd(**a)

    def bwd(**kw):
        a = {**dict(q=q, k=k, v=k, out=q, dout=q, lse=lse, offsets=off, delta=lse, dq=q, dk=k, dv=k, workspace=work, max_len=15, window=3), **kw}
        return lambda: sa.sa_attn_window_bwd(**a)
    wrong = [fwd(q=q[:19]), fwd(k=k[..., :32]), fwd(v=k[:, :1]), fwd(offsets=off.long()), fwd(offsets=off[:0]), fwd(out=q.float()), fwd(lse=lse[:, :19]),
             fwd(q=q.cpu()), fwd(window=2.5), fwd(sinks=None), bwd(dq=k), bwd(dk=q), bwd(dv=k.float()), bwd(dout=q[:10]), bwd(delta=lse.double()),
             bwd(workspace=work[:, ::2]), bwd(workspace=work.cpu())]
    for i, call in enumerate(wrong):
        with pytest.raises((ValueError, TypeError, ctypes.ArgumentError)):
            call()
            pytest.fail("case %d was taken" % i)
    for call in (fwd(window=0), fwd(sinks=-1), bwd(window=0), fwd(q=q[:, :3], out=q[:, :3], lse=lse[:3])):
        with pytest.raises(sa.StripedAttnError):
            call()
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(sa, "_here", lambda: 1)
    x, i, lse = torch.zeros(4, 2, 64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(2, 4, device="cuda")
    for call in (lambda: sa.sa_attn_window_fwd(x, x, x, i, x, lse, 4, 2), lambda: sa.sa_attn_window_bwd(x, x, x, x, x, lse, i, lse, x, x, x, None, 4, 2)):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_lengths_beyond_32_bits():
    """The binding's max_len, window and sinks: a number that 32 bits do not hold is the nearest one that they do, none of its bits are dropped."""
    q, k, off = torch.empty(20000, 4, 64, dtype=torch.bfloat16), torch.empty(20000, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    size = lambda *a: sa.sa_attn_window_bwd_workspace(q, k, off, *a)      # noqa: E731
    assert size(20000, 10, 2) > 0 and size(20000, 20000, 2) == 0
    for beyond in (2 ** 31, 2 ** 32, 2 ** 32 + 10, 2 ** 63 - 1, 2 ** 63, 2 ** 64 + 10, 10 ** 40):
        assert size(20000, beyond, 2) == 0                              # no window: nothing is seen from far
        assert size(beyond, 10, 2) == size(20000, 10, 2)                # as long as the tensors
        assert size(20000, 10, beyond) == size(20000, 10, 20000)        # every key is a first one
        for low in ((20000, -beyond, 2), (20000, 10, -beyond), (-beyond, 10, 2)):
            with pytest.raises(sa.StripedAttnError) as e:
                size(*low)
            assert e.value.status == E_SHAPE
    for bad in (10.0, "10", None):
        with pytest.raises((TypeError, ctypes.ArgumentError)):
            size(20000, bad, 2)
    assert size(20000, ctypes.c_int32(10), 2) == size(20000, 10, 2)

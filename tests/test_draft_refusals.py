"""What the entry points for windowed decoding, drafts and moves in the cache refuse, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2311_09431_amd import binding as sa
from tests.test_sequence_refusals import BAD_CACHE, E_ALIGN, E_NULL, E_SHAPE, NULL, ODD, OK, P, cache, decode
from tests.test_window_refusals import Window

REF = ctypes.byref


class Tree(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "H", "max_pages")] + [
        (n, ctypes.c_int64) for n in ("stride_b", "stride_t", "stride_h", "stat_stride_b", "stat_stride_t", "table_stride", "seen_stride")] + [
        ("softmax_scale", ctypes.c_float)]


class Accept(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "max_pages")] + [(n, ctypes.c_int64) for n in ("table_stride", "chosen_stride")]


def tree(**kw):
    return Tree(**{**dict(B=2, T=5, H=4, max_pages=5, stride_b=5 * 256, stride_t=256, stride_h=64, stat_stride_b=20, stat_stride_t=4, table_stride=5,
                          seen_stride=5), **kw})


def accept(**kw):
    return Accept(**{**dict(B=2, T=5, max_pages=5, table_stride=5, chosen_stride=5), **kw})


def play_tree(s=None, c=None, at=None, size=1 << 40):
    return sa.lib().sa_attn_tree(*(at or [P] * 10), size, REF(s or tree()), REF(c or cache()), None)


def play_accept(s=None, c=None, at=None):
    return sa.lib().sa_cache_accept(*(at or [P] * 7), REF(s or accept()), REF(c or cache()), None)


def play_copy(n=3, c=None, at=None):
    return sa.lib().sa_cache_copy(*(at or [P] * 5), n, REF(c or cache()), None)


def play_decode(s=None, c=None, w=Window(10, 2), at=None, size=1 << 40):
    return sa.lib().sa_attn_window_decode(*(at or [P] * 8), size, REF(s or decode()), REF(c or cache()), REF(w), None)


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_cache_shapes(kw, status):
    c = cache(**kw)
    for call in (play_tree, play_accept, play_copy, play_decode):
        assert call(c=c) == status
    assert sa.lib().sa_attn_tree_workspace(REF(tree()), REF(c)) == status


@pytest.mark.parametrize("kw,status", [(dict(B=-1), E_SHAPE), (dict(T=0), E_SHAPE), (dict(T=65, stride_b=65 * 256, stat_stride_b=260, seen_stride=65), E_SHAPE),
                                       (dict(H=3), E_SHAPE), (dict(H=0), E_SHAPE), (dict(max_pages=-1), E_SHAPE), (dict(max_pages=1 << 26, table_stride=1 << 26), E_SHAPE),
                                       (dict(stride_h=60), E_SHAPE), (dict(stride_t=252), E_SHAPE), (dict(stride_b=1276), E_SHAPE), (dict(stride_b=1282), E_ALIGN),
                                       (dict(stride_t=258, stride_b=2000), E_ALIGN), (dict(stride_h=66, stride_t=400, stride_b=4000), E_ALIGN),
                                       (dict(stat_stride_t=3), E_SHAPE), (dict(stat_stride_b=19), E_SHAPE), (dict(table_stride=4), E_SHAPE),
                                       (dict(seen_stride=4), E_SHAPE), (dict(B=1 << 21), E_SHAPE), (dict(B=1 << 12, max_pages=1 << 24, table_stride=1 << 24), E_SHAPE)])
def test_tree_shapes(kw, status):
    assert play_tree(tree(**kw)) == status
    if "seen_stride" not in kw:
        assert sa.lib().sa_attn_tree_workspace(REF(tree(**kw)), REF(cache())) == status


def test_tree_pointers():
    L, s, c = sa.lib(), tree(), cache()
    size = L.sa_attn_tree_workspace(REF(s), REF(c))
    assert size > 0 and size == L.sa_attn_tree_workspace(REF(tree(B=9)), REF(c))
    # q, k_cache, v_cache, table, lens, drafts, seen, out, lse, workspace
    for i in range(10):
        at = [P] * 10
        at[i] = NULL
        if i not in (5, 8):
            assert play_tree(at=at, size=size) == E_NULL
        at[i] = ctypes.c_void_p(0x1002)
        assert play_tree(at=at, size=size) == E_ALIGN
        if i not in (3, 4, 5, 8):
            at[i] = ODD
            assert play_tree(at=at, size=size) == E_ALIGN
    assert play_tree(size=size - 1) == E_SHAPE
    assert L.sa_attn_tree(*[P] * 10, size, None, REF(c), None) == E_NULL and L.sa_attn_tree(*[P] * 10, size, REF(s), None, None) == E_NULL
    assert play_tree(tree(B=0), at=[NULL] * 10, size=0) == OK


def test_tree_workspace_grows_with_the_rows():
    sizes = [sa.lib().sa_attn_tree_workspace(REF(tree(T=t, H=h, B=1, stride_t=64 * h, stat_stride_t=h)), REF(cache())) for t, h in ((1, 2), (8, 2), (16, 4), (64, 8))]
    assert sizes == sorted(sizes) and sizes[0] < sizes[-1] < 1 << 27


@pytest.mark.parametrize("kw", [dict(B=-1), dict(T=0), dict(T=65, chosen_stride=65), dict(max_pages=-1), dict(max_pages=1 << 26, table_stride=1 << 26),
                                dict(table_stride=4), dict(chosen_stride=4), dict(B=(1 << 22) + 1)])
def test_accept_shapes(kw):
    assert play_accept(accept(**kw)) == E_SHAPE


def test_accept_pointers():
    # k_cache, v_cache, table, lens, chosen, accepted, lens_after
    for i in range(7):
        at = [P] * 7
        at[i] = NULL
        if i != 6:
            assert play_accept(at=at) == E_NULL
        at[i] = ctypes.c_void_p(0x1002)
        assert play_accept(at=at) == E_ALIGN
        if i < 2:
            at[i] = ODD
            assert play_accept(at=at) == E_ALIGN
    assert sa.lib().sa_cache_accept(*[P] * 7, None, REF(cache()), None) == E_NULL and sa.lib().sa_cache_accept(*[P] * 7, REF(accept()), None, None) == E_NULL
    assert play_accept(accept(B=0), at=[NULL] * 7) == OK


def test_copy_arguments():
    for i in range(5):
        at = [P] * 5
        at[i] = NULL
        if i != 4:
            assert play_copy(at=at) == E_NULL
        at[i] = ctypes.c_void_p(0x1002)
        assert play_copy(at=at) == E_ALIGN
        if i < 2:
            at[i] = ODD
            assert play_copy(at=at) == E_ALIGN
    assert play_copy(-1) == E_SHAPE and play_copy((1 << 22) + 1) == E_SHAPE and play_copy(0, at=[NULL] * 5) == OK
    assert sa.lib().sa_cache_copy(*[P] * 5, 3, None, None) == E_NULL
    # a page of 2^34 bytes
    big = cache(n_pages=1, page_size=1 << 20, H_kv=64, d=128, stride_h=128, stride_s=64 * 128, stride_page=1 << 33)
    assert play_copy(c=big) == E_SHAPE


@pytest.mark.parametrize("kw,status", [(dict(B=-1), E_SHAPE), (dict(H=3), E_SHAPE), (dict(max_pages=-1), E_SHAPE), (dict(stride_b=258), E_ALIGN),
                                       (dict(table_stride=4), E_SHAPE), (dict(stat_stride_b=3), E_SHAPE)])
def test_window_decode_shapes(kw, status):
    assert play_decode(decode(**kw)) == status


def test_window_decode_arguments():
    for w in (Window(0, 0), Window(-4, 1), Window(3, -1)):
        assert play_decode(w=w) == E_SHAPE
    size = sa.lib().sa_attn_decode_workspace(REF(decode()), REF(cache()))
    for i in range(8):
        at = [P] * 8
        at[i] = NULL
        if i != 6:
            assert play_decode(at=at, size=size) == E_NULL
        at[i] = ctypes.c_void_p(0x1002)
        assert play_decode(at=at, size=size) == E_ALIGN
    assert play_decode(size=size - 1) == E_SHAPE and play_decode(decode(B=0), at=[NULL] * 8, size=0) == OK
    assert sa.lib().sa_attn_window_decode(*[P] * 8, size, REF(decode()), REF(cache()), None, None) == E_NULL


def test_the_binding_wants_gpu_tensors(monkeypatch):
    monkeypatch.setattr(sa, "_here", lambda: 0)
    monkeypatch.setattr(sa, "_stream", lambda: 0)
    x, i, c, m = torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.int32), torch.zeros(2, 16, 2, 64), torch.zeros(4, 1, dtype=torch.int64)
    for call in (lambda: sa.sa_attn_window_decode(x, c, c, i.view(4, 1), i, x, None, c, 3), lambda: sa.sa_attn_tree(x[:, None], c, c, i.view(4, 1), i, m, x[:, None], None, c),
                 lambda: sa.sa_cache_accept(c, c, i.view(4, 1), i, i.view(4, 1), i), lambda: sa.sa_cache_copy(c, c, i, i)):
        with pytest.raises(TypeError, match="GPU tensor"):
            call()


@pytest.mark.gpu
def test_the_binding_looks_at_its_tensors():
    cuda = dict(device="cuda", dtype=torch.bfloat16)
    B, T, H, H_kv, d = 3, 5, 4, 2, 64
    q, c, i = torch.zeros(B, T, H, d, **cuda), torch.zeros(3, 16, H_kv, d, **cuda), torch.zeros(B, dtype=torch.int32, device="cuda")
    table, seen, lse = torch.zeros(B, 2, dtype=torch.int32, device="cuda"), torch.zeros(B, T, dtype=torch.int64, device="cuda"), torch.zeros(B, T, H, device="cuda")
    work, chosen = torch.zeros(sa.sa_attn_tree_workspace(q, c), dtype=torch.uint8, device="cuda"), torch.zeros(B, T, dtype=torch.int32, device="cuda")

    def tr(**kw):
        a = {**dict(q=q, k_cache=c, v_cache=c, table=table, lens=i, seen=seen, out=q, lse=lse, workspace=work, drafts=i), **kw}
        return lambda: sa.sa_attn_tree(**a)

    def ac(**kw):
        a = {**dict(k_cache=c, v_cache=c, table=table, lens=i, chosen=chosen, accepted=i, lens_after=i), **kw}
        return lambda: sa.sa_cache_accept(**a)

    def cp(**kw):
        a = {**dict(k_cache=c, v_cache=c, src=i, dst=i, tokens=i), **kw}
        return lambda: sa.sa_cache_copy(**a)

    def de(**kw):
        a = {**dict(q=q[:, 0], k_cache=c, v_cache=c, table=table, lens=i, out=q[:, 0], lse=lse[:, 0], workspace=work, window=3), **kw}
        return lambda: sa.sa_attn_window_decode(**a)
    wrong = [tr(q=q[0]), tr(q=q.float(), out=q.float()), tr(out=q.float()), tr(out=q[:2]), tr(table=table.long()), tr(table=table[:2]), tr(lens=i.long()), tr(lens=i[:2]),
             tr(drafts=i.long()), tr(drafts=i[:2]), tr(seen=seen.int()), tr(seen=seen[:, :4]), tr(seen=seen.t().contiguous().t()), tr(lse=lse.double()),
             tr(lse=lse[:, :4]), tr(lse=lse[:, 0]), tr(workspace=work[::2]), tr(v_cache=c.float()), tr(q=q[..., :32], out=q[..., :32]), tr(q=q.cpu()),
             ac(v_cache=c[:2]), ac(table=table[:2]), ac(lens=i[:2]), ac(lens=i.long()), ac(chosen=chosen.long()), ac(chosen=chosen[:2]), ac(accepted=i[:2]),
             ac(accepted=i.float()), ac(lens_after=i[:2]), ac(lens_after=i.long()), ac(lens=table), ac(chosen=chosen.t().contiguous().t()),
             cp(src=i.long()), cp(dst=i[:2]), cp(tokens=i[:2]), cp(tokens=i.long()), cp(src=table, dst=table), cp(v_cache=c.float()), cp(k_cache=c[0], v_cache=c[0]),
             de(window=1.5), de(q=q), de(lens=i[:2]), de(lse=lse[:, 0].double()), de(out=q[:2, 0])]
    for n, call in enumerate(wrong):
        with pytest.raises((ValueError, TypeError, ctypes.ArgumentError)):
            call()
            pytest.fail("case %d was taken" % n)
    for call in (tr(workspace=work[:-16]), tr(q=q[:, :, :3], out=q[:, :, :3], lse=None), de(window=0), de(sinks=-1),
                 tr(q=torch.zeros(1, 65, 2, d, **cuda), out=torch.zeros(1, 65, 2, d, **cuda), table=table[:1], lens=i[:1], drafts=None, lse=None,
                    seen=torch.zeros(1, 65, dtype=torch.int64, device="cuda")), ac(chosen=torch.zeros(B, 65, dtype=torch.int32, device="cuda"))):
        with pytest.raises(sa.StripedAttnError):
            call()
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_tensors_of_another_device_are_refused(monkeypatch):
    """The current device stands in for another one: the tensors' is 0."""
    monkeypatch.setattr(sa, "_here", lambda: 1)
    x, i = torch.zeros(4, 2, 64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    c, m = torch.zeros(2, 16, 2, 64, device="cuda"), torch.zeros(4, 1, dtype=torch.int64, device="cuda")
    for call in (lambda: sa.sa_attn_window_decode(x, c, c, i.view(4, 1), i, x, None, c, 3), lambda: sa.sa_attn_tree(x[:, None], c, c, i.view(4, 1), i, m, x[:, None], None, c),
                 lambda: sa.sa_cache_accept(c, c, i.view(4, 1), i, i.view(4, 1), i), lambda: sa.sa_cache_copy(c, c, i, i)):
        with pytest.raises(ValueError, match="current device"):
            call()

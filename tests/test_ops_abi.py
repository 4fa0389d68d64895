"""Host-side checks of the standalone operators: bad calls are refused before
any HIP call (no GPU needed; the pointers are never read)."""
import ctypes as C

import pytest

from paper_2603_18599_amd import sjd

P = 1 << 20  # aligned to every requirement, never read


def call(fn, *args):
    return getattr(sjd.load_library(), fn)(*args)


def given(par=None, io=None):
    p = dict(B=2, L=4, V=50, flags=0, vis_lo=0, p_row=50, p_win=250, q_row=50, q_win=200)
    i = dict(d_p=P, d_q=P, d_draft=P, d_n=P, d_u=P, d_r=P, d_meta=P, d_tok=P, d_next=P)
    p.update(par or {})
    i.update(io or {})
    return call("sjd_verify_given", C.byref(sjd.GivenParams(**p)), C.byref(sjd.GivenIO(**i)), None)


@pytest.mark.parametrize("par", [dict(B=0), dict(B=65536), dict(L=0), dict(L=65), dict(V=0), dict(V=(1 << 24) + 1),
                                 dict(flags=2), dict(flags=4), dict(p_row=49), dict(q_row=49), dict(p_win=-1),
                                 dict(q_win=-1)])
def test_given_refuses_parameters(par):
    assert given(par) == -1


@pytest.mark.parametrize("io", [dict(d_p=None), dict(d_draft=None), dict(d_u=None), dict(d_r=None),
                                dict(d_meta=None), dict(d_tok=None), dict(d_p=P + 2), dict(d_q=P + 1),
                                dict(d_meta=P + 4)])
def test_given_refuses_buffers(io):
    assert given(None, io) == -1


def test_given_needs_next_for_continuation():
    assert given(dict(flags=1), dict(d_next=None)) == -1
    assert call("sjd_verify_given", None, None, None) == -1


def rope(par=None, io=None, axis=None, freq=None):
    p = dict(T=3, H=4, Hkv=2, head_dim=64, pairs=32, axes=3, dtype=1, inverse=0, q_row=256, k_row=128, out_q_row=256,
             out_k_row=128)
    i = dict(d_q=P, d_k=P, d_pos=P, d_out_q=2 * P, d_out_k=2 * P)
    p.update(par or {})
    i.update(io or {})
    n = max(p["pairs"], 1)
    f, a = (C.c_double * n)(*[1.0] * n), (C.c_uint8 * n)()
    for k, v in (axis or {}).items():
        a[k] = v
    for k, v in (freq or {}).items():
        f[k] = v
    p.setdefault("h_freq", C.addressof(f))
    p.setdefault("h_axis", C.cast(a, C.c_char_p))
    return call("sjd_rope_axes", C.byref(sjd.RopeParams(**p)), C.byref(sjd.RopeIO(**i)), None)


@pytest.mark.parametrize("par", [dict(T=-1), dict(T=(1 << 24) + 1), dict(H=-1), dict(H=0, Hkv=0), dict(H=2000),
                                 dict(head_dim=0), dict(head_dim=65), dict(head_dim=258), dict(pairs=0),
                                 dict(pairs=33), dict(axes=0), dict(axes=5), dict(dtype=2), dict(inverse=2),
                                 dict(q_row=255), dict(k_row=127), dict(out_q_row=255), dict(out_k_row=0)])
def test_rope_refuses_parameters(par):
    assert rope(par) == -1


def test_rope_refuses_tables_and_buffers():
    assert rope(axis={31: 3}) == -1
    assert rope(freq={0: float("inf")}) == -1
    assert rope(dict(h_freq=None)) == -1 and rope(dict(h_axis=None)) == -1
    for io in (dict(d_q=None), dict(d_k=None), dict(d_pos=None), dict(d_out_q=None), dict(d_out_k=None),
               dict(d_q=P + 1), dict(d_out_k=P + 1), dict(d_pos=P + 2)):
        assert rope(None, io) == -1, io
    assert rope(dict(out_q_row=512), dict(d_out_q=P)) == -1  # in place with another stride
    assert rope(dict(T=0), dict(d_q=None)) == 0  # nothing to do


PAGES = dict(d_pool=P, n_pages=4, page_len=64, n_kv_heads=2, head_dim=64, dtype=2)
WIN = dict(B=2, T=40, max_rows=20, max_cached=70, table_len=2, d_seq=P, d_table=P)


def append(fn="sjd_kv_append", pages=None, win=None, rows=None):
    p, w, r = dict(PAGES), dict(WIN), dict(d_k=P, d_v=P, k_row=128, v_row=128, dtype=1)
    p.update(pages or {})
    w.update(win or {})
    r.update(rows or {})
    return call(fn, C.byref(sjd.PagesDesc(**p)), C.byref(sjd.WindowsDesc(**w)), C.byref(sjd.KvRows(**r)), None)


def attend(pages=None, win=None, io=None, ws=P, size=1 << 40):
    p, w = dict(PAGES), dict(WIN)
    i = dict(H=4, scale=0.125, d_q=P, d_out=2 * P, q_row=256, out_row=256, d_anc=None)
    p.update(pages or {})
    w.update(win or {})
    i.update(io or {})
    return call("sjd_paged_attention", C.byref(sjd.PagesDesc(**p)), C.byref(sjd.WindowsDesc(**w)),
                C.byref(sjd.AttentionIO(**i)), ws, size, None)


BAD_PAGES = [dict(d_pool=None), dict(d_pool=P + 128), dict(n_pages=0), dict(page_len=16), dict(page_len=48),
             dict(page_len=2048), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(dtype=0), dict(dtype=3)]
BAD_WIN = [dict(B=-1), dict(B=65536), dict(T=-1), dict(T=(1 << 24) + 1), dict(max_rows=41), dict(max_rows=-1),
           dict(max_cached=-1), dict(max_cached=1 << 30), dict(table_len=-1), dict(table_len=0), dict(d_seq=None),
           dict(d_table=None), dict(d_seq=P + 4)]


@pytest.mark.parametrize("fn", ["sjd_kv_append", "sjd_kv_read"])
def test_cache_refusals(fn):
    for b in BAD_PAGES:
        assert append(fn, pages=b) == -1, b
    for b in BAD_WIN:
        assert append(fn, win=b) == -1, b
    for b in (dict(d_k=None), dict(d_v=None), dict(d_k=P + 8), dict(k_row=120), dict(v_row=129), dict(dtype=2)):
        assert append(fn, rows=b) == -1, b
    assert append(fn, pages=dict(head_dim=96)) == -5
    assert append(fn, win=dict(B=0)) == 0 and append(fn, win=dict(max_rows=0)) == 0  # nothing to do


def test_attention_refusals():
    for b in BAD_PAGES:
        assert attend(pages=b) == -1, b
    for b in BAD_WIN:
        assert attend(win=b) == -1, b
    for b in (dict(H=3), dict(H=0), dict(H=2000), dict(scale=float("nan")), dict(scale=float("inf")), dict(d_q=None),
              dict(d_out=None), dict(d_q=P + 8), dict(d_out=P + 2), dict(q_row=252), dict(out_row=248),
              dict(d_anc=P + 4)):
        assert attend(io=b) == -1, b
    assert attend(win=dict(max_rows=65, T=80), io=dict(d_anc=P)) == -1  # a mask has 64 bits
    assert attend(pages=dict(head_dim=32)) == -5
    big = dict(T=1 << 24, max_rows=1 << 24, table_len=1 << 20)
    assert attend(win=big, io=dict(H=128, q_row=1 << 20, out_row=1 << 20)) == -5  # query slots of a window
    assert attend(win=dict(B=0)) == 0
    assert call("sjd_paged_attention", None, None, None, None, 0, None) == -1


def test_attention_refuses_a_scale_that_overflows_as_a_power_of_two():
    import math
    most = 3.4028234e38 / math.log2(math.e)
    for s in (3.4e38, -3.4e38, most * 1.000001):
        assert attend(io=dict(scale=s)) == -1, s
    for s in (most * 0.999999, -0.0, 1e-45):
        assert attend(win=dict(B=0), io=dict(scale=s)) == 0, s


def test_attention_needs_its_workspace():
    w = dict(B=1, T=1, max_rows=1, max_cached=8000, table_len=200)
    lib = sjd.load_library()
    need = lib.sjd_paged_attention_workspace(C.byref(sjd.PagesDesc(**PAGES)), C.byref(sjd.WindowsDesc(**{**WIN, **w})), 4)
    assert need > 0  # a long cache of one sequence is split
    assert attend(win=w, ws=None) == -1
    assert attend(win=w, size=need - 1) == -1
    assert attend(win=w, ws=P + 16) == -1
    assert lib.sjd_paged_attention_workspace(C.byref(sjd.PagesDesc(**PAGES)), C.byref(sjd.WindowsDesc(**WIN)), 3) == 0


def test_page_bytes():
    # data of both parts and every head, one exponent byte a row, 256-byte steps
    assert sjd.page_bytes(64, 2, 64, "bf16") == 2 * 2 * 64 * 64 * 2
    assert sjd.page_bytes(32, 3, 64, "e4m3") == (2 * 3 * 32 * 64 + 2 * 3 * 32 + 255) // 256 * 256
    assert sjd.page_bytes(48, 2, 64, "bf16") == 0


def test_python_side_refuses_tensors_that_do_not_fit():
    import torch
    q, pos = torch.zeros(3, 2, 64), torch.zeros(3, 2, dtype=torch.int32)
    for args in ((q, None, pos, [1.0], [0]), (q.double(), None, pos, [1.0], [0]), (q, None, pos.long(), [1.0], [0]),
                 (q, None, pos, [1.0], [2]), (q, None, pos[:2], [1.0], [0]), (q.transpose(0, 1), None, pos, [1.0], [0])):
        with pytest.raises(sjd.SjdError):  # (the first: tensors that are not on the GPU)
            sjd.sjd_rope_axes(*args)
    with pytest.raises(sjd.SjdError):
        sjd.Pages(torch.zeros(100, dtype=torch.uint8), 1, 32, 1, 64, "e4m3")  # too small
    with pytest.raises(sjd.SjdError):
        sjd.Windows(torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32), 4, 1, 1)


def test_attention_workspace_follows_the_windows():
    """A window of few rows needs no more scratch in large row tensors than in small ones,
    ragged windows no more than their tensors' rows."""
    def need(**w):
        return sjd.load_library().sjd_paged_attention_workspace(C.byref(sjd.PagesDesc(**PAGES)),
                                                                C.byref(sjd.WindowsDesc(**{**WIN, **w})), 4)

    one = dict(B=1, max_rows=1, max_cached=8000, table_len=200)
    assert 0 < need(T=1, **one) == need(T=1 << 20, **one) == need(T=1 << 24, **one)
    few = dict(B=3, max_rows=16, max_cached=8000, table_len=200)
    assert 0 < need(T=20, **few) < need(T=48, **few) == need(T=49, **few)

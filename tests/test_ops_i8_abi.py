"""Host-side checks of the 8-bit projections and of rows placed and appended in
one call: bad calls are refused before any HIP call (no GPU needed; the pointers
are never read)."""
import ctypes as C

import pytest

from paper_2603_18599_amd import sjd
from test_ops_abi import BAD_PAGES, BAD_WIN, P, PAGES, WIN, call


def quantise(par=None, io=None):
    p = dict(T=3, K=50, dtype=1, norm_dtype=0, eps=1e-5, x_row=50, gate_row=50, code_row=64)
    i = dict(d_x=P, d_norm=None, d_gate=None, d_code=2 * P, d_scale=P)
    p.update(par or {})
    i.update(io or {})
    return call("sjd_quantise_rows", C.byref(sjd.QuantiseParams(**p)), C.byref(sjd.QuantiseIO(**i)), None)


@pytest.mark.parametrize("par", [dict(T=-1), dict(T=(1 << 24) + 1), dict(K=0), dict(K=65537), dict(dtype=2), dict(dtype=3),
                                 dict(x_row=49), dict(code_row=48), dict(code_row=65), dict(code_row=56)])
def test_quantise_refuses_parameters(par):
    assert quantise(par) == -1


def test_quantise_refuses_forms_and_buffers():
    for io in (dict(d_x=None), dict(d_code=None), dict(d_scale=None), dict(d_x=P + 1), dict(d_code=P + 8),
               dict(d_scale=P + 2), dict(d_norm=P, d_gate=P), dict(d_norm=P + 2), dict(d_gate=P + 1)):
        assert quantise(None, io) == -1, io
    for par in (dict(norm_dtype=2), dict(eps=0.0), dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(eps=1e-40)):
        assert quantise(par, dict(d_norm=P)) == -1, par
    assert quantise(dict(gate_row=49), dict(d_gate=P)) == -1
    assert quantise(dict(T=0), dict(d_x=None, d_code=None)) == 0  # nothing to do
    assert call("sjd_quantise_rows", None, None, None) == -1


WEIGHTS = dict(N=40, K=50, d_w=P, d_scale=P)


def pack(w=None, src=P, dtype=3, row=50):
    return call("sjd_pack_i8", C.byref(sjd.I8WeightsDesc(**{**WEIGHTS, **(w or {})})), src, dtype, row, None)


def matmul(w=None, io=None, ws=P, size=1 << 40):
    i = dict(T=3, dtype=1, d_code=P, d_code_scale=P, d_out=2 * P, d_add=None, code_row=64, out_row=40, add_row=40)
    i.update(io or {})
    return call("sjd_matmul_i8", C.byref(sjd.I8WeightsDesc(**{**WEIGHTS, **(w or {})})), C.byref(sjd.MatmulIO(**i)), ws,
                size, None)


BAD_WEIGHTS = [dict(N=0), dict(N=(1 << 20) + 1), dict(K=0), dict(K=65537), dict(d_w=None), dict(d_w=P + 128),
               dict(d_scale=None), dict(d_scale=P + 2)]


def test_weights_refusals():
    lib = sjd.load_library()
    for b in BAD_WEIGHTS:
        assert pack(b, row=1 << 20) == -1 and matmul(b, dict(code_row=1 << 20, out_row=1 << 21)) == -1, b
    assert pack(src=None) == -1 and pack(dtype=2) == -1 and pack(dtype=4) == -1 and pack(row=49) == -1
    assert pack(src=P + 2, dtype=0) == -1 and pack(src=P + 1, dtype=1) == -1
    assert lib.sjd_i8_weight_bytes(0, 5) == 0 == lib.sjd_i8_weight_bytes(5, 0) == lib.sjd_i8_weight_bytes(5, 65537)
    assert lib.sjd_i8_weight_bytes(1, 1) >= 32 * 32
    assert lib.sjd_i8_weight_bytes(1 << 20, 65536) == 1 << 36  # no 32-bit size


def test_matmul_refusals():
    for io in (dict(T=-1), dict(T=(1 << 24) + 1), dict(dtype=2), dict(dtype=3), dict(d_code=None), dict(d_code=P + 8),
               dict(d_code_scale=None), dict(d_code_scale=P + 1), dict(d_out=None), dict(d_out=P + 1), dict(code_row=48),
               dict(code_row=72), dict(out_row=39), dict(d_add=P + 1), dict(d_add=P, add_row=39),
               dict(d_add=2 * P, add_row=48), dict(dtype=0, d_out=P + 2)):
        assert matmul(None, io) == -1, io
    assert matmul(None, dict(T=0, d_code=None)) == 0
    assert call("sjd_matmul_i8", None, None, None, 0, None) == -1


def append(pages=None, win=None, rows=None, par=None, axis=None, freq=None):
    p, w, r = dict(PAGES), dict(WIN), dict(d_k=P, d_v=P, k_row=128, v_row=128, dtype=1)
    o = dict(H=4, pairs=32, axes=3, out_dtype=1, d_pos=P, d_q=P, d_out_q=2 * P, q_row=256, out_q_row=256)
    p.update(pages or {})
    w.update(win or {})
    r.update(rows or {})
    o.update(par or {})
    n = max(o["pairs"], 1)
    f, a = (C.c_double * n)(*[1.0] * n), (C.c_uint8 * n)()
    for k, v in (axis or {}).items():
        a[k] = v
    for k, v in (freq or {}).items():
        f[k] = v
    o.setdefault("h_freq", C.addressof(f))
    o.setdefault("h_axis", C.cast(a, C.c_char_p))
    return call("sjd_kv_append_rope", C.byref(sjd.PagesDesc(**p)), C.byref(sjd.WindowsDesc(**w)), C.byref(sjd.KvRows(**r)),
                C.byref(sjd.AppendRope(**o)), None)


def test_append_rope_refusals():
    for b in BAD_PAGES:
        assert append(pages=b) == -1, b
    for b in BAD_WIN:
        assert append(win=b) == -1, b
    for b in (dict(d_k=None), dict(d_v=None), dict(d_k=P + 8), dict(k_row=120), dict(v_row=129), dict(dtype=2)):
        assert append(rows=b) == -1, b
    for b in (dict(H=-1), dict(H=1025), dict(pairs=0), dict(pairs=33), dict(axes=0), dict(axes=5), dict(out_dtype=2),
              dict(out_dtype=3), dict(h_freq=None), dict(h_axis=None), dict(d_pos=None), dict(d_pos=P + 2), dict(d_q=None),
              dict(d_out_q=None), dict(d_q=P + 8), dict(d_out_q=P + 8), dict(q_row=248), dict(q_row=260),
              dict(out_q_row=255), dict(d_out_q=P, out_q_row=264), dict(d_out_q=P, out_dtype=0)):
        assert append(par=b) == -1, b
    assert append(axis={31: 3}) == -1 and append(freq={0: float("nan")}) == -1
    assert append(pages=dict(head_dim=96)) == -5
    assert append(win=dict(B=0)) == 0 and append(win=dict(max_rows=0)) == 0  # nothing to do
    assert call("sjd_kv_append_rope", None, None, None, None, None) == -1


def test_python_side_refuses_tensors_that_do_not_fit():
    import torch
    x, code, scale = torch.zeros(3, 50), torch.zeros(3, 64, dtype=torch.int8), torch.zeros(3)
    for a, kw in (((x, code, scale), {}),  # (tensors that are not on the GPU)
                  ((x, code[:, :50], scale), {}), ((x, code.float(), scale), {}), ((x, code, scale[:2]), {}),
                  ((x.double(), code, scale), {}), ((x[0], code, scale), {}), ((x, code, scale), dict(gate=x.bfloat16())),
                  ((x, code, scale), dict(norm=torch.zeros(49))), ((x.t(), code, scale), {})):
        with pytest.raises(sjd.SjdError):
            sjd.sjd_quantise_rows(*a, **kw)
    with pytest.raises(sjd.SjdError):
        sjd.I8Weights(0, 5, torch.zeros(0))
    with pytest.raises(sjd.SjdError):
        sjd.I8Weights(4, 5, torch.zeros(3))
    w = sjd.I8Weights(40, 50, torch.zeros(40))
    out, ws = torch.zeros(3, 40), torch.zeros(0, dtype=torch.uint8)
    for a, kw in (((code, scale, out, ws), {}), ((code, scale, out[:, :39], ws), {}), ((code[:2], scale, out, ws), {}),
                  ((code, scale, out, ws), dict(add=out.bfloat16())), ((code, scale, out, ws), dict(add=out[:2])),
                  ((code, scale, out, ws.float()), {})):
        with pytest.raises(sjd.SjdError):
            sjd.sjd_matmul_i8(w, *a, **kw)
    with pytest.raises(sjd.SjdError):
        sjd.sjd_pack_i8(w, torch.zeros(40, 49))


def test_workspace_of_products():
    """Split inputs need 32-bit sums: a call without room for them is refused."""
    lib = sjd.load_library()
    w = dict(N=4096, K=11008)
    io = dict(T=128, code_row=11008, out_row=4096, add_row=4096)
    need = lib.sjd_matmul_i8_workspace(C.byref(sjd.I8WeightsDesc(**{**WEIGHTS, **w})), 128)
    assert need >= 2 * 128 * 4096 * 4 and need % (128 * 4096 * 4) == 0
    for ws, size in ((None, need), (None, 0), (P, 0), (P, need - 1), (P + 8, need), (P, -1)):
        assert matmul(w, io, ws, size) == -1, (ws, size)
    for b in BAD_WEIGHTS:
        assert lib.sjd_matmul_i8_workspace(C.byref(sjd.I8WeightsDesc(**{**WEIGHTS, **b})), 128) <= 0, b
    small = sjd.I8WeightsDesc(**WEIGHTS)
    assert lib.sjd_matmul_i8_workspace(C.byref(small), 0) == 0 == lib.sjd_matmul_i8_workspace(C.byref(small), 1)
    assert lib.sjd_matmul_i8_workspace(C.byref(small), -1) <= 0 and lib.sjd_matmul_i8_workspace(None, 1) <= 0


@pytest.mark.parametrize("freq, axis", [([1.0] * 4, [0] * 3), ([1.0] * 4, [0, 0, 0, 256]), ([1.0] * 4, [0, -1, 0, 0]),
                                        ([1.0, 1.0, 1.0, "1"], [0] * 4), ([1.0] * 4, [0, 0, 0.5, 0])])
def test_pairs_of_other_kinds_are_refused(freq, axis):
    with pytest.raises(sjd.SjdError):
        sjd._pairs("sjd_kv_append_rope", freq, axis)


def test_pairs_take_any_sequence_of_numbers():
    import struct

    import numpy as np
    import torch
    want = (3, struct.pack("3d", 1.0, 0.5, -0.25), bytes([2, 0, 1]))
    f, a = [1.0, 0.5, -0.25], [2, 0, 1]
    for freq, axis in ((f, a), (tuple(f), bytes(a)), (np.float32(f), np.int64(a)), (torch.tensor(f), torch.tensor(a))):
        assert sjd._pairs("sjd_kv_append_rope", freq, axis) == want
    assert sjd._pairs("sjd_kv_append_rope", [1.0], torch.tensor([1])) == (1, struct.pack("d", 1.0), b"\1")

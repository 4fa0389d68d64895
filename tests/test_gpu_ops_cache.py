"""Rotary axes, and writing and reading back a cache in pages, against plain
64-bit forms."""
import numpy as np
import pytest
import torch

import paper_2603_18599_amd as sjd
from ops_util import Pool, quantise, table_for

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def rope_reference(x, pos, freq, axis, inverse):
    x = x.double().cpu().numpy()
    y, P = x.copy(), len(freq)
    for i in range(P):
        phi = pos[:, axis[i]].astype(np.float64) * freq[i] * (-1 if inverse else 1)
        z = (x[:, :, i] + 1j * x[:, :, i + P]) * np.exp(1j * phi)[:, None]
        y[:, :, i], y[:, :, i + P] = z.real, z.imag
    return y


def rope_tolerance(x, P, dtype):
    """Angles are reduced in 64 bits (2^-52 of up to 2^31 revolutions: 2^-21 of
    one at most, here positions stay below 2^17: nothing) and kept as 32-bit
    fractions of a turn (2^-25 of a half: 2 pi 2^-26); cos and sin, the two
    products and the sum round by some 2^-22 of the pair's length, and bf16 rounds
    the result once (2^-8 of it, which is at most the length)."""
    x = x.double().cpu().numpy()
    t = np.zeros_like(x)
    size = np.hypot(x[..., :P], x[..., P:2 * P])
    t[..., :P] = t[..., P:2 * P] = size
    return t * (2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0.0))


@pytest.mark.parametrize("T,H,Hkv,hd,P,axes,dtype,inverse", [
    (1, 4, 2, 128, 64, 3, "bf16", False), (7, 3, 1, 64, 32, 1, "fp32", False), (33, 2, 2, 80, 40, 2, "bf16", True),
    (300, 1, 1, 128, 20, 4, "fp32", True), (5, 2, 1, 66, 5, 2, "bf16", False), (9, 1, 1, 2, 1, 1, "fp32", False),
    (4, 2, 1, 256, 128, 3, "bf16", False), (2100, 2, 1, 64, 32, 3, "bf16", False), (3, 2, 0, 64, 32, 2, "fp32", False)])
def test_rope(T, H, Hkv, hd, P, axes, dtype, inverse):
    g = np.random.RandomState(T + hd)
    q, k = (torch.randn(T, n, hd, device="cuda").to(DT[dtype]) for n in (H, Hkv))
    pos = g.randint(-50000, 100000, (T, axes)).astype(np.int32)
    freq, axis = [10000.0 ** (-i / P) for i in range(P)], [int(a) for a in g.randint(0, axes, P)]
    oq, ok = torch.empty_like(q), torch.empty_like(k)
    args = (k, torch.from_numpy(pos).cuda(), freq, axis) if Hkv else (None, torch.from_numpy(pos).cuda(), freq, axis)
    sjd.sjd_rope_axes(q, *args, out_q=oq, out_k=ok if Hkv else None, inverse=inverse)
    for x, o in ((q, oq), (k, ok)):
        want = rope_reference(x, pos, freq, axis, inverse)
        err = np.abs(o.double().cpu().numpy() - want)
        assert (err <= rope_tolerance(x, P, dtype)).all(), err.max()
    # in place
    sjd.sjd_rope_axes(q, *args, inverse=inverse)
    assert torch.equal(q, oq) and (not Hkv or torch.equal(k, ok))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rope_on_rows_of_a_wider_tensor(dtype):
    """q and k inside rows of a joint projection, also from an odd element on
    (no 16-byte accesses), leave their neighbours as they are."""
    T, H, Hkv, hd = 19, 3, 2, 64
    for off, width in ((0, (H + 2 * Hkv) * hd), (1, (H + 2 * Hkv) * hd + 3)):
        rows = torch.randn(T, width, device="cuda").to(DT[dtype])
        before = rows.clone()
        q = rows[:, off:off + H * hd].view(T, H, hd)
        k = rows[:, off + H * hd:off + (H + Hkv) * hd].view(T, Hkv, hd)
        pos = torch.arange(T, dtype=torch.int32, device="cuda")[:, None].contiguous()
        freq, axis = [10000.0 ** (-i / 32) for i in range(32)], [0] * 32
        sjd.sjd_rope_axes(q, k, pos, freq, axis)
        want = rope_reference(before[:, off:off + (H + Hkv) * hd].reshape(T, H + Hkv, hd), pos.cpu().numpy(), freq, axis,
                              False)
        got = rows[:, off:off + (H + Hkv) * hd].reshape(T, H + Hkv, hd)
        tol = rope_tolerance(before[:, off:off + (H + Hkv) * hd].reshape(T, H + Hkv, hd), 32, dtype)
        assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()
        for part in (slice(0, off), slice(off + (H + Hkv) * hd, None)):
            assert torch.equal(rows[:, part], before[:, part])


def test_one_row_of_any_stride():
    """The stride of a single row separates nothing: any value of it is taken."""
    H, hd = 2, 64
    odd = [torch.randn(1, H * hd + 5, device="cuda").bfloat16() for _ in range(4)]
    k, v, k2, v2 = (x[:, :H * hd].unflatten(1, (H, hd)) for x in odd)
    pages = sjd.Pages(torch.zeros(sjd.page_bytes(32, H, hd, "bf16"), dtype=torch.uint8, device="cuda"), 1, 32, H, hd, "bf16")
    seq, table = torch.tensor([[0, 1, 0, 0]], dtype=torch.int32, device="cuda"), torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    win = sjd.Windows(seq, table, 1, 1, 0)
    sjd.sjd_kv_append(pages, win, k, v)
    sjd.sjd_kv_read(pages, win, k2, v2)
    assert torch.equal(k2, k) and torch.equal(v2, v)
    ws, out = sjd.attention_workspace(pages, win, H), torch.zeros(1, H * hd + 3, device="cuda").bfloat16()
    sjd.sjd_paged_attention(pages, win, k, out[:, :H * hd].unflatten(1, (H, hd)), ws, scale=0.125)
    assert torch.equal(out[:, :H * hd], v.flatten(1)) and not out[:, H * hd:].any()
    sjd.sjd_rope_axes(k, None, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), [1.0], [0])
    assert torch.equal(k, k2)


def rows_for(seqs, gap=3):
    """Sequence descriptions with rows nobody owns between them."""
    seq, at = [], gap
    for r, n in seqs:
        seq.append([at, r, n, 0])
        at += r + gap
    return seq, at


CASES = [  # (rows, cached) of each sequence; page length; heads; head size
    ([(1, 0)], 32, 1, 64), ([(1, 31), (1, 32), (1, 33), (0, 5)], 32, 2, 128), ([(70, 0), (33, 95), (5, 27)], 64, 3, 64),
    ([(300, 17)], 128, 2, 128), ([(32, 32), (64, 0), (31, 1)], 32, 1, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("seqs,plen,Hkv,hd", CASES)
def test_append_and_read(seqs, plen, Hkv, hd, cache, dtype):
    table, n_pages = table_for(seqs, plen)
    pool = Pool(n_pages, plen, Hkv, hd, cache)
    seq, T = rows_for(seqs)
    g = torch.Generator(device="cuda").manual_seed(T)
    size = torch.exp2(torch.randint(-20, 20, (T, Hkv, 1), generator=g, device="cuda").float())
    k, v = ((torch.randn(T, Hkv, hd, generator=g, device="cuda") * size).to(DT[dtype]) for _ in range(2))
    k[seq[0][0], 0] = 0.0  # a row of zeros
    before = pool.t.clone()
    st, tt = torch.tensor(seq, dtype=torch.int32).cuda(), torch.from_numpy(table).cuda()
    win = sjd.Windows(st, tt, T, max(r for r, _ in seqs), max(n for _, n in seqs))
    sjd.sjd_kv_append(pool.pages, win, k, v)
    pool.sync()
    kn, vn = k.double().cpu().numpy(), v.double().cpu().numpy()
    back = {d: [torch.full((T, Hkv, hd), 7.0, device="cuda", dtype=DT[d]) for _ in range(2)] for d in DT}
    for d in DT:
        sjd.sjd_kv_read(pool.pages, win, *back[d])
    owned = set()
    for z, (row0, r, n, _) in enumerate(seq):
        for i in range(r):
            page, inside = int(table[z, (n + i) // plen]), (n + i) % plen
            owned.add((page, inside))
            got = pool.decode(page, inside)
            for x, y, j in ((kn, got[0], 0), (vn, got[1], 1)):
                x = x[row0 + i]
                want = quantise(x)[0] if cache == "e4m3" else torch.from_numpy(x).to(torch.bfloat16).double().numpy()
                assert np.array_equal(y, want), (z, i, j)
                for d in DT:  # (both types hold a cached value exactly)
                    assert np.array_equal(back[d][j][row0 + i].double().cpu().numpy(), want), (z, i, j, d)
    named = [row0 + i for row0, r, _, _ in seq for i in range(r)]
    rest = torch.tensor([t for t in range(T) if t not in named], device="cuda")
    for d in DT:
        assert all(bool((b[rest] == 7.0).all()) for b in back[d])
    # other positions keep their bytes: as many changed bytes at most as rows hold
    changed = int((pool.t != before).sum())
    assert changed <= len(owned) * 2 * Hkv * (hd * (1 if cache == "e4m3" else 2) + 1)
    if cache == "bf16":  # every other position still reads as the fill (NaN)
        for page in range(n_pages):
            for inside in range(plen):
                if (page, inside) not in owned:
                    assert np.isnan(np.concatenate(pool.decode(page, inside))).all()


def test_quantiser_borders():
    """Largest magnitudes around 448 * 2^e, non-finite elements, subnormal and
    largest floats."""
    hd = 64
    rows = []
    for top in (448.0, 448.0 * (1 + 2.0 ** -23), 447.9, 1.75, 1.7500002, 0.875, 2.0 ** -126, 2.0 ** -140, 3.4028234e38, 3.0e38, 0.0):
        x = np.linspace(-1, 1, hd).astype(np.float32) * np.float32(top)
        x[0] = top
        rows.append(x)
    for put in ((np.inf,), (-np.inf, np.inf), (np.nan,), (np.nan, np.inf)):
        x = np.linspace(-3, 3, hd).astype(np.float32)
        x[5:5 + len(put)] = put
        rows.append(x)
    rows.append(np.full(hd, np.nan, np.float32))
    x = torch.from_numpy(np.stack(rows))[:, None].contiguous()
    T = len(rows)
    table, n_pages = table_for([(T, 0)], 32)
    pool = Pool(n_pages, 32, 1, hd, "e4m3")
    win = sjd.Windows(torch.tensor([[0, T, 0, 0]], dtype=torch.int32).cuda(), torch.from_numpy(table).cuda(), T, T, 0)
    sjd.sjd_kv_append(pool.pages, win, x.cuda(), x.flip(0).contiguous().cuda())
    pool.sync()
    for i in range(T):
        k, v = pool.decode(int(table[0, 0]), i)
        assert np.array_equal(k, quantise(x[i].numpy())[0], equal_nan=True), i
        assert np.array_equal(v, quantise(x[T - 1 - i].numpy())[0], equal_nan=True), i


def test_pages_outside_the_pool_and_wrong_sequences():
    """Positions of a page id that the pool does not have are not written and
    read as zeros; a sequence whose numbers break the call's bounds is left
    out."""
    hd, plen = 64, 32
    pool = Pool(4, plen, 1, hd, "bf16", fill=0)
    table = torch.tensor([[2, 7, 1], [-1, 3, 0], [3, 3, 3], [3, 3, 3], [3, 3, 3], [3, 3, 3]], dtype=torch.int32).cuda()
    # the last four: rows past T, more rows than the bound, a negative count, behind the table
    seq = torch.tensor([[0, 80, 4, 0], [80, 40, 0, 0], [100, 40, 0, 0], [0, 90, 0, 0], [0, 10, -1, 0],
                        [0, 80, 50, 0]], dtype=torch.int32).cuda()
    T = 120
    k = torch.randn(T, 1, hd, device="cuda").to(torch.bfloat16)
    win = sjd.Windows(seq, table, T, 80, 60)
    sjd.sjd_kv_append(pool.pages, win, k, -k)
    ok, ov = torch.full_like(k, 5.0), torch.full_like(k, 5.0)
    sjd.sjd_kv_read(pool.pages, win, ok, ov)
    want = k.clone()
    want[28:60] = 0.0        # page 7
    want[80:112] = 0.0       # page -1
    assert torch.equal(ok, want) and torch.equal(ov, -want)
    pool.sync()
    assert not pool.raw[0].any() and np.array_equal(pool.decode(3, 7)[0][0], k[119, 0].double().cpu().numpy())
    assert not np.concatenate(pool.decode(3, 8)).any()


def test_single_positions_build_up_a_tile():
    """One row at a time, as decoding writes them: the neighbours stay."""
    hd = 128
    pool = Pool(1, 32, 2, hd, "e4m3")
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    k, v = (torch.randn(32, 2, hd, device="cuda") for _ in range(2))
    for i in np.random.RandomState(0).permutation(32):
        seq = torch.tensor([[0, 1, int(i), 0]], dtype=torch.int32, device="cuda")
        sjd.sjd_kv_append(pool.pages, sjd.Windows(seq, table, 1, 1, 31), k[i:i + 1].contiguous(), v[i:i + 1].contiguous())
    pool.sync()
    for i in range(32):
        a, b = pool.decode(0, i)
        assert np.array_equal(a, quantise(k[i].double().cpu().numpy())[0])
        assert np.array_equal(b, quantise(v[i].double().cpu().numpy())[0])

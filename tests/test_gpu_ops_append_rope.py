"""Rows placed and appended in one call against plain 64-bit forms, and a layer of
8-bit projections around it and the attention."""
import numpy as np
import pytest
import torch

import paper_2603_18599_amd as sjd
from ops_util import Pool, attention, attention_tolerance, quantise, table_for
from test_gpu_ops_cache import rope_reference
from test_gpu_ops_i8 import check_product, check_rows, product, rows_reference

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def turn_error(x, P):
    """Angles are reduced in 64 bits; cos and sin are within 2^-22 (two steps of the library
    function and a correction), two products and a sum round by 2^-23 of the pair's
    length: together below 2^-21 of it."""
    x = x.double().cpu().numpy()
    t = np.zeros_like(x)
    t[..., :P] = t[..., P:2 * P] = np.hypot(x[..., :P], x[..., P:2 * P]) * 2.0 ** -21
    return t


def check_cached(got, want, err, e4):
    """A cached row [hd] against its exact values, which are `err` off before their rounding:
    half a step of bf16, or of e4m3 under the row's power of two (which may be the next one
    where the largest value is at its border)."""
    if not e4:
        assert (np.abs(got - want) <= err + 2.0 ** -8 * (np.abs(want) + err)).all()
        return
    fits = False
    for top in (max(np.abs(want).max() - err.max(), 0.0), np.abs(want).max(), np.abs(want).max() + err.max()):
        _, E = quantise(np.array([top, 0.0]))
        unit = 2.0 ** (float(E) - 127)
        fits |= bool((np.abs(got - want) <= err + np.maximum(2.0 ** -4 * (np.abs(want) + err), unit * 2.0 ** -10)).all())
    assert fits


def setup(seqs, plen, Hkv, hd, cache, extra=0):
    """Sequences (rows, cached) one behind the other in row tensors with `extra` rows more."""
    table, n = table_for(seqs, plen, seed=3)
    pool = Pool(n, plen, Hkv, hd, cache)
    seq, first = [], 0
    for r, c in seqs:
        seq.append([first, r, c, 0])
        first += r
    T = first + extra
    win = sjd.Windows(torch.tensor(seq, dtype=torch.int32).cuda(), torch.from_numpy(table).cuda(), T,
                      max(r for r, _ in seqs), max(c for _, c in seqs))
    return pool, table, seq, T, win


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("hd,Hkv,H,P,axes,dtype,out,plen,seqs", [
    (64, 1, 1, 32, 1, "bf16", "bf16", 32, [(1, 0)]),
    (128, 2, 8, 64, 3, "bf16", "bf16", 64, [(1, 63), (1, 64), (1, 0), (1, 200)]),
    (64, 3, 7, 24, 2, "fp32", "bf16", 64, [(5, 30), (70, 61), (33, 0)]),  # heads that do not divide
    (128, 1, 3, 5, 4, "fp32", "fp32", 128, [(40, 120), (1, 31)]),         # pairs off every alignment
    (64, 2, 2, 1, 1, "bf16", "fp32", 32, [(31, 1), (32, 32), (2, 63)]),
    (128, 2, 0, 40, 2, "bf16", "bf16", 64, [(9, 60), (64, 64)]),          # no queries
    (128, 16, 16, 64, 3, "fp32", "bf16", 64, [(3, 10)]),
    (64, 2, 1, 32, 2, "bf16", "bf16", 1024, [(130, 1000)]),               # fewer query heads than groups
    (64, 8, 32, 16, 3, "bf16", "bf16", 64, [(100, 500), (0, 10), (37, 0), (64, 128)])])
def test_append_rope(hd, Hkv, H, P, axes, dtype, out, plen, seqs, cache):
    g = np.random.RandomState(hd + H + P)
    pool, table, seq, T, win = setup(seqs, plen, Hkv, hd, cache, extra=3)
    before = pool.t.clone()
    q, k, v = (torch.randn(T, n, hd, device="cuda").to(DT[dtype]) for n in (H, Hkv, Hkv))
    pos = g.randint(-70000, 3000000, (T, axes)).astype(np.int32)
    pos[0], pos[T // 2] = 2 ** 31 - 1, -2 ** 31
    freq, axis = [10000.0 ** (-i / P) for i in range(P)], [int(a) for a in g.randint(0, axes, P)]
    oq = torch.full((T, H, hd), 7.0, device="cuda").to(DT[out]) if H else None
    sjd.sjd_kv_append_rope(pool.pages, win, k, v, torch.from_numpy(pos).cuda(), freq, axis, q=q if H else None, out_q=oq)
    used = T - 3
    if H:
        want, err = rope_reference(q, pos, freq, axis, False), turn_error(q, P)
        # (positions of 2^31: the revolutions round by 3 steps of 2^-53, as angles below 2^-50 of the position)
        err = err + np.abs(pos.astype(np.float64)).max(1)[:, None, None] * 2.0 ** -50 * np.abs(q.double().cpu().numpy()).max()
        got = oq.double().cpu().numpy()
        tol = err + ((np.abs(want) + err) * 2.0 ** -8 if out == "bf16" else 0)
        assert (np.abs(got - want)[:used] <= tol[:used]).all()
        assert (got[used:] == 7).all()  # rows that no sequence names
    pool.sync()
    kw, kerr = rope_reference(k, pos, freq, axis, False), turn_error(k, P)
    kerr = kerr + np.abs(pos.astype(np.float64)).max(1)[:, None, None] * 2.0 ** -50 * np.abs(k.double().cpu().numpy()).max()
    vw = v.double().cpu().numpy()
    for z, (first, r, c, _) in enumerate(seq):
        for i in range(r):
            p = c + i
            kk, vv = pool.decode(table[z, p // plen], p % plen)
            for h in range(Hkv):
                check_cached(kk[h], kw[first + i, h], kerr[first + i, h], pool.e4)
                check_cached(vv[h], vw[first + i, h], np.zeros(hd), pool.e4)
    # every other byte is as it was: those that sjd_kv_append leaves, too
    ones, zero = torch.full_like(before, 0x11), torch.zeros_like(k)
    sjd.sjd_kv_append(sjd.Pages(ones, pool.n_pages, plen, Hkv, hd, cache), win, zero, zero)
    untouched = ones == 0x11
    assert torch.equal(pool.t[untouched], before[untouched])
    # in place, and again: the same bits
    if H and out == dtype:
        first = pool.t.clone()
        sjd.sjd_kv_append_rope(pool.pages, win, k, v, torch.from_numpy(pos).cuda(), freq, axis, q=q)
        assert torch.equal(q[:used], oq[:used]) and torch.equal(pool.t, first)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("hd,Hkv,H,P,dtype,cache", [(128, 16, 32, 64, "bf16", "e4m3"), (128, 16, 16, 16, "fp32", "bf16"),
                                                    (64, 24, 48, 5, "bf16", "bf16"), (64, 16, 33, 32, "bf16", "e4m3")])
def test_large_calls_give_the_bits_of_small_ones(hd, Hkv, H, P, dtype, cache, inplace):
    """Calls large enough that a workgroup has several heads and positions, against a call
    for each sequence, and the queries against the formula."""
    seqs = [(600, 70), (511, 0), (577, 33), (1, 5), (640, 64)]
    pool, table, seq, T, win = setup(seqs, 64, Hkv, hd, cache, extra=2)
    q, k, v = (torch.randn(T, n, hd, device="cuda").to(DT[dtype]) for n in (H, Hkv, Hkv))
    pos = torch.randint(0, 100000, (T, 2), dtype=torch.int32, device="cuda")
    freq, axis = [10000.0 ** (-i / P) for i in range(P)], [i % 2 for i in range(P)]
    before = pool.t.clone()

    def place(w, x):
        out = None if inplace else torch.full_like(x, 7.0)
        sjd.sjd_kv_append_rope(pool.pages, w, k, v, pos, freq, axis, q=x, out_q=out)
        return x if inplace else out

    got, pages = place(win, q.clone()), pool.t.clone()
    pool.t.copy_(before)
    one, x = q.clone(), q.clone()
    for z, (first, r, c, _) in enumerate(seq):
        w = sjd.Windows(torch.tensor([seq[z]], dtype=torch.int32).cuda(), torch.from_numpy(table[z:z + 1]).cuda(), T, r, c)
        one[first:first + r] = place(w, x)[first:first + r]
    used = T - 2
    assert torch.equal(got[:used], one[:used]) and torch.equal(pages, pool.t)
    assert torch.equal(got[used:], q[used:] if inplace else torch.full_like(q[used:], 7.0))
    want, err = rope_reference(q, pos.cpu().numpy(), freq, axis, False), turn_error(q, P)
    err = err + 1e5 * 2.0 ** -50 * np.abs(q.double().cpu().numpy()).max()
    tol = err + ((np.abs(want) + err) * 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24 * np.abs(want))
    assert (np.abs(got.double().cpu().numpy() - want)[:used] <= tol[:used]).all()


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
def test_rows_of_a_joint_projection(cache):
    """q, k and v inside the rows of one product, queries turned in place."""
    H, Hkv, hd, P = 4, 2, 64, 32
    pool, table, seq, T, win = setup([(37, 50), (3, 0)], 64, Hkv, hd, cache)
    rows = torch.randn(T, (H + 2 * Hkv) * hd + 8, device="cuda").to(torch.bfloat16)
    q, k, v = (rows[:, a * hd:b * hd].view(T, b - a, hd) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
    before, pos = rows.clone(), torch.arange(T, dtype=torch.int32, device="cuda")[:, None].contiguous()
    freq, axis = [10000.0 ** (-i / P) for i in range(P)], [0] * P
    sjd.sjd_kv_append_rope(pool.pages, win, k, v, pos, freq, axis, q=q)
    assert torch.equal(rows[:, H * hd:], before[:, H * hd:])
    x = before[:, :H * hd].view(T, H, hd)
    want, err = rope_reference(x, pos.cpu().numpy(), freq, axis, False), turn_error(x, P)
    assert (np.abs(q.double().cpu().numpy() - want) <= err + 2.0 ** -8 * (np.abs(want) + err)).all()
    dense = Pool(pool.n_pages, 64, Hkv, hd, cache)
    sjd.sjd_kv_append_rope(dense.pages, win, k.contiguous(), v.contiguous(), pos, freq, axis)
    assert torch.equal(dense.t, pool.t)


def test_bad_sequences_and_pages_are_left_out():
    """Numbers that break the call's bounds leave a sequence out, queries too; a page outside
    the pool keeps its rows out of the cache, and their queries are placed."""
    H, Hkv, hd, P = 2, 1, 64, 32
    pool, table, seq, T, win = setup([(40, 20), (40, 20), (40, 20), (40, 20)], 32, Hkv, hd, "e4m3")
    seq[0][1] = 41      # more rows than max_rows
    seq[1][2] = -1      # negative
    seq[2][0] = T - 39  # past the row tensors
    table[3, 0], table[3, 1] = pool.n_pages, -5
    win = sjd.Windows(torch.tensor(seq, dtype=torch.int32).cuda(), torch.from_numpy(table).cuda(), T, 40, 20)
    q, k, v = (torch.randn(T, n, hd, device="cuda") for n in (H, Hkv, Hkv))
    out = torch.full((T, H, hd), 7.0, device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda")[:, None].contiguous()
    freq, axis = [10000.0 ** (-i / P) for i in range(P)], [0] * P
    sjd.sjd_kv_append_rope(pool.pages, win, k, v, pos, freq, axis, q=q, out_q=out)
    assert (out[:120] == 7).all()
    want = rope_reference(q, pos.cpu().numpy(), freq, axis, False)
    assert (np.abs(out.double().cpu().numpy() - want)[120:] <= turn_error(q, P)[120:]).all()
    # (positions 20 .. 59 of the last one lie on pages 0 and 1: nothing was written)
    assert (pool.t == 0xFF).all()


def test_special_values_keep_to_their_rows():
    """Infinities and NaN in one row of k, q or v change no other row's bytes."""
    H, Hkv, hd, P = 2, 2, 128, 64
    freq, axis = [10000.0 ** (-i / P) for i in range(P)], [0] * P
    for cache in ("e4m3", "bf16"):
        pools = []
        q, k, v = (torch.randn(70, n, hd, device="cuda") for n in (H, Hkv, Hkv))
        outs = []
        for bad in (False, True):
            pool, table, seq, T, win = setup([(70, 10)], 64, Hkv, hd, cache)
            if bad:
                q[33, 0, 3], k[33, 1, 5], v[33, 0, 7], k[33, 0, 2] = float("nan"), float("inf"), -float("inf"), float("nan")
            out = torch.empty_like(q)
            pos = torch.arange(T, dtype=torch.int32, device="cuda")[:, None].contiguous()
            sjd.sjd_kv_append_rope(pool.pages, win, k, v, pos, freq, axis, q=q, out_q=out)
            kk, vv = (torch.empty(T, Hkv, hd, device="cuda") for _ in range(2))
            sjd.sjd_kv_read(pool.pages, win, kk, vv)
            outs.append((out, kk, vv))
        others = torch.arange(70, device="cuda") != 33
        for a, b in zip(*outs):
            assert torch.equal(a[others], b[others])
        assert torch.isnan(outs[1][1][33, 0, 2]) and torch.isnan(outs[1][0][33, 0, 3])


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,Hkv,P", [(64, 1, 5), (64, 3, 16), (64, 2, 24), (128, 1, 5), (128, 2, 16), (128, 9, 40), (64, 2, 31)])
def test_dims_that_pass_through_keep_their_values(hd, Hkv, P, dtype, cache):
    """Infinities, NaN and zeros of either sign in key and query dims behind the pairs: the bytes
    of sjd_rope_axes and then sjd_kv_append. (At position 0, whose angles are exactly 0 in both, whole
    pages; elsewhere, in bf16 pages, the dims that pass through.)"""
    H = 3
    q, k, v = (torch.randn(45, n, hd, device="cuda") for n in (H, Hkv, Hkv))
    values = torch.tensor([float("inf"), -float("inf"), float("nan"), -0.0, 0.0, 3e38, -1e-40])
    for i, x in enumerate(values):
        for t in (q, k, v):
            t[3 * i + 1, i % t.shape[1], 2 * P + (5 * i + 1) % (hd - 2 * P)] = x
    k[40, 0, 2 * P:], k[41, 0, 2 * P:], q[41, 0, 2 * P:] = float("inf"), -0.0, -0.0
    q, k, v = (t.to(DT[dtype]) for t in (q, k, v))
    freq, axis = [10000.0 ** (-i / P) for i in range(P)], [i % 2 for i in range(P)]
    bits = lambda t: t.view(torch.int16 if t.dtype is torch.bfloat16 else torch.int32)  # noqa: E731
    for at in (0, 1):
        one, table, seq, T, win = setup([(45, 20)], 64, Hkv, hd, cache)
        two, pos = Pool(one.n_pages, 64, Hkv, hd, cache), torch.arange(T, dtype=torch.int32, device="cuda")
        pos = (at * pos[:, None] + torch.zeros(1, 2, dtype=torch.int32, device="cuda")).contiguous()
        oq, q2, k2 = (torch.empty_like(t) for t in (q, q, k))
        sjd.sjd_kv_append_rope(one.pages, win, k, v, pos, freq, axis, q=q, out_q=oq)
        sjd.sjd_rope_axes(q, k, pos, freq, axis, out_q=q2, out_k=k2)
        sjd.sjd_kv_append(two.pages, win, k2, v)
        assert torch.equal(bits(oq[..., 2 * P:]), bits(q[..., 2 * P:]))
        if at == 0:
            assert torch.equal(bits(oq), bits(q2)) and torch.equal(one.t, two.t)
            continue
        got = []
        for pool in (one, two):
            out = [torch.empty(T, Hkv, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            sjd.sjd_kv_read(pool.pages, win, *out)
            got.append(out)
        assert torch.equal(bits(got[0][1]), bits(got[1][1]))
        if cache == "bf16":
            assert torch.equal(bits(got[0][0][..., 2 * P:]), bits(got[1][0][..., 2 * P:]))
            assert torch.equal(bits(got[0][0][..., 2 * P:]), bits(k[..., 2 * P:].to(torch.bfloat16)))


def layer(d, T, seed):
    """A decoder layer's tensors: 8-bit weights of q, k, v; output; gate and up; down."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(norm=[1 + 0.1 * torch.randn(d["d"], generator=g, device="cuda") for _ in range(2)])
    for name, N, K in (("qkv", (d["H"] + 2 * d["Hkv"]) * d["hd"], d["d"]), ("o", d["d"], d["H"] * d["hd"]),
                       ("gu", 2 * d["F"], d["d"]), ("down", d["d"], d["F"])):
        w = torch.randn(N, K, generator=g, device="cuda") * K ** -0.5
        s[name] = sjd.I8Weights(N, K)
        sjd.sjd_pack_i8(s[name], w)
        code, scale = torch.empty(N, sjd.code_columns(K), dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
        sjd.sjd_quantise_rows(w, code, scale)
        s[name + "_codes"] = code[:, :K]
        s[name + "_ws"] = sjd.matmul_workspace(s[name], T)
        s[name + "_in"] = (torch.empty(T, sjd.code_columns(K), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"))
    return s


@pytest.mark.parametrize("tree", [False, True])
def test_a_layer_of_8_bit_projections(tree):
    """A window of two sequences through a layer as a program runs it: quantise behind the norm,
    q, k, v in one product, place and append, attend, output, gate and up, down; the residual
    rows in fp32. Each stage against 64 bits on what it was given, and the whole captured and
    replayed between eager runs."""
    d = dict(d=256, H=4, Hkv=2, hd=64, F=704)
    seqs = [(21, 75), (13, 40)]
    pool, table, seq, T, win = setup(seqs, 64, d["Hkv"], d["hd"], "e4m3")
    s = layer(d, T, 5)
    H, Hkv, hd, F, P = d["H"], d["Hkv"], d["hd"], d["F"], d["hd"] // 2
    # what is cached
    old = sjd.Windows(torch.tensor([[0, 75, 0, 0], [75, 40, 0, 0]], dtype=torch.int32).cuda(), win.table, 115, 75, 0)
    sjd.sjd_kv_append(pool.pages, old, *(torch.randn(115, Hkv, hd, device="cuda") for _ in range(2)))
    start, x0 = pool.t.clone(), torch.randn(T, d["d"], device="cuda")
    pos = torch.cat([torch.arange(c, c + r) for r, c in seqs]).to(torch.int32).cuda()[:, None].contiguous()
    freq, axis = [10000.0 ** (-i / P) for i in range(P)], [0] * P
    anc = None
    if tree:
        anc = torch.tensor([(1 << (i + 1)) - 1 if i < 8 else 1 | 1 << i for r, _ in seqs for i in range(r)],
                           dtype=torch.int64).cuda()
    x = x0.clone()
    qkv = torch.empty(T, (H + 2 * Hkv) * hd, device="cuda")
    q, k, v = (qkv[:, a * hd:b * hd].view(T, b - a, hd) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
    qr, att = (torch.empty(T, H, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gu = torch.empty(T, 2 * F, dtype=torch.bfloat16, device="cuda")
    ws = sjd.attention_workspace(pool.pages, win, H)
    mid = torch.empty_like(x)

    def run():
        pool.t.copy_(start)
        x.copy_(x0)
        sjd.sjd_quantise_rows(x, *s["qkv_in"], norm=s["norm"][0], eps=1e-5)
        sjd.sjd_matmul_i8(s["qkv"], *s["qkv_in"], qkv, s["qkv_ws"])
        sjd.sjd_kv_append_rope(pool.pages, win, k, v, pos, freq, axis, q=q, out_q=qr)
        sjd.sjd_paged_attention(pool.pages, win, qr, att, ws, scale=hd ** -0.5, anc=anc)
        sjd.sjd_quantise_rows(att.view(T, H * hd), *s["o_in"])
        sjd.sjd_matmul_i8(s["o"], *s["o_in"], x, s["o_ws"], add=x)
        mid.copy_(x)
        sjd.sjd_quantise_rows(x, *s["gu_in"], norm=s["norm"][1], eps=1e-5)
        sjd.sjd_matmul_i8(s["gu"], *s["gu_in"], gu, s["gu_ws"])
        sjd.sjd_quantise_rows(gu[:, F:], *s["down_in"], gate=gu[:, :F])
        sjd.sjd_matmul_i8(s["down"], *s["down_in"], x, s["down_ws"], add=x)

    run()
    torch.cuda.synchronize()

    def stage(name, rows, out, add=None):
        y, off = rows
        check_rows(y, off, s[name + "_in"][0], s[name + "_in"][1], s[name + "_in"][0].shape[1])
        check_product(out, *product(*s[name + "_in"], s[name + "_codes"], s[name].scale, add))

    stage("qkv", rows_reference(x0, s["norm"][0]), qkv)
    want, err = rope_reference(q, pos.cpu().numpy(), freq, axis, False), turn_error(q, P)
    assert (np.abs(qr.double().cpu().numpy() - want) <= err + 2.0 ** -8 * (np.abs(want) + err)).all()
    pool.sync()
    qn, an = qr.double().cpu().numpy(), att.double().cpu().numpy()
    kw, kerr = rope_reference(k, pos.cpu().numpy(), freq, axis, False), turn_error(k, P)
    for z, (first, r, c, _) in enumerate(seq):
        kv = [pool.decode(table[z, p // 64], p % 64) for p in range(c + r)]
        kk, vv = np.stack([a for a, _ in kv]), np.stack([b for _, b in kv])
        for i in range(r):
            for h in range(Hkv):
                check_cached(kk[c + i, h], kw[first + i, h], kerr[first + i, h], True)
        seen = np.ones((r, c + r), bool)
        for i in range(r):
            bits = int(anc[first + i]) if tree else (1 << (i + 1)) - 1
            seen[i, c:] = [bits >> j & 1 for j in range(r)]
        for h in range(H):
            o, mag = attention(qn[first:first + r, h], kk[:, h // 2], vv[:, h // 2], hd ** -0.5, seen)
            tol = attention_tolerance(qn[first:first + r, h], kk[:, h // 2], hd ** -0.5, mag, o, c + r)
            assert (np.abs(an[first:first + r, h] - o) <= tol).all()
    stage("o", rows_reference(att.view(T, H * hd)), mid, x0)
    stage("gu", rows_reference(mid, s["norm"][1]), gu)
    stage("down", rows_reference(gu[:, F:], None, gu[:, :F]), x, mid)

    keep = x.clone(), pool.t.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(3):
        x0.copy_(torch.randn_like(x0))
        graph.replay()
        torch.cuda.synchronize()
        got = x.clone(), pool.t.clone()
        run()
        torch.cuda.synchronize()
        assert torch.equal(got[0], x) and torch.equal(got[1], pool.t)
    assert not torch.equal(keep[0], x)

"""sjd_paged_attention against the plain 64-bit form, over the cache as it
was written (values decoded from the pages' bytes)."""
import numpy as np
import pytest
import torch

import paper_2603_18599_amd as sjd
from ops_util import Pool, attention, attention_tolerance, quantise, table_for, val_elem

pytestmark = pytest.mark.gpu


class Case:
    """Sequences (rows, cached), their pages filled by sjd_kv_append, and q.
    many: with so many empty sequences behind them that a launch counts as one of
    many query slots (keys shared by 128 slots rather than shared out)."""

    def __init__(self, seqs, plen, Hkv, G, hd, cache, seed=0, gap=2, scale=1.0, fill=0xFF, many=False):
        if many:
            tiles = Hkv * -(-max(r for r, _ in seqs) * G // 32)
            seqs = seqs + [(0, 0)] * (1536 // tiles + 1)
        self.seqs, self.Hkv, self.G, self.H, self.hd, self.cache = seqs, Hkv, G, Hkv * G, hd, cache
        self.plen = plen
        self.table, n_pages = table_for(seqs, plen, seed)
        self.pool = Pool(n_pages, plen, Hkv, hd, cache, fill)
        g = torch.Generator().manual_seed(seed + 1)
        self.k, self.v = ([torch.randn(r + n, Hkv, hd, generator=g).to(torch.bfloat16) for r, n in seqs] for _ in range(2))
        self.seq, at = [], gap
        for r, n in seqs:
            self.seq.append([at, r, n, 0])
            at += r + gap
        self.T = at
        self.q = (torch.randn(self.T, self.H, hd, generator=g) * scale).to(torch.bfloat16)
        self.st = torch.tensor(self.seq, dtype=torch.int32).cuda()
        self.tt = torch.from_numpy(self.table).cuda()
        self.scale = hd ** -0.5
        self.fill_pages()

    def fill_pages(self):
        rows = [r + n for r, n in self.seqs]
        if not sum(rows):
            return
        whole = torch.tensor([[sum(rows[:z]), m, 0, 0] for z, m in enumerate(rows)], dtype=torch.int32).cuda()
        win = sjd.Windows(whole, self.tt, sum(rows), max(rows), 0)
        sjd.sjd_kv_append(self.pool.pages, win, torch.cat(self.k).cuda(), torch.cat(self.v).cuda())

    def windows(self, slack=0):
        return sjd.Windows(self.st, self.tt, self.T, max(r for r, _ in self.seqs), max(n for _, n in self.seqs) + slack)

    def run(self, anc=None, q=None, slack=0):
        win = self.windows(slack)
        ws = sjd.attention_workspace(self.pool.pages, win, self.H)
        ws.fill_(0xFF)  # (NaN: nothing of it may be read before it is written)
        out = torch.full((self.T, self.H, self.hd), 3.0, dtype=torch.bfloat16, device="cuda")
        sjd.sjd_paged_attention(self.pool.pages, win, self.q.cuda() if q is None else q, out, ws, scale=self.scale,
                                anc=anc)
        return out

    def value(self, x):
        x = x.double().numpy()
        return quantise(x)[0] if self.cache == "e4m3" else x

    def seen(self, z, anc=None, left_out=()):
        r, n = self.seqs[z]
        p = np.arange(n + r)
        s = (p[None] - n) <= np.arange(r)[:, None]
        if anc is not None:
            first = self.seq[z][0]
            s = np.array([[x < n or (int(anc[first + i]) >> int(x - n)) & 1 for x in p] for i in range(r)], bool).reshape(r, n + r)
        for a, b in left_out:
            s[:, a:b] = False
        return s

    def check(self, out, anc=None, left_out=(), skip=()):
        got = out.double().cpu().numpy()
        named = np.zeros(self.T, bool)
        for z, (first, r, n, _) in enumerate(self.seq):
            if z in skip or r == 0:
                continue
            named[first:first + r] = True
            k, v = self.value(self.k[z]), self.value(self.v[z])
            seen = self.seen(z, anc, left_out)
            for h in range(self.H):
                qh = self.q[first:first + r, h].double().numpy()
                kh, vh = k[:, h // self.G], v[:, h // self.G]
                want, mag = attention(qh, kh, vh, self.scale, seen)
                tol = attention_tolerance(qh, kh[seen.any(0)], self.scale, mag, want, n + r)
                err = np.abs(got[first:first + r, h] - want)
                assert (err <= tol).all(), (z, h, float((err - tol).max()))
        assert (got[~named] == 3.0).all()  # rows that nobody names


SEQS = [
    [(1, 0)], [(1, 1239)], [(1, 31), (1, 32), (1, 95), (0, 40), (1, 0), (1, 700)],
    [(32, 333), (7, 64), (31, 0)], [(64, 5), (33, 1000)], [(130, 0), (1, 259)], [(300, 421)]]


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("hd,Hkv,G,plen", [(128, 2, 4, 64), (64, 3, 1, 32), (128, 1, 7, 128), (64, 2, 16, 1024)])
@pytest.mark.parametrize("seqs", SEQS, ids=[str(i) for i in range(len(SEQS))])
def test_causal(seqs, hd, Hkv, G, plen, cache):
    c = Case(seqs, plen, Hkv, G, hd, cache, scale=2.0)
    c.check(c.run())


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("hd,Hkv,G,plen", [(128, 2, 4, 64), (64, 3, 3, 32), (128, 1, 7, 128), (64, 2, 16, 1024)])
@pytest.mark.parametrize("seqs", [[(32, 333), (7, 64), (31, 0)], [(33, 1000), (64, 5), (0, 9)], [(130, 0), (1, 259)],
                                  [(300, 421)], [(65, 64), (64, 128)]], ids=[str(i) for i in range(5)])
def test_causal_many_slots(seqs, hd, Hkv, G, plen, cache):
    c = Case(seqs, plen, Hkv, G, hd, cache, scale=2.0, many=True)
    assert sjd.attention_workspace(c.pool.pages, c.windows(), c.H).numel() == 0
    c.check(c.run())


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("hd,Hkv,G", [(128, 1, 4), (64, 2, 2), (128, 2, 1)])
def test_tree(hd, Hkv, G, cache, many):
    """Ancestor masks: any of them, also of later rows, rows without any bit
    (and, with nothing cached, without any key: zeros), bits behind the window."""
    c = Case([(64, 700), (5, 0), (33, 31), (64, 0)], 32, Hkv, G, hd, cache, many=many)
    g = np.random.RandomState(3)
    anc = g.randint(0, 2 ** 32, c.T).astype(np.uint64) << np.uint64(32) | g.randint(0, 2 ** 32, c.T).astype(np.uint64)
    anc[c.seq[0][0]:c.seq[0][0] + 40] = [(1 << (i + 1)) - 1 for i in range(40)]
    anc[c.seq[0][0] + 50] = 0
    anc[c.seq[1][0] + 2] = 0
    anc[c.seq[1][0] + 3] = 1 << 60
    anc[c.seq[3][0] + 7] = 0
    out = c.run(torch.from_numpy(anc.astype(np.int64)).cuda())
    c.check(out, anc)
    assert not out[c.seq[1][0] + 2].any() and not out[c.seq[1][0] + 3].any() and not out[c.seq[3][0] + 7].any()


def test_long_cache_is_split():
    for seqs in ([(1, 20000)], [(3, 6000), (1, 17), (2, 0)]):
        c = Case(seqs, 256, 1, 4, 128, "e4m3", scale=3.0)
        assert sjd.attention_workspace(c.pool.pages, c.windows(), c.H).numel() > 0
        c.check(c.run())


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("scale", [-0.3, 0.0])
def test_negative_and_zero_scale(scale, many):
    c = Case([(40, 200), (3, 0)], 32, 2, 2, 64, "e4m3", many=many)
    c.scale = scale
    c.check(c.run())


def test_offsets_past_32_bits():
    """Pages behind the first 4 GiB of a pool, and rows behind element 2^31 of
    tensors with wide rows: the same bits as from small ones."""
    small = Case([(40, 130), (1, 300)], 64, 2, 2, 128, "e4m3")
    want = small.run()
    n = (1 << 32) // small.pool.size + small.pool.n_pages + 1
    pool = torch.empty(n * small.pool.size, dtype=torch.uint8, device="cuda")
    pages = sjd.Pages(pool, n, 64, 2, 128, "e4m3")
    shift = n - small.pool.n_pages
    assert shift * small.pool.size > 1 << 32
    table = torch.where(small.tt >= 0, small.tt + shift, small.tt)
    wide, T = 1 << 20, 2049 + small.T
    rows = torch.empty(T, wide, dtype=torch.bfloat16, device="cuda")
    q = rows[:, :small.H * 128].view(T, small.H, 128)
    q[2049:] = small.q.cuda()
    seq = small.st.clone()
    seq[:, 0] += 2049
    win = sjd.Windows(seq, table, T, 40, 300)
    # all keys and values through rows of the same wide tensor
    both = [r + m for r, m in small.seqs]
    k, v = (rows[:, a:a + 256].view(T, 2, 128) for a in (1024, 2048))
    at = T - sum(both)
    k[at:], v[at:] = torch.cat(small.k).cuda(), torch.cat(small.v).cuda()
    whole = torch.tensor([[at, both[0], 0, 0], [at + both[0], both[1], 0, 0]], dtype=torch.int32).cuda()
    every = sjd.Windows(whole, table, T, max(both), 0)
    sjd.sjd_kv_append(pages, every, k, v)
    out = rows[:, 4096:4096 + small.H * 128].view(T, small.H, 128)
    out[2049:] = 3.0
    ws = sjd.attention_workspace(pages, win, small.H)
    sjd.sjd_paged_attention(pages, win, q, out, ws, scale=small.scale)
    assert torch.equal(out[2049:], want)
    kb, vb = (rows[:, a:a + 256].view(T, 2, 128) for a in (8192, 9216))
    sjd.sjd_kv_read(pages, every, kb, vb)
    got = torch.cat([kb[at:], vb[at:]]).double().cpu().numpy()
    assert np.array_equal(got, np.concatenate([quantise(torch.cat(x).double().numpy())[0] for x in (small.k, small.v)]))
    pos = torch.arange(T, dtype=torch.int32, device="cuda")[:, None].contiguous()
    freq, axis = [1e4 ** (-i / 64) for i in range(64)], [0] * 64
    alone = q[2049:].contiguous()
    sjd.sjd_rope_axes(q, None, pos, freq, axis)
    sjd.sjd_rope_axes(alone, None, pos[2049:].contiguous(), freq, axis)
    assert torch.equal(q[2049:], alone)


def test_two_calls_at_once():
    """Two streams with a workspace each, and one stream twice with one."""
    c, d = (Case([(8, 900), (1, 2000)], 64, 2, 4, 128, "e4m3", seed=s) for s in (0, 5))
    want = [c.run(), d.run()]
    streams = [torch.cuda.Stream() for _ in range(2)]
    state = []
    for x in (c, d):
        win = x.windows()
        state.append((x, win, x.q.cuda(), torch.full_like(want[0], 3.0), sjd.attention_workspace(x.pool.pages, win, x.H)))
    torch.cuda.synchronize()
    for _ in range(20):
        for (x, win, q, out, ws), s in zip(state, streams):
            sjd.sjd_paged_attention(x.pool.pages, win, q, out, ws, scale=x.scale, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(s[3], w) for s, w in zip(state, want))
    for x, win, q, out, _ in state:
        out.fill_(3.0)
        sjd.sjd_paged_attention(x.pool.pages, win, q, out, state[0][4], scale=x.scale)
    assert all(torch.equal(s[3], w) for s, w in zip(state, want))


def test_bounds_larger_than_the_data():
    c = Case([(3, 77), (1, 200)], 64, 2, 4, 128, "e4m3")
    a, b = c.run(), c.run(slack=5000)
    c.check(a)
    c.check(b)


def test_strided_rows():
    """q inside the rows of a joint projection, out inside wider rows."""
    c = Case([(20, 100), (1, 3)], 32, 2, 2, 64, "bf16")
    wide = torch.randn(c.T, 7 * 64 + 8, device="cuda").to(torch.bfloat16)
    q = wide[:, 8:8 + c.H * 64].view(c.T, c.H, 64)
    q.copy_(c.q.cuda())
    win = c.windows()
    out = torch.full((c.T, c.H * 64 + 24), 3.0, dtype=torch.bfloat16, device="cuda")
    o = out[:, 16:16 + c.H * 64].view(c.T, c.H, 64)
    ws = sjd.attention_workspace(c.pool.pages, win, c.H)
    sjd.sjd_paged_attention(c.pool.pages, win, q, o, ws, scale=c.scale)
    c.check(o)
    assert bool((out[:, :16] == 3.0).all()) and bool((out[:, 16 + c.H * 64:] == 3.0).all())


@pytest.mark.parametrize("many", [False, True])
def test_pages_outside_the_pool_are_left_out(many):
    c = Case([(40, 130), (1, 300)], 64, 2, 4, 64, "e4m3", many=many)
    c.tt[:, 1] = 1 << 28
    c.check(c.run(), left_out=[(64, 128)])
    c.tt.fill_(-1)
    out = c.run()
    for first, r, _, _ in c.seq:
        assert not out[first:first + r].any()


@pytest.mark.parametrize("many", [False, True])
def test_wrong_sequences_are_left_out(many):
    c = Case([(40, 60), (3, 10), (2, 5), (1, 9)], 32, 1, 2, 64, "bf16", many=many)
    c.st[1] = torch.tensor([c.T - 2, 3, 10, 0])
    c.st[2] = torch.tensor([c.seq[2][0], 2, -1, 0])
    c.check(c.run(), skip=(1, 2))


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("rows,many", [(40, False), (200, False), (40, True), (200, True)])
def test_non_finite_values_reach_only_rows_that_attend(cache, rows, many):
    c = Case([(rows, 70)], 32, 1, 2, 64, cache, many=many)
    clean = c.run()
    bad = 23  # window row whose key and value are not finite
    p = 70 + bad
    for x in (float("nan"),) if cache == "e4m3" else (float("nan"), float("inf"), float("-inf")):
        keep_k, keep_v = c.k[0].clone(), c.v[0].clone()
        c.v[0][p, 0, 11] = x
        c.v[0][p, 0, 40] = x
        c.fill_pages()
        out = c.run()
        first = c.seq[0][0]
        assert torch.equal(out[first:first + bad], clean[first:first + bad])
        hit = out[first + bad:first + rows]
        want = torch.tensor(x).expand_as(hit[..., 11])
        assert torch.equal(torch.nan_to_num(hit[..., 11].float().cpu(), 1e9), torch.nan_to_num(want, 1e9))
        assert bool(torch.isfinite(hit[..., [0, 10, 12, 39, 41, 63]].float()).all())
        c.k[0], c.v[0] = keep_k.clone(), keep_v.clone()
        c.k[0][p, 0, 3] = x  # a key: whole rows, of those that attend
        c.fill_pages()
        out = c.run()
        assert torch.equal(out[first:first + bad], clean[first:first + bad])
        c.k[0] = keep_k
        c.fill_pages()
    # masked by a tree: nobody attends to it
    if rows <= 64:
        c.v[0][p] = float("nan")
        c.k[0][p] = float("nan")
        c.fill_pages()
        anc = np.array([((1 << 64) - 1) & ~(1 << bad)] * c.T, np.uint64)
        out = c.run(torch.from_numpy(anc.astype(np.int64)).cuda())
        assert bool(torch.isfinite(out.float()).all())


@pytest.mark.parametrize("many", [False, True])
def test_large_scores_and_lowest_values(many):
    """Scores of some thousands (one key takes all), and keys of bf16's lowest
    value, whose scores are huge or minus infinity."""
    c = Case([(33 if many else 3, 200)], 32, 1, 3 if many else 1, 64, "bf16", scale=200.0, many=many)
    c.check(c.run())
    c.q.abs_()
    c.k[0][5:60] = torch.finfo(torch.bfloat16).min
    c.fill_pages()
    out = c.run()
    c.check(out, left_out=[(5, 60)])


def test_runs_agree_and_follow_their_stream():
    """The same call twice, and on another stream behind its inputs' copies:
    the same bits."""
    c = Case([(32, 900), (1, 2000)], 64, 2, 4, 128, "e4m3")
    m = Case([(32, 900), (1, 2000)], 64, 2, 4, 128, "e4m3", many=True)
    assert torch.equal(m.run(), m.run())
    a = c.run()
    assert torch.equal(a, c.run())
    s = torch.cuda.Stream()
    q = torch.zeros_like(c.q, device="cuda")
    win = c.windows()
    ws, out = sjd.attention_workspace(c.pool.pages, win, c.H), torch.full_like(a, 3.0)
    torch.cuda.synchronize()
    src = c.q.pin_memory()
    with torch.cuda.stream(s):
        q.copy_(src, non_blocking=True)
        sjd.sjd_paged_attention(c.pool.pages, win, q, out, ws, scale=c.scale)
    s.synchronize()
    assert torch.equal(a, out)


def test_the_operators_together_and_captured():
    """A serving step: rows placed, written, attended to. Captured once and
    replayed while the sequences grow (their numbers live in device memory), each
    replay against the same calls made eagerly and against the plain form."""
    B, rows, Hkv, G, hd, plen = 3, 5, 2, 4, 128, 64
    H, T, steps = Hkv * G, 3 * 5, 6
    for cache in ("e4m3", "bf16"):
        table, n_pages = table_for([(rows * steps, 100 * z) for z in range(B)], plen)
        pools = [Pool(n_pages, plen, Hkv, hd, cache, fill=0) for _ in range(2)]
        tt = torch.from_numpy(table).cuda()
        seq = torch.tensor([[rows * z, rows, 100 * z, 0] for z in range(B)], dtype=torch.int32).cuda()
        g = torch.Generator().manual_seed(1)
        P = hd // 2
        freq, axis = [1e4 ** (-i / P) for i in range(P)], [i % 3 for i in range(P)]
        io = {}
        for e in range(2):
            io[e] = dict(qkv=torch.zeros(T, (H + 2 * Hkv) * hd, dtype=torch.bfloat16, device="cuda"),
                         pos=torch.zeros(T, 3, dtype=torch.int32, device="cuda"),
                         out=torch.zeros(T, H, hd, dtype=torch.bfloat16, device="cuda"),
                         win=sjd.Windows(seq.clone(), tt, T, rows, 100 * B + rows * steps))
            io[e]["ws"] = sjd.attention_workspace(pools[e].pages, io[e]["win"], H)
        past = []
        for z in range(B):  # what is cached already
            past.append([torch.randn(100 * z, Hkv, hd, generator=g).to(torch.bfloat16) for _ in range(2)])
        for pool in pools:
            m = [100 * z for z in range(B)]
            whole = torch.tensor([[sum(m[:z]), m[z], 0, 0] for z in range(B)], dtype=torch.int32).cuda()
            sjd.sjd_kv_append(pool.pages, sjd.Windows(whole, tt, sum(m), max(m), 0),
                              *(torch.cat([p[i] for p in past]).cuda() for i in range(2)))

        def step(e):
            x, c = io[e]["qkv"], io[e]
            q, k, v = (x[:, a * hd:b * hd].view(T, b - a, hd) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
            sjd.sjd_rope_axes(q, k, c["pos"], freq, axis)
            sjd.sjd_kv_append(pools[e].pages, c["win"], k, v)
            sjd.sjd_paged_attention(pools[e].pages, c["win"], q, c["out"], c["ws"], scale=hd ** -0.5)

        step(0)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(0)
        kept = [[p[0].double().numpy(), p[1].double().numpy()] for p in past]
        val = lambda x: quantise(x)[0] if cache == "e4m3" else x  # noqa: E731
        for i in range(steps):
            x = torch.randn(T, (H + 2 * Hkv) * hd, generator=g).to(torch.bfloat16)
            pos = torch.randint(0, 5000, (T, 3), generator=g, dtype=torch.int32)
            for e in range(2):
                io[e]["qkv"].copy_(x)
                io[e]["pos"].copy_(pos)
            graph.replay()
            step(1)
            torch.cuda.synchronize()
            assert torch.equal(io[0]["out"], io[1]["out"]) and torch.equal(io[0]["qkv"], io[1]["qkv"])
            assert torch.equal(pools[0].t, pools[1].t)
            rot = io[1]["qkv"].double().cpu().numpy()
            for z in range(B):
                r = slice(rows * z, rows * z + rows)
                q = rot[r, :H * hd].reshape(rows, H, hd)
                kv = [rot[r, (H + a * Hkv) * hd:(H + a * Hkv + Hkv) * hd].reshape(rows, Hkv, hd) for a in (0, 1)]
                kept[z] = [np.concatenate([o, n]) for o, n in zip(kept[z], kv)]
                n = len(kept[z][0])
                seen = np.arange(n)[None] - (n - rows) <= np.arange(rows)[:, None]
                for h in range(H):
                    k, v = (val(y[:, h // G]) for y in kept[z])
                    want, mag = attention(q[:, h], k, v, hd ** -0.5, seen)
                    tol = attention_tolerance(q[:, h], k, hd ** -0.5, mag, want, n)
                    assert (np.abs(io[1]["out"][r, h].double().cpu().numpy() - want) <= tol).all(), (i, z, h)
            for e in range(2):
                io[e]["win"].seq[:, 2] += rows


HOW = ["split", "whole", "shared"]  # keys split over workgroups, or not; keys shared by 128 slots


def stepped(cache, how, later, cached=8100):
    """Keys whose scores (log2 domain) are 0 in one half of every 256 positions and
    `later` in the other, which a wave that takes more than one tile meets after the
    first; one dim of a key differs from zero, so the scores are exact in 32 bits up to
    their scaling."""
    rows = 65 if how == "shared" else 3
    c = Case([(rows, cached)] + [(0, 0)] * (0 if how == "split" else 600), 64, 1, 1, 64, cache, many=how == "shared")
    assert (sjd.attention_workspace(c.pool.pages, c.windows(), 1).numel() > 0) == (how == "split")
    n = cached + rows
    c.k[0].zero_()
    c.k[0][:, 0, 0] = (torch.arange(n) // 128 % 2).to(torch.bfloat16)
    c.q.zero_()
    c.q[:, 0, 0] = later / (1.4426950408889634 * c.scale)
    return c, n


@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
def test_values_up_to_the_number_of_keys_below_the_largest_float(cache, how):
    """Values of up to 2^127 / (number of keys), most of them behind scores that are
    2^7.9 times as likely as the first ones'."""
    c, n = stepped(cache, how, 7.9)
    assert n <= 1 << 13
    c.v[0] = torch.sign(c.v[0].float()).to(torch.bfloat16) * 2.0 ** (127 - 13)
    c.v[0][:, 0, ::2] = 2.0 ** (127 - 13)  # (all of one sign: the largest sums)
    c.fill_pages()
    out = c.run()
    assert bool(torch.isfinite(out.float()).all())
    c.check(out)


@pytest.mark.parametrize("how", HOW)
def test_value_rows_with_the_largest_exponents(how):
    """Rows that the caller wrote with exponent byte 254: codes of at most 2^-8
    (values of 2^119 at most), zeros among them."""
    c, n = stepped("e4m3", how, 7.9, cached=180)
    assert n <= 1 << 8
    c.fill_pages()
    code = np.random.RandomState(2).randint(0, 3, (n, 64)).astype(np.uint8)  # 0, 2^-9, 2^-8
    raw = c.pool.t.cpu().numpy().reshape(c.pool.n_pages, -1)
    for p in range(n):
        page, i = raw[c.table[0][p // 64]], p % 64
        page[[64 * 64 + i // 32 * 32 * 64 + val_elem(i % 32, j, 64, True) for j in range(64)]] = code[p]
        page[2 * 64 * 64 + 64 + i] = 254
    c.pool.t.copy_(torch.from_numpy(raw.reshape(-1)))
    c.v[0] = torch.from_numpy(code * 2.0 ** (127 - 9)).to(torch.bfloat16)[:, None]
    c.pool.sync()
    assert np.array_equal(c.pool.decode(c.table[0][2], 3)[1], c.v[0][131].double().numpy())
    out = c.run()
    assert bool(torch.isfinite(out.float()).all())
    c.check(out)


@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("top", [2.0 ** 26, 3e9, 1e20, 1e35])
def test_huge_finite_scores(top, cache, how):
    """The largest score is far past what its own rounding leaves of a power of two:
    the keys that have it share the row, the others have nothing."""
    c, n = stepped(cache, how, 1.0, cached=1000)
    # products that are no floats times the scale, of either sign by the row
    c.q[:, 0, 0] = (torch.tensor(top).log2().div(2).exp2() * torch.tensor([1.37, -1.11, 1.93]).repeat(c.T)[:c.T]).to(torch.bfloat16)
    c.k[0][:, 0, 0] *= torch.tensor(top).sqrt().to(torch.bfloat16) * 1.21
    c.scale = 0.3
    c.fill_pages()
    out = c.run()
    assert bool(torch.isfinite(out.float()).all())
    got = out.double().cpu().numpy()
    k, v = c.value(c.k[0])[:, 0, 0], c.value(c.v[0])[:, 0]
    first = c.seq[0][0]
    for i in range(c.seqs[0][0]):
        s = float(c.q[first + i, 0, 0]) * k[:1000 + i + 1]
        share = v[:1000 + i + 1][s == s.max()]
        want, mag = share.mean(0), np.abs(share).mean(0)
        # (bf16 weights and output, a sum over the keys in 32 bits)
        assert (np.abs(got[first + i, 0] - want) <= (2.0 ** -8 + n * 2.0 ** -22) * mag + 2.0 ** -8 * np.abs(want)).all()


def test_few_rows_of_large_tensors():
    """Windows far apart in row tensors of a million rows: the bits, and the workspace, of
    the same ones in small tensors."""
    c = Case([(2, 5000), (3, 900)], 64, 1, 2, 64, "e4m3")
    want, T = c.run(), 1 << 20
    q = torch.zeros(T, 2, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 3.0)
    seq, at = c.st.clone(), [70000, T - 3]
    for z, (first, r, _, _) in enumerate(c.seq):
        q[at[z]:at[z] + r] = c.q[first:first + r].cuda()
        seq[z, 0] = at[z]
    win = sjd.Windows(seq, c.tt, T, 3, 5000)
    ws = sjd.attention_workspace(c.pool.pages, win, 2)
    assert 0 < ws.numel() <= sjd.attention_workspace(c.pool.pages, c.windows(), 2).numel()
    ws.fill_(0xFF)
    sjd.sjd_paged_attention(c.pool.pages, win, q, out, ws, scale=c.scale)
    for z, (first, r, _, _) in enumerate(c.seq):
        assert torch.equal(out[at[z]:at[z] + r], want[first:first + r])
        out[at[z]:at[z] + r] = 3.0
    assert bool((out == 3.0).all())


@pytest.mark.parametrize("how", HOW)
def test_scores_of_minus_infinity(how):
    """Keys with such scores have no weight; a row with no others gives zeros."""
    c, n = stepped("bf16", how, 1.0, cached=1000)
    c.k[0][300:, 0, 5], c.k[0][:40, 0, 5] = -float("inf"), -float("inf")
    c.q[:, 0, 5] = 0.5
    c.q[c.seq[0][0], 0, 5] = 2.0
    c.fill_pages()
    out, rows = c.run(), c.seqs[0][0]
    keep = c.k[0].clone()
    c.k[0][300:, 0, 5], c.k[0][:40, 0, 5] = 0, 0  # (the plain form leaves them out)
    c.check(out, left_out=[(0, 40), (300, n)])
    c.k[0] = keep
    c.k[0][:, 0, 5] = -float("inf")
    c.fill_pages()
    out = c.run()
    assert not out[c.seq[0][0]:c.seq[0][0] + rows].any()

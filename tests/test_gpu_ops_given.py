"""sjd_verify_given against the plain 64-bit form: whole numbers, equal."""
import numpy as np
import pytest
import torch

import paper_2603_18599_amd as sjd
from ops_util import given

pytestmark = pytest.mark.gpu


def call(p, q, draft, n, u, r, flags, vis_lo=0, stream=None):
    B, L = draft.shape
    d = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    out = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((B, 4), (B, L + 1), (B, L))]
    p = p if isinstance(p, torch.Tensor) else d(p)
    q = q if isinstance(q, torch.Tensor) else d(q)
    args = (p, q, d((draft + vis_lo).astype(np.int32)), d(n), d(u), d(r))
    sjd.sjd_verify_given(*args, *out, flags=flags, vis_lo=vis_lo)
    return [o.cpu().numpy() for o in out]


def inputs(B, L, V, seed, bonus, support=None, agree=1.0):
    g = np.random.RandomState(seed)
    rows = L + (1 if bonus else 0)
    z = g.randn(B, rows, V) * 2
    zq = z[:, :L] + agree * g.randn(B, L, V)
    if support and support < V:
        for x in (z, zq):
            x[x < np.sort(x, -1)[..., -support][..., None]] = -np.inf
    e = lambda x: np.exp(x - x.max(-1, keepdims=True))  # noqa: E731
    p, q = ((y / y.sum(-1, keepdims=True)).astype(np.float32) for y in (e(z), e(zq)))
    draft = (np.log(np.maximum(q, 1e-30)) + g.gumbel(size=q.shape)).argmax(-1).astype(np.int32)
    u, r = g.rand(B, L).astype(np.float32), g.rand(B, L + 1).astype(np.float32)
    return p, q, draft, g.randint(0, L + 1, B).astype(np.int32), np.minimum(u, 0.9999999), np.minimum(r, 0.9999999)


@pytest.mark.parametrize("ac", [False, True])
@pytest.mark.parametrize("bonus", [False, True])
@pytest.mark.parametrize("B,L,V,support", [(1, 1, 1, None), (3, 1, 7, None), (5, 8, 65, None), (9, 4, 1023, 5),
                                           (2, 33, 1025, None), (2, 64, 4096, 300), (3, 2, 65536, None), (2, 3, 70001, 9),
                                           (40, 64, 1024, 40), (2, 3, 4097, None), (2, 2, 12288, 2000),
                                           (2, 2, 12289, None), (1, 2, 262145, None)])
def test_given(B, L, V, support, bonus, ac):
    for certain in (False, True):
        p, q, draft, n, u, r = inputs(B, L, V, B * V + L, bonus, support)
        if certain:
            q = None
        flags = (sjd.SJD_AC if ac else 0) | (sjd.SJD_BONUS if bonus else 0)
        meta, tok, nxt = call(p, q, draft, n, u, r, flags, vis_lo=11)
        for b in range(B):
            m, t, x = given(p[b], None if q is None else q[b], draft[b], n[b], u[b], r[b], ac, bonus)
            up = lambda y: [e + 11 if e >= 0 else e for e in y]  # noqa: E731
            assert list(meta[b]) == m and list(tok[b]) == up(t) and list(nxt[b]) == up(x), b


def test_given_edges():
    """Uniforms of 0 and next to 1, q = 0, p = q, no mass at all, NaN and
    negative weights, drafts that are no tokens, counts out of range."""
    V, L = 200, 6
    p = np.full((1, L, V), 1.0 / 256, np.float32)
    q = p.copy()
    draft = np.array([[3, 4, 199, 0, 5, 6]], np.int32)
    top = np.float32(1 - 2.0 ** -24)
    u, r = np.full((1, L), 0.5, np.float32), np.array([[0.0, top, top, 0.0, 0.5, top, 0.5]], np.float32)
    q[0, 0, 3] = 0.0                      # q = 0 and p > 0: accepted whatever u
    u[0, 0] = top
    u[0, 1] = 0.0                         # u = 0: accepted where p > 0
    p[0, 2] = 0.0                         # no mass: -1
    p[0, 3, :] = 0.0
    p[0, 3, 150] = 0.25                   # q elsewhere: certain rejection, one token left
    p[0, 4, :] = np.nan
    p[0, 4, 7] = -1.0
    p[0, 4, 9:11] = 0.5                   # NaN and negative weights count as zero
    u[0, 4] = u[0, 5] = top               # p = q and u < 1: accepted at row 5
    for ac in (False, True):
        meta, tok, nxt = call(p, q, draft, None, u, r, sjd.SJD_AC if ac else 0)
        want = given(np.nan_to_num(p[0], nan=0.0), q[0], draft[0], L, u[0], r[0], ac, False)
        assert (list(meta[0]), list(tok[0]), list(nxt[0])) == tuple(want), ac
    # a residual without mass draws from p; drafts outside the row are rejected and draw from p
    p = np.full((2, 2, V), 1.0 / 256, np.float32)
    q = p * 2
    draft = np.array([[3, 4], [-1, V]], np.int32)
    u = np.full((2, 2), 0.9, np.float32)
    r = np.array([[0.25, 0.99, 0], [0.5, 0.0, 0]], np.float32)
    meta, tok, nxt = call(p, q, draft, None, u, r, sjd.SJD_AC)
    assert tok[0, 0] == 50 and nxt[0, 0] == 198 and tok[1, 0] == 100 and nxt[1, 0] == 0
    # counts out of range: left out
    meta, tok, nxt = call(p, q, draft, np.array([-1, 3], np.int32), u, r, sjd.SJD_AC)
    assert (meta == [-1, -1, 0, 0]).all() and (tok == -9).all() and (nxt == -9).all()
    meta, tok, nxt = call(p, q, draft, np.array([3, -5], np.int32), u, r, 0)
    assert (meta == [-1, -1, 0, 0]).all() and (tok == -9).all()
    # no drafts: the bonus alone, or nothing
    p3 = np.full((2, 3, V), 1.0 / 256, np.float32)
    meta, tok, nxt = call(p3, q, draft, np.zeros(2, np.int32), u, r, sjd.SJD_BONUS)
    assert meta[:, 0].tolist() == [1, 1] and tok[:, 0].tolist() == [50, 100]
    meta, tok, nxt = call(p, q, draft, np.zeros(2, np.int32), u, r, 0)
    assert meta[:, 0].tolist() == [0, 0] and (tok == -1).all()


@pytest.mark.parametrize("offset", [0, 1])
def test_given_strides(offset):
    """Rows and windows inside larger tensors, at any alignment; padding behind
    a row is not part of it."""
    B, L, V = 3, 5, 997
    p, q, draft, n, u, r = inputs(B, L, V, 5, True)
    wide = []
    for x in (p, q):
        t = torch.full((B, 9, V + 15), 3.0e38, device="cuda")
        t[:, 1:1 + x.shape[1], offset:offset + V] = torch.from_numpy(x).cuda()
        wide.append(t[:, 1:1 + x.shape[1], offset:offset + V])
    flags = sjd.SJD_AC | sjd.SJD_BONUS
    got = call(*wide, draft, n, u, r, flags)
    for a, b in zip(got, call(p, q, draft, n, u, r, flags)):
        assert np.array_equal(a, b)


def test_given_law():
    """Committed first tokens follow p whatever q is (the rejection sampling
    lemma): chi-square over 20000 windows, 7 degrees of freedom, 1e-4 tail."""
    B, V = 20000, 8
    g = np.random.RandomState(2)
    p1, q1 = (x / x.sum() for x in (g.rand(V), g.rand(V)))
    p, q = (np.tile(x.astype(np.float32), (B, 1, 1)) for x in (p1, q1))
    draft = g.choice(V, (B, 1), p=q1).astype(np.int32)
    u, r = (np.minimum(g.rand(B, k).astype(np.float32), 0.9999999) for k in (1, 2))
    _, tok, _ = call(p, q, draft, None, u, r, 0)
    seen = np.bincount(tok[:, 0], minlength=V)
    assert ((seen - B * p1) ** 2 / (B * p1)).sum() < 29.9


def test_given_largest_batch():
    """65535 windows of 64 drafts and a bonus row, 16 waves to a row: more threads
    than 32 bits count. All windows share their probabilities."""
    B, L, V = 65535, 64, 12289
    p, _, _, _, _, _ = inputs(1, L, V, 8, True)
    g = np.random.RandomState(9)
    draft, n = g.randint(0, V, (B, L)).astype(np.int32), g.randint(0, L + 1, B).astype(np.int32)
    u, r = (np.minimum(g.rand(B, k).astype(np.float32), 0.9999999) for k in (L, L + 1))
    u[:, ::3] = 0.0  # (accepted)
    meta, tok, nxt = call(torch.from_numpy(p).cuda().expand(B, L + 1, V), None, draft, n, u, r, sjd.SJD_AC | sjd.SJD_BONUS)
    for b in (0, 1, 40000, 64526, 64527, 64528, 65533, 65534):
        want = given(p[0], None, draft[b], n[b], u[b], r[b], True, True)
        assert (list(meta[b]), list(tok[b]), list(nxt[b])) == tuple(want), b

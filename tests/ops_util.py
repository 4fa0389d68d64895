"""Plain 64-bit forms of the standalone operators, for their tests: numpy, one
sequence, row and head at a time, from the definitions in include/sjd.h."""
import numpy as np
import torch


def key_elem(i, j, hd, e4m3):
    """Element of position i and dim j in a key tile."""
    h2 = hd // 2
    sw = (i & ~12) | ((i & 4) << 1) | ((i & 8) >> 1)
    lane, t = sw + 32 * (j // h2), j % h2 // 8
    return (64 * (t // 2) + lane) * 16 + 8 * (t % 2) + j % 8 if e4m3 else (64 * t + lane) * 8 + j % 8


def val_elem(i, j, hd, e4m3):
    lane = j % 32 + 32 * (i // 8 % 2)
    return ((64 * (j // 32) + lane) * 16 + 8 * (i // 16) + i % 8 if e4m3
            else ((j // 32 * 2 + i // 16) * 64 + lane) * 8 + i % 8)


def e4m3_values():
    """The value of each code (OCP e4m3: 1 sign, 4 exponent bits biased by 7, 3
    of mantissa, no infinities, all ones NaN)."""
    v = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = np.nan if e == 15 and m == 7 else m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = -x if c & 128 else x
    return v


E4M3 = e4m3_values()


def quantise(x):
    """(values, exponent bytes) of rows [..., hd]: the nearest code, ties to
    the even one, of x / 2^(E - 127)."""
    x = np.asarray(x, np.float64)
    fin = np.where(np.isfinite(x), np.abs(x), 0.0)
    amax = fin.max(-1)
    E = np.full(amax.shape, 127)
    for idx in np.ndindex(amax.shape):
        if amax[idx] > 0:
            e = 27
            while e < 246 and amax[idx] > 448 * 2.0 ** (e - 127):
                e += 1
            E[idx] = e
    s = 2.0 ** (E - 127.0)[..., None]
    y = np.clip(x / s, -448, 448)
    size = np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -40))), -6)
    step = 2.0 ** (np.where(np.isnan(size), 0, size) - 3)
    return np.round(y / step) * step * s, E


class Pool:
    """A pool of pages filled with a byte, its description, and the plain form
    of what its positions hold."""

    def __init__(self, n_pages, page_len, Hkv, hd, dtype, fill=0xFF):
        import paper_2603_18599_amd as sjd
        self.n_pages, self.plen, self.Hkv, self.hd, self.e4 = n_pages, page_len, Hkv, hd, dtype == "e4m3"
        self.size = sjd.page_bytes(page_len, Hkv, hd, dtype)
        self.t = torch.full((n_pages * self.size,), fill, dtype=torch.uint8, device="cuda")
        self.pages = sjd.Pages(self.t, n_pages, page_len, Hkv, hd, dtype)

    def decode(self, page, inside):
        """k, v [Hkv, hd] of one position, from the bytes (call sync first)."""
        raw = self.raw[page]
        es, P, hd = (1 if self.e4 else 2), self.plen, self.hd
        out = []
        for kv, elem in ((0, key_elem), (1, val_elem)):
            rows = []
            for h in range(self.Hkv):
                at = (2 * h + kv) * P * hd + inside // 32 * 32 * hd
                idx = np.array([at + elem(inside % 32, j, hd, self.e4) for j in range(hd)])
                if self.e4:
                    E = int(raw[2 * self.Hkv * P * hd + (2 * h + kv) * P + inside])
                    rows.append(E4M3[raw[idx]] * 2.0 ** (E - 127))
                else:
                    u = raw.view(np.uint16)[idx].astype(np.uint32) << 16
                    rows.append(u.view(np.float32).astype(np.float64))
            out.append(np.stack(rows))
        return out

    def sync(self):
        self.raw = self.t.cpu().numpy().reshape(self.n_pages, self.size)


def table_for(seqs, page_len, seed=0, spare=2):
    """Pages of (rows, cached) sequences in a scattered order: table [B, width]
    (-1 behind the last) and how many pages the pool needs."""
    need = [-(-(r + n) // page_len) for r, n in seqs]
    order = np.random.RandomState(seed).permutation(sum(need) + spare)
    table = np.full((len(seqs), max(max(need), 1)), -1, np.int32)
    at = 0
    for z, k in enumerate(need):
        table[z, :k] = order[at:at + k]
        at += k
    return table, sum(need) + spare


def attention(q, k, v, scale, seen):
    """One head: q [r, hd], k, v [n, hd], seen [r, n] -> out [r, hd] and the
    weighted mean of |v| (for tolerances)."""
    s = q @ k.T * scale
    out, mag = np.zeros((len(q), v.shape[1])), np.zeros((len(q), v.shape[1]))
    for i in range(len(q)):
        m = seen[i]
        if not m.any():
            continue
        w = np.exp(s[i, m] - s[i, m].max())
        w /= w.sum()
        out[i], mag[i] = w @ v[m], w @ np.abs(v[m])
    return out, mag


def attention_tolerance(q, k, scale, mag, out, keys):
    """Bound of the difference that the operator's roundings allow:
      - probabilities enter the value product as bf16 (half a step, 2^-8 of
        each), the output is rounded once more (2^-8);
      - scores are sums of head_dim products in 32 bits and a few roundings
        after, an error d of a score moves its weight by e^d - 1 in the
        numerator and in the denominator;
      - sums over the keys in 32 bits, with a rescaling for each tile.
    (Sums are given 2^-23 a term: the matrix unit need not round to nearest.)"""
    size = scale * (np.abs(q) @ np.abs(k).T).max(-1, initial=0.0)
    d = (q.shape[1] + 8) * 2.0 ** -23 * size
    return (2.0 ** -8 + 2 * np.expm1(d) + 2 * keys * 2.0 ** -23)[:, None] * mag + 2.0 ** -8 * np.abs(out) + 1e-30


def given(p, q, draft, n, u, r, ac, bonus):
    """One window of sjd_verify_given (entries as tokens): meta, tok, next."""
    L = len(draft)

    def draw(w, x):
        w = np.where(w > 0, w, 0.0)
        cum = np.cumsum(w)
        if not cum[-1] > 0:
            return None
        above = np.nonzero((cum > float(x) * cum[-1]) & (w > 0))[0]
        return int(above[0]) if len(above) else int(np.nonzero(w)[0][-1])

    rows, first = [], None
    for j in range(n):
        x = int(draft[j])
        inside = 0 <= x < p.shape[1]
        qx = 1.0 if q is None else float(q[j, x]) if inside else 0.0
        if inside and float(u[j]) * qx < float(p[j, x]):
            rows.append(x)
            continue
        first = j if first is None else first
        t = None
        pj = p[j].astype(np.float64)
        if inside:
            w = np.where(np.arange(len(pj)) == x, 0.0, pj) if q is None else pj - q[j].astype(np.float64)
            t = draw(w, r[j])
        if t is None:
            t = draw(pj, r[j])
        rows.append(-1 if t is None else t)
    if bonus:
        t = draw(p[n].astype(np.float64), r[n])
        rows.append(-1 if t is None else t)
    n_c = len(rows) if first is None else first + 1
    nxt = rows[n_c:] if ac else []
    return ([n_c, -1 if first is None else first, n if first is None else first, len(nxt)],
            rows[:n_c] + [-1] * (L + 1 - n_c), nxt + [-1] * (L - len(nxt)))

"""The operators whose speed is measured, in their plain form and through the
library's entry points: what a program that serves image windows with its own
model asks of them around its projections.

Four kinds of case:
  rope    rotary positions with several axes on the rows of q and k
          (sjd_rope_axes);
  cache   new key and value rows into the pages of a cache, in 8 bits or as
          bf16, and every cached row of those sequences read back
          (sjd_kv_append, sjd_kv_read);
  attend  attention of the new rows (a token, a tree window, a prompt) over
          the pages (sjd_paged_attention);
  given   verification of drafted tokens against the target's probabilities
          from given uniforms (sjd_verify_given).

Head counts, head sizes, window lengths, cache lengths and vocabulary sizes
are those of the repository's decoder configurations or lie between them.
"""
import math

import torch

own = False

_PAGE = 64


def listed():
    return [
        # one row of a decoding step, placed on time, height and width: a launch
        dict(name="rope_token", kind="rope", T=1, H=32, Hkv=8, hd=128, axes=3, pairs=64, dtype="bf16", inverse=False),
        # a window of one image on the mid shape, fp32 rows, two axes, part of each head rotated
        dict(name="rope_window", kind="rope", T=32, H=16, Hkv=16, hd=64, axes=2, pairs=24, dtype="fp32", inverse=False),
        # an image of 90 x 91 tokens given as context: memory traffic
        dict(name="rope_image", kind="rope", T=8190, H=32, Hkv=8, hd=128, axes=3, pairs=64, dtype="bf16",
             inverse=False),
        # four requests decode a token each over short caches: latency
        dict(name="cache_tokens", kind="cache", B=4, rows=1, cached=77, Hkv=8, hd=128, cache="e4m3", dtype="bf16"),
        # ragged windows of fp32 rows (a projection's output) into bf16 pages
        dict(name="cache_windows", kind="cache", B=8, rows=48, cached=1239, Hkv=16, hd=64, cache="bf16", dtype="fp32"),
        # prompts into 8 bits
        dict(name="cache_prompts", kind="cache", B=4, rows=4096, cached=1500, Hkv=32, hd=128, cache="e4m3",
             dtype="bf16"),
        # one token half-way through an image (7B heads): latency and few rows
        dict(name="attend_token", kind="attend", B=1, rows=1, cached=1239, H=32, Hkv=32, hd=128, cache="e4m3",
             tree=False),
        # many requests decode a token each, their caches ragged: memory traffic
        dict(name="attend_tokens", kind="attend", B=64, rows=1, cached=8190, H=32, Hkv=8, hd=128, cache="e4m3",
             tree=False),
        # tree windows of the speculative step (8B heads)
        dict(name="attend_windows", kind="attend", B=4, rows=32, cached=4172, H=32, Hkv=8, hd=128, cache="e4m3",
             tree=True),
        # a long prompt's chunk over what is cached of it: matrix rate
        dict(name="attend_prompt", kind="attend", B=1, rows=4096, cached=4172, H=32, Hkv=8, hd=128, cache="bf16",
             tree=False),
        # one window of 32 drafts: latency
        dict(name="given_window", kind="given", B=1, L=32, V=16384, top_k=2000, ac=True, bonus=False, delta=False),
        # a serving batch, the first rejection ends a window
        dict(name="given_batch", kind="given", B=256, L=8, V=65536, top_k=0, ac=False, bonus=True, delta=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "cache", "attend", "attend", "given"])
    if kind == "rope":
        hd = rng.choice([64, 64, 80, 128, 128, 256])
        Hkv = rng.choice([1, 4, 8, 16])
        return dict(kind="rope", T=_log_int(rng, 1, 8190 * 128 // hd // 2), H=Hkv * rng.choice([1, 2, 4][:2 if Hkv > 8 else 3]),
                    Hkv=Hkv, hd=hd, axes=rng.randint(1, 4), pairs=rng.choice([hd // 2, hd // 2, hd // 4, 5]),
                    dtype=rng.choice(["bf16", "fp32"]), inverse=rng.random() < 0.25)
    if kind == "cache":
        B = _log_int(rng, 1, 32)
        return dict(kind="cache", B=B, rows=_log_int(rng, 1, 4096 * 4 // B // 2), cached=rng.randint(0, 1000 if B > 4 else 4000),
                    Hkv=rng.choice([1, 2, 8, 16]), hd=rng.choice([64, 128]), cache=rng.choice(["e4m3", "bf16"]),
                    dtype=rng.choice(["bf16", "fp32"]))
    if kind == "attend":
        tree = rng.random() < 0.4
        B = _log_int(rng, 1, 64)
        rows = rng.randint(1, 64) if tree else _log_int(rng, 1, max(1, 4096 // B))
        Hkv = rng.choice([1, 2, 8, 16])
        most = 8190 if B <= 16 and B * rows <= 2048 else 4096
        return dict(kind="attend", B=B, rows=rows, cached=rng.choice([0] + 3 * [_log_int(rng, 1, most)]),
                    H=Hkv * rng.choice([1, 2, 4, 7] if Hkv <= 4 else [1, 2]), Hkv=Hkv, hd=rng.choice([64, 128]),
                    cache=rng.choice(["e4m3", "bf16"]), tree=tree)
    V, L = _log_int(rng, 64, 65536), _log_int(rng, 1, 32)
    return dict(kind="given", B=_log_int(rng, 1, min(1024, 256 * 8 * 65536 // (V * L))), L=L, V=V,
                top_k=rng.choice([0, 0, max(1, V // 8)]), ac=rng.random() < 0.5, bonus=rng.random() < 0.5,
                delta=rng.random() < 0.2)


# ---- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _ragged(total, count, seed, least):
    """count lengths of up to total, the first of them total itself."""
    g = torch.Generator().manual_seed(int(seed) * 7919 + 13)
    v = [total]
    for _ in range(count - 1):
        v.append(max(least, int(total * (0.25 + 0.75 * float(torch.rand(1, generator=g))))))
    return v


def _lengths(case):
    """Window rows and cached rows of each sequence (the same for every seed:
    the work of a case does not depend on it)."""
    return _ragged(case["rows"], case["B"], 1, 1), _ragged(case["cached"], case["B"], 2, 0)


def _pages_for(total):
    return -(-total // _PAGE)


_SWAP = [(i & ~12) | ((i & 4) << 1) | ((i & 8) >> 1) for i in range(32)]


def _page_bytes(Hkv, hd, cache):
    e = 1 if cache == "e4m3" else 2
    return -(-(2 * Hkv * _PAGE * hd * e + (2 * Hkv * _PAGE if e == 1 else 0)) // 256) * 256


def _places(page, inside, Hkv, hd, cache):
    """Where a page's parts hold position `inside` (of the page) of sequence
    pages `page`: element offsets of keys and of values [rows, Hkv, hd] and
    byte offsets of the two exponents [rows, Hkv], from the pool's start."""
    dev = page.device
    e = 1 if cache == "e4m3" else 2
    h = torch.arange(Hkv, device=dev)[None, :]
    j = torch.arange(hd, device=dev)[None, None, :]
    base = (page * (_page_bytes(Hkv, hd, cache) // e))[:, None] + h * (2 * _PAGE * hd)
    i = (inside % 32)[:, None, None]
    tile = (base + (inside // 32 * 32 * hd)[:, None])[:, :, None]
    lane = torch.tensor(_SWAP, device=dev)[i] + 32 * (j // (hd // 2))
    t = j % (hd // 2) // 8
    vl = j % 32 + 32 * (i // 8 % 2)
    if e == 1:
        k = ((t // 2) * 64 + lane) * 16 + (t % 2) * 8 + j % 8
        v = (j // 32 * 64 + vl) * 16 + i // 16 * 8 + i % 8
    else:
        k = (t * 64 + lane) * 8 + j % 8
        v = (j // 32 * 2 + i // 16) * 512 + vl * 8 + i % 8
    scales = (page * _page_bytes(Hkv, hd, cache))[:, None] + 2 * Hkv * _PAGE * hd + h * (2 * _PAGE) + inside[:, None]
    return tile + k, tile + _PAGE * hd + v, scales, scales + _PAGE


def _quantise(x):
    """Codes and biased exponents of rows [..., hd] (fp32)."""
    amax = x.abs().amax(-1)
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(-100, 119)
    e = torch.where(amax == 0, torch.zeros_like(e), e)
    code = torch.ldexp(x, -e[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    return code.view(torch.uint8), (e + 127).to(torch.uint8)


def _store(pool, k, v, page, inside, Hkv, hd, cache):
    """Rows k, v [rows, Hkv, hd] into the pool (its bytes)."""
    pk, pv, sk, sv = _places(page, inside, Hkv, hd, cache)
    if cache == "e4m3":
        (ck, ek), (cv, ev) = _quantise(k.float()), _quantise(v.float())
        pool[pk], pool[pv], pool[sk], pool[sv] = ck, cv, ek, ev
    else:
        flat = pool.view(torch.bfloat16)
        flat[pk], flat[pv] = k.to(torch.bfloat16), v.to(torch.bfloat16)


def _load(pool, page, inside, Hkv, hd, cache):
    """Rows of keys and of values [rows, Hkv, hd] as fp32."""
    pk, pv, sk, sv = _places(page, inside, Hkv, hd, cache)
    if cache != "e4m3":
        flat = pool.view(torch.bfloat16)
        return flat[pk].float(), flat[pv].float()
    k, v = pool[pk].view(torch.float8_e4m3fn).float(), pool[pv].view(torch.float8_e4m3fn).float()
    return torch.ldexp(k, (pool[sk].int() - 127)[..., None]), torch.ldexp(v, (pool[sv].int() - 127)[..., None])


_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _prepare_rope(c, g):
    T, dt = c["T"], _TYPES[c["dtype"]]
    q = torch.randn(T, c["H"], c["hd"], generator=g, device="cuda").to(dt)
    k = torch.randn(T, c["Hkv"], c["hd"], generator=g, device="cuda").to(dt)
    # an image of rows of 91 behind a prompt, many frames on
    t = torch.arange(T, device="cuda") + int(torch.randint(0, 64, (1,), generator=g, device="cuda"))
    first = int(torch.randint(0, 60000, (1,), generator=g, device="cuda"))
    pos = torch.stack([first + t // 8190, t // 91 % 90, t % 91, first + t][:c["axes"]], 1).to(torch.int32)
    # frequencies in order, sections of pairs per axis
    freq = [10000.0 ** (-i / c["pairs"]) for i in range(c["pairs"])]
    axis = [min(c["axes"] - 1, i * c["axes"] // c["pairs"]) for i in range(c["pairs"])]
    return dict(q=q, k=k, pos=pos, freq=freq, axis=axis, out_q=torch.zeros_like(q), out_k=torch.zeros_like(k))


def _sequences(c, seed):
    """Sequence descriptions, pages in a scattered order, and where each
    cached position is."""
    rows, cached = _lengths(c)
    need = [_pages_for(r + n) for r, n in zip(rows, cached)]
    width, total = max(max(need), 1), sum(need) + 3
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(seed) + 5))
    table = torch.full((c["B"], width), -1, dtype=torch.int64)
    at = first = 0
    seq = []
    for b in range(c["B"]):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        seq.append([first, rows[b], cached[b], 0])
        first += rows[b]
    return rows, cached, table, seq, total


def _positions(table, rows, cached, new):
    """Page and place inside it of every position of every sequence: the
    cached ones, or the window's."""
    pages, inside = [], []
    for b, (r, n) in enumerate(zip(rows, cached)):
        p = torch.arange(n, n + r) if new else torch.arange(n)
        pages.append(table[b][p // _PAGE])
        inside.append(p % _PAGE)
    return torch.cat(pages).cuda(), torch.cat(inside).cuda()


def _fill(pool, table, rows, cached, c, g, new_too):
    """Cached rows into the pool, in pieces."""
    for new in ((False, True) if new_too else (False,)):
        page, inside = _positions(table, rows, cached, new)
        for a in range(0, len(page), 16384):
            p, i = page[a:a + 16384], inside[a:a + 16384]
            k, v = (torch.randn(len(p), c["Hkv"], c["hd"], generator=g, device="cuda") for _ in range(2))
            _store(pool, k.to(torch.bfloat16), v.to(torch.bfloat16), p, i, c["Hkv"], c["hd"], c["cache"])


def _prepare_paged(c, seed, g):
    rows, cached, table, seq, total = _sequences(c, seed)
    T, Hkv, hd = sum(rows), c["Hkv"], c["hd"]
    pool = torch.zeros(total * _page_bytes(Hkv, hd, c["cache"]), dtype=torch.uint8, device="cuda")
    _fill(pool, table, rows, cached, c, g, c["kind"] == "attend")
    s = dict(pool=pool, total=total, table=table.to(torch.int32).cuda(), seq=torch.tensor(seq, dtype=torch.int32).cuda(),
             T=T, max_rows=max(rows), max_cached=max(cached))
    if c["kind"] == "cache":
        dt = _TYPES[c["dtype"]]
        s["k"], s["v"] = (torch.randn(T, Hkv, hd, generator=g, device="cuda").to(dt) for _ in range(2))
        # every row of every sequence, one sequence behind the other
        both = [r + n for r, n in zip(rows, cached)]
        first = [sum(both[:b]) for b in range(c["B"])]
        s["all"] = torch.tensor([[f, m, 0, 0] for f, m in zip(first, both)], dtype=torch.int32).cuda()
        s["total_rows"], s["max_both"] = sum(both), max(both)
        s["out_k"], s["out_v"] = (torch.zeros(sum(both), Hkv, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return s
    s["q"] = (torch.randn(T, c["H"], hd, generator=g, device="cuda") * 1.5).to(torch.bfloat16)
    s["out"] = torch.zeros(T, c["H"], hd, dtype=torch.bfloat16, device="cuda")
    s["scale"] = hd ** -0.5
    if c["tree"]:
        anc = []
        w = torch.Generator().manual_seed(int(seed) + 9)
        for r in rows:  # a spine, and siblings that branch off its start
            spine = r - min(9, r // 3)
            for i in range(r):
                if i < spine:
                    anc.append((1 << (i + 1)) - 1)
                else:
                    depth = int(torch.randint(0, max(1, min(4, spine)), (1,), generator=w))
                    anc.append((1 << depth) - 1 | 1 << i)
        s["anc"] = torch.tensor([a - (1 << 64) if a >> 63 else a for a in anc], dtype=torch.int64).cuda()
    else:
        s["anc"] = None
    return s


def _prepare_given(c, g):
    B, L, V = c["B"], c["L"], c["V"]
    n = torch.tensor(_ragged(L, B, 3, 0), dtype=torch.int32).cuda()
    logits = torch.randn(B, L + 1, V, generator=g, device="cuda") * 2
    if not c["bonus"]:
        logits = logits[:, :L].contiguous()
    draft_logits = logits[:, :L] + 0.5 * torch.randn(B, L, V, generator=g, device="cuda")
    for x in (logits, draft_logits):
        if c["top_k"]:
            x.masked_fill_(x < x.topk(c["top_k"], dim=-1).values[..., -1:], -math.inf)
    p, q = torch.softmax(logits, -1), torch.softmax(draft_logits, -1)
    race = -torch.log1p(-torch.rand(B, L, V, generator=g, device="cuda")) / q
    draft = race.argmin(-1).to(torch.int32)
    u = torch.rand(B, L, generator=g, device="cuda")
    r = torch.rand(B, L + 1, generator=g, device="cuda")
    return dict(p=p, q=None if c["delta"] else q, draft=draft, n=n, u=u, r=r, ac=c["ac"], bonus=c["bonus"],
                meta=torch.zeros(B, 4, dtype=torch.int32, device="cuda"),
                tok=torch.zeros(B, L + 1, dtype=torch.int32, device="cuda"),
                next=torch.zeros(B, L, dtype=torch.int32, device="cuda"))


def prepare(case, seed):
    g = _gen(seed)
    if case["kind"] == "rope":
        s = _prepare_rope(case, g)
    elif case["kind"] == "given":
        s = _prepare_given(case, g)
    else:
        s = _prepare_paged(case, seed, g)
    s["case"] = case
    return s


# ---- plain forms

def _plain_rope(s):
    c, P = s["case"], len(s["freq"])
    freq = torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
    axis = torch.tensor(s["axis"], device="cuda")
    phi = s["pos"][:, axis].double() * freq
    co, si = phi.cos().float()[:, None], phi.sin().float()[:, None]
    if c["inverse"]:
        si = -si

    def turn(x):
        x = x.float()
        a, b = x[..., :P], x[..., P:2 * P]
        return torch.cat([a * co - b * si, b * co + a * si, x[..., 2 * P:]], -1).to(s["q"].dtype)

    return {"q": turn(s["q"]), "k": turn(s["k"])}


def _cover(seq, B):
    """Sequence and place in it of rows 0 .. of the sequences `seq`, which
    lie one behind the other."""
    rows = seq[:, 1].long()
    b = torch.repeat_interleave(torch.arange(B, device="cuda"), rows)
    return b, torch.arange(len(b), device="cuda") - seq[:, 0].long()[b]


def _plain_cache(s):
    c, B = s["case"], s["case"]["B"]
    b, i = _cover(s["seq"], B)
    p = s["seq"][:, 2].long()[b] + i
    _store(s["pool"], s["k"], s["v"], s["table"].long()[b, p // _PAGE], p % _PAGE, c["Hkv"], c["hd"], c["cache"])
    b, p = _cover(s["all"], B)
    k, v = _load(s["pool"], s["table"].long()[b, p // _PAGE], p % _PAGE, c["Hkv"], c["hd"], c["cache"])
    return {"k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def _plain_attend(s):
    c, B = s["case"], s["case"]["B"]
    Hkv, hd, G = c["Hkv"], c["hd"], c["H"] // c["Hkv"]
    R, N = s["max_rows"], s["max_rows"] + s["max_cached"]
    rows, n = s["seq"][:, 1].long(), s["seq"][:, 2].long()
    p = torch.arange(N, device="cuda")
    page = s["table"].long()[:, (p // _PAGE).clamp(max=s["table"].shape[1] - 1)].clamp(min=0)
    k, v = _load(s["pool"], page.reshape(-1), (p % _PAGE).repeat(B), Hkv, hd, c["cache"])
    k, v = (x.view(B, N, Hkv, hd).transpose(1, 2) for x in (k, v))
    b, i = _cover(s["seq"], B)
    q = torch.zeros(B, R, Hkv, G, hd, device="cuda")
    q[b, i] = s["q"].float().view(-1, Hkv, G, hd)
    q = q.permute(0, 2, 1, 3, 4).reshape(B, Hkv, R * G, hd)
    new = p[None, None, :] - n[:, None, None]  # the window row that a position holds
    row = torch.arange(R, device="cuda")[None, :, None]
    if s["anc"] is None:
        seen = new <= row
    else:
        anc = torch.zeros(B, R, dtype=torch.int64, device="cuda")
        anc[b, i] = s["anc"]
        seen = (new < 0) | ((anc[:, :, None] >> new.clamp(0, 63)) & 1 > 0)
    seen = seen & (p[None, None, :] < (n + rows)[:, None, None]) & (row < rows[:, None, None])
    seen = seen[:, None, :, None, :].expand(B, 1, R, G, N).reshape(B, 1, R * G, N)
    score = (torch.matmul(q, k.transpose(-1, -2).contiguous()) * s["scale"]).masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score, v.masked_fill(~(p < (n + rows)[:, None])[:, None, :, None], 0.0).contiguous())
    out = out / torch.where(total == 0, torch.ones_like(total), total)
    out = out.view(B, Hkv, R, G, hd).transpose(1, 2).reshape(B, R, c["H"], hd)
    return {"out": out[b, i].to(torch.bfloat16)}


def _pick(w, r):
    """Least x with cum(x) > r * total of the rows w (64 bits)."""
    cum = w.cumsum(-1)
    x = (cum <= r.double()[..., None] * cum[..., -1:]).sum(-1)
    last = w.shape[-1] - 1 - (w > 0).flip(-1).int().argmax(-1)
    return torch.minimum(x, last)


def _plain_given(s):
    c, p, q, draft = s["case"], s["p"], s["q"], s["draft"].long()
    B, L, n = c["B"], c["L"], s["n"].long()
    rows = torch.arange(L, device="cuda")
    at = p[:, :L].gather(-1, draft[..., None])[..., 0].double()
    under = s["u"].double() if q is None else s["u"].double() * q.gather(-1, draft[..., None])[..., 0].double()
    ok = (under < at) & (rows < n[:, None])
    bad = ~ok & (rows < n[:, None])
    first = torch.where(bad.any(1), bad.int().argmax(1), n)
    # what each row that is needed draws from: rejected ones the residual, row n (with a bonus) p itself
    if c["ac"]:
        b, j = torch.arange(B, device="cuda").repeat_interleave(L + 1), torch.arange(L + 1, device="cuda").repeat(B)
        need = (j < n[b]) & ~ok[b, j.clamp(max=L - 1)]
    else:
        b, j = torch.arange(B, device="cuda"), first
        need = first < n
    need = need | ((j == n[b]) & c["bonus"])
    b, j = b[need], j[need]
    res = j < n[b]
    w = p[b, j].double()
    jq = j.clamp(max=L - 1)
    if q is None:
        less = w.scatter(-1, draft[b, jq][:, None], 0.0)
    else:
        less = (w - q[b, jq].double()).clamp(min=0)
    w = torch.where((res & (less > 0).any(-1))[:, None], less, w)
    out = torch.zeros(B, L + 1, dtype=torch.int64, device="cuda")
    out[:, :L] = draft
    out[b, j] = _pick(w, s["r"][b, j])
    some = first < n
    n_c = torch.where(some, first + 1, n + (1 if c["bonus"] else 0))
    carried = torch.where(some, n - first - 1 + (1 if c["bonus"] else 0), 0) * (1 if c["ac"] else 0)
    k = torch.arange(L + 1, device="cuda")
    tok = torch.where(k < n_c[:, None], out, -1)
    nxt = torch.where(rows < carried[:, None], out.gather(1, (n_c[:, None] + rows).clamp(max=L)), -1)
    meta = torch.stack([n_c, torch.where(some, first, -1), first, carried], 1)
    return {"meta": meta.int(), "tok": tok.int(), "next": nxt.int()}


def run(state):
    if own:
        return _run_own(state)
    return {"rope": _plain_rope, "cache": _plain_cache, "attend": _plain_attend,
            "given": _plain_given}[state["case"]["kind"]](state)


# ---- the library's calls

def _run_own(s):
    import paper_2603_18599_amd as sjd
    kind, c = s["case"]["kind"], s["case"]
    if kind == "rope":
        sjd.sjd_rope_axes(s["q"], s["k"], s["pos"], s["freq"], s["axis"], out_q=s["out_q"], out_k=s["out_k"],
                          inverse=c["inverse"])
        return {"q": s["out_q"], "k": s["out_k"]}
    if kind == "given":
        sjd.sjd_verify_given(s["p"], s["q"], s["draft"], s["n"], s["u"], s["r"], s["meta"], s["tok"], s["next"],
                             flags=(sjd.SJD_AC if s["ac"] else 0) | (sjd.SJD_BONUS if s["bonus"] else 0))
        return {"meta": s["meta"], "tok": s["tok"], "next": s["next"]}
    if "pages" not in s:  # the handles that a program keeps beside its buffers
        s["pages"] = sjd.Pages(s["pool"], s["total"], _PAGE, c["Hkv"], c["hd"], c["cache"])
        s["windows"] = sjd.Windows(s["seq"], s["table"], s["T"], s["max_rows"], s["max_cached"])
        if kind == "cache":
            s["whole"] = sjd.Windows(s["all"], s["table"], s["total_rows"], s["max_both"], 0)
        else:
            s["ws"] = sjd.attention_workspace(s["pages"], s["windows"], c["H"])
    if kind == "cache":
        sjd.sjd_kv_append(s["pages"], s["windows"], s["k"], s["v"])
        sjd.sjd_kv_read(s["pages"], s["whole"], s["out_k"], s["out_v"])
        return {"k": s["out_k"], "v": s["out_v"]}
    sjd.sjd_paged_attention(s["pages"], s["windows"], s["q"], s["out"], s["ws"], scale=s["scale"], anc=s["anc"])
    return {"out": s["out"]}


# ---- work and exact values

def _keys(c):
    """Sum over window rows of the positions that a row attends to (a tree's
    as a chain)."""
    rows, cached = _lengths(c)
    return sum(r * n + r * (r + 1) // 2 for r, n in zip(rows, cached))


def work(case):
    c = case
    if c["kind"] == "rope":
        e = 2 if c["dtype"] == "bf16" else 4
        heads = c["T"] * (c["H"] + c["Hkv"])
        return {"bytes": 2 * heads * c["hd"] * e + 4 * c["T"] * c["axes"], "flops": 6 * heads * c["pairs"]}
    if c["kind"] == "given":
        # one row of p and of q for each rejected window (adaptive continuation: about a third of the rows)
        draws = c["B"] * c["L"] / 3 if c["ac"] else c["B"]
        return {"bytes": draws * c["V"] * 4 * (1 if c["delta"] else 2) + c["B"] * c["L"] * 32,
                "flops": 3 * draws * c["V"]}
    rows, cached = _lengths(c)
    T, total, hd = sum(rows), sum(rows) + sum(cached), c["hd"]
    row = 2 * c["Hkv"] * (hd + 1 if c["cache"] == "e4m3" else 2 * hd)  # a cached row's bytes
    if c["kind"] == "cache":
        new = 2 * c["Hkv"] * hd * (2 if c["dtype"] == "bf16" else 4)
        return {"bytes": T * (new + row) + total * (row + 4 * c["Hkv"] * hd), "flops": 2 * c["Hkv"] * hd * (T + total)}
    return {"bytes": total * row + 4 * T * c["H"] * hd + 4 * sum(_pages_for(r + n) for r, n in zip(rows, cached)),
            "flops": 4 * hd * c["H"] * _keys(c)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "cache": _exact_cache, "attend": _exact_attend, "given": _exact_given}[case["kind"]](s)


def _exact_rope(s):
    out = {}
    sign = -1.0 if s["case"]["inverse"] else 1.0
    P = len(s["freq"])
    for name in ("q", "k"):
        x = s[name].double()
        y = x.clone()
        for i in range(P):
            phi = sign * s["pos"][:, s["axis"][i]].double() * s["freq"][i]
            z = torch.complex(x[..., i], x[..., i + P]) * torch.polar(torch.ones_like(phi), phi)[:, None]
            y[..., i], y[..., i + P] = z.real, z.imag
        out[name] = y
    return out


def _nearest_e4m3(x):
    """x rounded to the nearest of e4m3's values (ties to the even code)."""
    size = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -30))).clamp(min=-6)
    step = torch.exp2(size - 3)
    return torch.round(x / step) * step


def _cached(s, c, b, count):
    """The first `count` key and value rows of sequence b, page by page:
    every part of a page unrolled in the order that it is stored in."""
    Hkv, hd = c["Hkv"], c["hd"]
    e4 = c["cache"] == "e4m3"
    raw = s["pool"].view(s["total"], -1)[s["table"][b, :_pages_for(count)].long()]
    np_, size = raw.shape[0], 2 * Hkv * _PAGE * hd * (1 if e4 else 2)
    data = raw[:, :size].contiguous()
    if e4:
        code = data.to(torch.int64)
        power, low = code // 8 % 16, (code % 8).double()
        val = torch.where(power == 0, low * 2.0 ** -9, (1 + low / 8) * torch.exp2(power.double() - 7))
        val = torch.where(code >= 128, -val, val)
    else:
        val = data.view(torch.bfloat16).double()
    k, v = val.view(np_, Hkv, 2, _PAGE // 32, -1).unbind(2)
    if e4:
        # keys: 16-dim chunk pair, half of the dims, position (two of its bits exchanged), chunk, dim
        k = k.view(np_, Hkv, -1, hd // 32, 2, 2, 2, 2, 4, 2, 8).permute(0, 2, 5, 7, 6, 8, 1, 4, 3, 9, 10)
        # values: 32 dims, position's bit 3, dim, position's bit 4, position
        v = v.view(np_, Hkv, -1, hd // 32, 2, 32, 2, 8).permute(0, 2, 6, 4, 7, 1, 3, 5)
    else:
        k = k.view(np_, Hkv, -1, hd // 16, 2, 2, 2, 2, 4, 8).permute(0, 2, 5, 7, 6, 8, 1, 4, 3, 9)
        v = v.view(np_, Hkv, -1, hd // 32, 2, 2, 32, 8).permute(0, 2, 4, 5, 7, 1, 3, 6)
    k, v = (x.reshape(np_ * _PAGE, Hkv, hd)[:count] for x in (k, v))
    if e4:
        power = raw[:, size:size + 2 * Hkv * _PAGE].double().view(np_, Hkv, 2, _PAGE).permute(2, 0, 3, 1) - 127
        k, v = (x * torch.exp2(y.reshape(-1, Hkv)[:count])[..., None] for x, y in zip((k, v), power))
    return k, v


def _exact_cache(s):
    c, ks, vs = s["case"], [], []
    for b, (first, r, n, _) in enumerate(s["seq"].tolist()):
        old = _cached(s, c, b, n)
        for x, dst, o in ((s["k"], ks, old[0]), (s["v"], vs, old[1])):
            x = x[first:first + r].double()
            if c["cache"] == "e4m3":
                e = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 448))
                x = _nearest_e4m3(x / torch.exp2(e)) * torch.exp2(e)
            dst += [o, x]
    return {"k": torch.cat(ks), "v": torch.cat(vs)}


def _exact_attend(s):
    c = s["case"]
    G, out = c["H"] // c["Hkv"], torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, (first, r, n, _) in enumerate(s["seq"].tolist()):
        k, v = _cached(s, c, b, n + r)
        new = torch.arange(n + r, device="cuda") - n
        if s["anc"] is None:
            seen = new[None, :] <= torch.arange(r, device="cuda")[:, None]
        else:
            seen = (new < 0)[None, :] | ((s["anc"][first:first + r, None] >> new.clamp(min=0, max=63)[None, :]) & 1 == 1)
        for h in range(c["H"]):
            for a in range(0, r, 1024):
                z = s["q"][first:first + r][a:a + 1024, h].double() @ k[:, h // G].t() * s["scale"]
                z = torch.softmax(z.masked_fill(~seen[a:a + 1024], -math.inf), -1)
                out[first + a:first + min(r, a + 1024), h] = z @ v[:, h // G]
    return {"out": out}


def _exact_given(s):
    return None  # whole numbers only

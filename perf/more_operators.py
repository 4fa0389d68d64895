"""The operators around the attention over pages whose speed is measured, in
their plain form and through the library's entry points: a layer's projections
in 8-bit integers, and new rows placed and appended in one call.

Three kinds of case:
  linear   rows quantised with a scale each (as they are, behind an RMSNorm, or
           gated) and their product with 8-bit weights, in bf16
           (sjd_quantise_rows, sjd_matmul_i8);
  product  the product alone, of rows that are quantised already, in fp32
           (sjd_matmul_i8);
  place    rows of queries and keys placed on their axes, keys and values into
           the pages of a cache (sjd_kv_append_rope), and the new rows read
           back (sjd_kv_read).

Widths, head counts, window lengths and cache lengths are those of the
repository's decoder configurations or lie between them.
"""
import math

import torch

own = False

_PAGE = 64


def listed():
    return [
        # one token through an output projection: two launches
        dict(name="linear_token", kind="linear", T=1, K=4096, N=4096, form="rows", dtype="bf16", add=True),
        # a window of drafts into q, k and v (7B heads): the weights once through memory
        dict(name="linear_window", kind="linear", T=32, K=4096, N=12288, form="norm", dtype="fp32", add=False),
        # four windows down from the feed-forward width: split over a long K
        dict(name="linear_down", kind="linear", T=128, K=11008, N=4096, form="gate", dtype="bf16", add=True),
        # a short prompt, sizes off every tile
        dict(name="linear_odd", kind="linear", T=77, K=2811, N=1003, form="rows", dtype="fp32", add=False),
        # a long prompt's chunk into the gate and up projections: matrix rate
        dict(name="linear_prompt", kind="linear", T=4096, K=4096, N=22016, form="norm", dtype="bf16", add=False),
        # one row of logits of an image vocabulary (8B head): memory
        dict(name="product_logits", kind="product", T=1, K=4096, N=32768, add=False),
        # an image given as context, added to the residual rows: matrix rate, a long K
        dict(name="product_image", kind="product", T=8190, K=14336, N=4096, add=True),
        # four requests decode a token each: latency
        dict(name="place_tokens", kind="place", B=4, rows=1, cached=77, H=32, Hkv=8, hd=128, axes=3, pairs=64,
             cache="e4m3", dtype="bf16"),
        # ragged windows on two axes, part of each head rotated, fp32 rows into bf16 pages
        dict(name="place_windows", kind="place", B=8, rows=48, cached=1239, H=16, Hkv=16, hd=64, axes=2, pairs=24,
             cache="bf16", dtype="fp32"),
        # prompts of grouped heads into 8 bits: memory traffic
        dict(name="place_prompts", kind="place", B=4, rows=4096, cached=1500, H=32, Hkv=8, hd=128, axes=3, pairs=64,
             cache="e4m3", dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "product", "place"])
    if kind == "place":
        hd, Hkv, B = rng.choice([64, 128]), rng.choice([1, 2, 8, 16]), _log_int(rng, 1, 64)
        return dict(kind="place", B=B, rows=_log_int(rng, 1, max(1, 4096 * 2 // B)), cached=rng.randint(0, 4000),
                    H=Hkv * rng.choice([1, 2, 4] if Hkv <= 8 else [1, 2]), Hkv=Hkv, hd=hd, axes=rng.randint(1, 4),
                    pairs=rng.choice([hd // 2, hd // 2, hd // 4, 5]), cache=rng.choice(["e4m3", "bf16"]),
                    dtype=rng.choice(["bf16", "fp32"]))
    T, K = _log_int(rng, 1, 4096), _log_int(rng, 64, 16384)
    K = K if rng.random() < 0.3 else max(64, K // 64 * 64)
    N = _log_int(rng, 64, max(64, min(32768, 4096 * 4096 * 22016 // (T * K), (1 << 27) // K)))
    N = N if rng.random() < 0.3 else N // 64 * 64
    if kind == "product":
        return dict(kind="product", T=T, K=K, N=N, add=rng.random() < 0.3)
    return dict(kind="linear", T=T, K=K, N=N, form=rng.choice(["rows", "norm", "gate"]),
                dtype=rng.choice(["bf16", "fp32"]), add=rng.random() < 0.3)


_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_EPS = 1e-5


# ---- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _padded(K):
    """Bytes of a row of codes (zeros behind the last)."""
    return -(-K // 16) * 16


def _prepare_linear(c, g):
    T, K, N = c["T"], c["K"], c["N"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    # weights of a trained layer's kind: channels of different size, symmetric codes
    w = normal(N, K)
    s = dict(w_scale=w.abs().amax(1) * (0.02 / 127) * (0.5 + torch.rand(N, generator=g, device="cuda")),
             w=(w * (127 / w.abs().amax(1, keepdim=True))).round_().to(torch.int8))
    out = torch.float32 if c["kind"] == "product" else torch.bfloat16
    s["out"] = torch.zeros(T, N, dtype=out, device="cuda")
    s["add"] = normal(T, N).to(out) if c["add"] else None
    if c["kind"] == "product":
        s["a"] = torch.zeros(T, _padded(K), dtype=torch.int8, device="cuda")
        s["a"][:, :K] = (normal(T, K) * 32).round_().clamp_(-127, 127).to(torch.int8)
        s["a_scale"] = 0.01 + 0.02 * torch.rand(T, generator=g, device="cuda")
        return s
    dt = _TYPES[c["dtype"]]
    # rows with a few channels far larger than the others
    size = torch.where(torch.rand(K, generator=g, device="cuda") < 0.002, 20.0, 1.0)
    s["x"] = (normal(T, K) * size).to(dt)
    s["norm"] = (1 + 0.2 * normal(K)).to(dt) if c["form"] == "norm" else None
    s["gate"] = (normal(T, K) * 1.5).to(dt) if c["form"] == "gate" else None
    s["a"] = torch.zeros(T, _padded(K), dtype=torch.int8, device="cuda")
    s["a_scale"] = torch.zeros(T, device="cuda")
    return s


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


def _page_bytes(Hkv, hd, cache):
    e = 1 if cache == "e4m3" else 2
    return -(-(2 * Hkv * _PAGE * hd * e + (2 * Hkv * _PAGE if e == 1 else 0)) // 256) * 256


def _prepare_place(c, seed, g):
    rows, cached = _lengths(c)
    need = [-(-(r + n) // _PAGE) for r, n in zip(rows, cached)]
    total, T, Hkv, hd = sum(need) + 3, sum(rows), c["Hkv"], c["hd"]
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(seed) + 5)).to(torch.int32)
    table = torch.full((c["B"], max(need)), -1, dtype=torch.int32)
    seq, at, first = [], 0, 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        seq.append([first, rows[b], cached[b], 0])
        at, first = at + n, first + rows[b]
    # a cached row's position on a time axis and on the rows and columns of images of 91 columns
    p = torch.cat([torch.arange(n, n + r) for r, n in zip(rows, cached)]).cuda()
    first = int(torch.randint(0, 60000, (1,), generator=g, device="cuda"))
    pos = torch.stack([first + p // 8190, p // 91 % 90, p % 91, first + p][:c["axes"]], 1).to(torch.int32)
    dt = _TYPES[c["dtype"]]
    q, k, v = (torch.randn(T, h, hd, generator=g, device="cuda").to(dt) for h in (c["H"], Hkv, Hkv))
    return dict(pool=torch.zeros(total * _page_bytes(Hkv, hd, c["cache"]), dtype=torch.uint8, device="cuda"), total=total,
                table=table.cuda(), seq=torch.tensor(seq, dtype=torch.int32).cuda(), T=T, max_rows=max(rows),
                max_cached=max(cached), q=q, k=k, v=v, pos=pos.contiguous(),
                freq=[10000.0 ** (-i / c["pairs"]) for i in range(c["pairs"])],
                axis=[min(c["axes"] - 1, i * c["axes"] // c["pairs"]) for i in range(c["pairs"])],
                out_q=torch.zeros(T, c["H"], hd, dtype=torch.bfloat16, device="cuda"),
                out_k=torch.zeros(T, Hkv, hd, dtype=torch.bfloat16, device="cuda"),
                out_v=torch.zeros(T, Hkv, hd, dtype=torch.bfloat16, device="cuda"))


def prepare(case, seed):
    g = _gen(seed)
    s = _prepare_place(case, seed, g) if case["kind"] == "place" else _prepare_linear(case, g)
    s["case"] = case
    return s


# ---- plain forms

def _plain_rows(s):
    """Codes (as fp32) and scales of the rows."""
    c, y = s["case"], s["x"].float()
    if c["form"] == "norm":
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + _EPS) * s["norm"].float()
    elif c["form"] == "gate":
        z = s["gate"].float()
        y = y * (z / (1 + torch.exp(-z)))
    top = y.abs().amax(-1, keepdim=True)
    none = top < 2.0 ** -100
    code = torch.round(y * torch.where(none, torch.zeros_like(top), 127 / top))
    return code, torch.where(none, torch.zeros_like(top), top / 127)[:, 0]


def _plain_linear(s):
    c = s["case"]
    a, scale = (s["a"][:, :c["K"]].float(), s["a_scale"]) if c["kind"] == "product" else _plain_rows(s)
    out = torch.matmul(a, s["w"].float().t()) * scale[:, None] * s["w_scale"]
    if s["add"] is not None:
        out = out + s["add"].float()
    out = out.to(s["out"].dtype)
    return {"out": out} if c["kind"] == "product" else {"out": out, "scale": scale}


_SWAP = [(i & ~12) | ((i & 4) << 1) | ((i & 8) >> 1) for i in range(32)]


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
    """e4m3 codes and biased exponents of rows [..., hd] (fp32)."""
    amax = x.abs().amax(-1)
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(-100, 119)
    e = torch.where(amax == 0, torch.zeros_like(e), e)
    code = torch.ldexp(x, -e[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    return code.view(torch.uint8), (e + 127).to(torch.uint8)


def _decode(code, power):
    return torch.ldexp(code.view(torch.float8_e4m3fn).float(), (power.int() - 127)[..., None])


def _plain_place(s):
    c, P = s["case"], len(s["freq"])
    Hkv, hd, cache = c["Hkv"], c["hd"], c["cache"]
    phi = s["pos"][:, torch.tensor(s["axis"], device="cuda")].double() * torch.tensor(s["freq"], dtype=torch.float64,
                                                                                      device="cuda")
    co, si = phi.cos().float()[:, None], phi.sin().float()[:, None]

    def turn(x):
        x = x.float()
        a, b = x[..., :P], x[..., P:2 * P]
        return torch.cat([a * co - b * si, b * co + a * si, x[..., 2 * P:]], -1)

    q, k, v = turn(s["q"]).to(torch.bfloat16), turn(s["k"]), s["v"].float()
    rows = s["seq"][:, 1].long()
    b = torch.repeat_interleave(torch.arange(c["B"], device="cuda"), rows)
    p = s["seq"][:, 2].long()[b] + torch.arange(len(b), device="cuda") - s["seq"][:, 0].long()[b]
    pk, pv, sk, sv = _places(s["table"].long()[b, p // _PAGE], p % _PAGE, Hkv, hd, cache)
    if cache == "e4m3":
        pool = s["pool"]
        pool[pk], pool[sk] = _quantise(k)
        pool[pv], pool[sv] = _quantise(v)
        k, v = _decode(pool[pk], pool[sk]), _decode(pool[pv], pool[sv])
    else:
        pool = s["pool"].view(torch.bfloat16)
        pool[pk], pool[pv] = k.to(torch.bfloat16), v.to(torch.bfloat16)
        k, v = pool[pk], pool[pv]
    return {"q": q, "k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def run(state):
    if own:
        return _run_own(state)
    return _plain_place(state) if state["case"]["kind"] == "place" else _plain_linear(state)


# ---- the library's calls

def _run_own(s):
    import paper_2603_18599_amd as sjd
    c = s["case"]
    if c["kind"] == "place":
        if "pages" not in s:  # the handles that a program keeps beside its buffers
            s["pages"] = sjd.Pages(s["pool"], s["total"], _PAGE, c["Hkv"], c["hd"], c["cache"])
            s["windows"] = sjd.Windows(s["seq"], s["table"], s["T"], s["max_rows"], s["max_cached"])
        sjd.sjd_kv_append_rope(s["pages"], s["windows"], s["k"], s["v"], s["pos"], s["freq"], s["axis"], q=s["q"],
                               out_q=s["out_q"])
        sjd.sjd_kv_read(s["pages"], s["windows"], s["out_k"], s["out_v"])
        return {"q": s["out_q"], "k": s["out_k"], "v": s["out_v"]}
    if "weights" not in s:  # laid out once
        s["weights"] = sjd.I8Weights(c["N"], c["K"], s["w_scale"])
        sjd.sjd_pack_i8(s["weights"], s["w"])
        s["ws"] = sjd.matmul_workspace(s["weights"], c["T"])
    if c["kind"] == "product":
        sjd.sjd_matmul_i8(s["weights"], s["a"], s["a_scale"], s["out"], s["ws"], add=s["add"])
        return {"out": s["out"]}
    sjd.sjd_quantise_rows(s["x"], s["a"], s["a_scale"], norm=s["norm"], gate=s["gate"], eps=_EPS)
    sjd.sjd_matmul_i8(s["weights"], s["a"], s["a_scale"], s["out"], s["ws"], add=s["add"])
    return {"out": s["out"], "scale": s["a_scale"]}


# ---- work and exact values

def work(case):
    c = case
    if c["kind"] == "place":
        rows, cached = _lengths(c)
        T, hd = sum(rows), c["hd"]
        e = 2 if c["dtype"] == "bf16" else 4
        row = 2 * c["Hkv"] * (hd + 1 if c["cache"] == "e4m3" else 2 * hd)  # a cached row's bytes, written and read back
        new = (c["H"] + 2 * c["Hkv"]) * hd
        pages = sum((r + n - 1) // _PAGE - n // _PAGE + 1 for r, n in zip(rows, cached))
        return {"bytes": T * (new * (e + 2) + 2 * row + 4 * c["axes"]) + 4 * pages,
                "flops": T * (6 * (c["H"] + c["Hkv"]) * c["pairs"] + 4 * c["Hkv"] * hd)}
    T, K, N = c["T"], c["K"], c["N"]
    if c["kind"] == "product":
        return {"bytes": N * K + T * K + 4 * T * N * (2 if c["add"] else 1) + 4 * (T + N), "flops": 2 * T * N * K}
    e = 2 if c["dtype"] == "bf16" else 4
    rows = T * K * e * (2 if c["form"] == "gate" else 1) + (K * e if c["form"] == "norm" else 0)
    return {"bytes": N * K + rows + 2 * T * N * (2 if c["add"] else 1) + 4 * (T + N), "flops": 2 * T * N * K}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_place(s) if case["kind"] == "place" else _exact_linear(s)


def _exact_linear(s):
    c = s["case"]
    if c["kind"] == "product":
        a = s["a"][:, :c["K"]].double() * s["a_scale"].double()[:, None]
    else:
        y = s["x"].double()
        if s["norm"] is not None:
            y = y * s["norm"].double() * torch.rsqrt(y.square().mean(1) + _EPS)[:, None]
        if s["gate"] is not None:
            y = y * s["gate"].double() * torch.sigmoid(s["gate"].double())
        unit = y.abs().max(1).values / 127
        a = torch.round(y / unit[:, None]) * unit[:, None]
    out = a @ (s["w"].double() * s["w_scale"].double()[:, None]).t()
    if s["add"] is not None:
        out += s["add"].double()
    return {"out": out} if c["kind"] == "product" else {"out": out, "scale": unit}


def _nearest_e4m3(x):
    """x rounded to the nearest of e4m3's values (ties to the even code)."""
    size = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -30))).clamp(min=-6)
    step = torch.exp2(size - 3)
    return torch.round(x / step) * step


def _exact_place(s):
    P, out = len(s["freq"]), {}
    for name in ("q", "k", "v"):
        y = s[name].double()
        if name != "v":
            x, y = y, y.clone()
            for i in range(P):
                phi = s["pos"][:, s["axis"][i]].double() * s["freq"][i]
                z = torch.complex(x[..., i], x[..., i + P]) * torch.polar(torch.ones_like(phi), phi)[:, None]
                y[..., i], y[..., i + P] = z.real, z.imag
        if name != "q" and s["case"]["cache"] == "e4m3":
            unit = torch.exp2(torch.ceil(torch.log2(y.abs().amax(-1, keepdim=True) / 448)))
            y = _nearest_e4m3(y / unit) * unit
        out[name] = y
    return out

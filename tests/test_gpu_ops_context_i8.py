"""Decoder contexts whose layers' projections are in 8-bit integers (SJD_W8A8): their
window logits against a plain 64-bit decoder that rounds where they do, after
prefill, after steps, for several streams, and at the refusals.

The bound is derived as for the other contexts with pages: a value that differs by
1e-6 before a rounding may fall to the other side of it, by a step of int8, e4m3
or bf16, and the context rounds probabilities to bf16. Both were put into the
plain decoder on the CPU (test_bounds_hold_against_noise: noise of 1e-6 on the
embeddings, probabilities off by up to 2^-9, four seeds): logits of standard deviation
0.64 (64-dim heads) and 0.90 (128) moved by up to MOVED[0], in the mean square by up
to MOVED[1] of a forward. The bounds are twice that. (8 bits themselves move them as much: a
forward whose inputs are not quantised is off by 0.026 and 0.043 in the mean square. What
each operator rounds is held exactly in its own tests and in those of a layer.) Mistakes are off
by more (tested): another row's scale, another channel's, a missing key, no grid."""
import ctypes as C

import pytest
import torch

import paper_2603_18599_amd as sjd
from model_util import make_engine, weights_device
from ops_util import quantise
from synth_inputs import model_weights
from test_gpu_ops_context import GQA, STD, bf16, causal, config, places, tokens, turn

MOVED = 0.163, 0.0336
W8 = sjd.SJD_W8A8 | sjd.SJD_KV_E4M3
FLAGS = [W8, W8 | sjd.SJD_ROPE_GRID]
MODELS = [dict(L=16), dict(L=16, **GQA)]


def off_by(a, b):
    d = a - b
    return d.abs().max().item(), d.square().mean().sqrt().item()


def check(got, want, label=""):
    most, rms = off_by(got.cpu().double(), want)
    print(label, "off by", most, "rms", rms, "of logits with std", want.std().item())
    assert most < 2 * MOVED[0] and rms < 2 * MOVED[1]


def q8(x):
    """Rows as the nearest of 255 multiples of max / 127."""
    unit = x.abs().amax(-1, keepdim=True) / 127
    return torch.round(x / torch.where(unit == 0, torch.ones_like(unit), unit)) * unit


def reference(cfg, w, toks, pl, seen, noise=None, inputs=q8, weights=q8):
    """Logits of every row (see test_gpu_ops_context.reference). noise: a generator, for the bound;
    inputs, weights: how a projection's are quantised (for mistakes)."""
    H, Hkv, hd, eps = cfg["n_heads"], cfg["n_kv_heads"], cfg["head_dim"], cfg["rms_eps"]
    grid = bool(cfg["flags"] & sjd.SJD_ROPE_GRID)
    D = lambda t: t.double()  # noqa: E731
    norm = lambda x, g: x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * D(g)  # noqa: E731
    lin = lambda x, m: inputs(x) @ weights(D(m)).T  # noqa: E731
    T = len(toks)
    x = D(w["embed"])[torch.tensor(toks).long()]
    if noise is not None:
        x = x * (1 + 1e-6 * torch.randn(x.shape, generator=noise, dtype=torch.float64))
    for l in w["layers"]:
        y = norm(x, l["attn_norm"])
        q, k, v = (lin(y, l[n]).view(T, -1, hd) for n in ("wq", "wk", "wv"))
        q, k = bf16(turn(q, pl, cfg["rope_theta"], grid)), turn(k, pl, cfg["rope_theta"], grid)
        k, v = (torch.from_numpy(quantise(t.numpy())[0]) for t in (k, v))
        k, v = (t.repeat_interleave(H // Hkv, 1) for t in (k, v))
        z = torch.einsum("ihd,jhd->hij", q, k) * hd ** -0.5
        z = torch.softmax(z.masked_fill(~seen[None], -float("inf")), -1)
        if noise is not None:
            z = z * (1 + 2.0 ** -9 * (2 * torch.rand(z.shape, generator=noise, dtype=torch.float64) - 1))
        x = x + lin(bf16(torch.einsum("hij,jhd->ihd", z, v)).reshape(T, H * hd), l["wo"])
        y = norm(x, l["ffn_norm"])
        g, u = bf16(lin(y, l["wg"])), bf16(lin(y, l["wu"]))
        x = x + lin(g * torch.sigmoid(g) * u, l["wd"])
    return (norm(x, w["final_norm"]) @ D(w["lm_head"]).T)[:, cfg["vis_lo"]:cfg["vis_lo"] + cfg["V"]]


def window(cfg, w, prompt, gen, drafts):
    """Window logits of a stream: its prompt, what was generated, the caller's drafts as a chain."""
    seq = prompt.tolist() + gen
    toks = seq + drafts.tolist()[:-1]
    return reference(cfg, w, toks, places(cfg, len(prompt), range(len(toks))), causal(len(toks)))[len(seq) - 1:]


@pytest.mark.gpu
@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("over", [dict(L=16), dict(L=1, K=1, D=0, n_prompt=1), dict(L=33, n_prompt=200), dict(L=16, **GQA),
                                  dict(L=64, n_prompt=300, **GQA), dict(L=16, weights_f32=True)])
def test_window_logits(over, flags):
    cfg = config(flags, **over)
    w = model_weights(cfg, 3, std=STD)
    prompt, drafts = tokens(cfg, cfg["n_prompt"], 4), tokens(cfg, cfg["L"], 5, vis=True)
    eng = make_engine(cfg, weights_device(w))
    eng.prefill(prompt.cuda(), 1)
    eng.set_drafts(drafts.cuda())
    out = torch.empty(cfg["L"], cfg["V"], device="cuda")
    eng.forward_window(out)
    check(out, window(cfg, w, prompt, [], drafts))
    eng.close()


@pytest.mark.gpu
@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("streams", [dict(), dict(batch=2), dict(cfg_w=0.5), dict(batch=2, cfg_w=0.5), dict(batch=4)],
                         ids=["one", "images", "guided", "guided-images", "four"])
def test_rows_of_every_stream_after_steps(streams, flags):
    """Steps with drafting trees (accepted siblings move through the pages), then every image's
    drafts as a chain."""
    B, cfg_w, L = streams.get("batch", 1), streams.get("cfg_w"), 16
    cfg = config(flags, L=L, K=4, D=3, **streams, n_gen=900)
    w = model_weights(cfg, 3, std=STD)
    eng = make_engine(cfg, weights_device(w))
    meta, tok = torch.zeros(B, 8, dtype=torch.int32, device="cuda"), torch.zeros(B, L, dtype=torch.int32, device="cuda")
    prompts = [[tokens(cfg, n, 100 * b + n) for n in pair] for b, pair in enumerate([(37, 12), (50, 90), (1, 3), (129, 40)][:B])]
    gen, siblings = [[] for _ in range(B)], 0
    for b, (text, uncond) in enumerate(prompts):
        if cfg_w:
            eng.prefill_cfg(text.cuda(), uncond.cuda(), 7 + b, image=b)
        else:
            eng.prefill_image(b, text.cuda(), 7 + b)
    for i in range(150):  # (25, and more until a sibling was accepted)
        if i >= 25 and siblings:
            break
        eng.step(0.5, 40, 5, i, out_meta=meta, out_tok=tok)
        for b, (m, t) in enumerate(zip(meta.tolist(), tok.tolist())):
            gen[b] += t[:m[0]]
            siblings += m[5] >= 2
            assert m[7] == len(prompts[b][0]) + len(gen[b]) - 1
    assert siblings > 0
    drafts = [tokens(cfg, L, 60 + b, vis=True) for b in range(B)]
    for b in range(B):
        # (a row end takes eol_id and counts as accepted whatever was fed)
        drafts[b][(torch.arange(L) + len(gen[b])) % (cfg["row_len"] + 1) == cfg["row_len"]] = cfg["eol_id"]
        eng.set_drafts(drafts[b].cuda(), image=b)
    out = torch.empty(32 * (B - 1) + L, cfg["V"], device="cuda")
    eng.forward_window(out)
    for b in range(B):
        ref = [window(cfg, w, p, gen[b], drafts[b]) for p in prompts[b][:2 if cfg_w else 1]]
        want = ref[1] + cfg_w * (ref[0] - ref[1]) if cfg_w else ref[0]
        check(out[32 * b:32 * b + L], want, f"image {b} after {len(gen[b])} tokens:")
    eng.close()


@pytest.mark.gpu
def test_eager_and_captured_steps_agree():
    runs = []
    for extra in (0, 4):  # SJD_EAGER
        cfg = config(W8 | extra, L=16)
        eng = make_engine(cfg, weights_device(model_weights(cfg, 3, std=STD)))
        eng.prefill(tokens(cfg, cfg["n_prompt"], 4).cuda(), 1)
        got = []
        meta, tok = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(16, dtype=torch.int32, device="cuda")
        for i in range(12):
            eng.step(1.0, 50, 9, i, out_meta=meta, out_tok=tok)
            got += [meta.cpu(), tok.cpu()]
        runs.append(torch.cat(got))
        eng.close()
    assert torch.equal(*runs)


@pytest.mark.gpu
def test_two_contexts_at_once():
    """Contexts of their own weights and streams, their steps in turn without a wait between them, as one
    after the other."""
    def build(seed):
        cfg = config(W8, L=16)
        eng = make_engine(cfg, weights_device(model_weights(cfg, seed, std=STD)))
        eng.prefill(tokens(cfg, cfg["n_prompt"], seed).cuda(), 1)
        return eng, torch.zeros(8, 16, dtype=torch.int32, device="cuda")

    def step(eng, toks, i, stream=None):
        eng.step(1.0, 50, 9, i, out_tok=toks[i], stream=stream)

    alone = []
    for seed in (3, 4):
        eng, toks = build(seed)
        for i in range(8):
            step(eng, toks, i)
        torch.cuda.synchronize()
        alone.append(toks.cpu())
        eng.close()
    pairs = [build(seed) for seed in (3, 4)]
    streams = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()
    for i in range(8):
        for (eng, toks), st in zip(pairs, streams):
            step(eng, toks, i, st)
    torch.cuda.synchronize()
    for (eng, toks), want in zip(pairs, alone):
        assert torch.equal(toks.cpu(), want)
        eng.close()


def of_operators(cfg, w, toks, n_prompt):
    """The residual rows (fp32) of a window behind the last layer, from the operators themselves: the prompt's
    cached rows as one window, then the rows from its last token on, a causal chain."""
    H, Hkv, hd, F, L = (cfg[k] for k in ("n_heads", "n_kv_heads", "head_dim", "ffn_dim", "L"))
    Nq, N, P, theta = H * hd, (H + 2 * Hkv) * hd, hd // 2, cfg["rope_theta"]
    grid = bool(cfg["flags"] & sjd.SJD_ROPE_GRID)
    freq = [float(theta) ** (-2.0 * i / hd) for i in range(P)]
    axis = [0 if not grid or i < P // 4 else 1 + i % 2 for i in range(P)]
    at = places(cfg, n_prompt, range(len(toks))).to(torch.int32)[:, :3 if grid else 1].contiguous().cuda()
    n_pages = -(-cfg["max_seq"] // 64) + 1
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()[None].contiguous()

    def pack(*parts):
        m = torch.cat(parts).cuda()
        h = sjd.I8Weights(*m.shape)
        sjd.sjd_pack_i8(h, m)
        return h

    layers = [dict(qkv=pack(l["wq"], l["wk"], l["wv"]), o=pack(l["wo"]), gu=pack(l["wg"], l["wu"]), down=pack(l["wd"]),
                   norm=[l[n].to(torch.bfloat16).cuda() for n in ("attn_norm", "ffn_norm")],
                   pool=torch.zeros(n_pages * sjd.page_bytes(64, Hkv, hd, "e4m3"), dtype=torch.uint8, device="cuda"))
              for l in w["layers"]]
    for first, T in ((0, n_prompt - 1), (n_prompt - 1, L)):
        if T == 0:
            continue
        seq = torch.tensor([[0, T, first, 0]], dtype=torch.int32).cuda()
        win = sjd.Windows(seq, table, T, T, cfg["max_seq"])
        x = w["embed"].to(torch.bfloat16).float()[torch.tensor(toks[first:first + T]).long()].cuda()
        qkv, q8 = torch.empty(T, N, device="cuda"), torch.empty(T, H, hd, dtype=torch.bfloat16, device="cuda")
        q, k, v = (qkv[:, a:b].view(T, -1, hd) for a, b in ((0, Nq), (Nq, Nq + Hkv * hd), (Nq + Hkv * hd, N)))
        att, gu = torch.empty_like(q8), torch.empty(T, 2 * F, dtype=torch.bfloat16, device="cuda")

        def project(h, rows, out, add=None, **kw):
            code, scale = torch.empty(T, h.K, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
            sjd.sjd_quantise_rows(rows, code, scale, eps=cfg["rms_eps"], **kw)
            sjd.sjd_matmul_i8(h, code, scale, out, sjd.matmul_workspace(h, T), add=add)

        for l in layers:
            pages = sjd.Pages(l["pool"], n_pages, 64, Hkv, hd, "e4m3")
            project(l["qkv"], x, qkv, norm=l["norm"][0])
            sjd.sjd_kv_append_rope(pages, win, k, v, at[first:first + T].contiguous(), freq, axis, q=q, out_q=q8)
            sjd.sjd_paged_attention(pages, win, q8, att, sjd.attention_workspace(pages, win, H), scale=hd ** -0.5)
            project(l["o"], att.view(T, Nq), x, x)
            project(l["gu"], x, gu, norm=l["norm"][1])
            project(l["down"], gu[:, F:], x, x, gate=gu[:, :F])
    return x


def head(cfg, w, x):
    """Logits of residual rows in 64 bits, and how far the context's head may be off them: its inputs are
    two bf16 parts (2^-18 of each left out), its sums and the squares' run over d_model terms in 32 bits
    (2^-23 a term: the matrix unit need not round to nearest), with a few roundings beside."""
    x, g = x.double().cpu(), w["final_norm"].double()
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + cfg["rms_eps"]) * g
    m = w["lm_head"].to(torch.bfloat16).double()[cfg["vis_lo"]:cfg["vis_lo"] + cfg["V"]]
    return y @ m.T, (2.0 ** -18 + (2 * cfg["d_model"] + 16) * 2.0 ** -23) * (y.abs() @ m.abs().T)


CHAINS = [dict(L=16), dict(L=1, K=1, D=0, n_prompt=1), dict(L=33, n_prompt=60), dict(L=16, n_prompt=120, **GQA),
          dict(L=16, weights_f32=True)]


@pytest.mark.gpu
@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("over", CHAINS)
def test_window_logits_are_those_of_the_operators(over, flags):
    """A context's layers are the operators' calls, bit for bit: its logits are the head's of the rows that
    the calls give. (What 8 bits round moves the logits by more than 20 times this bound:
    test_projections_in_more_bits_are_told_apart.)"""
    cfg = config(flags, **over)
    w = model_weights(cfg, 3, std=STD)
    prompt, drafts = tokens(cfg, cfg["n_prompt"], 4), tokens(cfg, cfg["L"], 5, vis=True)
    eng = make_engine(cfg, weights_device(w))
    eng.prefill(prompt.cuda(), 1)
    eng.set_drafts(drafts.cuda())
    out = torch.empty(cfg["L"], cfg["V"], device="cuda")
    eng.forward_window(out)
    want, tol = head(cfg, w, of_operators(cfg, w, prompt.tolist() + drafts.tolist()[:-1], cfg["n_prompt"]))
    err = (out.cpu().double() - want).abs()
    print("off by", err.max().item(), "of", tol.max().item())
    assert (err <= tol).all()
    eng.close()


def test_projections_in_more_bits_are_told_apart():
    """(CPU) The plain decoder without the projections' quantisation, as a context that ignored the flag
    would be, is off by more than 20 times the bound of the comparison with the operators (one is enough)."""
    for over in MODELS:
        for flags in FLAGS:
            cfg, run = config(flags, **over), case(over, flags)
            same = lambda x: x  # noqa: E731
            rms = off_by(run(inputs=same, weights=same), run())[1]
            x = torch.randn(8, cfg["d_model"], generator=torch.Generator().manual_seed(1))
            tol = head(cfg, model_weights(cfg, 3, std=STD), x)[1].max().item()  # (of normed rows: their size does not matter)
            print("rms", rms, "bound", tol)
            assert rms > 20 * tol


def case(over, flags):
    cfg = config(flags, **over)
    w = model_weights(cfg, 3, std=STD)
    toks = tokens(cfg, 37, 4).tolist() + tokens(cfg, 40, 5, vis=True).tolist()
    T = len(toks)

    def run(missing=False, text_only=False, **kw):
        seen = causal(T)
        if missing:
            seen[60:, 45] = False
        return reference(cfg, w, toks, places(cfg, 37, range(T), text_only=text_only), seen, **kw)[36:]

    return run


def test_bounds_hold_against_noise():
    """(CPU) What the bounds stand on."""
    most = [0.0, 0.0]
    for over in MODELS:
        for flags in FLAGS:
            run = case(over, flags)
            good = run()
            for seed in range(4):
                most = [max(p) for p in zip(most, off_by(run(noise=torch.Generator().manual_seed(seed)), good))]
    print("moved by", most)
    for m, bound in zip(most, MOVED):
        assert 0.9 * bound < m <= bound


def test_reference_tells_mistakes_apart():
    """(CPU) Planted mistakes are off by more than the bounds."""
    def neighbours(x):
        """Quantised, with the scale of the row before."""
        y, top = q8(x), x.abs().amax(-1)
        return torch.cat([y[:1], y[1:] * (top[:-1] / top[1:])[:, None]])

    for over in MODELS:
        run = case(over, W8 | sjd.SJD_ROPE_GRID)
        good = run()
        for kw in (dict(inputs=neighbours), dict(weights=neighbours), dict(text_only=True)):
            most, rms = off_by(run(**kw), good)
            print(list(kw), most, rms)
            assert rms > 2.5 * 2 * MOVED[1]
        assert off_by(run(missing=True), good)[0] > 2 * MOVED[0]


def test_flags_refused_on_host():
    from paper_2603_18599_amd import sjd as b
    lib = b.load_library()
    good = dict(n_layers=1, d_model=64, n_heads=1, n_kv_heads=1, head_dim=64, ffn_dim=64, vocab_size=64, vis_lo=0, V=32,
                max_seq=64, L=4, K=1, D=0, flags=W8, rms_eps=1e-5, rope_theta=1e4, eol_id=-1, row_len=0)
    w, h = b.Weights(), C.c_void_p()
    for over, rc in ((dict(flags=sjd.SJD_W8A8), -1), (dict(flags=W8 | 16), -1), (dict(flags=sjd.SJD_W8A8 | sjd.SJD_ROPE_GRID, row_len=3), -1),
                     (dict(d_model=65600), -5), (dict(ffn_dim=65600), -5), (dict(n_heads=1040), -5), (dict(rms_eps=1e-40), -1),
                     (dict(), -1)):  # (the last: no weights)
        c = b.Config(**{**good, **over})
        assert lib.sjd_init(C.byref(c), C.byref(w), None, C.byref(h)) == rc, over

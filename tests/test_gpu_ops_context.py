"""Decoder contexts whose caches are pages (SJD_KV_E4M3, SJD_ROPE_GRID): their
window logits against a plain 64-bit decoder that rounds where they do; after
prefill, and after steps whose accepted tokens (siblings among them) moved
through the pages.

The bound. Where the plain decoder and the context differ by 1e-6 before a
rounding, some value falls to the other side, by a step of bf16 or of e4m3; the
context also rounds probabilities to bf16 (2^-9 of each on average). Both were
put into the plain decoder on the CPU (noise of 1e-6 on the embeddings,
probabilities off by up to 2^-9, four seeds): logits of standard deviation 0.64
(64-dim heads) and 0.90 (128) moved by up to 0.015 with bf16 pages and 0.025 with
e4m3 ones. The bounds are twice that, and the framework's 3e-2 for bf16.
Mistakes are off by more (tested): image tokens without their grid 1.07, one
key missing 0.38, the default path's rounding against e4m3's 0.11."""
import numpy as np
import pytest
import torch

import paper_2603_18599_amd as sjd
from model_util import make_engine, weights_device
from ops_util import quantise
from synth_inputs import model_config, model_weights

TOL = {sjd.SJD_ROPE_GRID: 3e-2, sjd.SJD_KV_E4M3: 5e-2, sjd.SJD_KV_E4M3 | sjd.SJD_ROPE_GRID: 5e-2}
STD = 0.04
BASE = dict(n_prompt=37, n_gen=200, row_len=9, eol_id=1000, V=960, vis_lo=32, weights_f32=False)
GQA = dict(n_layers=2, d_model=512, n_heads=4, n_kv_heads=2, head_dim=128, ffn_dim=512)


def bf16(x):
    return x.float().to(torch.bfloat16).double()


def places(cfg, n_p, pos, text_only=False):
    """[rows, 3] time, row, column (or the position three times)."""
    out = []
    for p in pos:
        g = p - n_p
        if text_only or g < 0 or not cfg["flags"] & sjd.SJD_ROPE_GRID:
            out.append((p, p, p))
        else:
            out.append((n_p, n_p + g // (cfg["row_len"] + 1), n_p + g % (cfg["row_len"] + 1)))
    return torch.tensor(out, dtype=torch.float64)


def turn(x, pl, theta, grid):
    P = x.shape[-1] // 2
    ax = torch.tensor([0 if not grid or i < P // 4 else 1 + i % 2 for i in range(P)])
    f = torch.tensor([float(theta) ** (-i / P) for i in range(P)], dtype=torch.float64)
    phi = pl[:, ax] * f
    c, s = phi.cos()[:, None], phi.sin()[:, None]
    a, b = x[..., :P], x[..., P:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def reference(cfg, w, toks, pl, seen, rounds=True):
    """Logits of every row of a forward over tokens `toks` (places pl, row i
    attends where seen[i])."""
    H, Hkv, hd, eps = cfg["n_heads"], cfg["n_kv_heads"], cfg["head_dim"], cfg["rms_eps"]
    e4, grid = cfg["flags"] & sjd.SJD_KV_E4M3, bool(cfg["flags"] & sjd.SJD_ROPE_GRID)
    rd = bf16 if rounds else (lambda x: x)
    D = lambda t: t.double()  # noqa: E731
    norm = lambda x, g: x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * D(g)  # noqa: E731
    T = len(toks)
    x = D(w["embed"])[torch.tensor(toks).long()]
    for l in w["layers"]:
        y = norm(x, l["attn_norm"])
        q, k, v = (rd(y @ D(l[n]).T).view(T, -1, hd) for n in ("wq", "wk", "wv"))
        q, k = rd(turn(q, pl, cfg["rope_theta"], grid)), rd(turn(k, pl, cfg["rope_theta"], grid))
        if e4 and rounds:
            k, v = (torch.from_numpy(quantise(t.numpy())[0]) for t in (k, v))
        k, v = (t.repeat_interleave(H // Hkv, 1) for t in (k, v))
        z = torch.einsum("ihd,jhd->hij", q, k) * hd ** -0.5
        z = torch.softmax(z.masked_fill(~seen[None], -float("inf")), -1)
        x = x + rd(torch.einsum("hij,jhd->ihd", z, v)).reshape(T, H * hd) @ D(l["wo"]).T
        y = norm(x, l["ffn_norm"])
        g = y @ D(l["wg"]).T
        x = x + (g * torch.sigmoid(g) * (y @ D(l["wu"]).T)) @ D(l["wd"]).T
    return (norm(x, w["final_norm"]) @ D(w["lm_head"]).T)[:, cfg["vis_lo"]:cfg["vis_lo"] + cfg["V"]]


def causal(T):
    return torch.arange(T)[None] <= torch.arange(T)[:, None]


def config(flags, **over):
    return model_config("tiny", **{**BASE, **over}, flags=sjd.SJD_AC | sjd.SJD_PD | flags)


def tokens(cfg, n, seed, vis=False):
    g = torch.Generator().manual_seed(seed)
    lo, hi = (cfg["vis_lo"], cfg["vis_lo"] + cfg["V"]) if vis else (0, cfg["vocab_size"])
    return torch.randint(lo, hi, (n,), generator=g, dtype=torch.int32)


FLAGS = [sjd.SJD_KV_E4M3, sjd.SJD_ROPE_GRID, sjd.SJD_KV_E4M3 | sjd.SJD_ROPE_GRID]
CASES = [dict(L=16), dict(L=1, K=1, D=0, n_prompt=1), dict(L=33, n_prompt=200), dict(L=16, **GQA),
         dict(L=64, n_prompt=300, **GQA)]


@pytest.mark.gpu
@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("over", CASES, ids=[str(i) for i in range(len(CASES))])
def test_window_logits(over, flags):
    cfg = config(flags, **over)
    w = model_weights(cfg, 3, std=STD)
    prompt, drafts = tokens(cfg, cfg["n_prompt"], 4), tokens(cfg, cfg["L"], 5, vis=True)
    eng = make_engine(cfg, weights_device(w))
    eng.prefill(prompt.cuda(), 1)
    eng.set_drafts(drafts.cuda())
    out = torch.empty(cfg["L"], cfg["V"], device="cuda")
    eng.forward_window(out)
    toks = prompt.tolist() + drafts.tolist()[:-1]
    ref = reference(cfg, w, toks, places(cfg, len(prompt), range(len(toks))), causal(len(toks)))[len(prompt) - 1:]
    err = (out.cpu().double() - ref).abs().max().item()
    print("max error", err, "of logits with std", ref.std().item())
    assert err < TOL[flags]
    eng.close()


@pytest.mark.gpu
@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("over", [dict(L=16, K=4, D=3), dict(L=12, K=2, D=4, **GQA)], ids=["tiny", "gqa"])
def test_steps_keep_the_pages(over, flags):
    """Steps with drafting trees; then the caller's drafts as a chain, whose
    logits depend on every cached row and on its place."""
    cfg = config(flags, **over)
    w = model_weights(cfg, 3, std=STD)
    prompt = tokens(cfg, cfg["n_prompt"], 4)
    eng = make_engine(cfg, weights_device(w))
    L = cfg["L"]
    meta, tok = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (8, L))
    out = torch.empty(L, cfg["V"], device="cuda")
    siblings = 0
    for seed in range(3):
        eng.prefill(prompt.cuda(), seed)
        seq = prompt.tolist()
        for i in range(30):
            eng.step(0.5, 40, seed, i, out_meta=meta, out_tok=tok)
            m = meta.tolist()
            seq += tok.tolist()[:m[0]]
            siblings += m[5] >= 2
            assert m[7] == len(seq) - 1
        drafts = tokens(cfg, L, 50 + seed, vis=True)
        eng.set_drafts(drafts.cuda())
        eng.forward_window(out)
        toks = seq + drafts.tolist()[:-1]
        ref = reference(cfg, w, toks, places(cfg, len(prompt), range(len(toks))), causal(len(toks)))[len(seq) - 1:]
        assert (out.cpu().double() - ref).abs().max().item() < TOL[flags], seed
    assert siblings > 0  # (rows moved)
    eng.close()


@pytest.mark.gpu
@pytest.mark.parametrize("flags", FLAGS)
def test_images_and_guidance(flags):
    """Two guided images in one context: four streams with prompts of their own
    lengths in one forward."""
    cfg = config(flags, L=16, batch=2, cfg_w=3.0)
    w = model_weights(cfg, 3, std=STD)
    eng = make_engine(cfg, weights_device(w))
    out = torch.empty(32 + 16, cfg["V"], device="cuda")
    prompts = [(tokens(cfg, n, n), tokens(cfg, m, m)) for n, m in ((37, 12), (50, 90))]
    drafts = [tokens(cfg, 16, 60 + b, vis=True) for b in range(2)]
    for b, (p, u) in enumerate(prompts):
        eng.prefill_cfg(p.cuda(), u.cuda(), 7, image=b)
        eng.set_drafts(drafts[b].cuda(), image=b)
    eng.forward_window(out)
    for b, pair in enumerate(prompts):
        ref = []
        for p in pair:
            toks = p.tolist() + drafts[b].tolist()[:-1]
            ref.append(reference(cfg, w, toks, places(cfg, len(p), range(len(toks))), causal(len(toks)))[len(p) - 1:])
        want = ref[1] + 3.0 * (ref[0] - ref[1])
        assert (out[32 * b:32 * b + 16].cpu().double() - want).abs().max().item() < 5 * TOL[flags]  # |1 - w| + |w| = 5
    # a batch restarts one image and goes on with the other; steps run from a captured graph
    meta, tok = torch.zeros(2, 8, dtype=torch.int32, device="cuda"), torch.zeros(2, 16, dtype=torch.int32, device="cuda")
    for i in range(4):
        eng.step(1.0, 0, 3, i, out_meta=meta, out_tok=tok)
        assert (meta[:, 0] >= 1).all()
    eng.close()


@pytest.mark.gpu
@pytest.mark.parametrize("flags", FLAGS)
def test_eager_and_captured_steps_agree(flags):
    runs = []
    for extra in (0, 4):  # SJD_EAGER
        cfg = config(flags | extra, L=16)
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


def test_reference_tells_mistakes_apart():
    """(CPU) The bounds above are well below what planted mistakes do."""
    for over in (dict(L=16), dict(L=16, **GQA)):
        for flags in FLAGS:
            cfg, tol = config(flags, **over), TOL[flags]
            w = model_weights(cfg, 3, std=STD)
            toks = tokens(cfg, 37, 4).tolist() + tokens(cfg, 40, 5, vis=True).tolist()
            T = len(toks)
            pl, seen = places(cfg, 37, range(T)), causal(T)
            good = reference(cfg, w, toks, pl, seen)[36:]
            off = lambda p, s, **kw: (reference(cfg, w, toks, p, s, **kw)[36:] - good).abs().max().item()  # noqa: E731
            missing = seen.clone()
            missing[60:, 45] = False
            assert off(pl, missing) > 5 * tol
            if flags & sjd.SJD_ROPE_GRID:
                assert off(places(cfg, 37, range(T), text_only=True), seen) > 10 * tol
                assert off(pl[:, [0, 2, 1]], seen) > 4 * tol
            if flags & sjd.SJD_KV_E4M3:
                assert off(pl, seen, rounds=False) > 2 * tol


def test_flags_refused_on_host():
    import ctypes as C
    from paper_2603_18599_amd import sjd as b
    lib = b.load_library()
    good = dict(n_layers=1, d_model=64, n_heads=1, n_kv_heads=1, head_dim=64, ffn_dim=64, vocab_size=64, vis_lo=0, V=32,
                max_seq=64, L=4, K=1, D=0, flags=0, rms_eps=1e-5, rope_theta=1e4, eol_id=-1, row_len=0)
    w, h = b.Weights(), C.c_void_p()
    for over in (dict(flags=sjd.SJD_ROPE_GRID), dict(flags=sjd.SJD_ROPE_GRID, row_len=-1),
                 dict(flags=sjd.SJD_KV_E4M3 | 16), dict(flags=512)):
        c = b.Config(**{**good, **over})
        assert lib.sjd_init(C.byref(c), C.byref(w), None, C.byref(h)) == -1, over


# A context without e4m3 pages rounds activations, keys and values to pairs of bf16 (16
# bits, half a step of 2^-17), 2^-8 of what a single bf16 rounding does. Rounding q, k, v
# and the attention's output to bf16 moves these cases' logits by 0.0051 to 0.0193 (plain
# decoder, CPU); the GEMM inputs and probabilities are as many rounding points again, and
# more: 4 * 0.0193 * 2^-8 = 3e-4. Three times that is the bound, a fifth of what bf16 does.
PAIRS = 1e-3


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [0, sjd.SJD_ROPE_GRID])
@pytest.mark.parametrize("over", CASES, ids=[str(i) for i in range(len(CASES))])
def test_a_grid_alone_keeps_the_default_precision(over, flags):
    """Where tokens are placed says nothing about the bits of the caches and of the
    attention."""
    cfg = config(flags, **over)
    w = model_weights(cfg, 3, std=STD)
    prompt, drafts = tokens(cfg, cfg["n_prompt"], 4), tokens(cfg, cfg["L"], 5, vis=True)
    eng = make_engine(cfg, weights_device(w))
    eng.prefill(prompt.cuda(), 1)
    eng.set_drafts(drafts.cuda())
    out = torch.empty(cfg["L"], cfg["V"], device="cuda")
    eng.forward_window(out)
    toks = prompt.tolist() + drafts.tolist()[:-1]
    ref = reference(cfg, w, toks, places(cfg, len(prompt), range(len(toks))), causal(len(toks)), rounds=False)
    err = (out.cpu().double() - ref[len(prompt) - 1:]).abs().max().item()
    print("max error", err)
    assert err < PAIRS
    eng.close()


@pytest.mark.gpu
def test_pages_instead_of_the_default_buffers():
    """Device memory of a context of 60000 positions: e4m3 pages are a quarter of the
    default's caches, and what its attention alone needs is not there."""
    over = dict(L=16, n_layers=4, n_heads=4, n_kv_heads=4, head_dim=64, d_model=256, ffn_dim=256, max_seq=60000)
    used = []
    for flags in (0, sjd.SJD_KV_E4M3):
        cfg = config(flags, **over)
        w = weights_device(model_weights(cfg, 3, std=STD))
        torch.cuda.synchronize()
        free = torch.cuda.mem_get_info()[0]
        eng = make_engine(cfg, w)
        used.append(free - torch.cuda.mem_get_info()[0])
        eng.close()
    positions = -(-60000 // 128) * 128
    planes = 4 * 4 * positions * 64 * 8  # layers, heads, positions, dims; two planes of k and of v
    splits = 4 * (positions // 128) * 128 * (64 + 2) * 4  # the default attention's partial outputs
    # (allocations are rounded up: 2 MB each, some 40 of them)
    assert used[0] >= planes + splits
    assert used[1] <= planes // 4 * 1.04 + (used[0] - planes - splits) + (16 << 20), used

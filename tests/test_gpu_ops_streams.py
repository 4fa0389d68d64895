"""Contexts of several streams (images, unconditional streams) with SJD_KV_E4M3 and
SJD_ROPE_GRID, by value after steps that moved accepted siblings: every image's
logits depend on every row that its streams have cached, and on each row's place.
Between the two rounds of steps the second image starts again with other prompts
while the first goes on.

The bounds are those of test_gpu_ops_context.py: e4m3 pages against the plain decoder
that rounds where they do, a grid alone against the one without roundings. A guided
image's logits are (1 - w) of the one stream's and w of the other's (w = 1/2)."""
import pytest
import torch

import paper_2603_18599_amd as sjd
from model_util import make_engine, weights_device
from synth_inputs import model_weights
from test_gpu_ops_context import FLAGS, GQA, PAIRS, STD, TOL, causal, config, places, reference, tokens

STEPS, MOST = 20, 150
MODELS = [dict(L=16, K=4, D=3), dict(L=12, K=2, D=4, **GQA)]
STREAMS = [dict(batch=2), dict(cfg_w=0.5), dict(batch=2, cfg_w=0.5), dict(batch=4)]
# (text, unconditional) prompt lengths: of the images, and of the second one's restart
PROMPTS, AGAIN = [(37, 12), (50, 90), (1, 3), (129, 40)], (20, 61)


def bound(flags):
    return PAIRS if flags == sjd.SJD_ROPE_GRID else TOL[flags]


def window(cfg, w, prompt, gen, drafts, rounds):
    """The plain decoder's window logits of a stream: its prompt, what the image has
    generated, and the caller's drafts as a chain."""
    seq = prompt.tolist() + gen
    toks = seq + drafts.tolist()[:-1]
    ref = reference(cfg, w, toks, places(cfg, len(prompt), range(len(toks))), causal(len(toks)), rounds)
    return ref[len(seq) - 1:]


@pytest.mark.gpu
@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("streams", STREAMS, ids=["images", "guided", "guided-images", "four"])
@pytest.mark.parametrize("model", MODELS, ids=["tiny", "gqa"])
def test_rows_of_every_stream_after_steps(model, streams, flags):
    B, cfg_w, L = streams.get("batch", 1), streams.get("cfg_w"), model["L"]
    cfg = config(flags, **model, **streams, n_gen=900)
    w = model_weights(cfg, 3, std=STD)
    eng = make_engine(cfg, weights_device(w))
    out = torch.empty(32 * (B - 1) + L, cfg["V"], device="cuda")
    meta, tok = torch.zeros(B, 8, dtype=torch.int32, device="cuda"), torch.zeros(B, L, dtype=torch.int32, device="cuda")
    prompts, gen, siblings = [None] * B, [[] for _ in range(B)], [0] * B

    def begin(b, lengths):
        prompts[b] = [tokens(cfg, n, 100 * b + n) for n in lengths]
        gen[b] = []
        text, uncond = (p.cuda() for p in prompts[b])
        if cfg_w:
            eng.prefill_cfg(text, uncond, 7 + b, image=b)
        else:
            eng.prefill_image(b, text, 7 + b)

    def run(first):
        """STEPS of them, and more until every image has had a sibling accepted."""
        for i in range(first, first + MOST):
            if i >= first + STEPS and min(siblings) > 0:
                return
            eng.step(0.5, 40, 5, i, out_meta=meta, out_tok=tok)
            for b, (m, t) in enumerate(zip(meta.tolist(), tok.tolist())):
                gen[b] += t[:m[0]]
                siblings[b] += m[5] >= 2
                assert m[7] == len(prompts[b][0]) + len(gen[b]) - 1

    def check(seed):
        drafts = [tokens(cfg, L, seed + b, vis=True) for b in range(B)]
        for b in range(B):
            # (a row end takes eol_id and counts as accepted whatever was fed: steps go on
            # from here, so that is what the drafts hold there)
            at = (torch.arange(L) + len(gen[b])) % (cfg["row_len"] + 1) == cfg["row_len"]
            drafts[b][at] = cfg["eol_id"]
            eng.set_drafts(drafts[b].cuda(), image=b)
        eng.forward_window(out)
        for b in range(B):
            ref = [window(cfg, w, p, gen[b], drafts[b], flags != sjd.SJD_ROPE_GRID)
                   for p in prompts[b][:2 if cfg_w else 1]]
            want = ref[1] + cfg_w * (ref[0] - ref[1]) if cfg_w else ref[0]
            err = (out[32 * b:32 * b + L].cpu().double() - want).abs().max().item()
            print("image", b, "after", len(gen[b]), "tokens,", siblings[b], "siblings: max error", err)
            assert err < bound(flags), b

    for b in range(B):
        begin(b, PROMPTS[b])
    run(0)
    assert min(siblings) > 0
    check(60)
    if B > 1:
        begin(1, AGAIN)
        siblings[1] = 0
    run(1000)
    assert min(siblings) > 0
    check(80)
    eng.close()


def test_rows_that_did_not_move_show():
    """(CPU) What a sibling's row that stays behind does to the logits, planted in the
    plain decoder: the rejected draft's token in its place, in one stream of two."""
    for model in MODELS:
        for flags in FLAGS:
            cfg = config(flags, **model)
            w = model_weights(cfg, 3, std=STD)
            prompt, gen, drafts = tokens(cfg, 90, 1), tokens(cfg, 45, 2, vis=True).tolist(), tokens(cfg, 16, 3, vis=True)
            good = window(cfg, w, prompt, gen, drafts, flags != sjd.SJD_ROPE_GRID)
            for at in (3, 20, 40):
                wrong = list(gen)
                wrong[at] = cfg["vis_lo"] + (wrong[at] - cfg["vis_lo"] + 17) % cfg["V"]
                off = (window(cfg, w, prompt, wrong, drafts, flags != sjd.SJD_ROPE_GRID) - good).abs().max().item()
                assert 0.5 * off > 2 * bound(flags), (flags, at, off)

"""Generations over pages launch k + 1 rows in every step, whether a draft was found or not.  Rows without a token leave nothing in the cache: a sequence's logits are those of steps
without such rows, whatever ran on the context before."""
import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu
CFG = synth.ModelCfg("paddings", 2, 512, 8, 64, 1024, 1040, "bf16")


def scaled(w, by):
    """layer 1's V `by` times as large, its output projection as much smaller: the same model, with layers whose pages have other scales"""
    f32 = lambda b: (b.astype(np.uint32) << 16).view(np.float32)
    lw = w["layers"][1]
    for name, rows, x in (("wqkv", slice(2 * CFG.d_model, None), by), ("wo", slice(None), 1.0 / by)):
        a = f32(lw[name]).copy()
        a[rows] *= x
        lw[name] = (a.view(np.uint32) >> 16).astype(np.uint16)
    return w


@pytest.fixture(scope="module")
def made():
    import paper_2304_04487_amd as llma
    w = scaled(synth.make_weights(CFG, 17), 1024.0)
    return llma, lambda k: llma.Context(CFG, w, max_seq=200, max_batch=2, max_k=k, kv_paged=True)


@pytest.mark.parametrize("prompt", [3, 40])
@pytest.mark.parametrize("k", [12, 32])
def test_a_generation_does_not_depend_on_what_ran_before(made, prompt, k):
    llma, make = made
    rng = np.random.default_rng(prompt + k)
    p = rng.integers(0, CFG.vocab, prompt)
    ref = (rng.integers(0, CFG.vocab, 30), [0, 30])
    seen = []
    for before in ([], [90], [5, 150], [150, 2]):
        ctx = make(k)
        ctx.enable_logits_dump(k + 1)
        for n in before:
            ctx.prefill(rng.integers(0, CFG.vocab, n), seq=1)
            ctx.verify_step(rng.integers(0, CFG.vocab, k), seq=1)
            ctx.reset(1)
        y, trace = ctx.generate(p, *ref, 2, k, 6)
        ctx.verify_step([])
        seen.append((y.tolist(), trace, ctx.logits(1)))
        ctx.close()
    for s in seen[1:]:
        assert s[0] == seen[0][0] and s[1] == seen[0][1] and np.array_equal(s[2], seen[0][2]), float(np.abs(s[2] - seen[0][2]).max())


@pytest.mark.parametrize("prompt", [3, 40, 62])
def test_logits_are_those_of_single_steps(made, prompt):
    """a generation without drafts, k = 12, against steps of one row; attention cuts its pages by the rows of a call, so sums may be added in another order: 2^-16
    of the largest logit, four hundred times what one layer's rounding in the pages makes of it"""
    llma, make = made
    rng = np.random.default_rng(prompt)
    p = rng.integers(0, CFG.vocab, prompt)
    ctx, one = make(12), make(0)
    ctx.enable_logits_dump(13)
    one.enable_logits_dump(1)
    y, trace = ctx.generate(p, rng.integers(0, CFG.vocab, 30), [0, 30], 3, 12, 7)
    assert all(t[0] == 1 for t in trace)                                 # (no draft was found)
    one.prefill(p)
    got = [one.verify_step([])[1] for _ in range(7)]
    assert y.tolist() == got
    assert ctx.verify_step([])[1] == one.verify_step([])[1]
    want = one.logits(1)
    assert np.abs(ctx.logits(1) - want).max() <= 2.0 ** -16 * np.abs(want).max(), float(np.abs(ctx.logits(1) - want).max() / np.abs(want).max())
    ctx.close(), one.close()


def test_batched_generations_leave_no_padding_either(made):
    """three sequences without drafts, k = 12, against steps of one row.  Rows without a token carry token 0, whose V is here a thousand times any other's in layer 0: one feature
    that only its embedding has, with large weights"""
    llma, _ = made
    rng = np.random.default_rng(9)
    w = synth.make_weights(CFG, 17)
    w["embed"] = w["embed"].copy()
    w["embed"][0], w["embed"][:, 3] = 0, 0
    w["embed"][0, 3] = 0x3F80                                            # 1
    w["layers"][0]["wqkv"] = w["layers"][0]["wqkv"].copy()
    w["layers"][0]["wqkv"][2 * CFG.d_model:, 3] = 0x4248                 # 50
    ctx, one = llma.Context(CFG, w, max_seq=200, max_batch=3, max_k=12, kv_paged=True), llma.Context(CFG, w, max_seq=200, max_batch=1, max_k=0, kv_paged=True)
    one.enable_logits_dump(1)
    ctx.enable_logits_dump(39)
    prompts = [rng.integers(1, CFG.vocab, n) for n in (33, 60, 7)]
    none = (rng.integers(1, CFG.vocab, 30), [0, 30])
    out = ctx.generate_batch(prompts, [none] * 3, 4, 12, 9)
    for s, p in enumerate(prompts):
        one.reset()
        one.prefill(p)
        y = [one.verify_step([])[1] for _ in range(9)]
        assert out[s][0].tolist() == y
        want = one.verify_step([])
        logits = one.logits(1)
        got = ctx.verify_step([], seq=s)
        assert got[1] == want[1]
        assert np.abs(ctx.logits(1) - logits).max() <= 2.0 ** -16 * np.abs(logits).max(), float(np.abs(ctx.logits(1) - logits).max() / np.abs(logits).max())
    ctx.close(), one.close()


@pytest.mark.parametrize("prompt", [1, 30, 64, 150])
def test_steps_do_not_depend_on_what_ran_before(made, prompt):
    """prompts, steps of several widths, batches and imports on a context whose pages and buffers other sequences have used, and on a new one"""
    import torch
    llma, make = made
    rng = np.random.default_rng(prompt)
    p, drafts = rng.integers(0, CFG.vocab, prompt), rng.integers(0, CFG.vocab, (4, 12))
    shape = (CFG.n_heads, 70, CFG.head_dim)
    kv = [[torch.tensor(rng.standard_normal(shape), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    seen = []
    for used in (False, True):
        ctx = make(12)
        ctx.enable_logits_dump(26)
        if used:
            for s in range(2):
                ctx.prefill(rng.integers(0, CFG.vocab, 170 - 60 * s), seq=s)
                ctx.verify_step(rng.integers(0, CFG.vocab, 12), seq=s)
            ctx.generate_batch([rng.integers(0, CFG.vocab, 33)] * 2, [None] * 2, 1, 12, 20)
            for s in range(2):
                ctx.reset(s)
        out = []
        ctx.prefill(p, seq=1)
        for d in (drafts[0], drafts[1][:3], drafts[2][:0]):
            out.append(ctx.verify_step(d, seq=1))
            out.append(ctx.logits(len(d) + 1))
        for l in range(2):
            ctx.kv_import(0, l, *kv[l], 70)
        ctx.set_pending(5, 0)
        out.append([x.tolist() if hasattr(x, "tolist") else x for x in ctx.verify_step_batch([0, 1], drafts[:2])])
        out.append(ctx.logits(26))
        out.append(ctx.verify_step_sampled(drafts[3], 0.9, np.full(12, 0.01, np.float32), 0.37, seq=1))
        out.append(ctx.logits(13))
        seen.append(out)
        ctx.close()
    for a, b in zip(*seen):
        assert np.array_equal(a, b) if isinstance(a, np.ndarray) else a == b

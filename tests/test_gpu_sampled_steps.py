"""llma_verify_step_sampled: the tokens are those that the plain form draws from the very logits that the step computed (dumped), state and refusals are a
verification step's."""
import numpy as np
import pytest

import paged_oracle
import synth

pytestmark = pytest.mark.gpu
CFGS = {"fp32": synth.ModelCfg("s32", 2, 128, 4, 32, 256, 333, "fp32"), "bf16": synth.ModelCfg("s16", 2, 512, 8, 64, 1024, 1040, "bf16")}


@pytest.fixture(scope="module", params=["fp32", "bf16", "paged"])
def setup(request):
    import paper_2304_04487_amd as llma
    cfg = CFGS["fp32" if request.param == "fp32" else "bf16"]
    w = synth.make_weights(cfg, 31)
    make = lambda **kw: llma.Context(cfg, w, kv_paged=request.param == "paged", **kw)
    return llma, cfg, make


def test_tokens_are_those_of_the_dumped_logits(setup):
    llma, cfg, make = setup
    ctx, rng = make(max_seq=200, max_batch=1, max_k=9), np.random.default_rng(2)
    ctx.enable_logits_dump(10)
    prompt = rng.integers(0, cfg.vocab, 50)
    ctx.prefill(prompt)
    T, pending, accepted = 49, int(prompt[-1]), 0
    for step in range(14):
        k, temp = int(rng.integers(0, 10)), float(rng.choice([0.0, 0.05, 0.2, 1.0]))
        draft = rng.integers(0, cfg.vocab, k)
        if step:
            draft[:1] = last                                # likely: the favourite of a row before
        ua, us = rng.random(k, dtype=np.float32) * np.float32(0.01), float(rng.random(dtype=np.float32))
        a, nxt, emitted = ctx.verify_step_sampled(draft, temp, ua, us)
        logits = ctx.logits(k + 1).astype(np.float64)
        n, token, want, near = paged_oracle.verify(logits, draft, k, None, float(np.float32(temp)), ua, np.float32(us))
        assert near > 1e-13 and (a, nxt, emitted) == (n, token, want)
        T, pending, accepted = T + a + 1, nxt, accepted + a
        assert ctx.get_state() == (T, pending)
        last = int(logits[n].argmax())
    ctx.close()


def test_temperature_zero_is_the_greedy_step(setup):
    llma, cfg, make = setup
    a, b = (make(max_seq=150, max_batch=6, max_k=8) for _ in range(2))
    rng = np.random.default_rng(3)
    for ctx in (a, b):
        for s in range(6):
            ctx.prefill(np.arange(5 + s) * 7 % cfg.vocab, seq=s)
    for B, k in ((6, 8), (2, 3), (1, 0), (6, 8), (6, 8)):    # 54 rows and few; eager, captured, replayed
        seqs = [int(s) for s in rng.permutation(6)[:B]]
        drafts = rng.integers(0, cfg.vocab, (B, k))
        want = a.verify_step_batch(seqs, drafts)
        got = b.verify_step_sampled_batch(seqs, drafts, np.zeros(B), rng.random((B, k)) * 0.99, rng.random(B) * 0.99)
        assert got[0].tolist() == want[0].tolist() and got[1].tolist() == want[1].tolist() and got[2] == want[2]
        for s in range(6):
            assert a.get_state(s) == b.get_state(s)
    a.close(), b.close()


def test_mixed_with_greedy_steps_and_other_sizes(setup):
    """memory grows with the rows, graphs of earlier steps do not outlive it; a batch row per sequence against the plain form"""
    llma, cfg, make = setup
    ctx, rng = make(max_seq=150, max_batch=4, max_k=6), np.random.default_rng(4)
    for s in range(4):
        ctx.prefill(np.arange(3 + 9 * s) % cfg.vocab, seq=s)
    for turn in range(9):
        B, k = [(1, 2), (1, 2), (4, 6), (2, 0), (1, 2), (4, 6), (4, 6), (3, 5), (1, 2)][turn]
        if turn == 6:
            ctx.enable_logits_dump(28)
        seqs = [int(s) for s in rng.permutation(4)[:B]]
        drafts, ua, us = rng.integers(0, cfg.vocab, (B, k)), rng.random((B, k), dtype=np.float32), rng.random(B, dtype=np.float32)
        before = [ctx.get_state(s)[0] for s in seqs]
        na, nt, em = ctx.verify_step_sampled_batch(seqs, drafts, np.full(B, 0.7), ua, us)
        for b, s in enumerate(seqs):
            assert ctx.get_state(s) == (before[b] + na[b] + 1, nt[b]) and em[b][:-1] == drafts[b][:na[b]].tolist() and em[b][-1] == nt[b]
        if turn >= 6:
            logits = ctx.logits(B * (k + 1)).reshape(B, k + 1, -1).astype(np.float64)
            for b in range(B):
                n, token, want, near = paged_oracle.verify(logits[b], drafts[b], k, None, float(np.float32(0.7)), ua[b], us[b])
                assert near > 1e-13 and (na[b], nt[b], em[b]) == (n, token, want)
        ctx.verify_step(rng.integers(0, cfg.vocab, 2), seq=seqs[0])
    ctx.close()


def test_refusals_leave_the_context_as_it_was(setup):
    llma, cfg, make = setup
    ctx = make(max_seq=40, max_batch=2, max_k=4)
    with pytest.raises(llma.LlmaError) as e:
        ctx.verify_step_sampled([1], 1.0, [0.5], 0.5)
    assert e.value.code == llma.LLMA_E_STATE
    ctx.prefill(np.arange(9))
    nan = float("nan")
    for draft, t, ua, us in (([1], -0.5, [0.5], 0.5), ([1], nan, [0.5], 0.5), ([1], float("inf"), [0.5], 0.5), ([1], 1.0, [1.0], 0.5), ([1], 1.0, [-0.1], 0.5), ([1], 1.0, [0.5], 1.0),
                             ([1], 1.0, [0.5], nan), ([cfg.vocab], 1.0, [0.5], 0.5), ([1] * 5, 1.0, [0.5] * 5, 0.5)):
        with pytest.raises(llma.LlmaError) as e:
            ctx.verify_step_sampled(draft, t, ua, us)
        assert e.value.code == llma.LLMA_E_RANGE
    with pytest.raises(llma.LlmaError):
        ctx.verify_step_sampled([1, 2], 1.0, [0.5], 0.5)
    assert ctx.get_state() == (8, 8)
    ctx.verify_step_sampled([1], 1.0, [0.5], 0.5)
    ctx.close()

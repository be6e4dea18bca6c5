"""A batched step one of whose rows has no token (its logits are NaN): the call reports it, and all of its slots stay as they were, for what reads them and for the steps
that follow."""
import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu
CFGS = {"fp32": synth.ModelCfg("f32", 2, 128, 4, 32, 256, 333, "fp32"), "bf16": synth.ModelCfg("f16", 2, 512, 8, 64, 1024, 1040, "bf16")}
POISON = 7                                                               # a token whose embedding is NaN


@pytest.mark.parametrize("kind", ["fp32", "bf16", "paged"])
def test_a_failed_batch_leaves_its_slots_as_they_were(kind):
    import paper_2304_04487_amd as llma
    cfg = CFGS["fp32" if kind == "fp32" else "bf16"]
    w = synth.make_weights(cfg, 31)
    w["embed"] = w["embed"].copy()
    w["embed"][POISON] = np.float32("nan") if kind == "fp32" else 0x7FC0
    a, b = (llma.Context(cfg, w, max_seq=120, max_batch=3, max_k=4, kv_paged=kind == "paged") for _ in range(2))
    prompts = [np.array([9, 8, 11 + s, 20]) for s in range(3)]
    for ctx in (a, b):
        for s, p in enumerate(prompts):
            ctx.prefill(p, seq=s)
    rng = np.random.default_rng(3)
    for turn in range(4):                                                # eager, captured, replayed
        k = 3
        drafts, ua, us = rng.integers(10, cfg.vocab, (3, k)), rng.random((3, k), dtype=np.float32), rng.random(3, dtype=np.float32)
        before = [a.get_state(s) for s in range(3)]
        pending = before[1][1]
        a.set_pending(POISON, seq=1)
        with pytest.raises(llma.LlmaError) as e:
            a.verify_step_sampled_batch([0, 1, 2], drafts, np.full(3, 0.7), ua, us)
        assert e.value.code == llma.LLMA_E_HIP
        assert [a.get_state(s) for s in range(3)] == [before[0], (before[1][0], POISON), before[2]]
        a.set_pending(pending, seq=1)
        got, want = (c.verify_step_sampled_batch([0, 1, 2], drafts, np.full(3, 0.7), ua, us) for c in (a, b))
        assert got[0].tolist() == want[0].tolist() and got[1].tolist() == want[1].tolist() and got[2] == want[2]
        assert [a.get_state(s) for s in range(3)] == [b.get_state(s) for s in range(3)]
        if turn == 1:                                                    # a greedy step behind a failed one
            a.set_pending(POISON, seq=1)
            with pytest.raises(llma.LlmaError):
                a.verify_step_sampled_batch([2, 1], drafts[:2], np.full(2, 0.7), ua[:2], us[:2])
            a.set_pending(b.get_state(1)[1], seq=1)
            got, want = (c.verify_step_batch([2, 0, 1], drafts) for c in (a, b))
            assert got[0].tolist() == want[0].tolist() and got[1].tolist() == want[1].tolist() and got[2] == want[2]
    a.close(), b.close()

"""Contexts whose cache lies in 8-bit pages (kv_split = LLMA_KV_PAGED): logits of prompts, steps, imports and batches against the float64 oracle over a
cache that is rounded the same way, and generations whose text is known.

Rounding to codes is a step function: a value that the library has 1e-6 beside the oracle's may fall to the other side of a border, and in a second
layer such differences feed on themselves.  So the model of these tests has one layer whose K and V are known to lie far from any border:
embeddings are +-1 (their norm is 1), a K or V feature is a sum of five of them with weights 1, 1/2, 1/4, 1/8 and 1/32 -- a value of four significant bits and a quarter
of a step -- and the rotary base is so large that the features of K that are not zero are not rotated.

Tolerance: ATOL is what the tests of two layers of this width with a two-plane cache allow (four times their measured error)."""
import numpy as np
import pytest

import paged_oracle
import synth
from oracle import OracleModel

pytestmark = pytest.mark.gpu

CFG = synth.ModelCfg("paged", 1, 1152, 9, 128, 2848, 1040, "bf16", rope_theta=1e30)
CFG64 = synth.ModelCfg("paged64", 1, 512, 8, 64, 1024, 1040, "bf16", rope_theta=1e30)
GEN = synth.ModelCfg("pagedgen", 2, 512, 8, 64, 1024, 1040, "bf16")
ATOL = 1e-3
PAGE = 64
DOUBT = 2.0 ** -14         # the library's K and V against the oracle's, relative to the largest: operands kept to 16 bits, some hundred addends


def to_bf16(x):
    b = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((b + 0x7FFF + (b >> 16 & 1)) >> 16 << 16).astype(np.uint32).view(np.float32).astype(np.float64)


class Plane:
    """a layer's K or V [heads, capacity, dh] that is rounded, page by page, as it is written"""

    def __init__(self, heads, capacity, dh):
        blocks = (capacity + PAGE - 1) // PAGE
        self.values, self.scale = np.zeros((blocks, heads, PAGE, dh)), np.ones((blocks, heads))
        self.nudge, self.doubtful = None, []               # an element to move across its border; the elements next to one

    def __setitem__(self, key, rows):                      # [:, T:T+m, :] = [heads, m, dh]
        at, off = key[1], DOUBT * np.abs(rows).max()
        x = to_bf16(rows)
        if self.nudge is not None:
            x[self.nudge[0]] = self.nudge[1]
        paged_oracle.append(self.values, self.scale, x.transpose(1, 0, 2), np.arange(at.start, at.stop))
        unit = np.stack([self.scale[p // PAGE] for p in range(at.start, at.stop)], 1)[..., None]
        self.doubtful = [(tuple(i), v[tuple(i)]) for v in (to_bf16(rows - off), to_bf16(rows + off))
                         for i in np.argwhere(paged_oracle.to_e4m3(v / unit) != paged_oracle.to_e4m3(x / unit))]

    def __getitem__(self, key):
        v = self.values * self.scale[..., None, None]
        return v.transpose(1, 0, 2, 3).reshape(v.shape[1], -1, v.shape[3])[key]


class Oracle(OracleModel):
    def new_cache(self, capacity):
        c = super().new_cache(1)
        for planes in (c.k, c.v):
            planes[:] = [Plane(self.cfg.n_heads, capacity, self.cfg.head_dim) for _ in planes]
        return c


def bits(a):
    return (to_bf16(a).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def stepped(cfg):
    rng = np.random.default_rng(7)
    w = synth.make_weights(cfg, 31, gain_jitter=0.2)
    d, dh = cfg.d_model, cfg.head_dim
    w["embed"] = bits(rng.choice([-1.0, 1.0], (cfg.vocab, d)))
    for lw in w["layers"]:
        lw["norm1"][:] = 1.0
        kv = np.zeros((2 * d, d))
        for f in range(2 * d):
            if f >= d or f % dh % (dh // 2) >= int(0.35 * dh):         # (K: the pairs that turn are zero)
                kv[f, rng.choice(d, 5, replace=False)] = np.array([1, 0.5, 0.25, 0.125, 0.03125]) * 2.0 ** rng.integers(-2, 3)
        lw["wqkv"][d:] = bits(kv)
        lw["wqkv"][:d] = bits(0.15 * rng.standard_normal((d, d)))
        lw["wo"] = bits(0.1 * rng.standard_normal((d, d)))
    return w


@pytest.fixture(scope="module", params=[CFG, CFG64], ids=lambda c: c.name)
def setup(request):
    import paper_2304_04487_amd as llma
    cfg = request.param
    w = stepped(cfg)
    return llma, cfg, w, Oracle(cfg, w), OracleModel(cfg, w)


@pytest.mark.parametrize("prompt,k", [(1, 0), (40, 3), (64, 8), (65, 8), (130, 16), (260, 8)])
def test_prompt_and_steps(setup, prompt, k):
    """several steps, drafts accepted in part, the cache truncated behind them: eager, captured and replayed launches"""
    llma, cfg, w, om, plain = setup
    ctx = llma.Context(cfg, w, max_seq=prompt + 80, max_batch=2, max_k=16, kv_paged=True)
    ctx.enable_logits_dump(k + 1)
    p = synth.uniform_tokens(5, prompt, prompt, cfg.vocab)
    cache, T = om.new_cache(prompt + 80), prompt - 1
    unrounded = plain.new_cache(prompt + 80)
    if T:
        om.forward(p[:-1], cache, 0)
        plain.forward(p[:-1], unrounded, 0)
    ctx.prefill(p, seq=1)
    pending, away = int(p[-1]), 0.0
    for step in range(4):
        draft = synth.uniform_tokens(6, 10 * prompt + step, k, cfg.vocab)
        if k and step % 2 == 0:                            # the first draft is the model's own choice
            probe = om.new_cache(prompt + 80)
            for a, b in zip(probe.k + probe.v, cache.k + cache.v):
                a.values, a.scale = b.values.copy(), b.scale.copy()
            draft[0] = int(np.argmax(om.forward([pending], probe, T)[0]))
        want = om.forward([pending] + draft.tolist(), cache, T)
        away = max(away, float(np.abs(plain.forward([pending] + draft.tolist(), unrounded, T) - want).max()))
        a, nxt, emitted = ctx.verify_step(draft, seq=1)
        err = float(np.abs(ctx.logits(k + 1) - want).max())
        assert err <= ATOL, (step, err)
        top = np.argmax(want, axis=1)
        assert a >= (1 if k and step % 2 == 0 else 0) and nxt == top[a] and emitted == top[:a + 1].tolist()
        T, pending = T + a + 1, nxt
        assert ctx.get_state(1) == (T, pending)
    assert prompt < 40 or away > 2 * ATOL                  # (the rounding is there to be seen)
    ctx.close()


def test_batched_steps_and_shared_prompts(setup):
    llma, cfg, w, om, _ = setup
    lens, k = (66, 3, 130, 1, 64), 10
    B = len(lens)
    ctx = llma.Context(cfg, w, max_seq=170, max_batch=B + 2, max_k=k, kv_paged=True)
    ctx.enable_logits_dump(B * (k + 1))
    prompts = [synth.uniform_tokens(8, b, n, cfg.vocab) for b, n in enumerate(lens)]
    slots = [4, 0, 6, 2, 5]
    for turn in range(3):
        out = ctx.generate_batch(prompts, [None] * B, 1, k, 1, seqs=slots)
        caches = [om.new_cache(170) for _ in lens]
        first = [om.forward(p, c, 0)[-1] for p, c in zip(prompts, caches)]
        nxt = [int(t[0]) for t, _ in out]
        for f, y in zip(first, nxt):
            assert f.max() - f[y] <= 2 * ATOL
        drafts = np.stack([synth.uniform_tokens(9, 7 * turn + b, k, cfg.vocab) for b in range(B)])
        na, nt, _ = ctx.verify_step_batch(slots, drafts)
        got = ctx.logits(B * (k + 1)).reshape(B, k + 1, -1)
        for b in range(B):
            want = om.forward([nxt[b]] + drafts[b].tolist(), caches[b], lens[b])
            assert float(np.abs(got[b] - want).max()) <= ATOL, (turn, b)
            assert ctx.get_state(slots[b])[0] == lens[b] + 1 + na[b]
    ctx.close()


def test_imported_caches(setup):
    """the imported values are rounded as the append rounds them.  Two layers with K and V like any model's: the five rows that the step computes
    may have codes on the other side of a border.  What each of those next to one does to the logits is computed, and all of it together allowed"""
    import torch
    llma, cfg, _, _, _ = setup
    cfg = synth.ModelCfg(cfg.name, 2, cfg.d_model, cfg.n_heads, cfg.head_dim, cfg.d_ffn, cfg.vocab, "bf16")
    w = synth.make_weights(cfg, 31, gain_jitter=0.2)
    om = Oracle(cfg, w)
    n = 150
    rng = np.random.default_rng(4)
    ctx = llma.Context(cfg, w, max_seq=200, max_batch=3, max_k=4, kv_paged=True)
    ctx.enable_logits_dump(5)
    for seq, n in ((2, 150), (0, 64), (2, 31)):
        cache = om.new_cache(200)
        for l in range(cfg.n_layers):
            k, v = (torch.tensor(rng.standard_normal((cfg.n_heads, n, cfg.head_dim)), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            cache.k[l][:, 0:n, :], cache.v[l][:, 0:n, :] = k.double().cpu().numpy(), v.double().cpu().numpy()
            ctx.kv_import(seq, l, k, v, n)
        ctx.set_pending(7, seq)
        draft = [3, 9, 1, 500]
        planes = cache.k + cache.v
        before = [(x.values.copy(), x.scale.copy()) for x in planes]
        want = om.forward([7] + draft, cache, n)
        tol = np.full_like(want, ATOL)
        for plane, nudge in [(x, d) for x in planes for d in x.doubtful]:
            for x, (values, scale) in zip(planes, before):
                x.values, x.scale, x.nudge = values.copy(), scale.copy(), None
            plane.nudge = nudge
            tol += np.abs(om.forward([7] + draft, cache, n) - want)
        ctx.verify_step(draft, seq=seq)
        assert (np.abs(ctx.logits(5) - want) <= tol).all() and tol.mean() <= 20 * ATOL, n
    ctx.close()


def chain(cfg, seed):
    """weights whose favourite after token t is next(t), far above the rest: LM-head row next(v) is v's embedding"""
    w = synth.make_weights(cfg, seed)
    rng = np.random.default_rng(seed)
    e = to_bf16(rng.standard_normal((cfg.vocab, cfg.d_model)))
    order = rng.permutation(cfg.vocab)
    nxt = np.empty(cfg.vocab, int)
    nxt[order] = np.roll(order, -1)
    head = np.empty_like(e)
    head[nxt] = e / np.sqrt(cfg.d_model)
    w["embed"], w["lm_head"] = bits(e), bits(head)
    return w, nxt


def follow(nxt, t, n):
    out = []
    for _ in range(n):
        t = int(nxt[t])
        out.append(t)
    return out


def test_generations_over_reused_slots():
    """generations of all kinds, one after the other on the same slots: pages come back, text and traces are those of a two-plane cache"""
    import paper_2304_04487_amd as llma
    cfg = GEN
    w, nxt = chain(cfg, 3)
    ctx = llma.Context(cfg, w, max_seq=330, max_batch=6, max_k=12, kv_paged=True)
    planes = llma.Context(cfg, w, max_seq=330, max_batch=6, max_k=12)
    rng = np.random.default_rng(1)
    for turn in range(10):
        B = int(rng.integers(1, 7))
        k = int(rng.integers(0, 13))
        prompts = [rng.integers(0, cfg.vocab, int(rng.integers(1, 200))) for _ in range(B)]
        texts = [follow(nxt, int(p[-1]), 90) for p in prompts]
        refs = [(np.array(t[5:40] + list(rng.integers(0, cfg.vocab, 9)) + t[50:80]), [0, 30, 74]) for t in texts]
        seqs = [int(s) for s in rng.permutation(6)[:B]]
        got = ctx.generate_batch(prompts, refs, 1, k, 90, seqs=seqs)
        want = planes.generate_batch(prompts, refs, 1, k, 90, seqs=seqs)
        for (y, trace), (y2, trace2), t in zip(got, want, texts):
            assert y.tolist() == t and y2.tolist() == t
            assert trace == trace2
            assert k < 4 or len(trace) < 90
        one = ctx.generate(prompts[0], *refs[0], 1, k, 90, seq=seqs[0])
        assert one[0].tolist() == texts[0] and one[1] == got[0][1]
        for s in range(6):
            assert ctx.get_state(s) == planes.get_state(s)
    ctx.close()
    planes.close()


def test_a_third_of_the_cache_bytes():
    import paper_2304_04487_amd as llma
    w = synth.make_weights(GEN, 3)
    size = {}
    for paged in (False, True):
        a, b = (llma.Context(GEN, w, max_seq=n, max_batch=4, max_k=4, kv_paged=paged) for n in (2048, 4096))
        size[paged] = b.device_bytes() - a.device_bytes()
        a.close(), b.close()
    # per position, slot and layer: 3 bytes of K and V each against one and 8 / 64 bytes of scales; shared: rotary table, scratch of longer prompts
    assert size[True] < size[False] - 2048 * 4 * 2 * 512 * 3.9


def test_refusals():
    import paper_2304_04487_amd as llma
    w = synth.make_weights(CFG64, 3)
    with pytest.raises(llma.LlmaError) as e:
        llma.Context(CFG64, w, max_seq=128, max_batch=5000, max_k=4, kv_paged=True)
    assert e.value.code == llma.LLMA_E_INVAL and "paged" in str(e.value)
    ctx = llma.Context(CFG64, w, max_seq=64, max_batch=1, max_k=4, kv_paged=True)
    ctx.prefill(np.arange(62))
    with pytest.raises(llma.LlmaError) as e:
        ctx.verify_step([1, 2, 3, 4])
    assert e.value.code == llma.LLMA_E_RANGE
    ctx.verify_step([1, 2])
    ctx.close()

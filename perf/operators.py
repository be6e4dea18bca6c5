"""The stateless operators of serving on pages, as timed cases: pages and slots of a step from the sequences' lengths, the
write into the 8-bit paged cache, attention over that cache, and verification of drafts with given random numbers.

`run` computes each in a plain form (elementary torch operations) or, with `own`, through the package's public calls.

Cache: pages of 64 positions; k [pages, kv heads, 64, head_dim] and v [pages, kv heads, head_dim, 64] hold e4m3 codes,
k_scale and v_scale [pages, kv heads] powers of two; a cached value is code * scale.  table [slots, blocks] names a
sequence's pages in order.
"""
import math

import torch

own = False

PAGE = 64
F8 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


# ------------------------------------------------------------------------------------------------ what is measured
def listed():
    return [
        # pages and slots of one step: a handful of sequences, nine rows each (one copied span of eight)
        {"name": "map_step_16", "kind": "map", "seqs": 16, "past": 4096, "rows": 9},
        # prompts of many requests enter together: tens of thousands of rows, hundreds of fresh pages
        {"name": "map_prompts_512", "kind": "map", "seqs": 512, "past": 700, "rows": 130},
        # the rows of a verification step of 16 sequences, one layer of the 7B shape
        {"name": "append_step_7b", "kind": "append", "seqs": 16, "past": 4096, "rows": 9, "kv_heads": 32, "head_dim": 128, "type": "bf16"},
        # prompts of four requests, shared key/value heads, float32 rows straight from a projection
        {"name": "append_prompts_gqa", "kind": "append", "seqs": 4, "past": 100, "rows": 2011, "kv_heads": 8, "head_dim": 128, "type": "fp32"},
        # one sequence of the d 512 model, plain decoding: a few launches
        {"name": "attend_one_d512", "kind": "attend", "seqs": 1, "past": 1001, "rows": 1, "heads": 8, "kv_heads": 8, "head_dim": 64, "type": "bf16"},
        # the same model's verification step in float32
        {"name": "attend_six_f32", "kind": "attend", "seqs": 6, "past": 1300, "rows": 9, "heads": 8, "kv_heads": 8, "head_dim": 64, "type": "fp32"},
        # 16 long sequences of the 7B shape, k = 8
        {"name": "attend_16x4096_7b", "kind": "attend", "seqs": 16, "past": 4096, "rows": 9, "heads": 32, "kv_heads": 32, "head_dim": 128, "type": "bf16"},
        # many ragged sequences, four query heads to a key head
        {"name": "attend_gqa_ragged", "kind": "attend", "seqs": 61, "past": 8000, "rows": 5, "heads": 32, "kv_heads": 8, "head_dim": 128, "type": "fp16"},
        # prompt rows on top of a long cache: bound by the products
        {"name": "attend_prompt_2047", "kind": "attend", "seqs": 2, "past": 2900, "rows": 2047, "heads": 32, "kv_heads": 8, "head_dim": 128, "type": "bf16"},
        # one sequence's copied span of eight, sampled
        {"name": "verify_one", "kind": "verify", "seqs": 1, "k": 8, "vocab": 32000, "type": "fp32", "probs": False},
        # a batch with long spans and mixed temperatures
        {"name": "verify_16x33", "kind": "verify", "seqs": 16, "k": 32, "vocab": 32000, "type": "fp32", "probs": False},
        # a draft model's probabilities over a large vocabulary
        {"name": "verify_64_probs", "kind": "verify", "seqs": 64, "k": 5, "vocab": 128256, "type": "bf16", "probs": True},
    ]


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    kind = rng.choice(["map", "append", "attend", "attend", "attend", "verify", "verify"])
    if kind == "map":
        rows = log(1, 130)
        return {"kind": kind, "seqs": log(1, 60000 // rows if rows > 117 else 512), "past": log(16, 4096), "rows": rows}
    if kind == "append":
        heads, rows = rng.choice([1, 8, 32]), log(1, 2011)
        return {"kind": kind, "seqs": max(1, log(1, max(1.5, min(64, 64000 / (heads * rows))))), "past": log(16, 4096), "rows": rows, "kv_heads": heads,
                "head_dim": rng.choice([64, 128]), "type": rng.choice(["bf16", "fp16", "fp32"])}
    if kind == "attend":
        kv = rng.choice([1, 2, 8, 32])
        heads = kv * rng.choice([1, 4, 8] if kv < 32 else [1])
        rows = rng.choice([1, log(2, 33), log(34, 1500)])
        past = log(16, 8000)
        cost = heads * rows * (past + rows)
        seqs = max(1, min(log(1, 64), int(2.5e8 / cost), int(70000 * 32 / (kv * (past + rows)))))
        return {"kind": kind, "seqs": seqs, "past": past, "rows": rows, "heads": heads, "kv_heads": kv, "head_dim": rng.choice([64, 128]),
                "type": rng.choice(["bf16", "bf16", "fp16", "fp32"])}
    vocab, k = log(500, 128256), rng.randint(0, 32)
    probs = rng.random() < 0.4
    return {"kind": kind, "seqs": max(1, min(log(1, 64), int(4e7 / (vocab * (k + 1))))), "k": k, "vocab": vocab, "type": rng.choice(["bf16", "fp16", "fp32"]), "probs": probs and k > 0}


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 7919 + 11)


def _rand(shape, g, dtype=torch.float32):
    return torch.rand(shape, generator=g, device="cuda", dtype=dtype)


def _ints(lo, hi, shape, g):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)


def _offsets(n):
    z = torch.zeros(1, dtype=torch.int32, device=n.device)
    return torch.cat([z, torch.cumsum(n, 0, dtype=torch.int32)])


def _lengths(case, g):
    """lengths before the step and rows of it: ragged, the first sequence at the case's full size"""
    B, past, rows = case["seqs"], case["past"], case["rows"]
    lens = _ints(max(1, past // 3), past + 1, (B,), g)
    n = _ints(max(1, rows // 2), rows + 1, (B,), g)
    lens[0], n[0] = past, rows
    return lens, n


def _table(total, max_blocks, n_pages, g):
    """a table whose sequences own the pages of `total` positions, drawn from a shuffled pool; the rest of the pool in order"""
    perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    need = (total + PAGE - 1) // PAGE
    first = _offsets(need)[:-1]
    cols = torch.arange(max_blocks, device="cuda", dtype=torch.int32)
    at = (first[:, None] + cols[None]).clamp(max=n_pages - 1)
    return torch.where(cols[None] < need[:, None], perm[at.long()], -1).to(torch.int32), need, perm


def _powers(lo, hi, dtype):
    """2^lo .. 2^hi, exactly (the device's pow and ldexp are not)"""
    return torch.tensor([2.0 ** i for i in range(lo, hi + 1)], dtype=dtype, device="cuda")


def _pow2(amax, powers=None):
    """smallest power of two s with amax / s <= 448, between 2^-64 and 2^120"""
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(amax > 0, e, torch.full_like(e, -64)).clamp(-64, 120)
    return (_powers(-64, 120, torch.float32) if powers is None else powers)[e.long() + 64]


def _filled(n_pages, heads, dh, g):
    """codes and scales of a filled cache: normal values whose channels differ in size"""
    k = torch.empty((n_pages, heads, PAGE, dh), dtype=torch.uint8, device="cuda")
    v = torch.empty((n_pages, heads, dh, PAGE), dtype=torch.uint8, device="cuda")
    ks, vs = (torch.empty((n_pages, heads), device="cuda") for _ in range(2))
    size = torch.exp(0.4 * torch.randn((1, heads, 1, dh), generator=g, device="cuda"))
    step = max(1, (1 << 24) // (heads * PAGE * dh))
    for a in range(0, n_pages, step):
        x = torch.randn((min(step, n_pages - a), heads, PAGE, dh), generator=g, device="cuda")
        y = torch.randn((min(step, n_pages - a), heads, dh, PAGE), generator=g, device="cuda")
        x = x * size
        ks[a:a + step], vs[a:a + step] = _pow2(x.abs().amax((2, 3))), _pow2(y.abs().amax((2, 3)))
        k[a:a + step] = (x / ks[a:a + step, :, None, None]).to(F8).view(torch.uint8)
        v[a:a + step] = (y / vs[a:a + step, :, None, None]).to(F8).view(torch.uint8)
    return k, v, ks, vs


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    i32 = {"dtype": torch.int32, "device": "cuda"}
    if kind == "map":
        lens, rows = _lengths(case, g)
        B, blocks = case["seqs"], (case["past"] + case["rows"] + PAGE - 1) // PAGE
        n_pages = B * blocks
        table, owned, perm = _table(lens, blocks, n_pages, g)
        used = owned.sum()
        free = torch.full((n_pages,), -1, **i32)
        n_free = (n_pages - used).to(torch.int32).reshape(1)
        at = torch.arange(n_pages, device="cuda")
        free = torch.where(at < n_free, perm[(at + used).clamp(max=n_pages - 1)], free)
        accepted = torch.minimum((_rand((B,), g) * (rows + 1)).to(torch.int32), rows)       # rows of the step that stay
        cap = B * case["rows"]
        return {"kind": kind, "table": table, "owned": owned, "free": free, "n_free": n_free, "lens": lens, "rows": rows, "kept": lens + accepted,
                "none": torch.zeros_like(rows), "row_offsets": torch.empty(B + 1, **i32), "lens_after": torch.empty(B, **i32), "slot_map": torch.empty(cap, **i32),
                "row_pos": torch.empty(cap, **i32), "status": torch.empty(1, **i32), "row_offsets2": torch.empty(B + 1, **i32),
                "lens_after2": torch.empty(B, **i32), "status2": torch.empty(1, **i32)}
    if kind == "append":
        lens, rows = _lengths(case, g)
        B, H, dh = case["seqs"], case["kv_heads"], case["head_dim"]
        # the pool holds the pages that the step writes to and some of others
        first = lens // PAGE
        blocks = (lens + rows + PAGE - 1) // PAGE - first
        total = B * (case["rows"] // PAGE + 2) + 8
        perm = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
        off = _offsets(rows)
        n = B * case["rows"]                                                                # room for the most rows: padding behind the last sequence
        i = torch.arange(n, device="cuda", dtype=torch.int32)
        b = torch.searchsorted(off[1:], i, right=True).clamp(max=B - 1)
        pos = lens[b] + i - off[b]
        page = perm[(_offsets(blocks)[:-1][b] + pos // PAGE - first[b]).long().clamp(0, total - 1)]
        slot_map = torch.where(i < off[-1], page * PAGE + pos % PAGE, -1).to(torch.int32)
        cache = _filled(total, H, dh, g)
        # as a projection leaves them: keys and values side by side in one row; now and then a large value
        kv = torch.randn((n, 2, H, dh), generator=g, device="cuda")
        kv = (kv * torch.where(_rand((n, 2, H, 1), g) < 0.05, 40.0, 1.0)).to(TYPES[case["type"]])
        return {"kind": kind, "cache": cache, "k": kv[:, 0], "v": kv[:, 1], "slot_map": slot_map, "max_runs": n // PAGE + 2 * B,
                "powers": _powers(-64, 120, torch.float32)}
    if kind == "attend":
        lens, rows = _lengths(case, g)
        total = lens + rows
        B, H, dh, dt = case["seqs"], case["kv_heads"], case["head_dim"], TYPES[case["type"]]
        blocks = (case["past"] + case["rows"] + PAGE - 1) // PAGE
        n_pages = B * blocks
        table, need, _ = _table(total, blocks, n_pages, g)
        k, v, ks, vs = _filled(n_pages, H, dh, g)
        # what lies behind the last position of a sequence's last page is anything: NaN codes here
        last = table[torch.arange(B, device="cuda"), (need - 1).long()].long()
        behind = (torch.arange(PAGE, device="cuda")[None] >= ((total - 1) % PAGE + 1)[:, None])
        k[last] = torch.where(behind[:, None, :, None], 0x7F, k[last])
        v[last] = torch.where(behind[:, None, None, :], 0x7F, v[last])
        off = _offsets(rows)
        n = B * case["rows"]                                                                # room for the most rows: those behind the last sequence stay zero
        q = (1.5 * torch.randn((n, case["heads"], dh), generator=g, device="cuda")).to(dt)
        return {"kind": kind, "cache": (k, v, ks, vs), "table": table, "lens": total, "row_offsets": off, "q": q, "out": torch.zeros_like(q),
                "max_rows": case["rows"], "scale": 1.0 / math.sqrt(dh)}
    B, k, V = case["seqs"], case["k"], case["vocab"]
    logits = (2.0 * torch.randn((B, k + 1, V), generator=g, device="cuda")).to(TYPES[case["type"]])
    temperature = torch.where(_rand((B,), g) < 0.15, 0.0, 0.5 + _rand((B,), g))
    n_draft = _ints(max(0, k - 3), k + 1, (B,), g)
    n_draft[0] = k
    if case["probs"]:
        # a draft model that agrees with the target roughly, and tokens drawn from it
        q = torch.softmax(logits[:, :k].float() + 0.7 * torch.randn((B, k, V), generator=g, device="cuda"), -1)
        drafts = (torch.log(q) - torch.log(-torch.log(_rand((B, k, V), g).clamp(1e-20, 1 - 1e-7)))).argmax(-1).to(torch.int32)
    else:
        # copied tokens: mostly what the target likes best, some that it does not
        q = None
        drafts = torch.where(_rand((B, k), g) < 0.9, logits[:, :k].argmax(-1).to(torch.int32), _ints(0, V, (B, k), g))
        at = drafts.long()[..., None]
        logits[:, :k].scatter_(-1, at, (logits[:, :k].gather(-1, at).float() + 7.0).to(logits.dtype))
    i32 = {"dtype": torch.int32, "device": "cuda"}
    return {"kind": "verify", "logits": logits, "drafts": drafts, "n_draft": n_draft, "temperature": temperature, "probs": q, "u_accept": _rand((B, k), g),
            "u_sample": _rand((B,), g), "n_accepted": torch.empty(B, **i32), "next": torch.empty(B, **i32), "emitted": torch.empty((B, k + 1), **i32)}


# ------------------------------------------------------------------------------------------------ the plain forms
def _map_plain(s, lens, rows, n_rows):
    table, owned, free, n_free = s["table"], s["owned"], s["free"], s["n_free"]
    after = lens + rows
    need = (after + PAGE - 1) // PAGE
    back, more = (owned - need).clamp(min=0), (need - owned).clamp(min=0)
    back_at, more_at = _offsets(back), _offsets(more)
    R, G = back_at[-1], more_at[-1]
    short = (G - R - n_free[0]).clamp(min=0)
    ok = short == 0
    cols = torch.arange(table.shape[1], device="cuda", dtype=torch.int32)[None]
    # given back in the reverse order of granting: the list's end is the first sequence's first page
    gone = (cols >= need[:, None]) & (cols < owned[:, None])
    to = n_free[0] + R - 1 - (back_at[:-1, None] + cols - need[:, None])
    stack = torch.cat([free, free.new_zeros(1)])
    stack.scatter_(0, torch.where(gone & ok, to, free.numel()).reshape(-1).long(), table.reshape(-1))
    new = (cols >= owned[:, None]) & (cols < need[:, None])
    at = n_free[0] + R - 1 - (more_at[:-1, None] + cols - owned[:, None])
    fresh = stack[at.clamp(0, free.numel() - 1).long()]
    table.copy_(torch.where(ok & new, fresh, torch.where(ok & gone, -1, table)))
    free.copy_(stack[:-1])
    n_free.copy_(torch.where(ok, n_free + R - G, n_free))
    owned.copy_(torch.where(ok, need, owned))
    off = _offsets(torch.where(ok, rows, 0).to(torch.int32))
    i = torch.arange(n_rows, device="cuda", dtype=torch.int32)
    b = torch.searchsorted(off[1:], i, right=True).clamp(max=lens.numel() - 1)
    live = i < off[-1]
    pos = torch.where(live, lens[b] + i - off[b], 0)
    slot = torch.where(live, table[b, (pos // PAGE).long()] * PAGE + pos % PAGE, -1)
    return off, torch.where(ok, after, lens), slot.to(torch.int32), pos.to(torch.int32), short.reshape(1).to(torch.int32)


def _round(x, s):
    return (x.float() / s).clamp(-448, 448).to(F8).view(torch.uint8)


def _append_plain(s):
    k_pages, v_pages, k_scale, v_scale = s["cache"]
    slot, k, v, runs = s["slot_map"], s["k"].float(), s["v"].float(), s["max_runs"]
    live = slot >= 0                                                   # what lies behind the last row: that row once more
    row = torch.minimum(torch.arange(slot.numel(), device="cuda"), live.sum() - 1)
    slot, k, v = slot[row], k[row], v[row]
    page, off = (slot // PAGE).long(), (slot % PAGE).long()
    begins = live.clone()
    begins[1:] &= (slot[1:] != slot[:-1] + 1) | (off[1:] == 0)
    run = torch.cumsum(begins, 0) - 1                                  # run of consecutive slots inside one page, of each row
    run_page = page[:1].repeat(runs).scatter(0, run, page)
    run_off = off[:1].repeat(runs).scatter_reduce(0, run, off, "amin", include_self=False)
    kept = torch.arange(PAGE, device="cuda")[None] < run_off[:, None]
    for x, pages, scale, seen in ((k, k_pages, k_scale, kept[:, None, :, None]), (v, v_pages, v_scale, kept[:, None, None, :])):
        a = torch.where(torch.isfinite(x), x.abs(), 0).amax(-1)        # [rows, heads]
        need = _pow2(torch.zeros((scale.shape[0], scale.shape[1]), device="cuda").index_reduce(0, page, a, "amax"), s["powers"])[run_page]
        old = scale[run_page]
        new = torch.where(run_off[:, None] > 0, torch.maximum(need, old), need)
        was = pages[run_page]
        again = _round(was.view(F8).float(), (new / old)[:, :, None, None])
        pages[run_page] = torch.where(seen & (new != old)[:, :, None, None], again, was)
        scale[run_page] = new
        codes = _round(x, scale[page][..., None])
        if x is k:
            pages[page, :, off] = codes
        else:
            pages[page, :, :, off] = codes
    return k_pages.view(F8), v_pages.view(F8), k_scale, v_scale


def _attend_plain(s):
    k_pages, v_pages, k_scale, v_scale = s["cache"]
    table, lens, off, q, M = s["table"].long().clamp(min=0), s["lens"].long(), s["row_offsets"].long(), s["q"], s["max_rows"]
    B, nb = table.shape
    heads, dh, H = q.shape[1], q.shape[2], k_pages.shape[1]
    G, S = heads // H, nb * PAGE
    at = torch.arange(S, device="cuda")
    there = (at[None] < lens[:, None])[:, None, :, None]
    K = (k_pages[table].view(F8).float() * k_scale[table][..., None, None]).permute(0, 2, 1, 3, 4).reshape(B, H, S, dh)
    V = (v_pages[table].view(F8).float() * v_scale[table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(B, H, S, dh)
    K, V = torch.where(there, K, 0.0), torch.where(there, V, 0.0)
    j = torch.arange(M, device="cuda")
    n = off[1:] - off[:-1]
    row = (off[:-1, None] + j[None]).clamp(max=q.shape[0] - 1)
    Q = q.float()[row].reshape(B, M, H, G, dh).permute(0, 2, 3, 1, 4).reshape(B, H, G * M, dh)
    scores = torch.matmul(Q, K.transpose(2, 3).contiguous()) * s["scale"]
    sees = at[None, None] <= (lens - n)[:, None, None] + j[None, :, None]
    scores = scores.reshape(B, H, G, M, S).masked_fill(~sees[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(B, H, G * M, S), V).reshape(B, H, G, M, dh) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, M, heads, dh).to(q.dtype)
    i = torch.arange(q.shape[0], device="cuda")
    b = torch.searchsorted(off[1:], i, right=True).clamp(max=B - 1)
    return torch.where((i < off[-1])[:, None, None], o[b, (i - off[b]).clamp(max=M - 1)], s["out"])


def _verify_plain(s):
    drafts, n_draft, probs, T = s["drafts"].long(), s["n_draft"].long(), s["probs"], s["temperature"].double()
    B, k1, V = s["logits"].shape
    k = k1 - 1
    greedy = T <= 0
    z = s["logits"].double() / torch.where(greedy, 1.0, T)[:, None, None]
    z = torch.where(torch.isnan(z), -math.inf, z)
    best = z.argmax(-1)
    e = torch.exp(z - z.amax(-1, keepdim=True))
    p = e / e.sum(-1, keepdim=True)
    rows = torch.arange(B, device="cuda")
    if k > 0:
        x = drafts.clamp(0, V - 1)
        fits = (drafts >= 0) & (drafts < V)
        px = torch.where(greedy[:, None], (best[:, :k] == x).double(), p[:, :k].gather(-1, x[..., None])[..., 0])
        qx = probs.gather(-1, x[..., None])[..., 0].double() if probs is not None else torch.ones_like(px)
        qx = torch.where(greedy[:, None], 1.0, qx)
        ok = fits & (s["u_accept"].double() * qx < px) & (torch.arange(k, device="cuda")[None] < n_draft[:, None])
        n_acc = torch.cumprod(ok.long(), 1).sum(1)
    else:
        n_acc = torch.zeros(B, dtype=torch.long, device="cuda")
    w = p[rows, n_acc]
    if k > 0:
        at = n_acc.clamp(max=k - 1)
        if probs is not None:
            left = (w - probs[rows, at].double()).clamp(min=0)
        else:
            token = torch.where(fits[rows, at], x[rows, at], V)[:, None]
            left = torch.cat([w, w.new_zeros(B, 1)], 1).scatter(1, token, 0.0)[:, :V]
        w = torch.where(((n_acc < n_draft) & (left.sum(-1) > 0))[:, None], left, w)
    c = torch.cumsum(w, -1)
    last = V - 1 - (w.flip(-1) > 0).long().argmax(-1)
    token = torch.minimum((c <= s["u_sample"].double()[:, None] * c[:, -1:]).sum(-1), last)
    token = torch.where(greedy, best[rows, n_acc], token)
    j = torch.arange(k1, device="cuda")[None]
    padded = torch.cat([drafts, drafts.new_zeros(B, 1)], 1)
    emitted = torch.where(j < n_acc[:, None], padded, torch.where(j == n_acc[:, None], token[:, None], -1))
    return n_acc.to(torch.int32), token.to(torch.int32), emitted.to(torch.int32)


def run(s):
    kind = s["kind"]
    if own:
        import paper_2304_04487_amd as llma

        if kind == "map":
            # a step's pages, and, once the accepted rows are known, what only rejected drafts had goes back
            pages = llma.PageTable(s["table"], s["owned"], s["free"], s["n_free"])
            llma.llma_map_pages(pages, s["lens"], s["rows"], s["row_offsets"], s["lens_after"], s["slot_map"], s["row_pos"], s["status"])
            llma.llma_map_pages(pages, s["kept"], s["none"], s["row_offsets2"], s["lens_after2"], None, None, s["status2"])
            return [s[n] for n in ("row_offsets", "lens_after", "slot_map", "row_pos", "status", "lens_after2", "status2", "table", "owned", "n_free")]
        if kind == "append":
            k, v, ks, vs = s["cache"]
            llma.llma_append_paged(llma.PagedCache(k, v, ks, vs), s["k"], s["v"], s["slot_map"])
            return [k.view(F8), v.view(F8), ks, vs]
        if kind == "attend":
            llma.llma_attend_paged(llma.PagedCache(*s["cache"]), s["q"], s["table"], s["lens"], s["row_offsets"], s["max_rows"], s["scale"], s["out"])
            return s["out"]
        llma.llma_verify_sampled(s["logits"], s["drafts"], s["u_accept"], s["u_sample"], s["n_accepted"], s["next"], s["emitted"], n_draft=s["n_draft"],
                                 draft_probs=s["probs"], temperature=s["temperature"])
        return [s["n_accepted"], s["next"], s["emitted"]]
    if kind == "map":
        first = _map_plain(s, s["lens"], s["rows"], s["slot_map"].numel())
        second = _map_plain(s, s["kept"], s["none"], 0)
        return [*first, second[1], second[4], s["table"], s["owned"], s["n_free"]]
    if kind == "append":
        return list(_append_plain(s))
    if kind == "attend":
        return _attend_plain(s)
    return list(_verify_plain(s))


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind, B = case["kind"], case["seqs"]
    if kind == "map":
        # lengths, rows, kept lengths and owned counts in and out, one table entry in 64 positions, slot and position of every row
        rows = 0.75 * case["rows"] * B
        return {"bytes": 40 * B + 8 * rows + 8 * (rows / PAGE + B), "flops": 4 * rows}
    if kind != "verify":
        past, rows = (case["past"], case["rows"]) if B == 1 else (2 / 3 * case["past"], 0.75 * case["rows"])
    if kind == "append":
        n = B * rows * case["kv_heads"] * case["head_dim"]
        return {"bytes": 2 * n * (SIZE[case["type"]] + 1), "flops": 4 * n}
    if kind == "attend":
        cached = 2 * B * (past + rows) * case["kv_heads"] * (case["head_dim"] + 4 / PAGE)
        return {"bytes": cached + 2 * B * rows * case["heads"] * case["head_dim"] * SIZE[case["type"]],
                "flops": 4 * B * rows * (past + rows / 2) * case["heads"] * case["head_dim"]}
    n = B * (case["k"] + 1) * case["vocab"]
    return {"bytes": n * SIZE[case["type"]] + (4 * B * case["vocab"] if case["probs"] else 0), "flops": 4 * n}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _values(codes):
    """what e4m3 codes stand for: sign, four bits of exponent (bias 7), three of fraction; all ones: NaN"""
    c = torch.arange(256, device="cuda")
    e, f = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * _powers(-7, 8, torch.float64)[e])
    v = torch.where((c & 127) == 127, math.nan, torch.where(c >= 128, -v, v))
    return v[codes.long()]


def _nearest(x):
    """the e4m3 value next to x, ties to the even one"""
    a = x.abs().clamp(max=448.0)
    step = _powers(-9, 5, torch.float64)[(torch.frexp(a.clamp(min=2.0 ** -6))[1] + 5).long()]     # three bits behind the leading one
    return torch.sign(x) * torch.round(a / step) * step


def _exact_append(s):
    k_pages, v_pages, k_scale, v_scale = s["cache"]
    slots = s["slot_map"].tolist()
    out = []
    for pages, scale, rows, keys in ((k_pages, k_scale, s["k"], True), (v_pages, v_scale, s["v"], False)):
        val, sc = _values(pages if keys else pages.transpose(2, 3)), scale.double().clone()
        i = 0
        while i < len(slots):
            if slots[i] < 0:
                i += 1
                continue
            page, at, n = slots[i] // PAGE, slots[i] % PAGE, 1
            while i + n < len(slots) and slots[i + n] == slots[i] + n and slots[i + n] // PAGE == page:
                n += 1
            x = rows[i:i + n].double().transpose(0, 1)                                  # [heads, rows, head_dim]
            m, e = torch.frexp(x.abs().amax((1, 2)) / 448)
            need = _powers(-64, 120, torch.float64)[(torch.where(m == 0.5, e - 1, e).clamp(-64, 120) + 64).long()]
            new = torch.maximum(need, sc[page]) if at else need
            kept = _nearest(val[page, :, :at] * (sc[page] / new)[:, None, None])
            val[page, :, :at], val[page, :, at:at + n], sc[page] = kept, _nearest(x / new[:, None, None]), new
            i += n
        out += [val if keys else val.transpose(2, 3).contiguous(), sc]
    return [out[0], out[2], out[1], out[3]]


def _exact_attend(s):
    k_pages, v_pages, k_scale, v_scale = s["cache"]
    q, H = s["q"].double(), k_pages.shape[1]
    G = q.shape[1] // H
    out = torch.zeros_like(q)
    lens, off = s["lens"].tolist(), s["row_offsets"].tolist()
    for b, n in enumerate(lens):
        pages = s["table"][b, :(n + PAGE - 1) // PAGE].long()
        m = off[b + 1] - off[b]
        for h in range(H):
            K = (_values(k_pages[pages, h]) * k_scale[pages, h].double()[:, None, None]).reshape(-1, q.shape[2])[:n]
            V = (_values(v_pages[pages, h]) * v_scale[pages, h].double()[:, None, None]).transpose(1, 2).reshape(-1, q.shape[2])[:n]
            Q = q[off[b]:off[b + 1], h * G:(h + 1) * G].reshape(m * G, -1)
            t = (Q @ K.t()) * s["scale"]
            limit = (n - m + torch.arange(m, device="cuda")).repeat_interleave(G)
            t = t.masked_fill(torch.arange(n, device="cuda")[None] > limit[:, None], -math.inf)
            out[off[b]:off[b + 1], h * G:(h + 1) * G] = (torch.softmax(t, -1) @ V).reshape(m, G, -1)
    return out


def _exact_verify(s):
    B, k1, V = s["logits"].shape
    n_acc, nxt, emitted = [], [], []
    T, nd, dr, ua, us = (s[n].tolist() for n in ("temperature", "n_draft", "drafts", "u_accept", "u_sample"))
    for b in range(B):
        kept, token = [], None
        for j in range(nd[b] + 1):
            z = s["logits"][b, j].double()
            if T[b] <= 0:
                p = torch.zeros_like(z)
                p[z.argmax()] = 1
            else:
                z = z / s["temperature"][b].double()
                p = torch.exp(z - torch.logsumexp(z, 0))
            if j < nd[b]:
                x = dr[b][j]
                q = torch.zeros_like(p)
                q[x] = 1
                if s["probs"] is not None and T[b] > 0:
                    q = s["probs"][b, j].double()
                if ua[b][j] * float(q[x]) < float(p[x]):
                    kept.append(x)
                    continue
                left = (p - q).clamp(min=0)
                p = left if float(left.sum()) > 0 else p
            c = torch.cumsum(p, 0)
            token = int(torch.searchsorted(c, us[b] * c[-1], right=True)) if T[b] > 0 else int(z.argmax())
            break
        n_acc.append(len(kept))
        nxt.append(token)
        emitted.append(kept + [token] + [-1] * (k1 - 1 - len(kept)))
    return [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (n_acc, nxt, emitted)]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "map":
        return None                                                                      # whole numbers only
    if kind == "append":
        return _exact_append(s)
    if kind == "attend":
        big = 4 * case["seqs"] * case["rows"] * (case["past"] + case["rows"]) * case["heads"] * case["head_dim"]
        return None if big > 4e12 else _exact_attend(s)
    return _exact_verify(s)

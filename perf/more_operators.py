"""Operators of serving on pages with a cache of 4 bits a value, as timed cases: the write into that cache and the read back
(of it and of the 8-bit one), attention over it, and log probabilities of given tokens.

`run` computes each in a plain form (elementary torch operations) or, with `own`, through the package's public calls.

Pages hold 64 positions.  The 4-bit cache: e2m1 codes, and for every 32 neighbouring features of a position a power of two as
its exponent plus 127.  k [pages, kv heads, 64, head_dim / 2]: byte j of a position has feature 2j in its low half, 2j + 1 in its
high half; v [pages, kv heads, head_dim / 2, 64]: the same bytes, transposed; k_scale and v_scale [pages, kv heads, head_dim / 32, 64].
A cached value is code * 2^(scale - 127).  The 8-bit cache: e4m3 codes k [pages, kv heads, 64, head_dim], v [pages, kv heads,
head_dim, 64], and powers of two k_scale, v_scale [pages, kv heads] as float32.
table [slots, blocks] names a sequence's pages in order.
"""
import math

import torch

own = False

PAGE, BLOCK = 64, 32
F8 = torch.float8_e4m3fn
E8 = torch.float8_e8m0fnu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


# ------------------------------------------------------------------------------------------------ what is measured
def listed():
    return [
        # a verification step's rows of 16 sequences, one layer of the 7B shape: written, and read back as attention will see them
        {"name": "write_step_7b", "kind": "write", "seqs": 16, "past": 4096, "rows": 9, "kv_heads": 32, "head_dim": 128, "type": "bf16"},
        # prompts of four requests, shared key/value heads, float32 rows straight from a projection, on top of a common prefix
        {"name": "write_prompts_gqa", "kind": "write", "seqs": 4, "past": 100, "rows": 2011, "kv_heads": 8, "head_dim": 128, "type": "fp32"},
        # a short session of the d 512 model leaves the 8-bit pages
        {"name": "read_8bit_d512", "kind": "read", "bits": 8, "seqs": 1, "past": 1001, "kv_heads": 8, "head_dim": 64, "type": "bf16"},
        # prefixes of five sequences of the 7B shape go from 8-bit pages into a cache in planes
        {"name": "read_8bit_7b", "kind": "read", "bits": 8, "seqs": 5, "past": 4001, "kv_heads": 32, "head_dim": 128, "type": "bf16"},
        # ragged sequences out of 4-bit pages, for a program that computes in float32
        {"name": "read_4bit_ragged", "kind": "read", "bits": 4, "seqs": 37, "past": 1900, "kv_heads": 8, "head_dim": 128, "type": "fp32"},
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
        # what a step answered, with a few alternatives a token
        {"name": "logprobs_step", "kind": "logprobs", "rows": 9, "vocab": 32000, "top": 5, "type": "fp32", "temperature": False},
        # a scored prompt over a large vocabulary, twenty alternatives a token
        {"name": "logprobs_prompt_2000", "kind": "logprobs", "rows": 2000, "vocab": 128256, "top": 20, "type": "bf16", "temperature": True},
    ]


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    kind = rng.choice(["write", "read", "read", "attend", "attend", "attend", "attend", "logprobs", "logprobs"])
    if kind == "logprobs":
        vocab = log(500, 128256)
        return {"kind": kind, "rows": max(1, min(log(1, 2000), int(2.5e8 / vocab))), "vocab": vocab, "top": rng.choice([0, 1, rng.randint(2, 32), rng.randint(2, 32)]),
                "type": rng.choice(["bf16", "fp16", "fp32"]), "temperature": rng.random() < 0.5}
    dh, dt = rng.choice([64, 128]), rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if kind == "write":
        heads, rows = rng.choice([1, 8, 32]), log(1, 2011)
        return {"kind": kind, "seqs": max(1, log(1, max(1.5, min(64, 64000 / (heads * rows))))), "past": log(16, 4096), "rows": rows, "kv_heads": heads, "head_dim": dh, "type": dt}
    if kind == "read":
        heads, past = rng.choice([1, 2, 8, 32]), log(16, 16000)
        return {"kind": kind, "bits": rng.choice([4, 8]), "seqs": max(1, min(log(1, 64), int(600000 / (heads * past)))), "past": past, "kv_heads": heads, "head_dim": dh, "type": dt}
    kv = rng.choice([1, 2, 8, 32])
    heads = kv * rng.choice([1, 4, 8] if kv < 32 else [1])
    rows = rng.choice([1, log(2, 33), log(34, 1500)])
    past = log(16, 24000)
    seqs = max(1, min(log(1, 64), int(2.5e8 / (heads * rows * (past + rows))), int(70000 * 32 / (kv * (past + rows)))))
    return {"kind": kind, "seqs": seqs, "past": past, "rows": rows, "heads": heads, "kv_heads": kv, "head_dim": dh, "type": dt}


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 6247 + 17)


def _rand(shape, g):
    return torch.rand(shape, generator=g, device="cuda")


def _randn(shape, g):
    return torch.randn(shape, generator=g, device="cuda")


def _ints(lo, hi, shape, g):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)


def _offsets(n):
    return torch.cat([torch.zeros(1, dtype=torch.int32, device=n.device), torch.cumsum(n, 0, dtype=torch.int32)])


def _powers(dtype=torch.float32):
    """2^-64 .. 2^120, exactly (the device's pow and ldexp are not)"""
    return torch.tensor([2.0 ** i for i in range(-64, 121)], dtype=dtype, device="cuda")


def _exponent(amax, most):
    """exponent of the smallest power of two s from 2^-64 to 2^120 with amax <= 0.875 * 2^most * s (7: most = 3; 448: 9)"""
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - most + 1, e - most)
    return torch.where(amax > 0, e, -64).clamp(-64, 120)


def _codes4(a):
    """e2m1 codes of magnitudes a (in units of the scale): 0, 0.5, 1, 1.5, 2, 3, 4, 6, nearest, ties to the even code"""
    return torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, torch.round(a) + 2, torch.round(a / 2) + 4)).clamp(max=7).to(torch.uint8)


def _pack4(x, powers):
    """x [..., head_dim]: bytes [..., head_dim / 2] and scales [..., head_dim / 32]"""
    b = x.reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    e = _exponent(b.abs().amax(-1), 3)
    c = _codes4(b.abs() / powers[e.long() + 64][..., None]) | (torch.signbit(b).to(torch.uint8) << 3)
    c = c.reshape(x.shape)
    return c[..., 0::2] | (c[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _unpack4(c, s, values, powers):
    """c [..., head_dim / 2], s [..., head_dim / 32]: the values they stand for, [..., head_dim]"""
    v = torch.stack([values[(c & 15).long()], values[(c >> 4).long()]], -1)
    p = powers[(s.long() - 63).clamp(0, 184)]
    return (v.reshape(*s.shape, BLOCK) * p[..., None]).reshape(*c.shape[:-1], 2 * c.shape[-1])


def _values4(dtype=torch.float32):
    v = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return torch.tensor(v + [-x for x in v], dtype=dtype, device="cuda")


def _lengths(case, g):
    """lengths before the step and rows of it: ragged, the first sequence at the case's full size"""
    B, past, rows = case["seqs"], case["past"], case.get("rows", 0)
    lens = _ints(max(1, past // 3), past + 1, (B,), g)
    n = _ints(max(1, rows // 2), rows + 1, (B,), g) if rows else torch.zeros_like(lens)
    lens[0], n[0] = past, rows
    return lens, n


def _table(total, max_blocks, n_pages, g):
    """a table whose sequences own the pages of `total` positions, drawn from a shuffled pool"""
    perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    need = (total + PAGE - 1) // PAGE
    cols = torch.arange(max_blocks, device="cuda", dtype=torch.int32)
    at = (_offsets(need)[:-1, None] + cols[None]).clamp(max=n_pages - 1)
    return torch.where(cols[None] < need[:, None], perm[at.long()], -1).to(torch.int32), need


def _filled(bits, n_pages, heads, dh, g):
    """codes and scales of a filled cache: normal values whose channels differ in size"""
    if bits == 4:
        k = torch.empty((n_pages, heads, PAGE, dh // 2), dtype=torch.uint8, device="cuda")
        v = torch.empty((n_pages, heads, dh // 2, PAGE), dtype=torch.uint8, device="cuda")
        ks, vs = (torch.empty((n_pages, heads, dh // BLOCK, PAGE), dtype=torch.uint8, device="cuda") for _ in range(2))
    else:
        k = torch.empty((n_pages, heads, PAGE, dh), dtype=torch.uint8, device="cuda")
        v = torch.empty((n_pages, heads, dh, PAGE), dtype=torch.uint8, device="cuda")
        ks, vs = (torch.empty((n_pages, heads), device="cuda") for _ in range(2))
    size, powers = torch.exp(0.4 * _randn((1, heads, 1, dh), g)), _powers()
    step = max(1, (1 << 24) // (heads * PAGE * dh))
    for a in range(0, n_pages, step):
        n = min(step, n_pages - a)
        x, y = _randn((n, heads, PAGE, dh), g) * size, _randn((n, heads, PAGE, dh), g)
        for z, codes, scale, keys in ((x, k, ks, True), (y, v, vs, False)):
            if bits == 4:
                c, s = _pack4(z, powers)
                scale[a:a + n] = s.transpose(2, 3)
            else:
                e = _exponent(z.abs().amax((2, 3)), 9)
                scale[a:a + n] = powers[e.long() + 64]
                c = (z / scale[a:a + n, :, None, None]).to(F8).view(torch.uint8)
            codes[a:a + n] = c if keys else c.transpose(2, 3)
    return k, v, ks, vs


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    if kind == "logprobs":
        n, V, dt = case["rows"], case["vocab"], TYPES[case["type"]]
        logits = torch.empty((n, V), dtype=dt, device="cuda")
        tokens = torch.empty(n, dtype=torch.int32, device="cuda")
        for a in range(0, n, 256):
            # some tokens well above the rest, some masked; given tokens mostly likely ones
            z = 2.0 * _randn((min(256, n - a), V), g)
            z = z + torch.where(_rand(z.shape, g) < 20.0 / V, 6.0, 0.0)
            z = torch.where(_rand(z.shape, g) < 0.02, -math.inf, z).to(dt)
            logits[a:a + 256] = z
            tokens[a:a + 256] = torch.where(_rand((len(z),), g) < 0.7, (z.float() + 2.0 * _randn(z.shape, g)).argmax(-1).to(torch.int32), _ints(0, V, (len(z),), g))
        top = min(case["top"], V)
        f32, i32 = {"device": "cuda"}, {"device": "cuda", "dtype": torch.int32}
        return {"kind": kind, "logits": logits, "tokens": tokens, "temperature": 0.5 + _rand((n,), g) if case["temperature"] else None, "top": top,
                "logprob": torch.empty(n, **f32), "rank": torch.empty(n, **i32), "entropy": torch.empty(n, **f32),
                "top_tokens": torch.empty((n, top), **i32) if top else None, "top_logprobs": torch.empty((n, top), **f32) if top else None}
    lens, rows = _lengths(case, g)
    B, H, dh, dt = case["seqs"], case["kv_heads"], case["head_dim"], TYPES[case["type"]]
    total = lens + rows
    blocks = (case["past"] + case.get("rows", 0) + PAGE - 1) // PAGE
    s = {"kind": kind, "bits": case.get("bits", 4), "values": _values4(), "powers": _powers(), "slots": torch.randperm(B, generator=g, device="cuda").to(torch.int32)}
    if kind == "write":
        # the pool holds the pages that the step writes to; a sequence's earlier pages are other pools' (page 0 stands for them)
        first = lens // PAGE
        blocks_b = (total + PAGE - 1) // PAGE - first
        n_pages = B * (case["rows"] // PAGE + 2) + 8
        perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        cols = torch.arange(blocks + 1, device="cuda", dtype=torch.int32)[None]
        at = _offsets(blocks_b)[:-1, None] + cols - first[:, None]
        table = torch.where((cols >= first[:, None]) & (cols < (first + blocks_b)[:, None]), perm[at.clamp(0, n_pages - 1).long()], 0).to(torch.int32)
        off, n = _offsets(rows), B * case["rows"]                                           # room for the most rows: padding behind the last sequence
        i = torch.arange(n, device="cuda", dtype=torch.int32)
        b = torch.searchsorted(off[1:], i, right=True).clamp(max=B - 1)
        pos = (lens[b] + i - off[b]).clamp(max=PAGE * blocks - 1)
        slot_map = torch.where(i < off[-1], table[b, (pos // PAGE).long()] * PAGE + pos % PAGE, -1).to(torch.int32)
        # as a projection leaves them: keys and values side by side in one row; now and then a large value
        kv = _randn((n, 2, H, dh), g)
        kv = (kv * torch.where(_rand((n, 2, H, 1), g) < 0.05, 40.0, 1.0)).to(dt)
        by_slot = torch.zeros_like(table)
        by_slot[s["slots"].long()] = table
        return {**s, "cache": _filled(4, n_pages, H, dh, g), "k": kv[:, 0], "v": kv[:, 1], "slot_map": slot_map, "table": by_slot, "first": lens, "row_offsets": off,
                "k_out": torch.zeros((n, H, dh), dtype=dt, device="cuda"), "v_out": torch.zeros((n, H, dh), dtype=dt, device="cuda")}
    n_pages = B * blocks
    table, need = _table(total, blocks, n_pages, g)
    cache = _filled(s["bits"], n_pages, H, dh, g)
    by_slot = torch.zeros_like(table)
    by_slot[s["slots"].long()] = table
    if kind == "read":
        # from some position on (a prefix that the receiver has already), all heads, as rows or, as a cache in planes takes them, head by head
        start = torch.where(_rand((B,), g) < 0.5, 0, (_rand((B,), g) * 0.3 * lens).to(torch.int32)).to(torch.int32)
        start[0] = 0
        n = B * case["past"]
        off = _offsets(lens - start)
        k_out, v_out = (torch.zeros((H, n, dh), dtype=dt, device="cuda").transpose(0, 1) for _ in range(2))
        return {**s, "cache": cache, "table": by_slot, "first": start, "row_offsets": off, "k_out": k_out, "v_out": v_out}
    # what lies behind the last position of a sequence's last page is anything: scales that stand for NaN here
    last = table[torch.arange(B, device="cuda"), (need - 1).long()].long()
    behind = torch.arange(PAGE, device="cuda")[None] >= ((total - 1) % PAGE + 1)[:, None]
    for scale in cache[2:]:
        scale[last] = torch.where(behind[:, None, None, :], 255, scale[last])
    n = B * case["rows"]                                                                    # room for the most rows: those behind the last sequence stay zero
    q = (1.5 * _randn((n, case["heads"], dh), g)).to(dt)
    return {**s, "cache": cache, "table": by_slot, "lens": total, "row_offsets": _offsets(rows), "q": q, "out": torch.zeros_like(q), "max_rows": case["rows"],
            "scale": 1.0 / math.sqrt(dh)}


# ------------------------------------------------------------------------------------------------ the plain forms
def _write_plain(s):
    k_pages, v_pages, k_scale, v_scale = s["cache"]
    slot = s["slot_map"]
    live = slot >= 0                                                   # what lies behind the last row: that row once more
    row = torch.minimum(torch.arange(slot.numel(), device="cuda"), live.sum() - 1)
    slot = slot[row]
    page, at = (slot // PAGE).long(), (slot % PAGE).long()
    k, ks = _pack4(s["k"].float(), s["powers"])
    v, vs = _pack4(s["v"].float(), s["powers"])
    k_pages[page, :, at], k_scale[page, :, :, at] = k[row], ks[row]
    v_pages[page, :, :, at], v_scale[page, :, :, at] = v[row], vs[row]


def _read_plain(s):
    k_pages, v_pages, k_scale, v_scale = s["cache"]
    off, k_out, v_out = s["row_offsets"], s["k_out"], s["v_out"]
    n, B = k_out.shape[0], s["first"].numel()
    i = torch.arange(n, device="cuda", dtype=torch.int32)
    b = torch.searchsorted(off[1:], i, right=True).clamp(max=B - 1)
    table = s["table"][s["slots"].long()]
    pos = (s["first"][b] + i - off[b]).clamp(max=PAGE * table.shape[1] - 1)
    page, at = table[b, (pos // PAGE).long()].long().clamp(min=0), (pos % PAGE).long()
    live = (i < off[-1])[:, None, None]
    k, v = k_pages[page, :, at], v_pages[page, :, :, at]
    if s["bits"] == 4:
        k = _unpack4(k, k_scale[page, :, :, at], s["values"], s["powers"])
        v = _unpack4(v, v_scale[page, :, :, at], s["values"], s["powers"])
    else:
        k = k.view(F8).float() * k_scale[page][..., None]
        v = v.view(F8).float() * v_scale[page][..., None]
    k_out.copy_(torch.where(live, k.to(k_out.dtype), k_out))
    v_out.copy_(torch.where(live, v.to(v_out.dtype), v_out))
    return k_out, v_out


def _attend_plain(s):
    k_pages, v_pages, k_scale, v_scale = s["cache"]
    table, lens, off, q, M = s["table"][s["slots"].long()].long().clamp(min=0), s["lens"].long(), s["row_offsets"].long(), s["q"], s["max_rows"]
    B, nb = table.shape
    heads, dh, H = q.shape[1], q.shape[2], k_pages.shape[1]
    G, S = heads // H, nb * PAGE
    at = torch.arange(S, device="cuda")
    there = (at[None] < lens[:, None])[:, None, :, None]
    K = _unpack4(k_pages[table], k_scale[table].transpose(3, 4), s["values"], s["powers"]).permute(0, 2, 1, 3, 4).reshape(B, H, S, dh)
    V = _unpack4(v_pages[table].transpose(3, 4), v_scale[table].transpose(3, 4), s["values"], s["powers"]).permute(0, 2, 1, 3, 4).reshape(B, H, S, dh)
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


def _logprobs_plain(s):
    x, token = s["logits"].float(), s["tokens"].long()[:, None]
    V = x.shape[1]
    z = x if s["temperature"] is None else x / s["temperature"][:, None]
    z = z - z.amax(-1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(-1, keepdim=True)
    lse = torch.log(total)
    mean = torch.where(e > 0, e * z, 0.0).sum(-1, keepdim=True) / total
    given = x.gather(1, token)
    ids = torch.arange(V, device="cuda")
    rank = (x > given).sum(-1) + ((x == given) & (ids[None] < token)).sum(-1)
    out = [(z.gather(1, token) - lse)[:, 0], rank.to(torch.int32), (lse - mean)[:, 0]]
    if s["top"]:
        # the largest, ties to the lowest id: ordered as integers, the id below the value
        bits = x.view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() * (1 << 32) + (V - 1 - ids)[None]
        best = V - 1 - torch.topk(key, s["top"], -1).values % (1 << 32)
        out += [best.to(torch.int32), z.gather(1, best) - lse]
    return out


def run(s):
    kind = s["kind"]
    if own:
        import paper_2304_04487_amd as llma

        if kind == "write":
            cache = llma.PagedMxCache(*s["cache"])
            llma.llma_append_paged_mx(cache, s["k"], s["v"], s["slot_map"])
            llma.llma_read_paged_mx(cache, s["table"], s["first"], s["row_offsets"], s["k_out"], s["v_out"], slots=s["slots"])
            return [s["k_out"], s["v_out"], s["cache"][2].view(E8), s["cache"][3].view(E8)]
        if kind == "read":
            if s["bits"] == 4:
                llma.llma_read_paged_mx(llma.PagedMxCache(*s["cache"]), s["table"], s["first"], s["row_offsets"], s["k_out"], s["v_out"], slots=s["slots"])
            else:
                llma.llma_read_paged(llma.PagedCache(*s["cache"]), s["table"], s["first"], s["row_offsets"], s["k_out"], s["v_out"], slots=s["slots"])
            return [s["k_out"], s["v_out"]]
        if kind == "attend":
            llma.llma_attend_paged_mx(llma.PagedMxCache(*s["cache"]), s["q"], s["table"], s["lens"], s["row_offsets"], s["max_rows"], s["scale"], s["out"], slots=s["slots"])
            return s["out"]
        llma.llma_token_logprobs(s["logits"], s["tokens"], s["logprob"], rank=s["rank"], entropy=s["entropy"], top_tokens=s["top_tokens"], top_logprobs=s["top_logprobs"],
                                 temperature=s["temperature"])
        return [s["logprob"], s["rank"], s["entropy"]] + ([s["top_tokens"], s["top_logprobs"]] if s["top"] else [])
    if kind == "write":
        _write_plain(s)
        return [*_read_plain(s), s["cache"][2].view(E8), s["cache"][3].view(E8)]
    if kind == "read":
        return list(_read_plain(s))
    if kind == "attend":
        return _attend_plain(s)
    return _logprobs_plain(s)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "logprobs":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * SIZE[case["type"]] + case["rows"] * (16 + 8 * case["top"]), "flops": 6 * n}
    B, H, dh, size = case["seqs"], case["kv_heads"], case["head_dim"], SIZE[case["type"]]
    past, rows = (case["past"], case.get("rows", 0)) if B == 1 else (2 / 3 * case["past"], 0.75 * case.get("rows", 0))
    value4 = 0.5 + 1 / BLOCK
    if kind == "write":
        n = 2 * B * rows * H * dh                                                           # in, codes out, codes in, values out
        return {"bytes": n * (2 * size + 2 * value4), "flops": 4 * n}
    if kind == "read":
        n = 2 * B * past * H * dh * (1 if B == 1 else 0.92)
        return {"bytes": n * (size + (value4 if case["bits"] == 4 else 1)), "flops": n}
    cached = 2 * B * (past + rows) * H * dh * value4
    return {"bytes": cached + 2 * B * rows * case["heads"] * dh * size, "flops": 4 * B * rows * (past + rows / 2) * case["heads"] * dh}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _exact_pages(codes, scale, keys, bits):
    """[pages, heads, 64, head_dim] of what codes and scales stand for"""
    c = codes if keys else codes.transpose(2, 3)
    if bits == 8:
        n = torch.arange(256, device="cuda")
        e, f = (n >> 3) & 15, (n & 7).double()
        v = torch.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * _powers(torch.float64)[e - 7 + 64])
        return torch.where(n >= 128, -v, v)[c.long()] * scale.double()[:, :, None, None]
    out = torch.empty((*c.shape[:3], 2 * c.shape[3]), dtype=torch.float64, device="cuda")
    for odd in (0, 1):
        n = (c >> (4 * odd) & 15).long()
        e, f = (n >> 1) & 3, (n & 1).double()
        v = torch.where(e == 0, f / 2, (1 + f / 2) * _powers(torch.float64)[e - 1 + 64])
        out[..., odd::2] = torch.where(n >= 8, -v, v)
    by = _powers(torch.float64)[(scale.long() - 127 + 64).clamp(0, 184)]                    # (what stands for NaN lies where nobody looks)
    return out * by.transpose(2, 3).repeat_interleave(BLOCK, -1)


def _exact_write(s):
    cache = [c.clone() for c in s["cache"]]
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    slots = s["slot_map"].tolist()
    live = torch.tensor([i for i, at in enumerate(slots) if at >= 0], device="cuda")
    page, at = (s["slot_map"][live] // PAGE).long(), (s["slot_map"][live] % PAGE).long()
    out, scales = [], []
    for rows, scale, like in ((s["k"], cache[2], s["k_out"]), (s["v"], cache[3], s["v_out"])):
        x = rows[live].double().reshape(len(live), rows.shape[1], -1, BLOCK)
        m, e = torch.frexp(x.abs().amax(-1) / 7)
        e = torch.where(m == 0, -64, torch.where(m == 0.5, e - 1, e)).clamp(-64, 120)
        by = _powers(torch.float64)[e.long() + 64][..., None]
        a = x.abs() / by
        d = (a[..., None] - grid).abs()
        d = d + torch.tensor([0, 1e-12] * 4, dtype=torch.float64, device="cuda") * (d == d.amin(-1, keepdim=True))      # ties to the even code
        value = torch.sign(x) * grid[d.argmin(-1)] * by
        full = like.double().clone()
        full[live] = value.reshape(len(live), rows.shape[1], -1)
        out.append(full)
        scale[page, :, :, at] = (e + 127).to(torch.uint8)
        scales.append(scale.view(E8).double())
    return out + scales


def _exact_read(s):
    k, v = _exact_pages(s["cache"][0], s["cache"][2], True, s["bits"]), _exact_pages(s["cache"][1], s["cache"][3], False, s["bits"])
    out = [s["k_out"].double().clone(), s["v_out"].double().clone()]
    first, off, slots = s["first"].tolist(), s["row_offsets"].tolist(), s["slots"].tolist()
    for b, start in enumerate(first):
        pos = torch.arange(start, start + off[b + 1] - off[b], device="cuda")
        page = s["table"][slots[b]][pos // PAGE].long()
        for o, x in zip(out, (k, v)):
            o[off[b]:off[b + 1]] = x[page, :, pos % PAGE]
    return out


def _exact_attend(s):
    k_pages, v_pages, k_scale, v_scale = s["cache"]
    q, H = s["q"].double(), k_pages.shape[1]
    G, out = q.shape[1] // H, torch.zeros_like(q)
    lens, off, slots = s["lens"].tolist(), s["row_offsets"].tolist(), s["slots"].tolist()
    for b, n in enumerate(lens):
        pages = s["table"][slots[b], :(n + PAGE - 1) // PAGE].long()
        m = off[b + 1] - off[b]
        K = _exact_pages(k_pages[pages], k_scale[pages], True, 4)
        V = _exact_pages(v_pages[pages], v_scale[pages], False, 4)
        limit = (n - m + torch.arange(m, device="cuda")).repeat_interleave(G)
        for h in range(H):
            Q = q[off[b]:off[b + 1], h * G:(h + 1) * G].reshape(m * G, -1)
            t = (Q @ K[:, h].reshape(-1, q.shape[2])[:n].t()) * s["scale"]
            t = t.masked_fill(torch.arange(n, device="cuda")[None] > limit[:, None], -math.inf)
            out[off[b]:off[b + 1], h * G:(h + 1) * G] = (torch.softmax(t, -1) @ V[:, h].reshape(-1, q.shape[2])[:n]).reshape(m, G, -1)
    return out


def _exact_logprobs(s):
    lp, ent, top = [], [], []
    n = s["logits"].shape[0]
    for a in range(0, n, 64):
        x = s["logits"][a:a + 64].double()
        if s["temperature"] is not None:
            x = x / s["temperature"][a:a + 64].double()[:, None]
        x = x - torch.logsumexp(x, -1, keepdim=True)
        lp.append(x.gather(1, s["tokens"][a:a + 64].long()[:, None])[:, 0])
        ent.append(-torch.where(x == -math.inf, 0.0, torch.exp(x) * x).sum(-1))
        if s["top"]:
            top.append(torch.topk(x, s["top"], -1).values)
    return [torch.cat(lp), None, torch.cat(ent)] + ([None, torch.cat(top)] if s["top"] else [])


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "write":
        return _exact_write(s)
    if kind == "read":
        return _exact_read(s)
    if kind == "attend":
        big = 4 * case["seqs"] * case["rows"] * (case["past"] + case["rows"]) * case["heads"] * case["head_dim"]
        return None if big > 4e12 else _exact_attend(s)
    return _exact_logprobs(s)

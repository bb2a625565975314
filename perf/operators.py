"""Operators of a paged, quantized cache as cases that can be timed and compared: rotary positions with several axes, new
tokens quantized into pages and read back, attention of new tokens over the pages.

A layer of a serving engine runs them in this order.  The new tokens' queries and keys get their positions (`rope`; text has
one axis, images and video have time, height and width).  Full groups of keys and values are quantized into the pages that
the engine has given their sequences, and what later steps will see of them is read back (`write`; `read` alone is what a
recomputation or a move of sequences between engines does).  The new tokens attend to their sequences' pages and to the rows
that are still in full precision (`attend`): one token per sequence, a few drafted tokens, or a chunk of a prompt.

A page holds `page` tokens of all KV heads.  Codes: `bits` per element, low bits first, token by token.  Keys have a scale and
a zero-point per channel and `group` tokens, values per token and `group` channels:

    scale = (max - min) / L,  zero = min,  code = clamp(rint((x - zero) / scale), 0, L),  L = 2^bits - 1,  x' = zero + scale code

Values decide in IEEE binary32, operation by operation; keys as real arithmetic on the stored scale and zero-point would.
With 16-bit metadata scale and zero-point are rounded to binary16 first and the codes go by the rounded ones.

Head dimension 128, heads as in this library's own workloads (squat_inputs/configs.py); token counts are theirs or odd ones
between one token and theirs.
"""
import math
import random

import torch

own = False

D = 128
HEADS = ((8, 8), (32, 32), (32, 8))
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SECTIONS = {"text": (64,), "image": (32, 32), "video": (16, 24, 24), "partial": (8, 12, 12)}


# ------------------------------------------------------------------------------------------------ the cases
def _rope(tokens, heads, sections, dtype="bf16", inverse=False):
    return dict(kind="rope", tokens=tokens, q_heads=heads[0], kv_heads=heads[1], sections=sections, dtype=dtype, inverse=inverse)


def _write(tokens, kv_heads, bits, group, page, meta="f32", dtype="bf16", read="bf16"):
    return dict(kind="write", tokens=tokens, kv_heads=kv_heads, bits=bits, group=group, page=page, meta=meta, dtype=dtype, read=read)


def _read(tokens, kv_heads, bits, group, page, meta="f32", read="bf16"):
    return dict(kind="read", tokens=tokens, kv_heads=kv_heads, bits=bits, group=group, page=page, meta=meta, read=read)


def _attend(seqs, heads, cached, new, tail, bits, group, page, meta="f32", ragged=False, mixed=False):
    return dict(kind="attend", seqs=seqs, q_heads=heads[0], kv_heads=heads[1], cached=cached, new=new, tail=tail, bits=bits, group=group,
                page=page, meta=meta, ragged=ragged, mixed=mixed)


def listed():
    c = [
        # A decode step's 64 sequences, one token each, somewhere in videos: latency counts.
        ("rope_decode_64", _rope(64, (32, 8), "video")),
        # Prompts with images, queries and keys of the grouped-query workload's heads.
        ("rope_prompt_32k", _rope(32768, (32, 8), "video")),
        # One full group of 13 sequences moves from full precision into their pages.
        ("write_window_13x32", _write(13 * 32, 8, 2, 32, 64)),
        # The prompts of the grouped-query workload: 16 sequences of 8192 tokens, 8 KV heads.
        ("write_prompt_16x8192", _write(16 * 8192, 8, 2, 32, 128)),
        # Long groups, 4 bits and 16-bit metadata, from float32 keys and values.
        ("write_4bit_f32_21k", _write(165 * 128, 8, 4, 128, 128, meta="f16", dtype="f32", read="f32")),
        # One sequence of the tiny workload is read back for a recomputation.
        ("read_352", _read(352, 8, 4, 32, 32, meta="f16", read="f32")),
        # Sequences of the long-context workload leave for another engine.
        ("read_64k", _read(65536, 32, 2, 32, 64)),
        # The smallest step: one sequence, one token, the tiny workload's cache.
        ("attend_one", _attend(1, (8, 8), 256, 1, 4, 2, 32, 32)),
        # A decode step of 64 ragged sequences with up to 4096 tokens, every head with its own keys.
        ("attend_decode_64", _attend(64, (32, 32), 4096, 1, 16, 2, 32, 64, ragged=True)),
        # Six drafted tokens of 16 sequences are looked at together, four query heads to a KV head.
        ("attend_drafts_16x6", _attend(16, (32, 8), 8160, 6, 24, 2, 32, 128, ragged=True)),
        # A chunk of a long prompt: 2048 new tokens over 8192 in the pages.
        ("attend_chunk_2048", _attend(1, (32, 8), 8192, 2048, 0, 2, 32, 128)),
        # A step as an engine mixes it: chunks of two prompts among sequences that get one token each; 4 bits, 16-bit metadata.
        ("attend_mixed_24", _attend(24, (32, 8), 4032, 509, 7, 4, 64, 64, meta="f16", ragged=True, mixed=True)),
    ]
    return [dict(case, name=name) for name, case in c]


def _cost(case):
    w = work(case)
    return w["bytes"] / 6.5e12 + w["flops"] / 1.6e15


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    while True:
        kind = rng.choice(("rope", "write", "read", "attend", "attend", "attend"))
        bits, group, meta = rng.choice((2, 4)), rng.choice((32, 64, 128)), rng.choice(("f32", "f16"))
        page = group * rng.choice((1, 2, 3))
        heads = rng.choice(HEADS)
        if kind == "rope":
            case = _rope(_log(rng, 1, 32768), heads, rng.choice(sorted(SECTIONS)), rng.choice(("bf16", "f32")), rng.random() < 0.25)
        elif kind == "write":
            case = _write(group * _log(rng, 1, 131072 // group), heads[1], bits, group, page, meta, rng.choice(("bf16", "f32")), rng.choice(("bf16", "f32")))
        elif kind == "read":
            case = _read(group * _log(rng, 1, 131072 // group), heads[1], bits, group, page, meta, rng.choice(("bf16", "f32")))
        else:
            seqs = _log(rng, 1, 64)
            new = rng.choice((1, 1, rng.randint(2, 8), _log(rng, 9, 2048)))
            cached = group * (_log(rng, 1, 32768 // group) if rng.random() < 0.95 else 0)
            case = _attend(seqs, heads, cached, new, rng.randint(0, 40), bits, group, page, meta, rng.random() < 0.7, rng.random() < 0.3 and seqs > 2)
            # the plain form works on sequences padded to the longest one, in 32 bits
            padded = seqs * (cached + new + 40.0)
            if padded * heads[1] * D > 8e8 or padded * new * heads[0] > 2e9:
                continue
        if _cost(case) <= most[kind]:
            return case


def _lengths(case):
    """Cached tokens (multiples of the group), new tokens and rows in full precision before them, of each sequence."""
    n, g = case["seqs"], case["group"]
    rng = random.Random(n * 7919 + case["cached"] * 31 + case["new"])
    cached = [case["cached"]] + [g * rng.randint(0, case["cached"] // g) if case["ragged"] else case["cached"] for _ in range(n - 1)]
    new = [1 if case["mixed"] and i >= 2 else case["new"] for i in range(n)]
    tail = [rng.randint(0, case["tail"]) if case["ragged"] else case["tail"] for _ in range(n)]
    return cached, new, tail


def _row_bytes(case, tokens):
    """Bytes of `tokens` quantized keys and values of one head: codes, scales and zero-points."""
    meta = 4 if case["meta"] == "f32" else 2
    return 2 * tokens * (D * case["bits"] // 8 + 2 * meta * D // case["group"])


def work(case):
    kind = case["kind"]
    if kind == "rope":
        # queries and keys in and out, a position per axis; a turn is two products and a sum for each channel
        n, size = case["tokens"], 2 if case["dtype"] == "bf16" else 4
        heads, axes, turned = case["q_heads"] + case["kv_heads"], len(SECTIONS[case["sections"]]), 2 * sum(SECTIONS[case["sections"]])
        return {"bytes": n * (2 * heads * D * size + 4 * axes), "flops": n * heads * turned * 3}
    if kind in ("write", "read"):
        rows, read = case["tokens"] * case["kv_heads"], 2 if case["read"] == "bf16" else 4
        packed = _row_bytes(case, rows)
        if kind == "read":
            return {"bytes": packed + 2 * rows * D * read, "flops": 2 * rows * D * 2}
        # in, into the pages, out again (the pages' part is there to be read where it was just written)
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * rows * D * (size + read) + packed, "flops": 2 * rows * D * 8}
    cached, new, tail = _lengths(case)
    h, hq = case["kv_heads"], case["q_heads"]
    moved = sum(_row_bytes(case, c) for c in cached) * h + 2 * 2 * D * h * sum(n + t for n, t in zip(new, tail)) + 2 * 2 * D * hq * sum(new)
    pairs = sum(n * (c + t) + n * (n + 1) // 2 for c, n, t in zip(cached, new, tail))
    return {"bytes": moved, "flops": 4 * D * hq * pairs}


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _keys(gen, *shape):
    """Keys have a few channels with much larger values than the others."""
    k = _normal(gen, *shape)
    k[..., 5::32] *= 4.0
    return k


def _empty_pages(case, pages):
    h, p, g, meta = case["kv_heads"], case["page"], case["group"], DTYPES[case["meta"]]
    row = D * case["bits"] // 8
    z = lambda *shape, dtype: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    return [z(pages, h, p, row, dtype=torch.uint8), z(pages, h, p // g, D, dtype=meta), z(pages, h, p // g, D, dtype=meta),
            z(pages, h, p, row, dtype=torch.uint8), z(pages, h, p, D // g, dtype=meta), z(pages, h, p, D // g, dtype=meta)]


def _full_pages(case, pages, gen):
    """Pages that were written earlier, a few at a time."""
    to = _empty_pages(case, pages)
    g, bits, meta, step = case["group"], case["bits"], DTYPES[case["meta"]], max(1, (1 << 19) // (case["page"] * case["kv_heads"]))
    for a in range(0, pages, step):
        n = min(step, pages - a)
        k, v = _keys(gen, n, case["kv_heads"], case["page"], D), _normal(gen, n, case["kv_heads"], case["page"], D)
        c, to[1][a:a + n], to[2][a:a + n] = _key_codes(k.unflatten(2, (-1, g)), bits, meta)
        to[0][a:a + n] = _packed(c.flatten(2, 3), bits)
        c, to[4][a:a + n], to[5][a:a + n] = _value_codes(v.unflatten(3, (-1, g)), bits, meta)
        to[3][a:a + n] = _packed(c.flatten(3, 4), bits)
    return to


def prepare(case, seed):
    gen, kind = _generator(seed), case["kind"]
    s = dict(case)
    if kind == "rope":
        n, dtype, axes = case["tokens"], DTYPES[case["dtype"]], len(SECTIONS[case["sections"]])
        # as a fused projection leaves them: queries, keys and values of a token side by side
        qkv = _normal(gen, n, case["q_heads"] + 2 * case["kv_heads"], D).to(dtype)
        s["q"], s["k"] = qkv[:, :case["q_heads"]], qkv[:, case["q_heads"]:case["q_heads"] + case["kv_heads"]]
        s["q_out"], s["k_out"] = (torch.empty(x.shape, dtype=dtype, device="cuda") for x in (s["q"], s["k"]))
        start = torch.randint(0, 1 << 20, (1,), generator=gen, device="cuda")
        s["positions"] = (start + torch.randint(0, 4096, (axes, n), generator=gen, device="cuda")).to(torch.int32)
        if own:
            import paper_2503_24358_b200 as sq
            s["plan"] = sq.RopePlan(SECTIONS[case["sections"]], base=10000.0)
        return s
    if kind in ("write", "read"):
        n, h, g, p = case["tokens"], case["kv_heads"], case["group"], case["page"]
        pages = -(-n // p) + 2
        # the groups lie in pages in any order
        s["slots"] = (torch.randperm(pages * (p // g), generator=gen, device="cuda")[:n // g] * g).to(torch.int32)
        s["pages"] = _empty_pages(case, pages) if kind == "write" else _full_pages(case, pages, gen)
        if kind == "write":
            s["k"], s["v"] = _keys(gen, n, h, D).to(DTYPES[case["dtype"]]), _normal(gen, n, h, D).to(DTYPES[case["dtype"]])
        s["k_out"], s["v_out"] = (torch.empty((n, h, D), dtype=DTYPES[case["read"]], device="cuda") for _ in range(2))
    else:
        cached, new, tail = _lengths(case)
        n, hq, h, p = case["seqs"], case["q_heads"], case["kv_heads"], case["page"]
        need = [-(-c // p) for c in cached]
        s["pages"] = _full_pages(case, sum(need) + 1, gen)
        order = torch.randperm(sum(need) + 1, generator=gen, device="cuda").to(torch.int32)
        s["page_table"] = torch.zeros((n, max(1, max(need))), dtype=torch.int32, device="cuda")
        a = 0
        for i, m in enumerate(need):
            s["page_table"][i, :m] = order[a:a + m]
            a += m
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        sums = lambda x: [sum(x[:i]) for i in range(len(x) + 1)]  # noqa: E731
        s["q_start"], s["cached_len"] = ints(sums(new)), ints(cached)
        rows = [a + b for a, b in zip(new, tail)]
        s["new_start"], s["new_len"] = ints(sums(rows)[:-1]), ints(rows)
        s["max_q"], s["max_rows"] = max(new), max(rows)
        s["q"] = _normal(gen, sum(new), hq, D).to(torch.bfloat16)
        # keys and values of the rows in full precision, side by side
        kv = torch.cat((_keys(gen, sum(rows), h, D), _normal(gen, sum(rows), h, D)), 1).to(torch.bfloat16)
        s["k_new"], s["v_new"] = kv[:, :h], kv[:, h:]
        s["out"] = torch.empty((sum(new), hq, D), dtype=torch.bfloat16, device="cuda")
    if own:
        import paper_2503_24358_b200 as sq
        s["pool"] = sq.PagePool(*s["pages"])
        if kind == "attend":
            s["workspace"] = torch.empty(sq.squat_chunk_attention_workspace_bytes(s["q"].shape[0], hq, h, s["max_q"]), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _packed(codes, bits):
    """[..., d] codes as [..., d bits / 8] bytes, low bits first."""
    per = 8 // bits
    c = codes.to(torch.int32).unflatten(-1, (-1, per)) << torch.arange(0, 8, bits, device=codes.device, dtype=torch.int32)
    return c.sum(-1).to(torch.uint8)


def _unpacked(packed, bits):
    c = packed.unsqueeze(-1) >> torch.arange(0, 8, bits, device=packed.device, dtype=torch.uint8)
    return (c & ((1 << bits) - 1)).flatten(-2).float()


def _grid(x, dim, levels, meta):
    lo, hi = x.amin(dim, keepdim=True), x.amax(dim, keepdim=True)
    scale = (hi - lo) / levels
    return scale.to(meta), lo.to(meta)


def _key_codes(x, bits, meta):
    """x [..., groups, tokens, d] float32, a grid per channel: next to a border 32 bits would not say on which side a key lies."""
    levels = float(2 ** bits - 1)
    scale, zero = _grid(x, -2, levels, meta)
    codes = torch.round((x.double() - zero.double()) / scale.double()).clamp(0.0, levels)
    return torch.where(scale > 0, codes, 0.0), scale.squeeze(-2), zero.squeeze(-2)


def _value_codes(x, bits, meta):
    """x [..., groups, channels] float32, a grid per token, decided in 32 bits."""
    levels = float(2 ** bits - 1)
    scale, zero = _grid(x, -1, levels, meta)
    codes = torch.round((x - zero.float()) / scale.float()).clamp(0.0, levels)
    return torch.where(scale > 0, codes, 0.0), scale.squeeze(-1), zero.squeeze(-1)


def _slots(s):
    """Page, first group and first token in it of each slot."""
    slots = s["slots"].long()
    page, token = slots // s["page"], slots % s["page"]
    return page, token // s["group"], token.unsqueeze(1) + torch.arange(s["group"], device="cuda")


def _write_plain(s):
    g, bits, meta = s["group"], s["bits"], DTYPES[s["meta"]]
    page, group, token = _slots(s)
    kc, ks, kz, vc, vs, vz = s["pages"]
    codes, scale, zero = _key_codes(s["k"].float().unflatten(0, (-1, g)).transpose(1, 2), bits, meta)           # [slots, h, g, d]
    kc[page.unsqueeze(1), :, token] = _packed(codes, bits).transpose(1, 2)
    ks[page, :, group], kz[page, :, group] = scale, zero
    codes, scale, zero = _value_codes(s["v"].float().unflatten(0, (-1, g)).unflatten(3, (-1, g)), bits, meta)   # [slots, g, h, d / g, g]
    vc[page.unsqueeze(1), :, token] = _packed(codes.flatten(3, 4), bits)
    vs[page.unsqueeze(1), :, token], vz[page.unsqueeze(1), :, token] = scale, zero


def _read_plain(s):
    bits, g = s["bits"], s["group"]
    page, group, token = _slots(s)
    kc, ks, kz, vc, vs, vz = s["pages"]
    k = _unpacked(kc[page.unsqueeze(1), :, token], bits)                                                        # [slots, g, h, d]
    k = kz[page, :, group].float().unsqueeze(1) + ks[page, :, group].float().unsqueeze(1) * k
    v = _unpacked(vc[page.unsqueeze(1), :, token], bits).unflatten(3, (-1, g))
    v = vz[page.unsqueeze(1), :, token].float().unsqueeze(4) + vs[page.unsqueeze(1), :, token].float().unsqueeze(4) * v
    s["k_out"].copy_(k.flatten(0, 1))
    s["v_out"].copy_(v.flatten(3, 4).flatten(0, 1))
    return s["k_out"], s["v_out"]


def _rope_plain(s):
    sections = SECTIONS[s["sections"]]
    pairs = sum(sections)
    axis = torch.repeat_interleave(torch.arange(len(sections), device="cuda"), torch.tensor(sections, device="cuda"), output_size=pairs)
    theta = 10000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)
    angle = s["positions"][axis].double().T * theta                       # far positions: 32 bits would lose the angle
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    sin = -sin if s["inverse"] else sin

    def turned(x):
        x = x.float()
        a, b = x[..., :pairs], x[..., pairs:2 * pairs]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, x[..., 2 * pairs:]), -1)

    s["q_out"].copy_(turned(s["q"]))
    s["k_out"].copy_(turned(s["k"]))
    return s["q_out"], s["k_out"]


def _attend_plain(s):
    """All sequences at once, padded to the longest one."""
    n, hq, h, bits, g, max_q = s["seqs"], s["q_heads"], s["kv_heads"], s["bits"], s["group"], s["max_q"]
    kc, ks, kz, vc, vs, vz = (t[s["page_table"]].transpose(1, 2) for t in s["pages"])                          # [n, h, pages, ...]
    k = (kz.float().unsqueeze(4) + ks.float().unsqueeze(4) * _unpacked(kc, bits).unflatten(3, (-1, g))).flatten(2, 4)
    v = (vz.float().unsqueeze(5) + vs.float().unsqueeze(5) * _unpacked(vc, bits).unflatten(4, (-1, g))).flatten(4, 5).flatten(2, 3)
    row = torch.arange(s["max_rows"], device="cuda")
    rows = (s["new_start"].unsqueeze(1) + row).clamp(max=s["k_new"].shape[0] - 1)
    k = torch.cat((k, s["k_new"][rows].float().transpose(1, 2)), 2)                                             # [n, h, tokens, d]
    v = torch.cat((v, s["v_new"][rows].float().transpose(1, 2)), 2)
    query = torch.arange(max_q, device="cuda")
    first, many = s["q_start"][:-1], s["q_start"][1:] - s["q_start"][:-1]
    q = s["q"][(first.unsqueeze(1) + query).clamp(max=s["q"].shape[0] - 1)].float()                             # [n, max_q, hq, d]
    q = q.unflatten(2, (h, hq // h)).permute(0, 2, 3, 1, 4).flatten(2, 3)                                       # [n, h, heads x max_q, d]
    scores = (q @ k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    cache = s["page_table"].shape[1] * s["page"]
    seen = torch.cat(((torch.arange(cache, device="cuda") < s["cached_len"].unsqueeze(1)).unsqueeze(1).expand(n, max_q, cache),
                      row <= (query.unsqueeze(0) + (s["new_len"] - many).unsqueeze(1)).unsqueeze(2)), 2)        # [n, max_q, tokens]
    scores = scores.unflatten(2, (-1, max_q)).masked_fill_(~seen[:, None, None], -math.inf).flatten(2, 3)
    scores = torch.exp(scores - scores.amax(3, keepdim=True))
    out = (scores @ v) / scores.sum(3, keepdim=True)
    out = out.unflatten(2, (-1, max_q)).permute(0, 3, 1, 2, 4).flatten(2, 3)                                    # [n, max_q, hq, d]
    every = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(s["q_start"][1:], every, right=True)
    s["out"].copy_(out[seq, every - first[seq]])
    return s["out"]


def run(s):
    kind = s["kind"]
    if not own:
        if kind == "rope":
            return _rope_plain(s)
        if kind == "read":
            return _read_plain(s)
        if kind == "write":
            _write_plain(s)
            return (*_read_plain(s), *s["pages"][1:3], *s["pages"][4:])
        return _attend_plain(s)
    import paper_2503_24358_b200 as sq
    if kind == "rope":
        sq.squat_rope_apply(s["plan"], s["positions"], s["q"], s["k"], s["q_out"], s["k_out"], inverse=s["inverse"])
        return s["q_out"], s["k_out"]
    if kind == "attend":
        sq.squat_chunk_attention(s["q"], s["pool"], s["q_start"], s["cached_len"], s["page_table"], s["out"], s["workspace"], s["max_q"],
                                 s["k_new"], s["v_new"], s["new_start"], s["new_len"])
        return s["out"]
    if kind == "write":
        sq.squat_pages_write(s["pool"], s["slots"], s["k"], s["v"])
    sq.squat_pages_read(s["pool"], s["slots"], s["k_out"], s["v_out"])
    return (s["k_out"], s["v_out"]) if kind == "read" else (s["k_out"], s["v_out"], *s["pages"][1:3], *s["pages"][4:])


# ------------------------------------------------------------------------------------------------ in 64 bits
def _codes64(packed, bits):
    """Codes by division, one of a byte at a time."""
    p, base, found = packed.to(torch.float64), 2.0 ** bits, []
    for _ in range(8 // bits):
        found.append(torch.remainder(p, base))
        p = torch.floor(p / base)
    return torch.stack(found, -1).flatten(-2)


def _expanded(meta, group, dim):
    return meta.double().repeat_interleave(group, dim)


def _exact_pages(s, where):
    """Keys and values, [tokens, heads, d], of the pages' token places `where` (page x page size + token)."""
    kc, ks, kz, vc, vs, vz = s["pages"]
    g, d = s["group"], D
    flat = lambda t: t.transpose(1, 2).reshape(-1, t.shape[1], t.shape[3])  # noqa: E731
    at = where // g
    k = flat(kz)[at].double() + flat(ks)[at].double() * _codes64(flat(kc)[where], s["bits"])
    v = _expanded(flat(vz)[where], g, 2) + _expanded(flat(vs)[where], g, 2) * _codes64(flat(vc)[where], s["bits"])
    return k[..., :d], v[..., :d]


def _exact_rope(s):
    sections = SECTIONS[s["sections"]]
    half = sum(sections)
    bounds = [sum(sections[:i + 1]) for i in range(len(sections))]
    sign = -1.0 if s["inverse"] else 1.0
    outs = []
    for x in (s["q"], s["k"]):
        y = x.double().clone()
        for i in range(half):
            ax = next(a for a, b in enumerate(bounds) if i < b)
            turn = torch.polar(torch.ones_like(s["positions"][ax], dtype=torch.float64), sign * s["positions"][ax].double() * 10000.0 ** (-i / half))
            z = torch.complex(x[..., i].double(), x[..., half + i].double()) * turn.unsqueeze(1)
            y[..., i], y[..., half + i] = z.real, z.imag
        outs.append(y)
    return tuple(outs)


def _exact_write(s):
    """A slot's grids and the values that the nearest of their levels stand for."""
    g, levels, meta = s["group"], 2 ** s["bits"] - 1, DTYPES[s["meta"]]
    stored = lambda t: t.to(torch.float32).to(meta)  # noqa: E731  (as the definition stores them)
    k, v = s["k"].float(), s["v"].float()
    n, h = k.shape[0] // g, k.shape[1]
    k, v = k.reshape(n, g, h, D), v.reshape(n, g, h, D // g, g)
    outs, pages = [], [t.double() for t in (*s["pages"][1:3], *s["pages"][4:])]
    for x, dim, scales, zeros in ((k, 1, pages[0], pages[1]), (v, 4, pages[2], pages[3])):
        low, high = x.min(dim, keepdim=True).values, x.max(dim, keepdim=True).values
        step, zero = stored((high - low) / levels), stored(low)
        wide = torch.float64 if dim == 1 else torch.float32                # values: decided in 32 bits, by definition
        code = torch.round(torch.nan_to_num((x.to(wide) - zero.to(wide)) / step.to(wide), 0.0, 0.0, 0.0)).clamp(0, levels)
        outs.append((zero.double() + step.double() * code.double()).reshape(n * g, h, D))
        slots = s["slots"].long()
        page, place = slots // s["page"], slots % s["page"]
        for t, to in ((step, scales), (zero, zeros)):
            if dim == 1:
                to[page, :, place // g] = t.squeeze(1).double()
            else:
                for i in range(g):
                    to[page, :, place + i] = t[:, i].squeeze(-1).double()
    return (*outs, *pages)


def _exact_attend(s):
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    h, per = s["kv_heads"], s["q_heads"] // s["kv_heads"]
    starts, cached, first, many = (s[x].tolist() for x in ("q_start", "cached_len", "new_start", "new_len"))
    for i in range(s["seqs"]):
        at = torch.arange(cached[i], device="cuda")
        k, v = _exact_pages(s, s["page_table"][i, at // s["page"]].long() * s["page"] + at % s["page"])
        rows = slice(first[i], first[i] + many[i])
        k, v = torch.cat((k, s["k_new"][rows].double())), torch.cat((v, s["v_new"][rows].double()))
        q = s["q"][starts[i]:starts[i + 1]].double()
        hidden = torch.ones(q.shape[0], k.shape[0], dtype=torch.bool, device="cuda").triu(k.shape[0] - q.shape[0] + 1)
        for j in range(h):
            mine = q[:, j * per:(j + 1) * per]
            scores = torch.einsum("qhd,td->hqt", mine, k[:, j]).div(math.sqrt(D)).masked_fill(hidden, -math.inf)
            out[starts[i]:starts[i + 1], j * per:(j + 1) * per] = torch.einsum("hqt,td->qhd", torch.softmax(scores, 2), v[:, j])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "rope":
        return _exact_rope(s)
    if s["kind"] == "write":
        return _exact_write(s)
    if s["kind"] == "read":
        slots = s["slots"].long().unsqueeze(1) + torch.arange(s["group"], device="cuda")
        return _exact_pages(s, slots.reshape(-1))
    return _exact_attend(s)

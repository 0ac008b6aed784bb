"""More operators that answer from the selected frames, as they are timed: a cache of 8-bit pages, attention over it, and
attention for sequences that share a long prefix.

Kinds of case (the "op" of a case dict):

  append  the new tokens of a batch of sequences into 8-bit pages, keys rotated on the way (and queries, where the case
          has them); what was written is read back, as the numbers that it stands for
  attend  the new tokens' queries over what 8-bit pages hold of their sequences, causal; with "keep" a mask leaves about
          that share of the earlier frames visible, and one of the sequences nothing at all
  shared  groups of sequences (questions or answers about one stream): every sequence of a group sees the group's prefix,
          then its own cached tokens, causal among those; pages of 16 bits, 8 or 4; with "keep" each sequence has a mask
          over the prefix's frames, and one of them sees nothing of it

A sequence's cached tokens lie in pages of "page" tokens, whose numbers a table gives in no order; a group's prefix has a
row of such a table of its own. Pages hold rows [page][head][token][dim] of 16-bit values, of bytes, or of 4-bit codes, two
to a byte. Beside bytes and codes lies a word for every 64 of them. 8 bits: a byte u and a scale s, a power of two as a bf16
number, stand for (u - 128) s; s is the smallest that brings all 64 values to 127 at most (of those whose 127 the type
holds; past that, values are cut). 4 bits: the word is a bf16 scale
of 4 significant bits, with the zero point in its low 4 bits.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 64  # values that share a scale
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
LEAST = {"bf16": -100, "fp16": -24}  # exponents of the smallest scale of 8-bit codes
MOST = {"bf16": 121, "fp16": 9}      # and of the largest: the type holds 127 of it


def _append(name, seqs, new, before, **kw):
    return {"name": name, "op": "append", "seqs": seqs, "new": new, "before": before, "heads": 32, "kv_heads": 8,
            "head_dim": 128, "rotary_dim": 128, "layout": "half", "axes": 1, "queries": True, "page": 64, "bits": 8,
            "dtype": "bf16", **kw}


def _attend(name, seqs, new, longest, **kw):
    return {"name": name, "op": "attend", "seqs": seqs, "new": new, "longest": longest, "heads": 32, "kv_heads": 8,
            "head_dim": 128, "page": 64, "bits": 8, "dtype": "bf16", "keep": 1.0, "frame": 256, **kw}


def _shared(name, groups, seqs, new, prefix, own_tokens, **kw):
    return {"name": name, "op": "shared", "groups": groups, "seqs": seqs, "new": new, "prefix": prefix, "own": own_tokens,
            "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64, "bits": 16, "dtype": "bf16", "keep": 1.0, "frame": 256, **kw}


def listed():
    return [
        # one new token of each of 32 answers, with its queries
        _append("append_step_8bit", 32, 1, 1000),
        # nine streams' frames
        _append("append_frames_8bit", 9, 12544, 500, axes=3, queries=False),
        # the first token of an answer over a few frames: latency
        _attend("answer_short_8bit", 1, 1, 1111),
        # a server's step: 32 answers of very different lengths
        _attend("answer_batch_8bit", 32, 1, 16384),
        # three tokens at a time over the evidence alone
        _attend("answer_evidence_8bit", 24, 3, 20001, heads=28, kv_heads=4, dtype="fp16", keep=0.3, frame=196),
        # a question of 256 tokens over 256 frames
        _attend("question_8bit", 1, 256, 65792),
        # four answers about a short stream: latency
        _shared("shared_step", 1, 4, 1, 5000, 40),
        # 32 answers about one stream of 1024 frames of 256 tokens
        _shared("shared_answers", 1, 32, 1, 262144, 700),
        # the same with 8 bits
        _shared("shared_answers_8bit", 1, 32, 1, 262144, 700, bits=8),
        # five streams with up to nine answers each
        _shared("shared_streams_fp16", 5, 9, 1, 50001, 1500, heads=28, kv_heads=4, dtype="fp16", page=32),
        # sixteen questions, each with the frames that are its evidence
        _shared("shared_evidence_4bit", 1, 16, 24, 100001, 60, bits=4, keep=0.3),
        # eight questions of up to 200 tokens about one stream, the largest
        _shared("shared_questions_8bit", 1, 8, 200, 65792, 200, bits=8),
    ]


HEADS = ((32, 8, 128), (32, 8, 128), (28, 4, 128), (16, 8, 64), (16, 16, 64), (14, 2, 64), (8, 1, 128))


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "shared", "shared", "shared"))
    heads, kv_heads, head_dim = rng.choice(HEADS)
    dtype, page = rng.choice(("bf16", "bf16", "fp16")), rng.choice((16, 32, 64, 128))
    size = kv_heads * head_dim
    if op == "append":
        seqs, axes, queries = _log(rng, 1, 64), rng.choice((1, 1, 3)), rng.random() < 0.5
        most = 65536 * 8 * 128 // (size * seqs)
        c = _append("", seqs, _log(rng, 1, max(1, min(32768, most // 4 if queries else most))), _log(rng, 1, 2000),
                    heads=heads, kv_heads=kv_heads, head_dim=head_dim, layout=rng.choice(("half", "interleaved")), axes=axes,
                    rotary_dim=head_dim if rng.random() < 0.6 else rng.choice((16, 32, 48, head_dim // 2)),
                    queries=queries, page=page, dtype=dtype)
    elif op == "attend":
        seqs = _log(rng, 1, 48)
        new = 1 if rng.random() < 0.4 else _log(rng, 1, 400)
        # at most the largest listed cases' bytes and products, in the padded form too
        most = min(262144 * 8 * 128 // (seqs * size), 256 * 65792 * 32 * 128 // (seqs * new * heads * head_dim))
        c = _attend("", seqs, new, _log(rng, 1, max(1, most)), heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page,
                    dtype=dtype, keep=rng.choice((1.0, 1.0, 0.2, 0.5)), frame=rng.choice((49, 100, 144, 196, 256)))
    else:
        groups = 1 if rng.random() < 0.5 else _log(rng, 2, 12)
        seqs = _log(rng, 1, max(1, 64 // groups))
        new = 1 if rng.random() < 0.5 else _log(rng, 1, 256)
        own_tokens = _log(rng, 1, max(1, min(4000, 262144 // (groups * seqs))))
        most = min(262144 * 8 * 128 // (groups * size), 1024 * 65792 * 32 * 128 // (groups * seqs * new * heads * head_dim))
        c = _shared("", groups, seqs, new, _log(rng, 1, max(1, most)), own_tokens, heads=heads, kv_heads=kv_heads,
                    head_dim=head_dim, page=page, bits=rng.choice((4, 8, 8, 16)), dtype=dtype,
                    keep=rng.choice((1.0, 1.0, 1.0, 0.3)), frame=rng.choice((49, 100, 144, 196, 256)))
    del c["name"]
    return c


# ---- sizes ----------------------------------------------------------------------------------------------------------


def _spread(n, lo, hi):
    """n whole numbers from hi down to lo, in an order of their own; hi alone where n is 1."""
    step = next(s for s in (7, 5, 3, 11, 1) if math.gcd(s, n) == 1)
    return [hi - (hi - lo) * ((i * step) % n) // max(1, n - 1) for i in range(n)]


def _members(c):
    """Sequences of each group."""
    return _spread(c["groups"], max(1, c["seqs"] // 2), c["seqs"])


def _prefixes(c):
    return _spread(c["groups"], max(1, c["prefix"] // 3), c["prefix"])[::-1]


def _sizes(c):
    """(new tokens, cached tokens with them) of each sequence; behind the prefix, where there is one."""
    n = sum(_members(c)) if c["op"] == "shared" else c["seqs"]
    new = _spread(n, max(1, c["new"] // 3), c["new"])
    if c["op"] == "append":
        return new, [a + b for a, b in zip(new, _spread(n, c["before"] // 2, c["before"])[::-1])]
    if c["op"] == "shared":
        return new, [a + b for a, b in zip(new, _spread(n, 0, c["own"])[::-1])]
    return new, _spread(n, min(c["longest"], max(1, c["longest"] // 20)), c["longest"])[::-1]


def _row(c):
    """Bytes of one token's keys, or values, in the pages."""
    return c["kv_heads"] * (c["head_dim"] * c["bits"] // 8 + (2 * (c["head_dim"] // GROUP) if c["bits"] < 16 else 0))


def _pairs(n, m):
    return n * m - n * (n - 1) // 2 if m >= n else m * (m + 1) // 2


def work(case):
    c = case
    h, hk, d, row = c["heads"], c["kv_heads"], c["head_dim"], _row(c)
    new, have = _sizes(c)
    t = sum(new)
    if c["op"] == "append":
        moved = 2 * 2 * t * (2 * hk * d + row) + (4 * t * h * d if c["queries"] else 0)  # written, and read back
        return {"bytes": moved + 4 * c["axes"] * t, "flops": 3 * t * c["rotary_dim"] * (hk + (h if c["queries"] else 0)) + 4 * t * hk * d}
    outer = 4 * t * h * d + 4 * t * h  # queries, outputs and log-sum-exps
    if c["op"] == "attend":
        share = 1.0 if c["keep"] >= 1 else c["keep"] * (1 - 1 / c["seqs"] if c["seqs"] > 1 else 1)
        pairs = sum(_pairs(n, m) for n, m in zip(new, have)) * share
        return {"bytes": 2 * sum(have) * share * row + (sum(have) if share < 1 else 0) + outer, "flops": 4 * pairs * h * d}
    pairs, read, masks, at = sum(_pairs(n, m) for n, m in zip(new, have)), sum(have), 0, 0
    for many, p in zip(_members(c), _prefixes(c)):
        share = c["keep"] if c["keep"] < 1 else 1.0
        pairs += sum(new[at:at + many]) * p * share
        read += p * (1 - (1 - share) ** many)  # a frame is read where any of the group sees it
        masks += many * p if share < 1 else 0
        at += many
    return {"bytes": 2 * read * row + masks + outer, "flops": 4 * pairs * h * d}


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _frequencies(c):
    return [1e6 ** (-2 * i / c["rotary_dim"]) for i in range(c["rotary_dim"] // 2)]


def _axes(c):
    """The position axis of each pair: frame, row and column in turn."""
    return [i % c["axes"] for i in range(c["rotary_dim"] // 2)]


def _normal(shape, dtype, g, spread=None):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if spread is not None:
        x *= spread
    return x.to(dtype)


def _channels(c, g):
    """Keys differ from channel to channel: some carry a few times the others' size."""
    return torch.exp(0.3 * torch.randn((c["kv_heads"], c["head_dim"]), generator=g, device="cuda")).clamp(0.3, 2.5)


def _positions(c, n, g):
    if c["axes"] == 1:
        return torch.randint(0, 131072, (n,), generator=g, device="cuda", dtype=torch.int32)
    t = torch.arange(n, device="cuda", dtype=torch.int32)
    first = torch.randint(0, 4096, (1,), generator=g, device="cuda", dtype=torch.int32)
    return torch.stack([first + t // 256, first + t % 256 // 16, first + t % 16])[:c["axes"]].contiguous()


def _bytes_of(x, kind):
    """Bytes and words of x's last axis, in groups: [..., d] -> uint8 [..., d], int16 [..., d / GROUP]."""
    y = x.float().unflatten(-1, (-1, GROUP))
    top = y.abs().amax(-1)
    # top = f 2^e, f in [1, 2): 2^(e - 6) is enough for f up to 127 / 64; the sum carries into the exponent above that
    field = (((top.view(torch.int32) + 0x1FFFF) >> 23) - 6).clamp(127 + LEAST[kind], 127 + MOST[kind])
    inverse = ((254 - field) << 23).view(torch.float32)
    n = torch.round(y * inverse.unsqueeze(-1)).clamp(-127, 127)  # halves to even
    return (n + 128).to(torch.uint8).flatten(-2), (field << 7).to(torch.int16)


def _values_of(u, words):
    """What bytes and words stand for, in fp32."""
    scale = words.view(torch.bfloat16).float().unsqueeze(-1)
    return ((u.unflatten(-1, (-1, GROUP)).float() - 128.0) * scale).flatten(-2)


def _codes_of(x):
    """4-bit codes and words of x's last axis: [..., d] -> uint8 [..., d / 2], int16 [..., d / GROUP]."""
    y = x.float().unflatten(-1, (-1, GROUP))
    lo, hi = y.amin(-1).clamp(max=0.0), y.amax(-1).clamp(min=0.0)
    scale = (((hi - lo) / 15).view(torch.int32) + 0xFFFFF & ~0xFFFFF).view(torch.float32)
    zero = (0.5 - lo / scale).floor().clamp(0, 15)
    codes = ((y / scale.unsqueeze(-1)).round() + zero.unsqueeze(-1)).clamp(0, 15).to(torch.uint8).flatten(-2)
    return codes[..., 0::2] | codes[..., 1::2] << 4, scale.to(torch.bfloat16).view(torch.int16) | zero.to(torch.int16)


def _numbers_of(codes, words):
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, GROUP)).float()
    scale = (words & -16).view(torch.bfloat16).float().unsqueeze(-1)
    return ((n - (words & 15).unsqueeze(-1).float()) * scale).flatten(-2)


def _pages(pool, c):
    """The pool as pages of the case's bits: {"pages", "scales"}."""
    if c["bits"] == 16:
        return pool, None
    # in pieces: the fp32 copies of a whole long cache would be large
    parts = [_bytes_of(p, c["dtype"]) if c["bits"] == 8 else _codes_of(p) for p in pool.split(1024)]
    return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def _frames(c, seqs, longest, g):
    """uint8 [seqs, longest]: frames that each sequence sees, nothing for one of them."""
    kept = torch.rand((seqs, -(-longest // c["frame"])), generator=g, device="cuda") < c["keep"]
    mask = kept.repeat_interleave(c["frame"], 1)[:, :longest]
    if seqs > 1:
        mask[seqs // 2] = False
    return mask


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    h, hk, d, dtype, page = c["heads"], c["kv_heads"], c["head_dim"], TYPES[c["dtype"]], c["page"]
    new, have = _sizes(c)
    t, seqs = sum(new), len(new)
    prefixes = _prefixes(c) if c["op"] == "shared" else []
    each = [-(-m // page) for m in have + prefixes]
    pages = sum(each) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)

    def table_of(counts, numbers):
        table = torch.zeros((len(counts), max(counts)), dtype=torch.int32, device="cuda")
        table[torch.arange(max(counts), device="cuda") < torch.tensor(counts, device="cuda")[:, None]] = numbers
        return table

    lengths = torch.tensor(have, dtype=torch.int32, device="cuda")
    offsets = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.tensor(new, device="cuda").cumsum(0)
    spread = _channels(c, g)
    s = {"case": c, "table": table_of(each[:seqs], order[:sum(each[:seqs])]), "lengths": lengths, "offsets": offsets, "most": max(new)}
    s["k_pages"], s["k_scales"] = _pages(_normal((pages, page, hk, d), dtype, g, spread).transpose(1, 2).contiguous(), c)
    s["v_pages"], s["v_scales"] = _pages(_normal((pages, hk, page, d), dtype, g), c)
    s["mask"] = s["prefix_mask"] = None
    if c["op"] == "append":
        s["k"], s["v"] = _normal((t, hk, d), dtype, g, spread), _normal((t, hk, d), dtype, g)
        s["q"] = _normal((t, h, d), dtype, g) if c["queries"] else None
        s["qo"] = torch.empty_like(s["q"]) if c["queries"] else None
        s["positions"] = _positions(c, t, g)
        s["ro"] = [torch.empty((t, hk, d), dtype=dtype, device="cuda") for _ in range(2)]
        # the plain form's plan: each pair's turn per position as a 64-bit fraction, so that far positions keep their angle
        s["turns"] = torch.tensor([int(x / (2 * math.pi) * 2.0 ** 64) for x in _frequencies(c)], dtype=torch.int64, device="cuda")
        s["axis"] = torch.tensor(_axes(c), device="cuda")
    else:
        s["q"] = 1.3 * _normal((t, h, d), dtype, g)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((t, h), dtype=torch.float32, device="cuda")
        if c["op"] == "attend" and c["keep"] < 1:
            fresh = torch.arange(max(have), device="cuda") >= (lengths - offsets.diff())[:, None]  # the new tokens
            mask = _frames(c, seqs, max(have), g) | fresh
            if seqs > 1:
                mask[seqs // 2] = False  # nothing of this one
            s["mask"] = mask.to(torch.uint8).contiguous()
        if c["op"] == "shared":
            members = _members(c)
            s["groups"] = torch.zeros(len(members) + 1, dtype=torch.int32, device="cuda")
            s["groups"][1:] = torch.tensor(members, device="cuda").cumsum(0)
            s["prefix_table"] = table_of(each[seqs:], order[sum(each[:seqs]):sum(each)])
            s["prefix_lengths"] = torch.tensor(prefixes, dtype=torch.int32, device="cuda")
            ends = [sum(members[:i + 1]) for i in range(len(members))]
            s["most_shared"] = max(sum(new[e - m:e]) for e, m in zip(ends, members))
            if c["keep"] < 1:
                s["prefix_mask"] = _frames(c, seqs, max(prefixes), g).to(torch.uint8).contiguous()
    if own:
        from paper_2609_03675_gb300 import KVCache, Rotary

        rotary = None
        if c["op"] == "append":
            rotary = Rotary(d, rotary_dim=c["rotary_dim"], base=1e6, layout=c["layout"], axes=_axes(c) if c["axes"] > 1 else None)
        s["cache"] = KVCache(pages, page, h, hk, d, dtype=dtype, bits="int8" if c["bits"] == 8 else c["bits"], rotary=rotary,
                             k_pages=s["k_pages"], v_pages=s["v_pages"], k_scales=s["k_scales"], v_scales=s["v_scales"])
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    c, cache = s["case"], s["cache"]
    batch = s["table"], s["lengths"], s["offsets"]
    if c["op"] == "append":
        cache.append(s["k"], s["v"], *batch, positions=s["positions"], q=s["q"], q_out=s["qo"])
        return s["qo"], *cache.read(*batch, out=s["ro"])
    if c["op"] == "attend":
        return cache.attend(s["q"], *batch, max_new=s["most"], mask=s["mask"], out=s["out"], lse=s["lse"])
    return cache.attend_shared(s["q"], *batch, prefix_table=s["prefix_table"], prefix_lengths=s["prefix_lengths"],
                               groups=s["groups"], max_new=s["most"], max_shared=s["most_shared"], prefix_mask=s["prefix_mask"],
                               out=s["out"], lse=s["lse"])


def _plain(s):
    return {"append": _plain_append, "attend": _plain_attend, "shared": _plain_shared}[s["case"]["op"]](s)


def _rotated(x, s):
    """x [n, heads, d] in fp32, rotated."""
    c = s["case"]
    half = c["rotary_dim"] // 2
    p = s["positions"].long()
    p = p[s["axis"]].T if c["axes"] > 1 else p[:, None]
    a = ((p * s["turns"]) >> 32).float() * (math.pi / 2.0 ** 31)  # the products wrap, as turns do
    cos, sin = a.cos()[:, None], a.sin()[:, None]
    x = x.float()
    if c["layout"] == "half":
        x1, x2 = x[..., :half], x[..., half:2 * half]
        return torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin, x[..., 2 * half:]], -1)
    x1, x2 = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
    return torch.cat([torch.stack([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1).flatten(-2), x[..., 2 * half:]], -1)


def _plain_append(s):
    c = s["case"]
    dtype = s["k"].dtype
    t = torch.arange(int(s["k"].shape[0]), device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["offsets"], t, right=True) - 1
    at = (s["lengths"] - s["offsets"][1:])[seq] + t
    page, place = s["table"][seq, at // c["page"]].long(), (at % c["page"]).long()
    q = _rotated(s["q"], s).to(dtype) if c["queries"] else None
    k, kw = _bytes_of(_rotated(s["k"], s), c["dtype"])
    v, vw = _bytes_of(s["v"], c["dtype"])
    s["k_pages"][page, :, place], s["k_scales"][page, :, place] = k, kw
    s["v_pages"][page, :, place], s["v_scales"][page, :, place] = v, vw
    return (q, _values_of(s["k_pages"][page, :, place], s["k_scales"][page, :, place]).to(dtype),
            _values_of(s["v_pages"][page, :, place], s["v_scales"][page, :, place]).to(dtype))


def _cached(s, name, table):
    """[rows of the table, kv heads, tokens, d] in fp32, tokens up to whole pages."""
    at, bits = table.long(), s["case"]["bits"]
    x = s[name + "_pages"][at]
    x = x.float() if bits == 16 else (_values_of if bits == 8 else _numbers_of)(x, s[name + "_scales"][at])
    return x.transpose(1, 2).flatten(2, 3)


def _part(s, table, first, count, most, seen):
    """Attention of token rows first .. first + count of each row of the table over its tokens, `seen` [rows, most, tokens]:
    the maximum, the sum of exponentials above it and the sum of values, for each token of the call, [tokens, heads, ...]."""
    c = s["case"]
    h, hk, d = c["heads"], c["kv_heads"], c["head_dim"]
    i = torch.arange(most, device="cuda", dtype=torch.int32)
    real = i < count[:, None]
    rows = torch.where(real, first[:, None] + i, 0).long()
    q = s["q"].float()[rows].unflatten(2, (hk, h // hk)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [rows, kv heads, group x most, d]
    x = q @ _cached(s, "k", table).transpose(2, 3) * d ** -0.5
    x = x.unflatten(2, (h // hk, most)).masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    e = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = e.sum(-1, keepdim=True)
    o = (e.flatten(2, 3) @ _cached(s, "v", table)).unflatten(2, (h // hk, most))
    return [y.permute(0, 3, 1, 2, 4).flatten(2, 3)[real] for y in (top, total, o)]


def _own_part(s):
    count, first = s["offsets"].diff(), s["offsets"][:-1]
    tokens = torch.arange(s["table"].shape[1] * s["case"]["page"], device="cuda")
    i = torch.arange(s["most"], device="cuda", dtype=torch.int32)
    seen = tokens <= ((s["lengths"] - count)[:, None] + i)[..., None]  # [seqs, new, tokens]
    if s["mask"] is not None:
        seen &= torch.nn.functional.pad(s["mask"], (0, len(tokens) - s["mask"].shape[1])).bool()[:, None]
    return _part(s, s["table"], first, count, s["most"], seen)


def _finished(top, total, o, dtype):
    out = o / torch.where(total > 0, total, 1.0)
    return out.to(dtype), (top + total.log()).squeeze(-1)


def _plain_attend(s):
    return _finished(*_own_part(s), s["q"].dtype)


def _plain_shared(s):
    starts = s["offsets"][s["groups"].long()]
    first, count, most = starts[:-1], starts.diff(), s["most_shared"]
    tokens = torch.arange(s["prefix_table"].shape[1] * s["case"]["page"], device="cuda")
    seen = (tokens < s["prefix_lengths"][:, None])[:, None]  # [groups, 1, tokens]
    if s["prefix_mask"] is not None:
        mask = torch.nn.functional.pad(s["prefix_mask"], (0, len(tokens) - s["prefix_mask"].shape[1])).bool()
        row = (first[:, None] + torch.arange(most, device="cuda", dtype=torch.int32)).clamp(max=int(s["q"].shape[0]) - 1)
        seq = (torch.searchsorted(s["offsets"], row, right=True) - 1).clamp(max=len(mask) - 1)
        seen = seen & mask[seq]
    top_p, total_p, o_p = _part(s, s["prefix_table"], first, count, most, seen)
    top_o, total_o, o_o = _own_part(s)
    top = torch.maximum(top_p, top_o)
    base = torch.where(top == -math.inf, 0.0, top)
    by_p, by_o = (top_p - base).exp(), (top_o - base).exp()
    return _finished(top, total_p * by_p + total_o * by_o, o_p * by_p + o_o * by_o, s["q"].dtype)


# ---- the definition, in 64 bits -------------------------------------------------------------------------------------


def _exact_turn(x, positions, c):
    p = positions.double().reshape(c["axes"], -1)
    a = torch.stack([p[ax] * w for ax, w in zip(_axes(c), _frequencies(c))], 1)
    z = torch.polar(torch.ones_like(a), a)[:, None]
    y, half = x.double().clone(), c["rotary_dim"] // 2
    one, two = (slice(0, half), slice(half, 2 * half)) if c["layout"] == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    w = torch.complex(x[..., one].double(), x[..., two].double()) * z
    y[..., one], y[..., two] = w.real, w.imag
    return y


def _exact_eight_bits(x, kind):
    """The whole multiple of its group's scale nearest to each x."""
    y = x.double().reshape(*x.shape[:-1], -1, GROUP)
    part, power = torch.frexp(y.abs().max(-1, keepdim=True).values)
    power = torch.where(part <= 127 / 128, power - 7, power - 6).clamp(LEAST[kind], MOST[kind])
    step = (power.long() + 1023 << 52).view(torch.float64)  # 2^power to the last bit, which ldexp is not
    return (torch.round(y / step).clamp(-127, 127) * step).reshape(x.shape)


def _held(s, name, rows, c):
    """[kv heads, tokens, d] of one row of a table, in 64 bits."""
    x = s[name + "_pages"][rows.long()]
    if c["bits"] < 16:
        w = (s[name + "_scales"][rows.long()].int() & 0xFFFF)[..., None]
        codes = (x if c["bits"] == 8 else torch.stack([x % 16, x // 16], -1).reshape(*x.shape[:-1], -1))
        codes = codes.double().reshape(*x.shape[:-1], -1, GROUP)
        if c["bits"] == 8:  # the word's bits: 8 of exponent, 7 of nothing
            x = (codes - 128) * torch.exp2((w >> 7).double() - 127)
        else:  # 8 of exponent, 3 of mantissa, 4 of zero point
            x = (codes - w % 16) * ((8 + (w >> 4 & 7)).double() * torch.exp2((w >> 7).double() - 130))
        x = x.flatten(-2)
    return x.double().transpose(0, 1).reshape(c["kv_heads"], -1, c["head_dim"])


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    h, hk, d = c["heads"], c["kv_heads"], c["head_dim"]
    if c["op"] == "append":
        q = _exact_turn(s["q"], s["positions"], c) if c["queries"] else None
        return q, _exact_eight_bits(_exact_turn(s["k"], s["positions"], c), c["dtype"]), _exact_eight_bits(s["v"], c["dtype"])
    new, have = _sizes(c)
    members, prefixes = (_members(c), _prefixes(c)) if c["op"] == "shared" else ([c["seqs"]], [0])
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    b = t = 0
    for i, (many, p) in enumerate(zip(members, prefixes)):
        ahead = [_held(s, name, s["prefix_table"][i, :-(-p // c["page"])], c)[:, :p] for name in "kv"] if p else None
        for b in range(b, b + many):
            n, m = new[b], have[b]
            own_kv = [_held(s, name, s["table"][b, :-(-m // c["page"])], c)[:, :m] for name in "kv"]
            at, last = torch.arange(m, device="cuda"), torch.arange(m - n, m, device="cuda")
            seen = at[None] <= last[:, None]
            if s["mask"] is not None:
                seen = seen & (s["mask"][b, :m] != 0)[None]
            if p:
                before = s["prefix_mask"][b, :p] != 0 if s["prefix_mask"] is not None else torch.ones(p, dtype=torch.bool, device="cuda")
                seen = torch.cat([before[None].expand(n, -1), seen], 1)
            for j in range(h):
                k, v = [torch.cat([a[j // (h // hk)], o[j // (h // hk)]]) for a, o in zip(ahead, own_kv)] if p else [o[j // (h // hk)] for o in own_kv]
                x = torch.where(seen, s["q"][t:t + n, j].double() @ k.T / math.sqrt(d), -math.inf)
                lse[t:t + n, j] = torch.logsumexp(x, 1)
                w = torch.where(seen.any(1)[:, None], torch.softmax(x, 1), 0.0)
                out[t:t + n, j] = w @ v
            t += n
        b += 1
    return out, lse

"""The operators that answer a question from the selected frames, as they are timed: rotary positions, appending to a
paged key/value cache, and attention over that cache.

Kinds of case (the "op" of a case dict):

  rotary  queries and keys of some tokens rotated to their positions, or, with "backward", their gradients rotated back;
          with "fused" both are views of one projection's output
  append  the new tokens of a batch of sequences put into the cache: keys rotated on the way, and queries too where the
          case has them; pages of 4-bit codes are read back, as the numbers that they stand for
  attend  the new tokens' queries over what the cache holds of their sequences, causal; with "keep" a mask leaves about
          that share of the earlier frames visible, and one of the sequences nothing at all

A sequence's cached tokens lie in pages of "page" tokens, whose numbers a table gives in no order. Pages hold 16-bit
values [page][head][token][dim], or 4-bit codes, two to a byte, and for every 64 codes a word: the scale as a bf16 number
of 4 significant bits, and in the word's low 4 bits the zero point.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 64  # values that share a scale
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _rotary(name, tokens, heads, kv_heads, head_dim, **kw):
    return {"name": name, "op": "rotary", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "rotary_dim": head_dim, "layout": "half", "scaling": "none", "factor": 1.0, "axes": 1, "dtype": "bf16",
            "backward": False, "fused": False, "furthest": 131072, **kw}


def _append(name, seqs, new, before, **kw):
    return {"name": name, "op": "append", "seqs": seqs, "new": new, "before": before, "heads": 32, "kv_heads": 8,
            "head_dim": 128, "rotary_dim": 128, "layout": "half", "axes": 1, "queries": True, "page": 64, "bits": 16,
            "dtype": "bf16", **kw}


def _attend(name, seqs, new, longest, **kw):
    return {"name": name, "op": "attend", "seqs": seqs, "new": new, "longest": longest, "heads": 32, "kv_heads": 8,
            "head_dim": 128, "page": 64, "bits": 16, "dtype": "bf16", "keep": 1.0, "frame": 256, **kw}


def listed():
    return [
        # one step of a small batch of answers: eight tokens
        _rotary("rotate_step", 8, 32, 8, 128),
        # training: gradients of an odd number of tokens, part of the head, positions stretched to four times the length
        _rotary("rotate_grad_part", 10007, 28, 4, 128, rotary_dim=96, scaling="yarn", factor=4.0, dtype="fp16",
                backward=True, fused=True),
        # 256 frames of 256 tokens with frame, row and column positions
        _rotary("rotate_frames", 65536, 32, 8, 128, layout="interleaved", axes=3),
        # one new token of each of 32 answers
        _append("append_step", 32, 1, 1000),
        # the tokens of 64 frames behind what a stream has cached
        _append("append_frames", 1, 16384, 4096, axes=3, layout="interleaved"),
        # nine streams' frames into 4-bit pages
        _append("append_frames_4bit", 9, 12544, 500, axes=3, queries=False, bits=4),
        # the first token of an answer over a few frames: latency
        _attend("answer_short", 1, 1, 1111),
        # a server's step: 32 answers of very different lengths
        _attend("answer_batch", 32, 1, 16384),
        # one answer over 1024 frames of 256 tokens
        _attend("answer_long_4bit", 1, 1, 262144, bits=4),
        # three tokens at a time over the evidence alone
        _attend("answer_evidence_4bit", 24, 3, 20001, heads=28, kv_heads=4, bits=4, dtype="fp16", keep=0.3, frame=196),
        # a question of 256 tokens over 256 frames, the largest
        _attend("question_4bit", 1, 256, 65792, bits=4),
        # questions of several streams in one call
        _attend("question_batch", 7, 300, 9001, heads=16, kv_heads=8, head_dim=64, page=32),
    ]


HEADS = ((32, 8, 128), (32, 8, 128), (28, 4, 128), (16, 8, 64), (16, 16, 64), (14, 2, 64), (8, 1, 128))


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    op = rng.choice(("rotary", "append", "attend", "attend"))
    heads, kv_heads, head_dim = rng.choice(HEADS)
    dtype, layout, axes = rng.choice(("bf16", "bf16", "fp16")), rng.choice(("half", "interleaved")), rng.choice((1, 1, 3))
    rotary_dim = head_dim if rng.random() < 0.6 else rng.choice((16, 32, 48, head_dim // 2))
    if op == "rotary":
        scaling = rng.choice(("none", "none", "linear", "base", "yarn"))
        c = _rotary("", _log(rng, 1, 65536 * 40 * 128 // ((heads + kv_heads) * head_dim)), heads, kv_heads, head_dim,
                    rotary_dim=rotary_dim, layout=layout, scaling=scaling, axes=axes, dtype=rng.choice((dtype, "fp32")),
                    factor=1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0)), backward=rng.random() < 0.5,
                    fused=rng.random() < 0.5, furthest=rng.choice((4096, 131072, 1000000)))
        if c["dtype"] == "fp32":
            c["tokens"] = max(1, c["tokens"] // 2)
    elif op == "append":
        seqs = _log(rng, 1, 64)
        most = 65536 * 8 * 128 // (kv_heads * head_dim * seqs)
        queries = rng.random() < 0.5
        c = _append("", seqs, _log(rng, 1, max(1, min(32768, most // 4 if queries else most))), _log(rng, 1, 2000),
                    heads=heads, kv_heads=kv_heads, head_dim=head_dim, rotary_dim=rotary_dim, layout=layout, axes=axes,
                    queries=queries, page=rng.choice((16, 32, 64, 128)), bits=rng.choice((4, 16)), dtype=dtype)
    else:
        seqs = _log(rng, 1, 48)
        new = 1 if rng.random() < 0.4 else _log(rng, 1, 512)
        # at most the largest listed case's bytes and products, in the padded form too
        most = min(262144 * 8 * 128 // (seqs * kv_heads * head_dim), 256 * 65792 * 32 * 128 // (seqs * new * heads * head_dim))
        c = _attend("", seqs, new, _log(rng, 1, max(1, most)), heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                    page=rng.choice((16, 32, 64, 128)), bits=rng.choice((4, 16)), dtype=dtype,
                    keep=rng.choice((1.0, 1.0, 0.2, 0.5)), frame=rng.choice((49, 100, 144, 196, 256)))
    del c["name"]
    return c


# ---- sizes ----------------------------------------------------------------------------------------------------------


def _spread(n, lo, hi):
    """n whole numbers from hi down to lo, in an order of their own; hi alone where n is 1."""
    step = next(s for s in (7, 5, 3, 11, 1) if math.gcd(s, n) == 1)
    return [hi - (hi - lo) * ((i * step) % n) // max(1, n - 1) for i in range(n)]


def _sizes(c):
    """(new tokens, cached tokens with them) of each sequence."""
    n = c["seqs"]
    new = _spread(n, max(1, c["new"] // 3), c["new"])
    if c["op"] == "append":
        return new, [a + b for a, b in zip(new, _spread(n, c["before"] // 2, c["before"])[::-1])]
    return new, _spread(n, min(c["longest"], max(1, c["longest"] // 20)), c["longest"])[::-1]


def _visible_share(c):
    return 1.0 if c["keep"] >= 1 else c["keep"] * (1 - 1 / c["seqs"] if c["seqs"] > 1 else 1)


def work(case):
    c = case
    size = 4 if c.get("dtype") == "fp32" else 2
    h, hk, d = c["heads"], c["kv_heads"], c["head_dim"]
    if c["op"] == "rotary":
        n = c["tokens"] * (h + hk)
        return {"bytes": 2 * n * d * size + 4 * c["axes"] * c["tokens"], "flops": 3 * n * c["rotary_dim"]}
    new, have = _sizes(c)
    row = hk * (d * size if c["bits"] == 16 else d // 2 + 2 * (d // GROUP))  # bytes of one token's keys, or values
    if c["op"] == "append":
        t = sum(new)
        moved = 2 * t * (hk * d * size + row) + (2 * t * h * d * size if c["queries"] else 0)
        if c["bits"] == 4:  # read back
            moved += 2 * t * (hk * d * size + row)
        return {"bytes": moved + 4 * c["axes"] * t,
                "flops": 3 * t * c["rotary_dim"] * (hk + (h if c["queries"] else 0)) + (8 * t * hk * d if c["bits"] == 4 else 0)}
    share = _visible_share(c)
    pairs = sum(n * m - n * (n - 1) // 2 if m >= n else m * (m + 1) // 2 for n, m in zip(new, have)) * share
    return {"bytes": 2 * sum(have) * share * row + (sum(have) if share < 1 else 0) + 2 * sum(new) * h * d * size + 4 * sum(new) * h,
            "flops": 4 * pairs * h * d}


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _frequencies(c):
    """Each pair's turn per position, in double precision, and the factor on the rotated values."""
    rd, base, s = c["rotary_dim"], 1e6, c.get("factor", 1.0)
    kind = c.get("scaling", "none")
    if kind == "base":
        base *= s ** (rd / (rd - 2))
    f = [base ** (-2 * i / rd) for i in range(rd // 2)]
    m = 1.0
    if kind == "linear":
        f = [x / s for x in f]
    elif kind == "yarn":  # pairs of under 1 turn over the trained length are stretched, those of over 32 are not
        g = [min(1.0, max(0.0, (32768 * x / (2 * math.pi) - 1) / 31)) for x in f]
        f = [x * k + x / s * (1 - k) for x, k in zip(f, g)]
        m = 0.1 * math.log(s) + 1
    return f, m


def _axes(c):
    """The position axis of each pair: frame, row and column in turn."""
    return [i % c["axes"] for i in range(c["rotary_dim"] // 2)]


def _handle(c):
    from paper_2609_03675_gb300 import Rotary

    return Rotary(c["head_dim"], rotary_dim=c["rotary_dim"], base=1e6, layout=c["layout"], scaling=c.get("scaling", "none"),
                  factor=c.get("factor", 1.0), original_len=32768, axes=_axes(c) if c["axes"] > 1 else None)


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
        return torch.randint(0, c.get("furthest", 131072), (n,), generator=g, device="cuda", dtype=torch.int32)
    t = torch.arange(n, device="cuda", dtype=torch.int32)
    first = torch.randint(0, 4096, (1,), generator=g, device="cuda", dtype=torch.int32)
    return torch.stack([first + t // 256, first + t % 256 // 16, first + t % 16])[:c["axes"]].contiguous()


def _quantised(x):
    """Codes and words of x's last axis, in groups: [..., d] -> uint8 [..., d / 2], int16 [..., d / GROUP]."""
    y = x.float().unflatten(-1, (-1, GROUP))
    lo, hi = y.amin(-1).clamp(max=0.0), y.amax(-1).clamp(min=0.0)
    raw = (hi - lo) / torch.full_like(hi, 15.0)  # a plain 15 would be a product with its inverse
    scale = ((raw.view(torch.int32) + 0xFFFFF) & ~0xFFFFF).view(torch.float32)  # up to 4 significant bits
    scale = torch.where(raw < 2.0 ** -100, torch.zeros_like(scale), scale)
    by = torch.where(scale > 0, scale, torch.full_like(scale, math.inf))
    zero = (-lo / by + 0.5).floor().clamp(0, 15)
    steps = y / by.unsqueeze(-1)
    steps = steps.sign() * (steps.abs() + 0.5).floor()  # halves go away from zero
    codes = (steps + zero.unsqueeze(-1)).clamp(0, 15).to(torch.uint8).flatten(-2)
    words = scale.to(torch.bfloat16).view(torch.int16) | zero.to(torch.int16)
    return codes[..., 0::2] | codes[..., 1::2] << 4, words


def _numbers(codes, words):
    """What codes and words stand for, in fp32."""
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, GROUP)).float()
    scale = (words & -16).view(torch.bfloat16).float().unsqueeze(-1)
    return ((n - (words & 15).unsqueeze(-1).float()) * scale).flatten(-2)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    h, hk, d, dtype = c["heads"], c["kv_heads"], c["head_dim"], TYPES[c["dtype"]]
    if c["op"] == "rotary":
        n = c["tokens"]
        if c["fused"]:
            x = _normal((n, h + 2 * hk, d), dtype, g)
            q, k = x[:, :h], x[:, h:h + hk]
        else:
            q, k = _normal((n, h, d), dtype, g), _normal((n, hk, d), dtype, g)
        s = {"case": c, "q": q, "k": k, "positions": _positions(c, n, g), "qo": torch.empty((n, h, d), dtype=dtype, device="cuda"),
             "ko": torch.empty((n, hk, d), dtype=dtype, device="cuda")}
        if own:
            s["rotary"] = _handle(c)
        return _with_turns(s)
    new, have = _sizes(c)
    t, page, seqs = sum(new), c["page"], c["seqs"]
    each = [-(-m // page) for m in have]
    pages = sum(each) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((seqs, max(each)), dtype=torch.int32, device="cuda")
    lengths = torch.tensor(have, dtype=torch.int32, device="cuda")
    counts = torch.tensor(each, device="cuda")
    at = torch.arange(max(each), device="cuda")
    table[at < counts[:, None]] = order[:sum(each)]
    offsets = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.tensor(new, device="cuda").cumsum(0)
    spread = _channels(c, g)
    pool_k = _normal((pages, page, hk, d), dtype, g, spread).transpose(1, 2).contiguous()
    pool_v = _normal((pages, hk, page, d), dtype, g)
    s = {"case": c, "table": table, "lengths": lengths, "offsets": offsets, "most": max(new)}
    if c["bits"] == 4:
        # in pieces: the fp32 copies of a whole long cache would be large
        for name, pool in (("k", pool_k), ("v", pool_v)):
            parts = [_quantised(p) for p in pool.split(1024)]
            s[name + "_pages"], s[name + "_scales"] = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])
    else:
        s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"] = pool_k, pool_v, None, None
    if c["op"] == "append":
        s["k"], s["v"] = _normal((t, hk, d), dtype, g, spread), _normal((t, hk, d), dtype, g)
        s["q"] = _normal((t, h, d), dtype, g) if c["queries"] else None
        s["qo"] = torch.empty_like(s["q"]) if c["queries"] else None
        s["positions"] = _positions(c, t, g)
        s["ro"] = [torch.empty((t, hk, d), dtype=dtype, device="cuda") for _ in range(2)] if c["bits"] == 4 else None
        _with_turns(s)
    else:
        s["q"] = 1.3 * _normal((t, h, d), dtype, g)
        s["mask"] = None
        if c["keep"] < 1:
            frames = -(-max(have) // c["frame"])
            kept = torch.rand((seqs, frames), generator=g, device="cuda") < c["keep"]
            mask = kept.repeat_interleave(c["frame"], 1)[:, :max(have)]
            mask = mask | (torch.arange(max(have), device="cuda") >= (lengths - offsets.diff())[:, None])  # the new tokens
            if seqs > 1:
                mask[seqs // 2] = False  # nothing of this one
            s["mask"] = mask.to(torch.uint8).contiguous()
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((t, h), dtype=torch.float32, device="cuda")
    if own:
        from paper_2609_03675_gb300 import KVCache

        s["cache"] = KVCache(pages, page, h, hk, d, dtype=dtype, bits=c["bits"], rotary=_handle(c) if c["op"] == "append" else None,
                             k_pages=s["k_pages"], v_pages=s["v_pages"], k_scales=s["k_scales"], v_scales=s["v_scales"])
    return s


def _with_turns(s):
    """The plain form's plan: each pair's turn per position as a 64-bit fraction, so that far positions keep their angle."""
    f, s["amplitude"] = _frequencies(s["case"])
    s["turns"] = torch.tensor([int(x / (2 * math.pi) * 2.0 ** 64) for x in f], dtype=torch.int64, device="cuda")
    s["axis"] = torch.tensor(_axes(s["case"]), device="cuda")
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    c = s["case"]
    if c["op"] == "rotary":
        turn = s["rotary"].backward if c["backward"] else s["rotary"].apply
        return turn((s["q"], s["k"]), s["positions"], out=(s["qo"], s["ko"]))
    cache = s["cache"]
    if c["op"] == "append":
        cache.append(s["k"], s["v"], s["table"], s["lengths"], s["offsets"], positions=s["positions"], q=s["q"], q_out=s["qo"])
        if c["bits"] == 16:
            return s["qo"], s["k_pages"], s["v_pages"]
        return s["qo"], *cache.read(s["table"], s["lengths"], s["offsets"], out=s["ro"])
    return cache.attend(s["q"], s["table"], s["lengths"], s["offsets"], max_new=s["most"], mask=s["mask"], out=s["out"], lse=s["lse"])


def _plain(s):
    return {"rotary": _plain_rotary, "append": _plain_append, "attend": _plain_attend}[s["case"]["op"]](s)


def _rotated(x, s, back=False):
    """x [n, heads, d] in fp32, rotated."""
    c = s["case"]
    half = c["rotary_dim"] // 2
    p = s["positions"].long()
    p = p[s["axis"]].T if c["axes"] > 1 else p[:, None]
    a = ((p * s["turns"]) >> 32).float() * (math.pi / 2.0 ** 31)  # the products wrap, as turns do
    cos, sin = (a.cos() * s["amplitude"])[:, None], (a.sin() * s["amplitude"])[:, None]
    if back:
        sin = -sin
    x = x.float()
    if c["layout"] == "half":
        x1, x2 = x[..., :half], x[..., half:2 * half]
        return torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin, x[..., 2 * half:]], -1)
    x1, x2 = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
    return torch.cat([torch.stack([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1).flatten(-2), x[..., 2 * half:]], -1)


def _plain_rotary(s):
    back = s["case"]["backward"]
    return _rotated(s["q"], s, back).to(s["q"].dtype), _rotated(s["k"], s, back).to(s["k"].dtype)


def _slots(s):
    """(page, place in the page) of every new token."""
    t = torch.arange(int(s["k"].shape[0]), device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["offsets"], t, right=True) - 1
    at = (s["lengths"] - s["offsets"][1:])[seq] + t
    return s["table"][seq, at // s["case"]["page"]].long(), (at % s["case"]["page"]).long()


def _plain_append(s):
    c = s["case"]
    dtype = s["k"].dtype
    page, place = _slots(s)
    k, v = _rotated(s["k"], s), s["v"]
    q = _rotated(s["q"], s).to(dtype) if c["queries"] else None
    if c["bits"] == 16:
        s["k_pages"][page, :, place] = k.to(dtype)
        s["v_pages"][page, :, place] = v
        return q, s["k_pages"], s["v_pages"]
    for name, x in (("k", k), ("v", v)):
        s[name + "_pages"][page, :, place], s[name + "_scales"][page, :, place] = _quantised(x)
    return (q, _numbers(s["k_pages"][page, :, place], s["k_scales"][page, :, place]).to(dtype),
            _numbers(s["v_pages"][page, :, place], s["v_scales"][page, :, place]).to(dtype))


def _cached(s, name):
    """[seqs, kv heads, tokens, d] in fp32, tokens up to whole pages."""
    x = s[name + "_pages"][s["table"].long()]
    x = _numbers(x, s[name + "_scales"][s["table"].long()]) if s["case"]["bits"] == 4 else x.float()
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attend(s):
    c = s["case"]
    h, hk, d = c["heads"], c["kv_heads"], c["head_dim"]
    k, v = _cached(s, "k"), _cached(s, "v")
    count, first = s["offsets"].diff(), s["offsets"][:-1]
    i = torch.arange(s["most"], device="cuda", dtype=torch.int32)
    real = i < count[:, None]
    rows = torch.where(real, first[:, None] + i, 0).long()
    q = s["q"].float()[rows].unflatten(2, (hk, h // hk)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [seqs, kv heads, group x new, d]
    at = torch.arange(k.shape[2], device="cuda")
    seen = at <= ((s["lengths"] - count)[:, None] + i)[..., None]  # [seqs, new, tokens]
    if s["mask"] is not None:
        seen &= torch.nn.functional.pad(s["mask"], (0, k.shape[2] - s["mask"].shape[1])).bool()[:, None]
    seen = seen[:, None, None].expand(-1, -1, h // hk, -1, -1).flatten(2, 3)
    x = (q @ k.transpose(2, 3) * d ** -0.5).masked_fill(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    o = (e @ v) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log()).squeeze(-1)
    o = o.unflatten(2, (h // hk, -1)).permute(0, 3, 1, 2, 4).flatten(2, 3)[real]
    return o.to(s["q"].dtype), lse.unflatten(2, (h // hk, -1)).permute(0, 3, 1, 2).flatten(2, 3)[real]


# ---- the definition, in 64 bits -------------------------------------------------------------------------------------


def _exact_turn(x, positions, c, back=False):
    f, m = _frequencies(c)
    p = positions.double().reshape(c["axes"], -1)
    a = torch.stack([p[ax] * w for ax, w in zip(_axes(c), f)], 1)
    z = torch.polar(torch.full_like(a, m), -a if back else a)[:, None]
    y, half = x.double().clone(), c["rotary_dim"] // 2
    one, two = (slice(0, half), slice(half, 2 * half)) if c["layout"] == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    w = torch.complex(x[..., one].double(), x[..., two].double()) * z
    y[..., one], y[..., two] = w.real, w.imag
    return y


def _exact_four_bits(x):
    """The values nearest to x that its groups' scales and zero points allow."""
    y = x.double().reshape(*x.shape[:-1], -1, GROUP)
    lo, hi = y.min(-1, keepdim=True).values.clamp(max=0), y.max(-1, keepdim=True).values.clamp(min=0)
    part, power = torch.frexp((hi - lo) / 15)
    s = torch.ldexp(torch.ceil(part * 16) / 16, power)
    u = torch.where(s > 0, s, 1.0)
    n, low = torch.trunc(y / u + torch.copysign(torch.full_like(y, 0.5), y)), torch.trunc(0.5 - lo / u).clamp(0, 15)
    return (torch.minimum(torch.maximum(n, -low), 15 - low) * s).reshape(x.shape)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] == "rotary":
        return tuple(_exact_turn(x, s["positions"], c, c["backward"]) for x in (s["q"], s["k"]))
    new, have = _sizes(c)
    table, page = s["table"].long(), c["page"]
    if c["op"] == "append":
        k, v = _exact_turn(s["k"], s["positions"], c), s["v"].double()
        q = _exact_turn(s["q"], s["positions"], c) if c["queries"] else None
        if c["bits"] == 4:
            return q, _exact_four_bits(k), _exact_four_bits(v)
        pools, t = (s["k_pages"].double(), s["v_pages"].double()), 0
        for b, (n, m) in enumerate(zip(new, have)):
            at = torch.arange(m - n, m, device="cuda")
            for pool, x in zip(pools, (k, v)):
                pool.transpose(1, 2)[table[b, at // page], at % page] = x[t:t + n]
            t += n
        return q, *pools
    h, hk, d = c["heads"], c["kv_heads"], c["head_dim"]
    out, lse, t = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda"), 0
    for b, (n, m) in enumerate(zip(new, have)):
        held = []
        for name in ("k", "v"):
            x = s[name + "_pages"][table[b, :-(-m // page)]]
            if c["bits"] == 4:
                w = s[name + "_scales"][table[b, :-(-m // page)]].int() & 0xFFFF
                # the word's bits: 8 of exponent, 3 of mantissa, 4 of zero point
                scale = torch.where(w >> 4 > 0, (8 + (w >> 4 & 7)).double() * torch.exp2((w >> 7).double() - 130), 0.0)
                codes = torch.stack([x % 16, x // 16], -1).reshape(*x.shape[:-1], d // GROUP, GROUP)
                x = ((codes.double() - (w % 16)[..., None]) * scale[..., None]).reshape(*x.shape[:-1], d)
            held.append(x.double().transpose(0, 1).reshape(hk, -1, d)[:, :m])
        at, last = torch.arange(m, device="cuda"), torch.arange(m - n, m, device="cuda")
        seen = at[None] <= last[:, None]
        if s["mask"] is not None:
            seen = seen & (s["mask"][b, :m] != 0)[None]
        for j in range(h):
            x = s["q"][t:t + n, j].double() @ held[0][j // (h // hk)].T / math.sqrt(d)
            x = torch.where(seen, x, -math.inf)
            lse[t:t + n, j] = torch.logsumexp(x, 1)
            w = torch.softmax(x, 1)
            out[t:t + n, j] = torch.where(seen.any(1)[:, None], w, 0.0) @ held[1][j // (h // hk)]
        t += n
    return out, lse

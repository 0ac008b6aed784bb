"""Pages of bytes: what is written, to the bit, and attention over it to the bounds that hold the other pages' too.

The definition (include/cofie_kv.h), restated here in 64 bits: s the smallest power of two with max |x| <= 127 s, from
2^-100 to 2^121 (bf16) or 2^-24 to 2^9 (fp16); u = 128 + the whole number nearest to x / s, halves to the even one, cut to
-127..127. Attention sees (u - 128) s, which both types hold exactly, so tests/kv_bounds.py applies with one change: few rows
over fp16 caches round weight times scale to fp16 with the largest scale of the group at 2^10 or more, off by 2^-35 of it at
most, and a value by 127 of that, where 127 s < 2 max |v| (s is the smallest power of two, unless it is the least allowed, where
127 s is below 2^-17): less than the m 2^-32 max |v| that the bound has for 4-bit codes, or 2^-52 a token."""
import math

import pytest
import torch

from tests import kv_bounds as B
from tests import kv_oracle as K
from tests.test_gpu_kv import BATCHES, HEADS, _offsets, _table

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def quantise(x, dtype):
    """x [..., d] -> (bytes uint8 [..., d], words int16 [..., d / 64]); groups of finite values."""
    y = x.detach().double().cpu().unflatten(-1, (-1, 64))
    top = y.abs().amax(-1)
    lo, hi = (-100, 121) if dtype == torch.bfloat16 else (-24, 9)
    e = torch.full(top.shape, lo, dtype=torch.int64)
    for k in range(lo, hi):  # one more for each power that is too small; 127 2^k is exact
        e += (top > 127.0 * 2.0 ** k).long()
    s = torch.tensor([2.0 ** k for k in range(lo, hi + 1)], dtype=torch.float64)[e - lo]
    n = torch.round(y / s[..., None]).clamp(-127, 127)  # on the CPU: halves to even
    return (n + 128).to(torch.uint8).flatten(-2), ((e + 127) << 7).to(torch.int16)


def numbers(u, words):
    s = torch.exp2((words.cpu().long() >> 7).double() - 127)[..., None]
    return ((u.cpu().double().unflatten(-1, (-1, 64)) - 128) * s).flatten(-2)


def make(n_pages, page, heads, kv, d, dtype, rotary=None):
    """A cache whose pages are NaN until they are written."""
    from paper_2609_03675_gb300 import KVCache
    c = KVCache(n_pages, page, heads, kv, d, dtype=dtype, bits="int8", rotary=rotary)
    c.k_pages.fill_(0x5A)
    c.v_pages.fill_(0xA5)
    c.k_scales.fill_(0x7FC0)
    c.v_scales.fill_(0x7FC0)
    return c


def fill(cache, table, lengths, g, seen=None):
    """Random tokens put into the pages by hand; (k, v) of each sequence as the pages' numbers."""
    page, kv, d, held = cache.page_size, cache.n_kv_heads, cache.head_dim, []
    for s, m in enumerate(lengths):
        k = (torch.randn((m, kv, d), generator=g) * torch.exp(0.3 * torch.randn((kv, d), generator=g))).to(cache.dtype)
        v = torch.randn((m, kv, d), generator=g).to(cache.dtype)
        at = torch.arange(m) if seen is None else torch.arange(m)[seen[s, :m]]
        p, o = table[s].cpu().long()[at // page].cuda(), (at % page).cuda()
        out = []
        for x, pages, scales in ((k, cache.k_pages, cache.k_scales), (v, cache.v_pages, cache.v_scales)):
            u, w = quantise(x, cache.dtype)
            pages[p, :, o], scales[p, :, o] = u[at].cuda(), w[at].cuda()
            out.append(numbers(u, w))
        held.append(out)
    return held


def check(cache, q, table, lengths, new, held, mask=None, causal=True, max_new=None, scale=0.0):
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    cache.attend(q, table, lens, _offsets(new), max_new=max(new) if max_new is None else max_new, mask=mask, causal=causal, scale=scale,
                 out=out, lse=lse)
    cache.status()
    out, lse, t = out.cpu(), lse.cpu(), 0
    for s, (n, m) in enumerate(zip(new, lengths)):
        seen = torch.ones((n, m), dtype=torch.bool)
        if causal:
            seen = torch.arange(m)[None] <= (m - n + torch.arange(n))[:, None]
        if mask is not None:
            w = torch.zeros(m, dtype=torch.bool)
            w[:mask.shape[1]] = mask[s, :m].cpu() != 0
            seen = seen & w[None]
        if n:
            bad = B.exceeds(out[t:t + n], lse[t:t + n], B.attend(q[t:t + n], *held[s], seen, scale or cache.head_dim ** -0.5, q.dtype))
            assert not bool(bad[0].any()), (s, "out")
            assert not bool(bad[1].any()), (s, "lse")
        t += n
    assert bool((out[t:] == 7.0).all()) and bool((lse[t:] == 7.0).all()), "rows past the batch were written"


# ---- append and read ------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,page,kv,rd,layout", [(128, 64, 2, 128, "half"), (128, 32, 3, 128, "interleaved"), (128, 16, 1, 96, "interleaved"),
                                                 (128, 256, 2, 48, "half"), (64, 128, 3, 48, "half"), (64, 64, 2, 6, "interleaved"), (64, 16, 5, 64, "half")])
def test_append_then_read(dtype, d, page, kv, rd, layout):
    """Values: the definition's bytes. Keys: the definition's bytes of a key within fp32's error of the rotated one."""
    from paper_2609_03675_gb300 import Rotary
    g = torch.Generator().manual_seed(d + page)
    new, before = [5, 0, 1, 70, 3], [0, 4, page - 1, page, 200]
    lengths = [a + b for a, b in zip(new, before)]
    table, n_pages = _table(lengths, page, 2, g)
    offsets, n, heads = _offsets(new), sum(new), 2 * kv
    cache = make(n_pages, page, heads, kv, d, dtype, Rotary(d, rotary_dim=rd, layout=layout))
    old = [x.clone() for x in (cache.k_pages, cache.v_pages, cache.k_scales, cache.v_scales)]
    x = (torch.randn((n, heads + 2 * kv, d), generator=g) * torch.exp(0.5 * torch.randn((heads + 2 * kv, d), generator=g))).to(dtype).cuda()
    q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    v[0, 0, :64] = 0.0
    v[1, 0, :64] = v[1, 0, :64].abs()
    pos = torch.randint(0, 100000, (n,), generator=g).to(torch.int32).cuda()
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    qr = cache.append(k, v, table, lens, offsets, positions=pos, q=q)
    rk, rv = cache.read(table, lens, offsets, n_tokens=n)
    cache.status()
    freq, m = K.frequencies(rd, 1e4)
    want, slack = K.rotate(q, pos, freq, m, layout)
    assert bool(((qr.double().cpu() - want).abs() <= slack + K.UNIT[dtype] * want.abs() + 2.0 ** -25).all())
    written = torch.zeros((n_pages, page), dtype=torch.bool)
    u, w = quantise(v, dtype)
    t = 0
    for s in range(len(new)):
        for i in range(before[s], lengths[s]):
            p, o = int(table[s, i // page]), i % page
            written[p, o] = True
            assert torch.equal(cache.v_pages[p, :, o].cpu(), u[t]) and torch.equal(cache.v_scales[p, :, o].cpu(), w[t])
            t += 1
    for now, was in zip((cache.k_pages, cache.v_pages, cache.k_scales, cache.v_scales), old):
        a, b = now.transpose(1, 2).cpu(), was.transpose(1, 2).cpu()
        assert torch.equal(a[~written], b[~written]), "a place outside the batch was written"
    assert torch.equal(rv.double().cpu(), numbers(u, w))
    want, slack = K.rotate(k, pos, freq, m, layout)
    _, w = quantise(want, dtype)
    step = torch.exp2((w.long() >> 7).double() - 127).repeat_interleave(64, -1)
    assert bool(((rk.double().cpu() - want).abs() <= 0.5 * step + slack).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_bytes_without_rotary_from_odd_strides(dtype):
    """Single tokens; keys as they come are the definition's bytes too; rows that allow no wide loads."""
    g = torch.Generator().manual_seed(5)
    lengths = [1, 17, 33, 2]
    table, n_pages = _table(lengths, 16, 0, g)
    for d in (64, 128):
        cache = make(n_pages, 16, 4, 2, d, dtype)
        wide = torch.randn((4, 2 * 2 * d + 1), generator=g).to(dtype).cuda()
        k, v = (wide[:, 1 + o:1 + o + 2 * d].unflatten(1, (2, d)) for o in (0, 2 * d))
        lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        cache.append(k, v, table, lens)
        got = cache.read(table, lens)
        cache.status()
        for x, y in zip(got, (k, v)):
            assert torch.equal(x.double().cpu(), numbers(*quantise(y, dtype)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_extremes_of_a_group(dtype, d):
    """Borders of the scales, halves, the smallest and the largest values; a neighbouring group is not touched."""
    finite = [[127.0, 0.5, 1.5, 2.5, -0.5, -1.5], [127.5, 1.0, 3.0, 5.0], [-127.0, 126.5], [-128.0, 1.0], [3.0], [0.0],
              [127.0 / 64, 1.0 / 128, 3.0 / 128], [2.0 ** -14, 2.0 ** -24, -(2.0 ** -24)], [2.0 ** -24], [65024.0, 256.0, 768.0, -1.0]]
    finite += [[65280.0, 65024.0], [65504.0, -65504.0, 100.0]] if dtype == torch.float16 else \
              [[3.0e38, -3.0e38], [3.38e38, 1e36], [2.0 ** -99, 2.0 ** -101, 3 * 2.0 ** -101, 2.0 ** -102], [2.0 ** -126], [2.0 ** -93, 2.0 ** -100]]
    rows = finite + [[math.inf, 1.0], [math.nan, 2.0], [-math.inf], [1.0, math.nan]]
    x = torch.zeros((len(rows), 1, d))
    for i, r in enumerate(rows):
        x[i, 0, :len(r)] = torch.tensor(r)
    if d == 128:
        x[:, 0, 64] = 1.0
    x = x.to(dtype)
    n = len(rows)
    cache = make(n, 16, 1, 1, d, dtype)
    table, ones = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous(), torch.ones(n, dtype=torch.int32, device="cuda")
    src = x.cuda()
    cache.append(src, src, table, ones)
    k, v = (y.double().cpu() for y in cache.read(table, ones))
    cache.status()
    for got in (k, v):
        for i in range(n):
            if i < len(finite):
                u, w = quantise(x[i], dtype)
                assert torch.equal(got[i], numbers(u, w)), rows[i]
                assert torch.equal(cache.v_scales[i, :, 0].cpu(), w) and torch.equal(cache.v_pages[i, :, 0].cpu(), u)
                assert bool(torch.isfinite(got[i]).all())
            else:
                assert bool(torch.isnan(got[i, 0, :64]).all()), rows[i]
            if d == 128:
                assert float(got[i, 0, 64]) == 1.0


# ---- attention ------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new,lengths,page", BATCHES + [([1, 40], [3000, 2000], 64)])
def test_every_token_counts(dtype, new, lengths, page):
    for i, (h, kv, d) in enumerate(HEADS):
        g = torch.Generator().manual_seed(11 * i + page)
        table, n_pages = _table(lengths, page, 1, g)
        cache = make(n_pages, page, h, kv, d, dtype)
        held = fill(cache, table, lengths, g)
        q = (1.5 * torch.randn((sum(new), h, d), generator=g)).to(dtype).cuda()
        check(cache, q, table, lengths, new, held)
        check(cache, q, table, lengths, new, held, causal=False, scale=0.07)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [4, 1, 3, 2], [20, 3, 40, 2]])
def test_masks(dtype, new):
    """Whole tiles masked, single places, nothing left, a mask shorter than the sequence; what is masked holds NaN."""
    lengths, width = [700, 40, 131, 64], 650
    for h, kv, d, page in ((8, 2, 128, 32), (4, 4, 64, 16)):
        g = torch.Generator().manual_seed(d)
        table, n_pages = _table(lengths, page, 1, g)
        mask = torch.rand((4, width), generator=g) < 0.5
        mask[0, 64:400] = False
        mask[1] = False
        mask[2, :128] = False
        mask[2, 128:] = True
        mask[3] = True
        seen = torch.zeros((4, 700), dtype=torch.bool)
        seen[:, :width] = mask
        for causal in (True, False):
            cache = make(n_pages, page, h, kv, d, dtype)
            held = fill(cache, table, lengths, g, seen)
            q = torch.randn((sum(new), h, d), generator=g).to(dtype).cuda()
            check(cache, q, table, lengths, new, held, mask=mask.cuda(), causal=causal)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 3, 30])
def test_scales_far_apart(dtype, n):
    """Values of one group 2^20 times those of the other, tokens whose scales rise and fall by 2^12: rows of the small ones'
    size, and of the large ones' where they weigh anything."""
    h, kv, d, page, m = 4, 1, 128, 64, 900
    g = torch.Generator().manual_seed(n)
    table, n_pages = _table([m], page, 0, g)
    cache = make(n_pages, page, h, kv, d, dtype)
    k = torch.randn((m, kv, d), generator=g) * 2.0 ** -3
    v = torch.randn((m, kv, d), generator=g)
    v[..., 64:] *= 2.0 ** -14
    v *= torch.exp2(torch.randint(-6, 7, (m, 1, 1), generator=g).float())
    k, v = k.to(dtype), v.to(dtype)
    lens, offsets = _ints(m), _ints(0, m)
    cache.append(k.cuda(), v.cuda(), table, lens, offsets)
    held = [[numbers(*quantise(x, dtype)) for x in (k, v)]]
    q = torch.randn((n, h, d), generator=g).to(dtype).cuda()
    out, lse = cache.attend(q, table, lens, _ints(0, n), max_new=n)
    cache.status()
    seen = torch.arange(m)[None] <= (m - n + torch.arange(n))[:, None]
    for lo in (0, 64):  # the bound of each group by its own values
        w = B.attend(q, held[0][0], held[0][1][..., lo:lo + 64], seen, d ** -0.5, dtype)
        bad = B.exceeds(out[..., lo:lo + 64], lse, w)
        assert not bool(bad[0].any()) and not bool(bad[1].any()), lo


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 17])
def test_every_byte_of_every_scale(dtype, d, new):
    """One cached token to a sequence, which all rows see: its values come out as they are, a weight of one being exact."""
    lo, hi = (-100, 121) if dtype == torch.bfloat16 else (-24, 9)
    S, kv = hi - lo + 1, 256 // d
    c = make(S, 16, kv, kv, d, dtype)
    u = torch.arange(256).clamp(min=1).view(kv, d).to(torch.uint8)  # a byte of zero stands for no number
    w = torch.arange(lo + 127, hi + 128) << 7
    c.k_pages[:, :, 0], c.k_scales[:, :, 0] = 128, 127 << 7
    c.v_pages[:, :, 0], c.v_scales[:, :, 0] = u.cuda(), w.to(torch.int16).view(S, 1, 1).cuda()
    table = torch.arange(S, dtype=torch.int32, device="cuda").view(S, 1)
    q = torch.randn((S * new, kv, d), device="cuda").to(dtype)
    out, _ = c.attend(q, table, torch.ones(S, dtype=torch.int32, device="cuda"), torch.arange(0, S * new + 1, new, dtype=torch.int32, device="cuda"),
                      max_new=new, causal=False)
    c.status()
    want = numbers(u.expand(S, kv, d), w.view(S, 1, 1).expand(S, kv, d // 64)).to(dtype)
    assert torch.equal(out.cpu().view(S, new, kv, d), want[:, None].expand(S, new, kv, d))


@pytest.mark.parametrize("n", [1, 40])
def test_pages_past_four_gigabytes(n):
    """The last pages of a pool of over 2^32 bytes: appended to, read, attended to."""
    h, kv, d, page, dtype = 4, 4, 128, 64, torch.bfloat16
    n_pages = (1 << 32) // (kv * page * d) + 40
    from paper_2609_03675_gb300 import KVCache
    cache = KVCache(n_pages, page, h, kv, d, bits="int8")
    m = 30 * page - 3
    table = torch.arange(n_pages - 1, n_pages - 31, -1, dtype=torch.int32, device="cuda").view(1, -1)
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn((m, kv, d), generator=g).to(dtype) for _ in range(2))
    cache.append(k.cuda(), v.cuda(), table, _ints(m), _ints(0, m))
    held = [[numbers(*quantise(x, dtype)) for x in (k, v)]]
    got = cache.read(table, _ints(m), _ints(0, m), n_tokens=m)
    assert all(torch.equal(a.double().cpu(), b) for a, b in zip(got, held[0]))
    q = torch.randn((n, h, d), generator=g).to(dtype).cuda()
    check(cache, q, table, [m], [n], held)


def test_pages_of_another_kind_are_refused():
    from paper_2609_03675_gb300 import KVCache
    for bits in (8, "8", "int4", torch.int8, True):
        with pytest.raises(ValueError, match="bits"):
            KVCache(2, 16, 2, 1, 64, bits=bits)
    with pytest.raises(ValueError, match="pages"):
        KVCache(2, 16, 2, 1, 64, bits="int8", k_pages=torch.zeros((2, 1, 16, 64), dtype=torch.int8, device="cuda"))
    with pytest.raises(ValueError, match="pages"):
        KVCache(2, 16, 2, 1, 64, bits="int8", k_pages=torch.zeros((2, 1, 16, 32), dtype=torch.uint8, device="cuda"))
    assert KVCache(2, 16, 2, 1, 64, bits="int8").bits == 8


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,rd,layout,start,axes", [(128, 128, "half", 0, 1), (128, 128, "interleaved", 0, 3), (128, 96, "half", 0, 1), (64, 64, "half", 0, 2),
                                                    (64, 48, "interleaved", 1, 1), (128, 64, "half", 1, 1)])
def test_bytes_of_rotated_keys_are_the_nearest(dtype, d, rd, layout, start, axes):
    """2 million rotated keys at far positions: the bytes of the keys turned in 64 bits, all of them. (fp32 puts one in 3 10^5
    on the wrong side of a half: about seven of these. In 64 bits as few as 10^-8 of the values are as close to a half as the
    oracle's angles are off: positions below 2^17 times a frequency rounded to 2^-53, 2^-36 turns.)"""
    from paper_2609_03675_gb300 import Rotary
    n, kv, page = 2048000 // d // 8, 8, 64
    g = torch.Generator().manual_seed(d + rd)
    flat = torch.zeros(n * kv * d + 1, dtype=dtype)
    k = flat[start:start + n * kv * d].view(n, kv, d)
    k.copy_(torch.randn((n, kv, d), generator=g) * torch.exp(0.3 * torch.randn((kv, d), generator=g)))
    pos = torch.randint(0, 131072, (axes, n), generator=g).to(torch.int32)
    of = [i % axes for i in range(rd // 2)]
    cache = make(-(-n // page), page, kv, kv, d, dtype, Rotary(d, rotary_dim=rd, layout=layout, base=1e6, axes=of if axes > 1 else None))
    table = torch.arange(-(-n // page), dtype=torch.int32, device="cuda").view(1, -1)
    dev = flat.cuda()[start:start + n * kv * d].view(n, kv, d)
    cache.append(dev, dev, table, _ints(n), _ints(0, n), positions=pos.cuda() if axes > 1 else pos[0].cuda())
    got, _ = cache.read(table, _ints(n), _ints(0, n), n_tokens=n)
    cache.status()
    freq, m = K.frequencies(rd, 1e6)
    want, _ = K.rotate(k, pos, freq, m, layout, of if axes > 1 else None)
    u, w = quantise(want, dtype)
    wrong = (got.double().cpu() != numbers(u, w)).sum()
    assert int(wrong) == 0, int(wrong)

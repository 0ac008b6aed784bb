"""The paged cache (append, read) and attention over it, against their
definitions in 64 bits: both kinds of pages, head layouts, page sizes, lengths
from zero, masks that leave rows empty, garbage in masked places, strides,
captured calls, and refusals."""
import math

import pytest
import torch

from tests import kv_oracle as K

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _table(lengths, page, spare, g):
    """Page table over as many pages as the lengths need, in no order; unused entries are out of range."""
    each = [-(-m // page) for m in lengths]
    n = sum(each) + spare
    order = torch.randperm(n, generator=g).to(torch.int32)
    t = torch.full((len(lengths), max(1, max(each, default=1))), -7, dtype=torch.int32)
    at = 0
    for s, e in enumerate(each):
        t[s, :e] = order[at:at + e]
        at += e
    return t.cuda(), n


def _offsets(new):
    return torch.tensor([0] + new).cumsum(0).to(torch.int32).cuda()


def _cache(n_pages, page, heads, kv, d, dtype, bits, rotary=None, fill=None):
    """A cache whose pages hold NaN until they are written."""
    from paper_2609_03675_gb300 import KVCache
    c = KVCache(n_pages, page, heads, kv, d, dtype=dtype, bits=bits, rotary=rotary)
    if bits == 16:
        c.k_pages.fill_(math.nan)
        c.v_pages.fill_(math.nan)
    else:
        c.k_pages.fill_(0x5A)
        c.v_pages.fill_(0xA5)
        c.k_scales.fill_(0x7FC3)  # a NaN scale
        c.v_scales.fill_(0x7FC3)
    return c


# ---- append and read ------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits,d,page,kv,rd,layout", [
    (16, 128, 64, 2, 128, "half"), (16, 64, 16, 3, 32, "interleaved"), (4, 128, 32, 2, 128, "half"),
    (4, 128, 16, 1, 96, "interleaved"), (4, 64, 128, 3, 48, "half"), (4, 64, 64, 2, 6, "interleaved"),
])
def test_append_then_read(dtype, bits, d, page, kv, rd, layout):
    from paper_2609_03675_gb300 import Rotary
    g = torch.Generator().manual_seed(d + page)
    new, before = [5, 0, 1, 70, 3], [0, 4, page - 1, page, 200]
    lengths = [a + b for a, b in zip(new, before)]
    table, n_pages = _table(lengths, page, 2, g)
    offsets, n, heads = _offsets(new), sum(new), 2 * kv
    rotary = Rotary(d, rotary_dim=rd, layout=layout, base=1e4)
    cache = _cache(n_pages, page, heads, kv, d, dtype, bits, rotary)
    old = [x.clone() for x in (cache.k_pages, cache.v_pages)]
    x = (torch.randn((n, heads + 2 * kv, d), generator=g) * torch.exp(0.5 * torch.randn((heads + 2 * kv, d), generator=g))).to(dtype).cuda()
    q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    v[0, 0, :64] = 0.0  # a group of zeros
    v[1, 0, :64] = v[1, 0, :64].abs()  # all of one sign
    pos = torch.randint(0, 100000, (n,), generator=g).to(torch.int32).cuda()
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    qr = cache.append(k, v, table, lens, offsets, positions=pos, q=q)
    rk, rv = cache.read(table, lens, offsets, n_tokens=n)
    cache.status()
    freq, m = K.frequencies(rd, 1e4)
    for y, src in ((qr, q), (rk, k) if bits == 16 else (qr, q)):
        want, slack = K.rotate(src, pos, freq, m, layout)
        err = (y.double().cpu() - want).abs()
        assert bool((err <= slack + K.UNIT[dtype] * want.abs() + 2.0 ** -25).all())
    # the places that the batch names, and no others, are written
    written = torch.zeros((n_pages, page), dtype=torch.bool)
    for s in range(len(new)):
        for i in range(before[s], lengths[s]):
            written[int(table[s, i // page]), i % page] = True
    for now, was in zip((cache.k_pages, cache.v_pages), old):
        a, b = now.transpose(1, 2).cpu(), was.transpose(1, 2).cpu()
        assert torch.equal(a[~written].view(torch.uint8), b[~written].view(torch.uint8)), "a place outside the batch was written"
    if bits == 16:
        assert torch.equal(rv, v)
        return
    # values: the codes of the definition, to the bit
    codes, scale, zero = K.quantise(v)
    t = 0
    for s in range(len(new)):
        for i in range(before[s], lengths[s]):
            p, o = int(table[s, i // page]), i % page
            b, w = K.pack(codes[t], scale[t], zero[t])
            assert torch.equal(cache.v_pages[p, :, o].cpu(), b) and torch.equal(cache.v_scales[p, :, o].cpu(), w)
            t += 1
    # keys: within half a step of the rotated keys, the step that of the definition; where fp32 rounds the extremes'
    # difference over a step of the scale, the next one
    want, slack = K.rotate(k, pos, freq, m, layout)
    _, s64, _ = K.quantise(want)
    err = (rk.double().cpu() - want).abs()
    step = s64.repeat_interleave(64, -1)
    assert bool((err <= 0.5 * step * (1 + 2.0 ** -10) + slack).float().mean() > 0.999)
    assert bool((err <= 0.5 * 1.125 * step * (1 + 2.0 ** -10) + slack).all())


def test_codes_of_single_tokens_keys_without_rotary_and_odd_strides():
    """offsets=None; keys without rotary are the definition's codes too; rows that allow no wide loads."""
    g = torch.Generator().manual_seed(5)
    lengths = [1, 17, 33, 2]
    table, n_pages = _table(lengths, 16, 0, g)
    cache = _cache(n_pages, 16, 4, 2, 64, torch.float16, 4)
    wide = torch.randn((4, 2 * 2 * 64 + 1), generator=g).half().cuda()
    k, v = (wide[:, 1 + o:129 + o].unflatten(1, (2, 64)) for o in (0, 128))
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    cache.append(k, v, table, lens)
    rk, rv = cache.read(table, lens)
    cache.status()
    for got, src in ((rk, k), (rv, v)):
        want, _ = K.unpack(*K.pack(*K.quantise(src)))
        assert torch.equal(got.double().cpu(), want)


def test_extremes_of_a_group():
    """Ties, one value alone, tiny and huge values, infinities and NaN, in a group each."""
    x = torch.zeros((1, 1, 128))
    rows = []
    for values in ([15.0, 0.5, 1.5, 2.5, 3.5, 14.5], [-7.5, 7.5, 0.5, -0.5, 1.0], [-15.0, -0.5], [3.0], [2.0 ** -120], [3.0e38, -3.0e38],
                   [2.0 ** -99, 2.0 ** -103], [math.inf, 1.0], [math.nan, 2.0], [-math.inf], [1.0, 1.0 / 15, 2.0 / 15]):
        y = x.clone()
        y[0, 0, :len(values)] = torch.tensor(values)
        y[0, 0, 64] = 1.0
        rows.append(y)
    src = torch.cat(rows).to(torch.bfloat16).cuda()
    n = src.shape[0]
    table = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous()
    cache = _cache(n, 16, 1, 1, 128, torch.bfloat16, 4)
    ones = torch.ones(n, dtype=torch.int32, device="cuda")
    cache.append(src, src, table, ones)
    rk, rv = cache.read(table, ones)
    cache.status()
    assert torch.equal(rk.view(torch.int16), rv.view(torch.int16))
    for i in range(n):
        finite = bool(torch.isfinite(src[i, 0, :64]).all()) and float(src[i, 0, :64].abs().max()) < 1e38
        if not finite:
            assert bool(torch.isnan(rv[i, 0, :64]).all()), i
        else:
            want, _ = K.unpack(*K.pack(*K.quantise(src[i])))
            assert torch.equal(rv[i].double().cpu(), want), i
        # the group beside it is not touched: 1 / 15 goes up to 9 / 128, of which 1 is nearest to 14
        assert float(rv[i, 0, 64]) == 14 * 9 / 128


# ---- attention ------------------------------------------------------------------------------------------------------


def _fill(cache, table, lengths, g, seen=None):
    """Writes random tokens (no rotation) through the pages; returns per sequence (k, v, |k| for the bound), fp64.
    seen [seqs, tokens]: places that stay NaN where it is False."""
    page, kv, d, dtype = cache.page_size, cache.n_kv_heads, cache.head_dim, cache.dtype
    held = []
    for s, m in enumerate(lengths):
        k = (torch.randn((m, kv, d), generator=g) * torch.exp(0.3 * torch.randn((kv, d), generator=g))).to(dtype)
        v = torch.randn((m, kv, d), generator=g).to(dtype)
        at = torch.arange(m) if seen is None else torch.arange(m)[seen[s, :m]]
        p, o = table[s].cpu().long()[at // page], at % page
        if cache.bits == 16:
            cache.k_pages[p.cuda(), :, o.cuda()] = k[at].cuda()
            cache.v_pages[p.cuda(), :, o.cuda()] = v[at].cuda()
            held.append((k.double(), v.double(), None))
            continue
        out = []
        for x, pages, scales in ((k, cache.k_pages, cache.k_scales), (v, cache.v_pages, cache.v_scales)):
            b, w = K.pack(*K.quantise(x))
            pages[p.cuda(), :, o.cuda()] = b[at].cuda()
            scales[p.cuda(), :, o.cuda()] = w[at].cuda()
            out.append(K.unpack(b, w))
        held.append((out[0][0], out[1][0], out[0][1] * (144 if dtype == torch.bfloat16 else 1040)))
    return held


def _check_attend(cache, q, table, lengths, new, held, mask=None, causal=True, scale=0.0, max_new=None, label="", call=None):
    offsets = _offsets(new)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    # what is not written keeps these
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
    if call is None:
        cache.attend(q, table, lens, offsets, max_new=max(new) if max_new is None else max_new, mask=mask, causal=causal, scale=scale,
                     out=out, lse=lse)
    else:
        call(q, table, lens, offsets, mask, out, lse)
    cache.status()
    t = 0
    for s, (n, m) in enumerate(zip(new, lengths)):
        seen = torch.ones((n, m), dtype=torch.bool)
        if causal:
            seen = torch.arange(m)[None] <= (m - n + torch.arange(n))[:, None]
        if mask is not None:
            w = torch.zeros(m, dtype=torch.bool)
            w[:mask.shape[1]] = mask[s, :m].cpu() != 0
            seen = seen & w[None]
        k, v, excess = held[s]
        want, l, b_out, b_lse = K.attend(q[t:t + n], k, v, seen, scale or cache.head_dim ** -0.5, q.dtype, excess)
        got, gl = out[t:t + n].double().cpu(), lse[t:t + n].double().cpu()
        empty = ~seen.any(1)
        assert bool((got[empty] == 0).all()) and bool((gl[empty] == -math.inf).all()), (label, s, "empty rows")
        err = (got - want).abs()
        assert bool(((err <= b_out) | empty[:, None, None]).all()), (label, s, "out", float((err - b_out).nan_to_num(9e9).max()))
        e2 = (gl - l).abs()
        assert bool(((e2 <= b_lse) | empty[:, None]).all()), (label, s, "lse", float((e2 - b_lse)[~empty].max()))
        t += n
    assert bool((out[t:] == 7.0).all()) and bool((lse[t:] == 7.0).all()), "rows past the batch were written"


HEADS = [(32, 8, 128), (28, 4, 128), (16, 8, 64), (5, 5, 64), (14, 2, 64), (8, 1, 128), (1, 1, 128)]
BATCHES = [
    # new tokens, cached tokens with them, page size
    ([1], [1], 16),
    ([1, 1, 1], [2, 0, 63], 64),
    ([1, 1, 1, 1, 1], [64, 65, 300, 1111, 17], 32),
    ([1, 0, 3, 2], [400, 9, 3, 1], 16),
    ([2, 4, 1], [257, 130, 1000], 128),
    ([9, 30, 1, 17], [9, 700, 90, 16], 64),
    ([70, 1, 129], [500, 2, 260], 256),
]


@pytest.mark.parametrize("bits,dtype", [(16, torch.bfloat16), (4, torch.bfloat16), (16, torch.float16), (4, torch.float16)])
@pytest.mark.parametrize("new,lengths,page", BATCHES)
def test_attend(bits, dtype, new, lengths, page):
    for i, (h, kv, d) in enumerate(HEADS):
        g = torch.Generator().manual_seed(100 * i + page)
        table, n_pages = _table(lengths, page, 1, g)
        cache = _cache(n_pages, page, h, kv, d, dtype, bits)
        held = _fill(cache, table, lengths, g)
        q = (1.5 * torch.randn((sum(new), h, d), generator=g)).to(dtype).cuda()
        _check_attend(cache, q, table, lengths, new, held, label=(h, kv, d))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("new,lengths", [([1, 1, 1, 1], [700, 40, 131, 64]), ([20, 3, 40, 2], [700, 40, 131, 64])])
def test_masks(bits, new, lengths):
    """Whole tiles masked, single places, nothing left, a mask shorter than the sequence; what is masked holds NaN."""
    h, kv, d, page = 8, 2, 128, 32
    g = torch.Generator().manual_seed(bits)
    table, n_pages = _table(lengths, page, 1, g)
    width = 650  # the first sequence goes on past the mask
    mask = torch.rand((4, width), generator=g) < 0.5
    mask[0, 64:400] = False
    mask[1] = False  # nothing of this one
    mask[2, :128] = False  # only its last places
    mask[2, 128:] = True
    mask[3] = True
    for causal in (True, False):
        cache = _cache(n_pages, page, h, kv, d, torch.bfloat16, bits)
        seen = torch.zeros((4, 700), dtype=torch.bool)
        seen[:, :width] = mask
        held = _fill(cache, table, lengths, g, seen)
        q = torch.randn((sum(new), h, d), generator=g).to(torch.bfloat16).cuda()
        _check_attend(cache, q, table, lengths, new, held, mask=mask.cuda(), causal=causal, label=causal)
        _check_attend(cache, q, table, lengths, new, held, mask=(mask * 3).to(torch.uint8).cuda(), causal=causal, scale=0.3)


@pytest.mark.parametrize("bits", [16, 4])
def test_long_and_short_in_one_call(bits):
    """Work that is split over many CTAs beside sequences of a few tokens; twice, the same bits."""
    h, kv, d, page = 8, 2, 64, 64
    new, lengths = [1, 2, 1, 1, 1], [20000, 3, 1, 4097, 64]
    g = torch.Generator().manual_seed(2)
    table, n_pages = _table(lengths, page, 1, g)
    cache = _cache(n_pages, page, h, kv, d, torch.bfloat16, bits)
    held = _fill(cache, table, lengths, g)
    q = (2 * torch.randn((sum(new), h, d), generator=g)).to(torch.bfloat16).cuda()
    _check_attend(cache, q, table, lengths, new, held)
    lens, offsets = torch.tensor(lengths, dtype=torch.int32, device="cuda"), _offsets(new)
    a, b = (cache.attend(q, table, lens, offsets, max_new=2) for _ in range(2))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("bits", [16, 4])
def test_many_rows_over_a_long_cache(bits):
    for (h, kv, d), new, lengths in (((8, 2, 128), [300], [3000]), ((7, 1, 64), [64, 150], [1500, 200])):
        g = torch.Generator().manual_seed(3)
        table, n_pages = _table(lengths, 64, 1, g)
        for dtype in (torch.bfloat16, torch.float16):
            cache = _cache(n_pages, 64, h, kv, d, dtype, bits)
            held = _fill(cache, table, lengths, g)
            q = (2 * torch.randn((sum(new), h, d), generator=g)).to(dtype).cuda()
            _check_attend(cache, q, table, lengths, new, held)
            _check_attend(cache, q, table, lengths, new, held, max_new=0)


@pytest.mark.parametrize("h,kv,d", [(16, 8, 64), (16, 2, 128)])
def test_row_blocks_of_one_and_of_two_tiles_in_turn(h, kv, d):
    """Items whose second tile of 128 rows is empty between items where it is not, long enough that the roles of a CTA
    run as far apart as they can; repeated, the same bits."""
    G = h // kv
    new, lengths = [300 // G, 100 // G, 600 // G, 40 // G + 5, 430 // G], [2500, 3000, 700, 2100, 5000]
    g = torch.Generator().manual_seed(11)
    table, n_pages = _table(lengths, 32, 1, g)
    for bits in (16, 4):
        cache = _cache(n_pages, 32, h, kv, d, torch.bfloat16, bits)
        held = _fill(cache, table, lengths, g)
        q = (2 * torch.randn((sum(new), h, d), generator=g)).to(torch.bfloat16).cuda()
        _check_attend(cache, q, table, lengths, new, held)
        lens, offsets = torch.tensor(lengths, dtype=torch.int32, device="cuda"), _offsets(new)
        first = cache.attend(q, table, lens, offsets, max_new=max(new))
        for _ in range(20):
            again = cache.attend(q, table, lens, offsets, max_new=max(new))
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
        cache.status()


@pytest.mark.parametrize("bits", [16, 4])
def test_pages_past_four_gigabytes(bits):
    """Places whose byte offsets pass 32 bits: the last pages of a large pool, read, appended to and attended to."""
    from paper_2609_03675_gb300 import Rotary
    h, kv, d, page = 8, 4, 128, 64
    each = kv * page * d * bits // 8
    n_pages = (1 << 32) // each + 40
    rotary = Rotary(d)
    cache = _cache(n_pages, page, h, kv, d, torch.bfloat16, bits, rotary)
    far = torch.arange(n_pages - 30, n_pages, dtype=torch.int32).view(2, 15).contiguous().cuda()
    near = torch.arange(30, dtype=torch.int32).view(2, 15).contiguous().cuda()
    g = torch.Generator(device="cuda").manual_seed(3)
    for new in ([1, 1], [60, 45]):
        lens = torch.tensor([900, 333], dtype=torch.int32, device="cuda")
        x = torch.randn((1233, h + 2 * kv, d), generator=g, device="cuda").to(torch.bfloat16)
        pos = torch.arange(1233, device="cuda", dtype=torch.int32)
        whole = torch.tensor([0, 900, 1233], dtype=torch.int32, device="cuda")
        got = []
        for table in (far, near):
            cache.append(x[:, h:h + kv], x[:, h + kv:], table, lens, whole, positions=pos)
            q = x[:sum(new), :h].contiguous()
            got.append((*cache.read(table, lens, whole, n_tokens=1233), *cache.attend(q, table, lens, _offsets(new), max_new=max(new))))
        cache.status()
        for a, b in zip(*got):
            assert torch.equal(a, b)


def test_large_scores_and_planted_keys():
    """Scores in the hundreds, rising along the sequence, so that the running maximum moves in every tile."""
    h, kv, d = 4, 2, 128
    new, lengths = [1, 3], [2000, 777]
    for bits in (16, 4):
        for n in (new, [40, 50]):
            g = torch.Generator().manual_seed(4)
            table, n_pages = _table(lengths, 64, 1, g)
            cache = _cache(n_pages, 64, h, kv, d, torch.bfloat16, bits)
            held = []
            for s, m in enumerate(lengths):
                k = (torch.randn((m, kv, d), generator=g) * 0.3 + torch.linspace(0, 6, m)[:, None, None]).to(torch.bfloat16)
                v = torch.randn((m, kv, d), generator=g).to(torch.bfloat16)
                at = torch.arange(m)
                p, o = table[s].cpu().long()[at // 64].cuda(), (at % 64).cuda()
                if bits == 16:
                    cache.k_pages[p, :, o], cache.v_pages[p, :, o] = k.cuda(), v.cuda()
                    held.append((k.double(), v.double(), None))
                else:
                    e = []
                    for x, pages, scales in ((k, cache.k_pages, cache.k_scales), (v, cache.v_pages, cache.v_scales)):
                        b, w = K.pack(*K.quantise(x))
                        pages[p, :, o], scales[p, :, o] = b.cuda(), w.cuda()
                        e.append(K.unpack(b, w))
                    held.append((e[0][0], e[1][0], e[0][1] * 144))
            q = (torch.randn((sum(n), h, d), generator=g) + 1.0).to(torch.bfloat16).cuda()
            _check_attend(cache, q, table, lengths, n, held)


def test_strided_queries_and_outputs():
    h, kv, d = 6, 3, 64
    new, lengths = [1, 2, 18], [100, 50, 300]
    g = torch.Generator().manual_seed(6)
    table, n_pages = _table(lengths, 16, 1, g)
    cache = _cache(n_pages, 16, h, kv, d, torch.float16, 16)
    held = _fill(cache, table, lengths, g)
    for pad in (0, 1, 8):
        wide = torch.randn((sum(new), h * d + 2 * kv * d + pad), generator=g).half().cuda()
        q = wide[:, pad:pad + h * d].unflatten(1, (h, d))
        dest = torch.empty((h, sum(new) + 3, d), dtype=torch.float16, device="cuda").transpose(0, 1)[:sum(new)]

        def call(q_, table_, lens, offsets, mask, out, lse):
            cache.attend(q_, table_, lens, offsets, max_new=18, out=dest, lse=lse)
            out.copy_(dest)
        _check_attend(cache, q, table, lengths, new, held, call=call, label=pad)


def test_capture_and_growing_lengths():
    """One captured step (append, attend) launched for several tokens: table and lengths are read on the device."""
    from paper_2609_03675_gb300 import Rotary
    h, kv, d, page, seqs = 8, 2, 64, 16, 3
    table = torch.arange(seqs * 4, dtype=torch.int32, device="cuda").view(seqs, 4).contiguous()
    rotary = Rotary(d)
    for bits in (16, 4):
        step = _cache(seqs * 4, page, h, kv, d, torch.bfloat16, bits, rotary)
        whole = _cache(seqs * 4, page, h, kv, d, torch.bfloat16, bits, rotary)
        g = torch.Generator(device="cuda").manual_seed(7)
        x = torch.randn((40, seqs, h + 2 * kv, d), generator=g, device="cuda").to(torch.bfloat16)
        now, pos = torch.zeros_like(x[0]), torch.zeros(seqs, dtype=torch.int32, device="cuda")
        lens = torch.ones(seqs, dtype=torch.int32, device="cuda")
        out, lse = torch.empty_like(now[:, :h]), torch.empty((seqs, h), device="cuda")
        qo = torch.empty_like(out)

        def run(c):
            c.append(now[:, h:h + kv], now[:, h + kv:], table, lens, positions=pos, q=now[:, :h], q_out=qo)
            c.attend(qo, table, lens, out=out, lse=lse)

        run(step)  # before the capture; its token is written again
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(step)
        for t in range(40):
            now.copy_(x[t])
            pos.fill_(t)
            lens.fill_(t + 1)
            graph.replay()
            a = out.clone(), lse.clone()
            run(whole)
            assert torch.equal(a[0], out) and torch.equal(a[1], lse), (bits, t)
        step.status()


def test_bad_device_data_is_reported_and_left_out():
    from paper_2609_03675_gb300 import NGFFError
    g = torch.Generator().manual_seed(8)
    for bits in (16, 4):
        for n in (1, 40):
            cache = _cache(4, 16, 2, 1, 64, torch.bfloat16, bits)
            k = torch.randn((2 * n, 1, 64), generator=g).to(torch.bfloat16).cuda()
            q = torch.randn((2 * n, 2, 64), generator=g).to(torch.bfloat16).cuda()
            offsets = _offsets([n, n])
            table = torch.tensor([[0, 1, 4], [2, 3, -1]], dtype=torch.int32, device="cuda")
            lens = torch.tensor([40, 48], dtype=torch.int32, device="cuda")
            cache.append(k, k, table, lens, offsets)
            with pytest.raises(NGFFError, match="page"):
                cache.status()
            cache.status()  # reported once
            cache.attend(q, table, lens, offsets, max_new=n)
            with pytest.raises(NGFFError, match="page"):
                cache.status()
            for bad in ([49, 40], [-1, 40]):
                lens = torch.tensor(bad, dtype=torch.int32, device="cuda")
                good = torch.tensor([[0, 1, 0], [2, 3, 2]], dtype=torch.int32, device="cuda")
                cache.attend(q, good, lens, offsets, max_new=n)
                with pytest.raises(NGFFError, match="length"):
                    cache.status()
            # offsets that do not rise, or pass the rows that there are
            for off in ([0, 5 * n, 2 * n], [0, n, 9 * n], [-3, n, 2 * n]):
                lens = torch.tensor([40, 40], dtype=torch.int32, device="cuda")
                cache.attend(q, good, lens, torch.tensor(off, dtype=torch.int32, device="cuda"), max_new=n)
                with pytest.raises(NGFFError, match="length|offset"):
                    cache.status()


def test_refusals():
    from paper_2609_03675_gb300 import KVCache, NGFFError, Rotary
    for args, msg in (((0, 16, 2, 1, 64), "n_pages"), ((2, 24, 2, 1, 64), "page_size"), ((2, 16, 3, 2, 64), "n_kv_heads"),
                      ((2, 16, 2, 1, 96), "head_dim")):
        with pytest.raises(NGFFError, match=msg):
            KVCache(*args)
    with pytest.raises(ValueError, match="bits"):
        KVCache(2, 16, 2, 1, 64, bits=8)
    with pytest.raises(ValueError, match="dtype"):
        KVCache(2, 16, 2, 1, 64, dtype=torch.float32)
    cache = KVCache(2, 16, 2, 1, 64)
    t, l = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    k = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(1, dtype=torch.int32, device="cuda")
    for call, msg in ((lambda: cache.append(k, k, t.long(), l), "table"), (lambda: cache.append(k, k, t, l.long()), "lengths"),
                      (lambda: cache.append(k, k[:0], t, l), "v must be"), (lambda: cache.append(q, k, t, l), "k must be"),
                      (lambda: cache.append(k.half(), k, t, l), "k must be"), (lambda: cache.append(k, k, t, l, positions=pos), "rotary"),
                      (lambda: cache.append(k, k, t, l, q=q), "rotary"), (lambda: cache.attend(k, t, l), "q must be"),
                      (lambda: cache.attend(q, t, l, mask=torch.ones(1, 2, device="cuda")), "mask"),
                      (lambda: cache.attend(q, t, l, lse=torch.zeros(1, 2, device="cuda").half()), "lse"),
                      (lambda: cache.attend(q.cpu(), t, l), "q must be"),
                      (lambda: cache.read(t, l, out=(k, k.half())), "out must be")):
        with pytest.raises(ValueError, match=msg):
            call()
    with pytest.raises(NGFFError, match="one new token"):
        cache.attend(q.expand(3, -1, -1), t, l)
    with pytest.raises(NGFFError, match="scale"):
        cache.attend(q, t, l, scale=-1.0)
    with pytest.raises(NGFFError, match="head_dim"):
        KVCache(2, 16, 2, 1, 64, rotary=Rotary(128)).append(k, k, t, l, positions=pos)
    assert cache.attend(q[:0], t[:0], l[:0])[0].shape == (0, 2, 64)

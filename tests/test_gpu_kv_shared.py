"""Attention of sequences behind shared prefixes, against its definition: attention over the prefix's tokens and the
sequence's own, in 64 bits, to the bounds of tests/kv_bounds.py (whose 2^-16 of sum p |v| and 2^-20 of the log-sum-exp have
room for the two roundings that joining the parts adds: factors good to 2^-22, two products and a sum)."""
import math

import pytest
import torch

from tests import kv_bounds as B
from tests import test_gpu_kv as T
from tests import test_gpu_kv_int8 as I
from tests.test_gpu_kv import _offsets, _table

pytestmark = pytest.mark.gpu

BITS = [16, "int8", 4]


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Shared:
    """A cache that holds sequences' own tokens and prefixes, what it holds as numbers, and the call."""

    def __init__(self, bits, dtype, heads, new, own, prefixes, groups, page, seed=0, prefix_mask=None, mask=None):
        """groups: the first sequence of each group, and the end of the last; masks [sequences, width], bool."""
        h, kv, d = heads
        g = self.g = torch.Generator().manual_seed(seed + page)
        self.new, self.own, self.prefixes, self.groups = new, own, prefixes, groups
        S = len(new)
        table, n_pages = _table(own + prefixes, page, 2, g)
        make, fill = (I.make, I.fill) if bits == "int8" else (lambda *a: T._cache(*a, bits), T._fill)
        self.cache = make(n_pages, page, h, kv, d, dtype)
        seen = torch.ones((S + len(prefixes), max(own + prefixes + [1])), dtype=torch.bool)
        if mask is not None:
            seen[:S] = False
            seen[:S, :mask.shape[1]] = mask[:, :seen.shape[1]]
        if prefix_mask is not None:  # what none of the group sees stays NaN
            seen[S:] = False
            for i in range(len(prefixes)):
                w = prefix_mask[groups[i]:groups[i + 1]].any(0)[:seen.shape[1]]
                seen[S + i, :len(w)] = w
        self.held = [x[:2] for x in fill(self.cache, table, own + prefixes, g, seen)]
        self.table, self.prefix_table = table[:S].contiguous(), table[S:].contiguous()
        self.lens, self.prefix_lens = _ints(*own), _ints(*prefixes)
        self.offsets, self.group_of = _offsets(new), _ints(*groups)
        self.mask, self.prefix_mask = mask, prefix_mask
        self.q = (1.5 * torch.randn((sum(new), h, d), generator=g)).to(dtype).cuda()

    def call(self, q=None, **kw):
        args = dict(prefix_table=self.prefix_table, prefix_lengths=self.prefix_lens, groups=self.group_of, max_new=max(self.new),
                    max_shared=max([sum(self.new[a:b]) for a, b in zip(self.groups, self.groups[1:])] + [1]),
                    mask=None if self.mask is None else self.mask.cuda(), prefix_mask=None if self.prefix_mask is None else self.prefix_mask.cuda())
        args.update(kw)
        return self.cache.attend_shared(self.q if q is None else q, self.table, self.lens, self.offsets, **args)

    def check(self, causal=True, scale=0.0, **kw):
        q, c = self.q, self.cache
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        self.call(out=out, lse=lse, causal=causal, scale=scale, **kw)
        c.status()
        self.compare(out, lse, causal, scale)
        return out, lse

    def compare(self, out, lse, causal=True, scale=0.0):
        q, c, S = self.q, self.cache, len(self.new)
        out, lse, t = out.cpu(), lse.cpu(), 0
        for s, (n, m) in enumerate(zip(self.new, self.own)):
            seen = torch.ones((n, m), dtype=torch.bool)
            if causal:
                seen = torch.arange(m)[None] <= (m - n + torch.arange(n))[:, None]
            if self.mask is not None:
                w = torch.zeros(m, dtype=torch.bool)
                w[:self.mask.shape[1]] = self.mask[s, :m]
                seen = seen & w
            k, v = self.held[s]
            for i in range(len(self.prefixes)):
                if self.groups[i] <= s < self.groups[i + 1]:
                    p = self.prefixes[i]
                    w = torch.ones(p, dtype=torch.bool)
                    if self.prefix_mask is not None:
                        w[:] = False
                        w[:self.prefix_mask.shape[1]] = self.prefix_mask[s, :p]
                    seen = torch.cat([w[None].expand(n, -1), seen], 1)
                    k, v = torch.cat([self.held[S + i][0], k]), torch.cat([self.held[S + i][1], v])
            if n:
                bad = B.exceeds(out[t:t + n], lse[t:t + n], B.attend(q[t:t + n], k, v, seen, scale or c.head_dim ** -0.5, q.dtype))
                assert not bool(bad[0].any()), (s, "out")
                assert not bool(bad[1].any()), (s, "lse")
            t += n
        assert bool((out[t:] == 7.0).all()) and bool((lse[t:] == 7.0).all()), "rows past the batch were written"


HEADS = [(32, 8, 128), (28, 4, 128), (16, 8, 64), (5, 5, 64), (14, 2, 64), (8, 1, 128), (1, 1, 128)]
BATCHES = [
    # new tokens, own cached tokens with them, prefixes, groups, page size
    ([1], [1], [1], [0, 1], 16),
    ([1, 1], [3, 40], [700], [0, 2], 64),
    ([1, 1, 1, 1], [1, 65, 2, 130], [64], [0, 4], 32),
    ([2, 1, 3], [2, 80, 9], [333, 65], [0, 1, 3], 16),  # two groups
    ([1] * 9, [5, 0, 1, 64, 65, 63, 1, 300, 2], [129, 0, 500], [1, 4, 5, 8], 128),  # no prefix, and an empty one
    ([20, 3, 40, 2], [20, 3, 90, 200], [450], [0, 4], 64),
    ([70, 1, 129, 5], [70, 100, 260, 5], [300, 200], [0, 2, 4], 256),
    ([1] * 70, [1 + 3 * i % 50 for i in range(70)], [1000], [0, 70], 64),
    ([3, 0, 2], [40, 7, 1], [90], [0, 3], 16),  # a sequence without new tokens, one of fewer cached than new
]


@pytest.mark.parametrize("bits,dtype", [(b, t) for b in BITS for t in (torch.bfloat16, torch.float16)])
@pytest.mark.parametrize("new,own,prefixes,groups,page", BATCHES)
def test_attend_shared(bits, dtype, new, own, prefixes, groups, page):
    for i, heads in enumerate(HEADS):
        x = Shared(bits, dtype, heads, new, own, prefixes, groups, page, seed=100 * i)
        x.check()
        if i in (1, 2):
            x.check(causal=False, scale=0.11)
            x.check(max_new=0, max_shared=0)  # no hints
            x.check(max_new=1, max_shared=1)  # wrong ones choose other kernels


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("heads", [(8, 2, 128), (16, 8, 64), (14, 2, 64)])
@pytest.mark.parametrize("new,own", [([1, 1, 1, 1, 1], [30, 1, 70, 64, 5]), ([3, 2, 1, 4, 2], [30, 2, 70, 64, 5]), ([30, 9, 25, 64, 2], [30, 9, 70, 64, 5])])
def test_masks(bits, heads, new, own):
    """Each sequence its own evidence: whole tiles, single places, nothing; masks shorter than the prefix, of every
    alignment; own tokens masked too; a row that sees nothing of either. What none of a group sees holds NaN."""
    prefixes, groups = [700, 333], [0, 3, 5]
    for width, own_width in ((704, 70), (700, 33), (697, 0), (64, 70)):
        g = torch.Generator().manual_seed(width)
        pm = torch.rand((5, width), generator=g) < 0.4
        pm[0, 64:640] = False
        pm[1] = False
        pm[2, 128:192] = False
        pm[0:3, 200:330] = False  # nobody of the first group
        pm[3] = True
        mask = torch.rand((5, own_width), generator=g) < 0.7
        mask[1] = False  # nothing at all
        x = Shared(bits, torch.bfloat16, heads, new, own, prefixes, groups, 32, seed=width, prefix_mask=pm, mask=mask)
        x.check()
        x.check(causal=False)
        x.mask = None
        if width == 704:
            y = Shared(bits, torch.float16, heads, new, own, prefixes, groups, 64, seed=1, prefix_mask=pm)
            y.check()
            y.check(prefix_mask=pm.to(torch.uint8).cuda() * 5, max_shared=0)


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("heads", [(8, 1, 128), (16, 2, 64), (7, 1, 128)])
@pytest.mark.parametrize("new", [[16, 16], [20, 20, 30], [10, 17, 5, 40], [64, 3]])
def test_evidence_of_one_half_of_a_block(bits, heads, new):
    """Runs of tiles that only the first or only the second 128 rows of a block see: long ones, every other one, the first
    of all, and a token whose heads lie in both halves (7 heads); blocks of their last rows alone."""
    S, width = len(new), 6001
    at = torch.arange(width)
    for run in (64, 192, 3000):
        for turn in (0, 1):
            pm = torch.stack([(at // run + turn) % S == s for s in range(S)])
            pm[:, 4000:4100] = False
            x = Shared(bits, torch.bfloat16, heads, new, new, [width], [0, S], 64, seed=run, prefix_mask=pm)
            x.check()
    y = Shared(bits, torch.float16, heads, new + new, new + new, [width, 700], [0, S, 2 * S], 32, prefix_mask=torch.cat([pm, ~pm]))
    y.check()
    y.check(max_shared=20)  # lists of the first block stand for those after it


def test_masked_sums_that_outlast_tensor_memory():
    """fp16 sums that leave tensor memory after 128 tiles, of which either half of a block's rows sees others."""
    G, width = 10, 12801  # 160 items of 201 tiles over 152 CTAs
    at = torch.arange(width)
    pm = torch.stack([at % 640 >= 192, at % 640 < 512])
    x = Shared(16, torch.float16, (128, 16, 64), [16, 16] * G, [16, 17] * G, [width] * G, list(range(0, 2 * G + 1, 2)), 64, prefix_mask=pm.repeat(G, 1))
    x.check()


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("n", [1, 9, 40])
def test_a_prefix_alone_and_none_at_all(bits, n):
    """One group of all without offsets; prefixes of no tokens give what attend gives, to the bit."""
    S, h, kv, d = 6, 8, 2, 128
    x = Shared(bits, torch.bfloat16, (h, kv, d), [n] * S, [n + 10 * s for s in range(S)], [900], [0, S], 64)
    x.check(groups=None)
    zero = _ints(0)
    a = x.call(groups=None, prefix_lengths=zero)
    b = x.cache.attend(x.q, x.table, x.lens, x.offsets, max_new=n)
    assert torch.equal(a[0], b[0]) and torch.allclose(a[1], b[1], rtol=2.0 ** -21, atol=2.0 ** -21)
    # own caches of nothing: the prefix alone, which attend gives for all rows as one sequence's
    none = torch.zeros_like(x.lens)
    a = x.cache.attend_shared(x.q, x.table, none, x.offsets, prefix_table=x.prefix_table, prefix_lengths=x.prefix_lens, max_new=n)
    b = x.cache.attend(x.q, x.prefix_table, x.prefix_lens, _ints(0, n * S), max_new=n * S, causal=False)
    x.cache.status()
    assert torch.allclose(a[0].float(), b[0].float(), rtol=2.0 ** -7, atol=2.0 ** -10) and torch.allclose(a[1], b[1], rtol=2.0 ** -20, atol=2.0 ** -20)
    if n == 1:
        a = x.cache.attend_shared(x.q, x.table, x.lens, prefix_table=x.prefix_table, prefix_lengths=x.prefix_lens)
        x.compare(*a)


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("new", [1, 30])
def test_long_prefixes_are_the_same_bits_again(bits, new):
    """Work split over all CTAs; repeated, on another stream, with other strides and in place: the same bits."""
    S, heads = 5, (8, 2, 128)
    x = Shared(bits, torch.bfloat16, heads, [new] * S, [new + 700 * s for s in range(S)], [20000], [0, S], 64)
    want = x.check()
    for _ in range(5):
        got = x.call()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = x.call(cuda_stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    n, h, d = x.q.shape
    wide = torch.zeros((n, h + 3, d + 1), dtype=x.q.dtype, device="cuda")
    q = wide[:, 1:h + 1, :d]
    q.copy_(x.q)
    out = torch.zeros((h, n, d + 2), dtype=x.q.dtype, device="cuda").transpose(0, 1)[..., 1:d + 1]
    got = x.call(q=q, out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q = x.q.clone()
    got = x.call(q=q, out=q)
    assert torch.equal(q, want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("new", [1, 20])
def test_captured_before_larger_calls(bits, new):
    """A graph's scratch stays its own when later calls need more; replayed with other queries, lengths and masks."""
    S, heads = 4, (8, 2, 64)
    pm = torch.rand((S, 512), generator=torch.Generator().manual_seed(1)) < 0.3
    x = Shared(bits, torch.bfloat16, heads, [new] * S, [new + 9 * s for s in range(S)], [500], [0, S], 16)
    mask = pm.cuda()
    out, lse = torch.empty_like(x.q), torch.empty(x.q.shape[:2], device="cuda")

    def call():
        x.call(prefix_mask=mask, out=out, lse=lse)

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    kept = []
    for seqs in (40, 300):  # more rows, and a larger mask
        one = _ints(*[1] * seqs)
        q = torch.randn((seqs, 8, 64), device="cuda").to(torch.bfloat16)
        for _ in range(2):
            x.cache.attend_shared(q, x.table[:1].expand(seqs, -1).contiguous(), one, prefix_table=x.prefix_table, prefix_lengths=x.prefix_lens,
                                  prefix_mask=mask[:1].expand(seqs, -1).contiguous())
        kept.append(torch.full((1 << 18,), 7, dtype=torch.int32, device="cuda"))
    for i in range(3):
        x.prefix_mask = torch.rand((S, 512), generator=torch.Generator().manual_seed(i + 5)) < 0.3
        mask.copy_(x.prefix_mask)
        x.q.copy_(torch.randn(x.q.shape, device="cuda"))
        x.prefix_lens.fill_(500 - 100 * i)
        x.prefixes[0] = 500 - 100 * i
        x.held[S] = [y[:x.prefixes[0]] for y in x.held[S]]
        out.fill_(9.0)
        graph.replay()
        got = out.clone(), lse.clone()
        x.compare(*got)
        call()
        assert torch.equal(got[0], out) and torch.equal(got[1], lse)
    x.cache.status()
    assert all(bool((y == 7).all()) for y in kept)


def test_growth_while_capturing_is_refused():
    from paper_2609_03675_gb300 import NGFFError
    x = Shared(16, torch.bfloat16, (2, 1, 64), [1], [1], [16], [0, 1], 16)
    torch.cuda.synchronize()
    out, lse, mask = torch.empty_like(x.q), torch.empty(x.q.shape[:2], device="cuda"), torch.ones((1, 16), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(NGFFError, match="capture"):
            x.call(out=out, lse=lse)
    x.call(out=out, lse=lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.call(out=out, lse=lse)
        with pytest.raises(NGFFError, match="capture"):
            x.call(out=out, lse=lse, prefix_mask=mask)
    graph.replay()
    x.compare(out, lse)


@pytest.mark.parametrize("new", [1, 20])
def test_bad_pages_lengths_and_groups_are_reported(new):
    """Left out, and reported by status; nothing outside is read."""
    from paper_2609_03675_gb300 import NGFFError
    x = Shared(16, torch.bfloat16, (8, 2, 64), [new] * 3, [new + 5] * 3, [300, 200], [0, 2, 3], 16)
    x.check()
    table = x.prefix_table.clone()
    table[0, 3] = x.cache.n_pages
    x.call(prefix_table=table)
    with pytest.raises(NGFFError, match="page"):
        x.cache.status()
    for kw in ({"prefix_lengths": _ints(-1, 200)}, {"prefix_lengths": _ints(300, 1 << 30)}, {"groups": _ints(0, 4, 3)}, {"groups": _ints(-1, 2, 3)},
               {"groups": _ints(0, 2, 9)}, {"groups": _ints(3, 0, 3)}):
        for mask in (None, torch.ones((3, 300), dtype=torch.uint8, device="cuda")):
            x.call(prefix_mask=mask, **kw)
            with pytest.raises(NGFFError, match="length|offset|group"):
                x.cache.status()
    x.check()


def test_pages_past_four_gigabytes_and_rows_past_two():
    """A prefix in the last pages of a large pool; scratch rows whose bytes pass 32 bits."""
    from paper_2609_03675_gb300 import KVCache
    h, kv, d, page = 64, 8, 128, 64
    n_pages = (1 << 32) // (kv * page * d * 2) + 40
    cache = KVCache(n_pages, page, h, kv, d)
    n = (1 << 32) // (h * d * 4) + 100  # rows of single tokens
    table = torch.arange(n_pages - 1, n_pages - 31, -1, dtype=torch.int32, device="cuda").view(1, -1)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((1500, kv, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    cache.append(k, v, table, _ints(1500), _ints(0, 1500))
    q = torch.randn((n, h, d), generator=g, device="cuda").to(torch.bfloat16)
    own = torch.zeros((n, 1), dtype=torch.int32, device="cuda")  # every sequence's own token is the pool's first page's first
    cache.append(k[:1], v[:1], own[:1], _ints(1))
    out, lse = cache.attend_shared(q, own, torch.ones(n, dtype=torch.int32, device="cuda"), prefix_table=table, prefix_lengths=_ints(1500))
    cache.status()
    last = torch.tensor([0, 1, n // 2, n - 2, n - 1], device="cuda")
    both = [torch.cat([x, x[:1]]).cpu() for x in (k, v)]
    bad = B.exceeds(out[last], lse[last], B.attend(q[last], *both, torch.ones((5, 1501), dtype=torch.bool), d ** -0.5, q.dtype))
    assert not bool(bad[0].any()) and not bool(bad[1].any())


def test_refusals():
    from paper_2609_03675_gb300 import NGFFError
    x = Shared(16, torch.bfloat16, (4, 2, 64), [1, 1], [1, 2], [20, 30], [0, 1, 2], 16)
    pt, pl, gr = x.prefix_table, x.prefix_lens, x.group_of
    for kw, msg in (({"prefix_table": pt.long()}, "prefix_table"), ({"prefix_table": pt[0]}, "prefix_table"), ({"prefix_table": pt.cpu()}, "prefix_table"),
                    ({"prefix_lengths": pl[:1]}, "prefix_lengths"), ({"prefix_lengths": pl.float()}, "prefix_lengths"), ({"groups": None}, "groups"),
                    ({"groups": gr[:2]}, "groups"), ({"prefix_mask": torch.ones((1, 30), dtype=torch.uint8, device="cuda")}, "prefix_mask"),
                    ({"prefix_mask": torch.ones((2, 30), device="cuda")}, "prefix_mask"), ({"mask": torch.ones((3, 30), dtype=torch.uint8, device="cuda")}, "mask"),
                    ({"lse": torch.empty((2, 4), device="cuda").half()}, "lse")):
        with pytest.raises(ValueError, match=msg):
            x.call(**kw)
    with pytest.raises(NGFFError, match="scale"):
        x.call(scale=math.nan)
    with pytest.raises(ValueError, match="gradient"):
        x.call(q=x.q.clone().requires_grad_())
    assert x.cache.attend_shared(x.q[:0], x.table[:0], x.lens[:0], prefix_table=pt, prefix_lengths=pl, groups=gr)[0].shape == (0, 4, 64)
    x.check()

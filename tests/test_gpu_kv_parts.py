"""Attention of many rows where a CTA works off an item of its own, whose sums outlast tensor memory and are kept in the CTA's
part, and then begins one that goes on into the next CTA, whose part lies in the same place."""
import pytest
import torch

from tests import kv_bounds as B

pytestmark = pytest.mark.gpu

CHAIN = {torch.float16: 128, torch.bfloat16: 1024}  # tiles of 64 tokens that tensor memory sums


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def pairs(ctas, seqs, new, m, kv, group, chain):
    """The walk of the items over the CTAs: (rows of the second item, its tiles here) wherever one with kept sums and more
    than 128 rows comes before one that goes on and that nothing else orders after it."""
    items = []
    for _ in range(seqs):
        rows = new * group
        for at in range(0, rows, 256):
            end = min(rows, at + 256)
            items += [(end - at, -(-(m - new + (end - 1) // group + 1) // 64))] * kv
    size = -(-sum(8 + t for _, t in items) // ctas)
    found, kept, at = [], set(), 0
    for rows, tiles in items:
        first, past = (at + 8) // size, (at + 8 + tiles - 1) // size
        here = min(at + 8 + tiles, (first + 1) * size) - (at + 8)
        if first == past and tiles > chain and rows > 128:
            kept.add(first)
        if first != past and first in kept and here <= chain:
            found.append((rows, here))
        at += 8 + tiles
    return found


@pytest.mark.parametrize("bits,dtype,seqs,new,m,kv,group", [(16, torch.float16, 40, 300, 9000, 2, 1), ("int8", torch.float16, 40, 75, 9000, 2, 4),
                                                           (4, torch.float16, 60, 300, 12800, 2, 1), (16, torch.bfloat16, 80, 130, 66000, 2, 1)])
def test_kept_sums_before_an_item_that_goes_on(bits, dtype, seqs, new, m, kv, group):
    """The sequences share their pages and queries; all of them against the one definition."""
    from paper_2609_03675_gb300 import KVCache
    d, page, h = 64, 64, kv * group
    ctas = torch.cuda.get_device_properties(0).multi_processor_count
    assert pairs(ctas, seqs, new, m, kv, group, CHAIN[dtype])
    g = torch.Generator().manual_seed(new)
    n_pages = -(-m // page)
    cache = KVCache(n_pages, page, h, kv, d, dtype=dtype, bits=bits)
    k, v = (torch.randn((m, kv, d), generator=g).to(dtype).cuda() for _ in range(2))
    one = torch.arange(n_pages, dtype=torch.int32, device="cuda").view(1, -1)
    all_of, offsets = torch.tensor([m], dtype=torch.int32, device="cuda"), torch.tensor([0, m], dtype=torch.int32, device="cuda")
    cache.append(k, v, one, all_of, offsets)
    k, v = cache.read(one, all_of, offsets, n_tokens=m)
    q = torch.randn((new, h, d), generator=g).to(dtype)
    out, lse = cache.attend(q.cuda().repeat(seqs, 1, 1), one.repeat(seqs, 1), all_of.repeat(seqs),
                            torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * new, max_new=new)
    cache.status()
    seen = torch.arange(m)[None] <= (m - new + torch.arange(new))[:, None]
    want = B.attend(q, k, v, seen, d ** -0.5, dtype)
    bad = B.exceeds(out.view(seqs, new, h, d), lse.view(seqs, new, h), want)
    assert not bool(bad[0].any()) and not bool(bad[1].any())


@pytest.mark.parametrize("bits", [16, "int8", 4])
@pytest.mark.parametrize("heads", [(8, 2, 128), (16, 8, 64), (4, 4, 64), (14, 2, 64)])
@pytest.mark.parametrize("new", [5, 20, 70])
def test_tables_of_every_width(bits, heads, new):
    """The table's width bounds the tokens and chooses whether items are cut, or taken by blocks of few rows: the same
    sequences under tables of 128 to 2048 tokens, with and without prefixes, masked and not, to the one definition."""
    from paper_2609_03675_gb300 import KVCache
    h, kv, d = heads
    page, dtype = 32, torch.bfloat16
    lengths, news = [new, 128, new + 1, 0, 77 + new // 2, 126], [new, 1, new, 0, new // 2, 2]
    g = torch.Generator().manual_seed(new)
    cache = KVCache(4 * len(lengths) + 1, page, h, kv, d, dtype=dtype, bits=bits)
    table = torch.randperm(4 * len(lengths), generator=g).to(torch.int32).view(-1, 4).cuda()
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    whole = torch.tensor([0] + lengths).cumsum(0).to(torch.int32).cuda()
    x = [torch.randn((sum(lengths), kv, d), generator=g).to(dtype).cuda() for _ in range(2)]
    cache.append(*x, table, lens, whole)
    k, v = cache.read(table, lens, whole, n_tokens=sum(lengths))
    q = torch.randn((sum(news), h, d), generator=g).to(dtype).cuda()
    offsets = torch.tensor([0] + news).cumsum(0).to(torch.int32).cuda()
    mask = torch.rand((len(lengths), 128), generator=g) < 0.6
    mask[1] = False
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    for masked in (False, True):
        want, t, at = [], 0, 0
        for s, (n, m) in enumerate(zip(news, lengths)):
            seen = torch.arange(m)[None] <= (m - n + torch.arange(n))[:, None]
            if masked:
                seen = seen & mask[s, :m]
            want.append(B.attend(q[t:t + n], k[at:at + m], v[at:at + m], seen, d ** -0.5, dtype) if n else None)
            t, at = t + n, at + m
        for width in (4, 12, 16, 17, 64):
            wide = torch.nn.functional.pad(table, (0, width - 4)).contiguous()
            kw = dict(max_new=new, mask=mask.cuda() if masked else None)
            for out, lse in (cache.attend(q, wide, lens, offsets, **kw),
                             cache.attend_shared(q, wide, lens, offsets, prefix_table=wide[:1], prefix_lengths=none, **kw)):
                cache.status()
                t = 0
                for n, w in zip(news, want):
                    if n:
                        bad = B.exceeds(out[t:t + n], lse[t:t + n], w)
                        assert not bool(bad[0].any()) and not bool(bad[1].any()), width
                    t += n


@pytest.mark.parametrize("bits", [16, "int8", 4])
@pytest.mark.parametrize("d", [64, 128])
def test_parts_of_more_rows_than_the_call_says(bits, d):
    """Long items that several CTAs share, 300 rows of them where the hint says 17 to 128, or fewer; rows past the batch."""
    from paper_2609_03675_gb300 import KVCache
    h, kv, page, dtype = 8, 2, 64, torch.bfloat16
    lengths, news = [9000, 70, 5000], [75, 3, 20]
    g = torch.Generator().manual_seed(d)
    each = [-(-m // page) for m in lengths]
    cache = KVCache(sum(each), page, h, kv, d, dtype=dtype, bits=bits)
    table = torch.zeros((3, max(each)), dtype=torch.int32)
    for s, e in enumerate(each):
        table[s, :e] = torch.arange(sum(each[:s]), sum(each[:s + 1]))
    table, lens = table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    whole = torch.tensor([0] + lengths).cumsum(0).to(torch.int32).cuda()
    x = [torch.randn((sum(lengths), kv, d), generator=g).to(dtype).cuda() for _ in range(2)]
    cache.append(*x, table, lens, whole)
    k, v = cache.read(table, lens, whole, n_tokens=sum(lengths))
    q = torch.randn((sum(news) + 5, h, d), generator=g).to(dtype).cuda()
    offsets = torch.tensor([0] + news).cumsum(0).to(torch.int32).cuda()
    want, t, at = [], 0, 0
    for n, m in zip(news, lengths):
        seen = torch.arange(m)[None] <= (m - n + torch.arange(n))[:, None]
        want.append(B.attend(q[t:t + n], k[at:at + m], v[at:at + m], seen, d ** -0.5, dtype))
        t, at = t + n, at + m
    for hint in (5, 8, 20, 32, 33, 75, 0):
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        cache.attend(q, table, lens, offsets, max_new=hint, out=out, lse=lse)
        cache.status()
        t = 0
        for n, w in zip(news, want):
            bad = B.exceeds(out[t:t + n], lse[t:t + n], w)
            assert not bool(bad[0].any()) and not bool(bad[1].any()), hint
            t += n
        assert bool((out[t:] == 7.0).all()) and bool((lse[t:] == 7.0).all())

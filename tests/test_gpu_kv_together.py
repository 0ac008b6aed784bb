"""Pages of bytes and shared prefixes as they are used together: a stream's frames appended once, questions behind them,
captured steps; long flat sums; calls that hint wrongly, leave rows over or run out of memory."""
import importlib.util
import os

import pytest
import torch

from tests import kv_bounds as B
from tests import test_gpu_kv_int8 as I
from tests.conftest import REPO
from tests.test_gpu_kv_shared import Shared, _ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("bits", ["int8", 16, 4])
def test_questions_about_one_stream(bits):
    """examples/questions.py: every output is attention, in 64 bits, of the rotated queries over what the cache holds of the
    question's evidence and of its own tokens so far."""
    spec = importlib.util.spec_from_file_location("questions_example", os.path.join(REPO, "examples", "questions.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    chosen, out, outs, made = ex.run(questions=4, steps=3, bits=bits)
    texts, evidence = made["texts"], made["evidence"].cpu() != 0
    assert len(chosen) == 4 and all(len(c) >= 1 for c in chosen)
    (pk, pv), (ok, ov) = made["held"]
    start, first = 0, 0
    for s, n in enumerate(texts):
        length = n + 3
        k, v = torch.cat([pk, ok[start:start + length]]).cpu(), torch.cat([pv, ov[start:start + length]]).cpu()
        for q, got, fresh, before in [(made["queries"][0][first:first + n], out[first:first + n], n, 0)] + \
                [(made["queries"][1 + t][s:s + 1], outs[t][s:s + 1], 1, n + t) for t in range(3)]:
            own = torch.arange(length)[None] <= (before + torch.arange(fresh))[:, None]
            seen = torch.cat([evidence[s][None].expand(fresh, -1), own], 1)
            want = B.attend(q, k, v, seen, ex.HEAD_DIM ** -0.5, torch.bfloat16)
            bad = B.exceeds(got, want[1].float(), want)
            assert not bool(bad[0].any()), (s, before)
        start += length
        first += n


# ---- long flat sums ---------------------------------------------------------------------------------------------------


def _flat(dtype, m, d, above, value, g):
    """Keys and values of which one lies `above` the others and has another value; tests/test_gpu_kv_peaks.py has the other pages."""
    k = torch.zeros((m, 1, d), dtype=dtype)
    k[1000, 0, 0] = 15.0
    v = (1.0 + 0.25 * torch.randn((m, 1, d), generator=g)).to(dtype)
    v[1000] = value
    return k, v


def _put(cache, k, v, page, d):
    held = []
    for x, pages, scales in ((k, cache.k_pages, cache.k_scales), (v, cache.v_pages, cache.v_scales)):
        u, w = I.quantise(x, cache.dtype)
        n = x.shape[0] // page
        pages[:n].copy_(u.view(n, page, 1, d).transpose(1, 2))
        scales[:n].copy_(w.view(n, page, 1, d // 64).transpose(1, 2))
        held.append(I.numbers(u, w))
    return held


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [1, 5, 17])
@pytest.mark.parametrize("above,value", [(0.0, 1.0), (12.0, 0.0), (14.3, 1.0), (17.5, 0.0)])
def test_long_flat_caches_of_bytes(dtype, n, above, value):
    """Neither log-sum-exps nor outputs lose what many small weights come to: 304 sequences share 262144 tokens."""
    from paper_2609_03675_gb300 import KVCache
    seqs, m, d, page, h = 304, 262144, 64, 256, 2
    g = torch.Generator().manual_seed(n)
    cache = KVCache(m // page, page, h, 1, d, dtype=dtype, bits="int8")
    k, v = _put(cache, *_flat(dtype, m, d, above, value, g), page, d)
    q = (0.5 * torch.randn((n, h, d), generator=g)).to(dtype)
    q[..., 0] = above * d ** 0.5 / 15.0
    table = torch.arange(m // page, dtype=torch.int32, device="cuda").repeat(seqs, 1)
    offsets = torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * n
    out, lse = cache.attend(q.cuda().repeat(seqs, 1, 1), table, torch.full((seqs,), m, dtype=torch.int32, device="cuda"), offsets, max_new=n)
    cache.status()
    seen = torch.arange(m)[None] <= (m - n + torch.arange(n))[:, None]
    chain = m // 8 if n * h <= 16 else 8192 if dtype == torch.float16 else 65536
    bad = B.exceeds(out.view(seqs, n, h, d), lse.view(seqs, n, h), B.attend(q, k, v, seen, d ** -0.5, dtype, chain))
    assert not bool(bad[0].any()) and not bool(bad[1].any())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("seqs", [3, 40, 700])
@pytest.mark.parametrize("above,value", [(0.0, 1.0), (14.3, 1.0), (17.5, 0.0)])
def test_long_flat_prefixes(dtype, seqs, above, value):
    """The same of a prefix, for few rows, rows that both streams of a CTA take, and many; own tokens join what is left."""
    from paper_2609_03675_gb300 import KVCache
    m, d, page, h, own = 262144, 64, 256, 2, 5
    g = torch.Generator().manual_seed(seqs)
    cache = KVCache(m // page + 1, page, h, 1, d, dtype=dtype, bits="int8")
    k, v = _flat(dtype, m + page, d, above, value, g)
    k, v = _put(cache, k, v, page, d)
    q = (0.5 * torch.randn((seqs, h, d), generator=g)).to(dtype)
    q[..., 0] = above * d ** 0.5 / 15.0
    stream = torch.arange(m // page, dtype=torch.int32, device="cuda").view(1, -1)
    table = torch.full((seqs, 1), m // page, dtype=torch.int32, device="cuda")  # all of them the last page's first tokens
    out, lse = cache.attend_shared(q.cuda(), table, torch.full((seqs,), own, dtype=torch.int32, device="cuda"), prefix_table=stream, prefix_lengths=_ints(m))
    cache.status()
    keep = slice(0, m + own)
    chain = m // 8 if seqs * h <= 16 else 8192 if dtype == torch.float16 else 65536
    some = torch.tensor(sorted({0, 1, seqs // 2, seqs - 1}))
    want = B.attend(q[some], k[keep], v[keep], torch.ones((len(some), m + own), dtype=torch.bool), d ** -0.5, dtype, chain)
    bad = B.exceeds(out[some.cuda()], lse[some.cuda()], want)
    assert not bool(bad[0].any()) and not bool(bad[1].any())


# ---- calls --------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("bits", [16, "int8", 4])
@pytest.mark.parametrize("new", [[1] * 9, [3, 40, 1, 70, 2, 9, 1, 5, 30]])
def test_masked_calls_with_hints_that_are_wrong_or_missing(bits, new):
    """Lists of tiles are made for as many blocks of rows as the hint gives; the rows past them are served all the same."""
    g = torch.Generator().manual_seed(3)
    pm = torch.zeros((9, 900), dtype=torch.bool)
    for s in range(9):  # frames of 90 tokens that few of the sequences see
        pm[s, 90 * s:90 * s + 90] = True
        pm[s, torch.randint(0, 900, (1,), generator=g)] = True
    x = Shared(bits, torch.bfloat16, (16, 2, 64), new, [n + 3 * i for i, n in enumerate(new)], [900, 700], [0, 6, 9], 32, prefix_mask=pm)
    x.check()
    for hint in (0, 1, 40, 5000):
        x.check(max_shared=hint)
        x.check(max_shared=hint, max_new=hint)


@pytest.mark.parametrize("new", [1, 20])
def test_rows_past_the_batch_are_left_alone(new):
    """More rows of queries than the offsets name, with and without a prefix mask."""
    x = Shared("int8", torch.bfloat16, (8, 2, 64), [new] * 3, [new + 4] * 3, [200], [0, 3], 16)
    q = torch.cat([x.q, x.q[:5]])
    for mask in (None, torch.ones((3, 200), dtype=torch.uint8, device="cuda")):
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        x.call(q=q, out=out, lse=lse, prefix_mask=mask, max_shared=0)
        x.cache.status()
        n = len(x.q)
        assert bool((out[n:] == 7.0).all()) and bool((lse[n:] == 7.0).all())
        x.compare(out[:n], lse[:n])


def test_own_tokens_of_wide_tables_and_of_narrow_ones():
    """The same sequences behind a prefix, their table padded past what one CTA is left to: equal to its bounds."""
    for new in ([1, 1, 1], [3, 1, 4]):
        x = Shared("int8", torch.bfloat16, (8, 2, 128), new, [n + 60 * i for i, n in enumerate(new)], [500], [0, 3], 64)
        a = x.check()
        x.table = torch.nn.functional.pad(x.table, (0, 160)).contiguous()
        b = x.check()
        assert torch.allclose(a[0].float(), b[0].float(), rtol=2.0 ** -6, atol=2.0 ** -8) and torch.allclose(a[1], b[1], rtol=2.0 ** -18, atol=2.0 ** -18)


def test_scratch_that_cannot_be_had():
    """COFIE_ENOMEM, nothing launched, and the next call works."""
    from paper_2609_03675_gb300 import NGFFError, _abi
    lib = _abi.load()
    x = Shared(16, torch.bfloat16, (4, 2, 64), [1, 1], [3, 2], [40], [0, 2], 16)
    mask = torch.ones((2, 40), dtype=torch.uint8, device="cuda")
    for after, kw in ((0, {}), (0, {"prefix_mask": mask})):
        out = torch.full_like(x.q, 7.0)
        lib.cofie_ngff_debug_fail_alloc(after)
        try:
            with pytest.raises(NGFFError) as e:
                x.call(out=out, **kw)
            assert e.value.code == _abi.ENOMEM
        finally:
            lib.cofie_ngff_debug_fail_alloc(-1)
        torch.cuda.synchronize()
        assert bool((out == 7.0).all())
        x.compare(*x.call(**kw))


def test_two_caches_share_pages_and_streams():
    """Two handles over the same pages attend at the same time on streams of their own; a capture of one is replayed beside
    the other's calls."""
    from paper_2609_03675_gb300 import KVCache
    x = Shared("int8", torch.bfloat16, (8, 2, 128), [1] * 20, [9 + i for i in range(20)], [3000], [0, 20], 64)
    want = x.check()
    c = x.cache
    other = KVCache(c.n_pages, 64, 8, 2, 128, bits="int8", k_pages=c.k_pages, v_pages=c.v_pages, k_scales=c.k_scales, v_scales=c.v_scales)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    out = [torch.empty_like(x.q) for _ in range(2)]
    lse = [torch.empty(x.q.shape[:2], device="cuda") for _ in range(2)]
    args = dict(prefix_table=x.prefix_table, prefix_lengths=x.prefix_lens)
    other.attend_shared(x.q, x.table, x.lens, out=out[1], lse=lse[1], **args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other.attend_shared(x.q, x.table, x.lens, out=out[1], lse=lse[1], **args)
    for _ in range(30):
        with torch.cuda.stream(one):
            c.attend_shared(x.q, x.table, x.lens, out=out[0], lse=lse[0], **args)
        with torch.cuda.stream(two):
            graph.replay()
    torch.cuda.synchronize()
    for o, l in zip(out, lse):
        assert torch.equal(o, want[0]) and torch.equal(l, want[1])
    c.status()
    other.status()

"""Values near the ends of their type's range, behind weights that grow: few rows and many see the same numbers."""
import pytest
import torch

from tests import kv_bounds as B
from tests import test_gpu_kv_int8 as I

pytestmark = pytest.mark.gpu

SEQS = 304


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cache(bits, k, v, heads):
    """A cache of one sequence's tokens k, v [tokens, 1, d], and what it holds of them."""
    from paper_2609_03675_gb300 import KVCache
    m, _, d = k.shape
    pages = -(-m // 16)
    cache = KVCache(pages, 16, heads, 1, d, dtype=k.dtype, bits=bits)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
    cache.append(k.cuda(), v.cuda(), table, _ints(m), _ints(0, m))
    return cache, table, *cache.read(table, _ints(m), _ints(0, m), n_tokens=m)


def _many(cache, q, table, m, scale, shared=False):
    """q's rows for SEQS sequences of the same tokens, or groups of one sequence each behind them: so many that a CTA takes
    all of a row's tokens (where several do, each has a maximum of its own)."""
    n, seqs = len(q), SEQS
    every, lens, offsets = q.cuda().repeat(seqs, 1, 1), _ints(*[m] * seqs), torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * n
    tables = table.expand(seqs, -1).contiguous()
    if shared:
        out, lse = cache.attend_shared(every, tables[:, :1].contiguous(), torch.zeros_like(lens), offsets, prefix_table=tables, prefix_lengths=lens,
                                       groups=torch.arange(seqs + 1, dtype=torch.int32, device="cuda"), max_new=n, max_shared=n, scale=scale)
    else:
        out, lse = cache.attend(every, tables, lens, offsets, max_new=n, causal=False, scale=scale)
    cache.status()
    return out.view(seqs, *q.shape), lse.view(seqs, *q.shape[:2])


@pytest.mark.parametrize("bits", [16, "int8"])
@pytest.mark.parametrize("rows", [4, 16, 20, 32, 40, 200])
@pytest.mark.parametrize("shared", [False, True])
def test_large_values_of_heavier_tokens(bits, rows, shared):
    """bf16: the token that weighs most by 2^7, after others, has values of 2^121 to 2^127 (bytes: up to 127 2^120, so that
    two of them are in range together), alone or beside light ones of that size. The bound is that of values of common size."""
    d, m, size = 64, 130, 2.0 ** 121
    g = torch.Generator().manual_seed(rows)
    k = torch.zeros((m, 1, d), dtype=torch.bfloat16)
    for at, bit in ((3, 0.0), (70, 3.0), (129, 7.0)):  # powers of two; a tile each
        k[at, 0, 0] = bit
    k[[i for i in range(m) if i not in (3, 70, 129)], 0, 0] = -40.0
    v = torch.zeros((m, 1, d))
    v[3] = torch.randn((1, d), generator=g)
    v[70] = torch.randn((1, d), generator=g).clamp(-3, 3)
    v[129] = torch.randn((1, d), generator=g).clamp(-3, 3) * (8.0 if bits == 16 else 1.0)
    v = (v * size).to(torch.bfloat16)
    cache, table, kh, vh = _cache(bits, k, v, 4)
    q = torch.zeros((rows // 4, 4, d), dtype=torch.bfloat16)
    q[..., 0] = 1.0
    scale, n = 0.6931471805599453, rows // 4
    got = _many(cache, q, table, m, scale, shared)
    want = B.attend(q, kh, vh.double() / size, torch.ones((n, m), dtype=torch.bool), scale, torch.bfloat16)
    bad = B.exceeds(got[0].double() / size, got[1], want)
    assert not bool(bad[0].any()) and not bool(bad[1].any())


@pytest.mark.parametrize("rows", [4, 20, 40, 200])
@pytest.mark.parametrize("size", [2.0 ** -126, 2.0 ** -120, 2.0 ** -110, 2.0 ** 127])
def test_one_value_of_any_size(rows, size):
    """bf16: one cached token, whose weight is one: its values come out as they are."""
    d = 64
    v = (torch.arange(d).view(1, 1, d) % 2 * -2 + 1) * torch.tensor(size)
    v = (v * (1.0 + torch.arange(d).view(1, 1, d) / 128.0)).to(torch.bfloat16)
    cache, table, _, vh = _cache(16, torch.ones_like(v), v, 4)
    q = torch.ones((rows // 4, 4, d), dtype=torch.bfloat16, device="cuda")
    out, _ = cache.attend(q, table, _ints(1), _ints(0, rows // 4), max_new=rows // 4, causal=False)
    cache.status()
    assert torch.equal(out.cpu(), vh.cpu().expand_as(out))


@pytest.mark.parametrize("dtype", I.TYPES)
@pytest.mark.parametrize("rows", [20, 200])
def test_maxima_that_rise_from_tile_to_tile(dtype, rows):
    """Each tile's heaviest token is 0.25 to 40 powers of two above the one before."""
    d, m = 64, 64 * 12
    for rise in (0.25, 1.0, 3.0, 6.0, 7.0, 8.0, 9.0, 40.0):
        g = torch.Generator().manual_seed(int(rise))
        k = torch.zeros((m, 1, d))
        k[:, 0, 0] = -8.0 * torch.rand(m, generator=g)
        k[::64, 0, 0] = 0.0
        k[:, 0, 1] = (rise * (torch.arange(m) // 64))
        v = torch.randn((m, 1, d), generator=g)
        cache, table, kh, vh = _cache(16, k.to(dtype), v.to(dtype), 4)
        q = 0.02 * torch.randn((rows // 4, 4, d), generator=g).to(dtype)
        q[..., :2] = 1.0
        n, scale = rows // 4, 0.6931471805599453
        bad = B.exceeds(*_many(cache, q, table, m, scale), B.attend(q, kh, vh, torch.ones((n, m), dtype=torch.bool), scale, dtype))
        assert not bool(bad[0].any()) and not bool(bad[1].any()), rise


@pytest.mark.parametrize("rows", [4, 16, 20, 32, 40, 200])
def test_the_lightest_weights_that_fp16_holds(rows):
    """fp16, 16-bit pages: weights of 2^-32.375 of the largest, whose token has no value, so that the output is theirs. With
    the largest at 2^8 they are 2^-24.375, off by half a spacing of the smallest numbers at most: 2^-33 of the largest each.
    (With it at 2^7 they are under half of the smallest number, and nothing.)"""
    d, m, value = 64, 4096, 1024.0
    k, v = torch.zeros((m, 1, d)), torch.full((m, 1, d), value)
    k[0, 0, 0], v[0] = 32.375, 0.0
    cache, table, _, _ = _cache(16, k.half(), v.half(), 4)
    q = torch.zeros((rows // 4, 4, d), dtype=torch.float16)
    q[..., 0] = 1.0
    out, lse = _many(cache, q, table, m, 0.6931471805599453)
    want = (m - 1) * value * 2.0 ** -32.375
    assert bool(((out.double().cpu() - want).abs() <= (m - 1) * value * 2.0 ** -33 + 2.0 ** -11 * want).all())


@pytest.mark.parametrize("dtype", I.TYPES)
@pytest.mark.parametrize("rows", [20, 200])
@pytest.mark.parametrize("size", [1100.0, 1300.0, 1500.0, 1700.0])
def test_scores_that_fp32_rounds_by_sixteen(dtype, rows, size):
    """Scores of 1.1 to 2.7 10^8 powers of two, of which a weight may be 2^8 off: the outputs stay among the values."""
    d, m = 64, 700
    g = torch.Generator().manual_seed(int(size))
    k = size + torch.randint(-3, 4, (m, 1, d), generator=g).float()
    v = 1.0 + torch.rand((m, 1, d), generator=g)
    cache, table, _, _ = _cache(16, k.to(dtype), v.to(dtype), 4)
    q = (size + torch.randint(-3, 4, (rows // 4, 4, d), generator=g)).to(dtype)
    out, lse = _many(cache, q, table, m, 1.0)
    assert bool(torch.isfinite(lse).all()) and bool(((out >= 0.99) & (out <= 2.01)).all())

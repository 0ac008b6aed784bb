"""Long flat caches below one key. Each of the flat keys' weights is small beside the largest, together they are not:
sums must not lose them. There are more sequences than the GPU holds at a time (they share their pages), so that few CTAs
see a row: where many do, each has a maximum and sums of its own."""
import functools

import pytest
import torch

from tests import kv_bounds as B
from tests import kv_oracle as K

pytestmark = pytest.mark.gpu

SEQS, D, PAGE = 304, 64, 256


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@functools.lru_cache(maxsize=1)
def _run(dtype, bits, n, above, value, M=262144, H=2, seqs=SEQS):
    """(outputs, log-sum-exps) of n new tokens that pass their bounds; key 1000 lies `above` the others, its value is
    `value`, theirs are about 1."""
    from paper_2609_03675_gb300 import KVCache
    g = torch.Generator().manual_seed(n)
    cache = KVCache(M // PAGE, PAGE, H, 1, D, dtype=dtype, bits=bits)
    k = torch.zeros((M, 1, D), dtype=dtype)
    k[1000, 0, 0] = 15.0
    v = (1.0 + 0.25 * torch.randn((M, 1, D), generator=g)).to(dtype)
    v[1000] = value
    for x, pages, scales in ((k, cache.k_pages, cache.k_scales), (v, cache.v_pages, cache.v_scales)):
        if bits == 16:
            pages.copy_(x.view(M // PAGE, PAGE, 1, D).transpose(1, 2))
        else:
            b, w = K.pack(*K.quantise(x))
            pages.copy_(b.view(M // PAGE, PAGE, 1, D // 2).transpose(1, 2))
            scales.copy_(w.view(M // PAGE, PAGE, 1, D // 64).transpose(1, 2))
    if bits == 4:
        k, v = (K.unpack(*K.pack(*K.quantise(x)))[0] for x in (k, v))
    q = (0.5 * torch.randn((n, H, D), generator=g)).to(dtype)
    q[..., 0] = above * D ** 0.5 / 15.0
    table = torch.arange(M // PAGE, dtype=torch.int32, device="cuda").repeat(seqs, 1)
    lens = torch.full((seqs,), M, dtype=torch.int32, device="cuda")
    offsets = torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * n
    out, lse = cache.attend(q.cuda().repeat(seqs, 1, 1), table, lens, offsets, max_new=n)
    cache.status()
    seen = torch.arange(M)[None] <= (M - n + torch.arange(n))[:, None]
    chain = M // 8 if n * H <= 32 else 8192 if dtype == torch.float16 else 65536
    return B.exceeds(out.view(seqs, n, H, D), lse.view(seqs, n, H), B.attend(q, k, v, seen, D ** -0.5, dtype, chain))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("n", [1, 5, 17])
@pytest.mark.parametrize("above", [0.0, 12.0, 17.5])
def test_sum_of_the_weights(dtype, bits, n, above):
    assert not bool(_run(dtype, bits, n, above, 0.0)[1].any())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_sum_of_the_weights_of_a_million_tokens(dtype):
    """A lane of the kernel of few rows sums 1 in 64 of a CTA's tokens."""
    assert not bool(_run(dtype, 16, 1, 17.5, 0.0, 1 << 20, 1)[1].any())
    _run.cache_clear()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("n", [1, 5, 17])
def test_weights_that_fp16_holds(bits, n):
    """Rounded to fp16 a weight under 2^-25 is nothing; the key above has no value, so that the outputs are the others'."""
    assert not bool(_run(torch.float16, bits, n, 17.5, 0.0)[0].any())


@pytest.mark.parametrize("n", [1, 17])
def test_scores_of_millions_in_fp16(n):
    """fp32 rounds such scores by whole units; weights formed from them stay finite."""
    from paper_2609_03675_gb300 import KVCache
    m, d = 700, 128
    g = torch.Generator(device="cuda").manual_seed(n)
    x = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    cache = KVCache(44, 16, 4, 2, d, dtype=torch.float16)
    table = torch.arange(44, dtype=torch.int32, device="cuda").view(1, -1)
    lens, offsets = (torch.tensor(y, dtype=torch.int32, device="cuda") for y in ([m], [0, m]))
    k = (900.0 * x(m, 2, d) + 1500.0).half()
    cache.append(k, x(m, 2, d).half(), table, lens, offsets)
    q = (900.0 * x(n, 4, d) + 1500.0).half()
    out, lse = cache.attend(q, table, lens, torch.tensor([0, n], dtype=torch.int32, device="cuda"), max_new=n)
    cache.status()
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    assert float(lse.min()) > 1e7


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("n", [1, 17])
@pytest.mark.parametrize("above,value", [(0.0, 1.0), (12.0, 0.0), (14.3, 1.0), (17.5, 1.0)])
def test_outputs_of_long_sums(dtype, bits, n, above, value):
    """Values that all point one way, so that nothing of a sum cancels."""
    assert not bool(_run(dtype, bits, n, above, value)[0].any())


def test_outputs_of_sums_of_a_million_in_bf16():
    assert not bool(_run(torch.bfloat16, 16, 33, 15.0, 1.0, 1 << 20, 1)[0].any())
    _run.cache_clear()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [1, 5, 17])
@pytest.mark.parametrize("larger", [0, 1])
def test_values_of_which_one_group_is_larger(dtype, n, larger):
    """4-bit values of a head's two groups, one 1024 times the other's size: each against its own bound."""
    from paper_2609_03675_gb300 import KVCache
    seqs, m, h, d = SEQS, 262144, 2, 128
    g = torch.Generator().manual_seed(n)
    k = torch.zeros((m, 1, d), dtype=dtype)
    k[1000, 0, 0] = 15.0
    v = 1.0 + 0.25 * torch.randn((m, 1, d), generator=g)
    v[1000] = 0.0
    v[..., 64 * larger:64 * larger + 64] *= 1024.0
    cache = KVCache(m // PAGE, PAGE, h, 1, d, dtype=dtype, bits=4)
    held = []
    for x, pages, scales in ((k, cache.k_pages, cache.k_scales), (v.to(dtype), cache.v_pages, cache.v_scales)):
        b, w = K.pack(*K.quantise(x))
        pages.copy_(b.view(m // PAGE, PAGE, 1, d // 2).transpose(1, 2))
        scales.copy_(w.view(m // PAGE, PAGE, 1, d // 64).transpose(1, 2))
        held.append(K.unpack(b, w)[0])
    q = (0.5 * torch.randn((n, h, d), generator=g)).to(dtype)
    q[..., 0] = 17.5 * d ** 0.5 / 15.0
    table = torch.arange(m // PAGE, dtype=torch.int32, device="cuda").repeat(seqs, 1)
    lens = torch.full((seqs,), m, dtype=torch.int32, device="cuda")
    offsets = torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * n
    out, lse = cache.attend(q.cuda().repeat(seqs, 1, 1), table, lens, offsets, max_new=n)
    cache.status()
    seen = torch.arange(m)[None] <= (m - n + torch.arange(n))[:, None]
    chain = m // 8 if n * h <= 32 else 8192 if dtype == torch.float16 else 65536
    for part in (slice(0, 64), slice(64, 128)):
        want = B.attend(q, held[0], held[1][..., part], seen, d ** -0.5, dtype, chain)
        bad = B.exceeds(out.view(seqs, n, h, d)[..., part], lse.view(seqs, n, h), want)
        assert not bool(bad[0].any()) and not bool(bad[1].any()), part


@pytest.mark.parametrize("n", [1, 17])
@pytest.mark.parametrize("size", [2.0 ** -90, 2.0 ** -60, 2.0 ** 60, 2.0 ** 100, 2.0 ** 118])
def test_values_of_any_size_in_4_bits(n, size):
    """bf16 has the exponents of fp32: values near either end (not so near that their sums pass it)."""
    from paper_2609_03675_gb300 import KVCache
    m, h, d = 90, 2, 64
    g = torch.Generator().manual_seed(n)
    k = torch.randn((m, 1, d), generator=g).to(torch.bfloat16)
    v = (torch.randn((m, 1, d), generator=g).clamp(-4, 4) * size).to(torch.bfloat16)
    cache = KVCache(6, 16, h, 1, d, bits=4)
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(1, -1)
    lens, offsets = torch.tensor([m], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    cache.append(k.cuda(), v.cuda(), table, lens, torch.tensor([0, m], dtype=torch.int32, device="cuda"))
    q = (0.3 * torch.randn((n, h, d), generator=g)).to(torch.bfloat16)
    out, lse = cache.attend(q.cuda(), table, lens, offsets, max_new=n)
    cache.status()
    k, v = (K.unpack(*K.pack(*K.quantise(x)))[0] for x in (k, v))
    seen = torch.arange(m)[None] <= (m - n + torch.arange(n))[:, None]
    bad = B.exceeds(out.double() / size, lse, B.attend(q, k, v / size, seen, d ** -0.5, torch.bfloat16))
    assert not bool(bad[0].any()) and not bool(bad[1].any())


@pytest.mark.parametrize("dtype,m", [(torch.float16, 96000), (torch.bfloat16, 640000)])
@pytest.mark.parametrize("bits", [16, 4])
def test_outputs_of_long_sums_that_are_joined(dtype, m, bits):
    """A row's tokens lie with several CTAs, with each more of them than a sum holds."""
    bad = _run(dtype, bits, 17, 15.0, 1.0, m, 2, 20)
    assert not bool(bad[0].any()) and not bool(bad[1].any())
    _run.cache_clear()

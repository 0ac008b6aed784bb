"""Calls of the cache and of the rotary that leave something out, come after a close, or want a gradient."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _normal(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def test_read_with_offsets_wants_a_count():
    """Offsets lie on the device: how many rows they name is the caller's to say."""
    from paper_2609_03675_gb300 import KVCache
    cache = KVCache(4, 16, 2, 1, 64)
    table, lens, offsets = _ints(0, 1, 2, 3).view(2, 2), _ints(20, 5), _ints(0, 20, 25)
    k = _normal(25, 1, 64)
    cache.append(k, k, table, lens, offsets)
    with pytest.raises(ValueError, match="n_tokens"):
        cache.read(table, lens, offsets)
    out = torch.empty_like(k), torch.empty_like(k)
    for got in (cache.read(table, lens, offsets, n_tokens=25), cache.read(table, lens, offsets, out=out)):
        assert torch.equal(got[0], k) and torch.equal(got[1], k)
    last = cache.read(table, lens)  # without offsets one row each, the last
    assert torch.equal(last[0], k[[19, 24]])
    cache.status()


@pytest.mark.parametrize("bits", [16, 4])
def test_append_after_the_rotary_is_closed(bits):
    """Without its rotary a cache would store keys that are not rotated."""
    from paper_2609_03675_gb300 import KVCache, NGFFError, Rotary
    rotary = Rotary(64)
    cache = KVCache(2, 16, 2, 1, 64, bits=bits, rotary=rotary)
    table, lens, pos = _ints(0, 1).view(1, 2), _ints(1), _ints(5)
    k, q = _normal(1, 1, 64), _normal(1, 2, 64)
    cache.append(k, k, table, lens, positions=pos)
    before = cache.k_pages.clone()
    rotary.close()
    for kw in ({}, {"q": q}):
        with pytest.raises(ValueError, match="closed"):
            cache.append(_normal(1, 1, 64, seed=1), k, table, lens, positions=pos, **kw)
    assert torch.equal(cache.k_pages, before)
    with pytest.raises(NGFFError):
        rotary.apply(q, pos)
    cache.close()
    with pytest.raises(NGFFError):
        cache.attend(q, table, lens)


@pytest.mark.parametrize("n", [1, 40])
def test_a_mask_of_no_tokens_hides_them_all(n):
    """A cached token past the mask counts as masked."""
    from paper_2609_03675_gb300 import KVCache
    cache = KVCache(4, 16, 2, 1, 64)
    table, lens, offsets = _ints(0, 1, 2, 3).view(1, 4), _ints(50), _ints(0, 50)
    k = _normal(50, 1, 64)
    cache.append(k, k, table, lens, offsets)
    for dtype in (torch.uint8, torch.bool):
        for width in (0, 1):
            mask = torch.zeros((1, width), dtype=dtype, device="cuda")
            out, lse = cache.attend(_normal(n, 2, 64), table, lens, _ints(0, n), max_new=n, mask=mask)
            assert bool((out == 0).all()) and bool((lse == -float("inf")).all())
    cache.status()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_joins_autograd(layout):
    """Against the transposed rotation called by hand, which has tests of its own against the formula and differences."""
    from paper_2609_03675_gb300 import Rotary
    r = Rotary(64, rotary_dim=48, layout=layout, scaling="yarn", factor=2.0, original_len=4096)
    n = 37
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 91
    x, y = _normal(n, 6, 64, dtype=torch.float32).requires_grad_(), _normal(n, 2, 64, seed=1, dtype=torch.float32).requires_grad_()
    w, u = _normal(n, 6, 64, seed=2, dtype=torch.float32), _normal(n, 2, 64, seed=3, dtype=torch.float32)
    a, b = r.apply((x, y), pos)
    with torch.no_grad():
        plain = r.apply((x, y), pos)
        want = r.backward((w, u), pos)
    assert not plain[0].requires_grad and torch.equal(a, plain[0]) and torch.equal(b, plain[1])
    gx, gy = torch.autograd.grad((a, b), (x, y), (w, u))
    assert torch.equal(gx, want[0]) and torch.equal(gy, want[1])
    # a single tensor, a gradient without strides, another without its own
    r.apply(x, pos).sum().backward()
    assert torch.equal(x.grad, r.backward(torch.ones_like(w), pos)) and y.grad is None
    z = y.detach()
    one, _ = r.apply((x, z), pos)
    assert torch.equal(torch.autograd.grad(one, x, w)[0], want[0])
    # backward is linear too: its own gradient is apply
    g = w.clone().requires_grad_()
    back, = torch.autograd.grad(r.apply(x, pos), x, g, create_graph=True)
    assert torch.equal(torch.autograd.grad(back, g, x.detach())[0], plain[0])
    assert torch.equal(torch.autograd.grad(r.backward(g, pos), g, x.detach())[0], plain[0])
    with pytest.raises(ValueError, match="out does not go"):
        r.apply(x, pos, out=torch.empty_like(w))
    kept = r.apply(x, pos)
    pos += 1  # the gradient would be that of other positions
    with pytest.raises(RuntimeError, match="modified"):
        kept.sum().backward()


def test_a_cache_has_no_gradient():
    """Refused, not lost."""
    from paper_2609_03675_gb300 import KVCache, Rotary
    cache = KVCache(2, 16, 2, 1, 64, rotary=Rotary(64))
    table, lens, pos = _ints(0, 1).view(1, 2), _ints(1), _ints(5)
    k, v, q = _normal(1, 1, 64), _normal(1, 1, 64, seed=1), _normal(1, 2, 64, seed=2)
    for i in range(3):
        kvq = [x.clone().requires_grad_(i == j) for j, x in enumerate((k, v, q))]
        call = lambda: cache.append(kvq[0], kvq[1], table, lens, positions=pos, q=kvq[2])  # noqa: E731
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    p = q.clone().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        cache.attend(p, table, lens)
    with torch.no_grad():
        out, _ = cache.attend(p, table, lens)
    assert torch.equal(out, cache.attend(p.detach(), table, lens)[0]) and not out.requires_grad


def test_a_new_cache_is_ready_on_every_stream():
    """Its counters are cleared on the default stream, for which a stream of the caller's need not wait."""
    from paper_2609_03675_gb300 import KVCache
    k, v = (torch.zeros((64, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    KVCache(64, 16, 2, 1, 64, k_pages=k, v_pages=v)  # the library is loaded
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)  # a tenth of a second of the default stream
    cache = KVCache(64, 16, 2, 1, 64, k_pages=k, v_pages=v)
    assert torch.cuda.default_stream().query()
    side = torch.cuda.Stream()
    x, y, q = _normal(1000, 1, 64), _normal(1000, 1, 64, seed=1), _normal(1, 2, 64, seed=2)
    table, lens, offsets = torch.arange(64, dtype=torch.int32, device="cuda").view(1, -1), _ints(1000), _ints(0, 1000)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.append(x, y, table, lens, offsets)
        a = cache.attend(q, table, lens)
        b = cache.attend(q, table, lens)
        cache.status()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and bool(torch.isfinite(a[1]).all())


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("n", [1, 5, 90])
def test_outputs_in_the_queries_place(bits, n):
    """With the queries' strides; with others it is refused, as for rotated queries."""
    from paper_2609_03675_gb300 import KVCache, NGFFError
    h, kv, d = 8, 2, 64
    cache = KVCache(64, 64, h, kv, d, bits=bits)
    table, lens, offsets = torch.arange(64, dtype=torch.int32, device="cuda").view(1, -1), _ints(4000), _ints(0, 4000)
    cache.append(_normal(4000, kv, d), _normal(4000, kv, d, seed=1), table, lens, offsets)
    q = _normal(n, h, d, seed=2)
    want = cache.attend(q, table, lens, _ints(0, n), max_new=n)
    with pytest.raises(NGFFError, match="in place"):
        cache.attend(q, table, lens, _ints(0, n), max_new=n, out=q.view(-1).as_strided((n, h, d), (d, n * d, 1) if n > 1 else (h * d, 0, 1)))
    if n == 1:  # a stride that nothing is at
        other = q.clone()
        out, lse = cache.attend(other, table, lens, out=other.as_strided((1, h, d), (h * d + 64, d, 1)))
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    out, lse = cache.attend(q, table, lens, _ints(0, n), max_new=n, out=q)
    cache.status()
    assert out is q and torch.equal(out, want[0]) and torch.equal(lse, want[1])

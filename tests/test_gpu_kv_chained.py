"""Calls one behind the other, none of them waited for: each reads the lists, tables and masks that were written just before
it, not what its predecessor found at the same addresses."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.fixture(autouse=True)
def _no_cache_left():
    """A cache that an exception's frames still hold would be freed whenever they are collected: in a capture, perhaps."""
    gc.collect()
    yield
    gc.collect()


@pytest.mark.parametrize("bits", [16, "int8", 4])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("shared", [False, True])
def test_masks_and_tables_that_change_from_call_to_call(bits, new, shared):
    from paper_2609_03675_gb300 import KVCache
    S, m, h, kv, d, page = 6, 3000, 8, 2, 128, 32
    g = torch.Generator(device="cuda").manual_seed(new)
    pages = -(-m // page)
    cache = KVCache(S * pages, page, h, kv, d, bits=bits)
    k, v = (torch.randn((S * m, kv, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    full = torch.arange(S * pages, dtype=torch.int32, device="cuda").view(S, pages)
    lens = torch.full((S,), m, dtype=torch.int32, device="cuda")
    cache.append(k, v, full, lens, torch.arange(0, S * m + 1, m, dtype=torch.int32, device="cuda"))
    q = torch.randn((S * new, h, d), generator=g, device="cuda").to(torch.bfloat16)
    offsets = torch.arange(0, S * new + 1, new, dtype=torch.int32, device="cuda")
    frames = torch.arange(m, device="cuda") // 100
    sets = []
    for i in range(4):  # frames of which other tiles are left, and other orders of the pages
        seen = torch.rand((S, 30), generator=g, device="cuda") < (0.1, 0.5, 0.9, 0.3)[i]
        sets.append((seen[:, frames].to(torch.uint8).contiguous(), full[torch.randperm(S, generator=g, device="cuda")].contiguous()))
    mask, table = sets[0][0].clone(), sets[0][1].clone()
    none = torch.zeros_like(lens)

    def call(out, lse):
        if shared:
            cache.attend_shared(q, table[:, :1].contiguous(), none, offsets, prefix_table=table[:1], prefix_lengths=lens[:1], prefix_mask=mask,
                                max_new=new, out=out, lse=lse)
        else:
            cache.attend(q, table, lens, offsets, max_new=new, mask=mask, causal=False, out=out, lse=lse)

    want = []
    for x, y in sets:
        mask.copy_(x)
        table.copy_(y)
        torch.cuda.synchronize()
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        call(out, lse)
        torch.cuda.synchronize()
        want.append((out, lse))
    cache.status()
    order = [i % 4 if i % 7 else 3 - i % 4 for i in range(60)]
    got = [(torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")) for _ in order]
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    for i, (out, lse) in zip(order, got):
        mask.copy_(sets[i][0])
        table.copy_(sets[i][1])
        call(out, lse)
    torch.cuda.synchronize()
    for i, pair in zip(order, got):
        assert all(torch.equal(a, b) for a, b in zip(pair, want[i]))
    again = [torch.empty_like(q) for _ in order[:8]], [torch.empty(q.shape[:2], device="cuda") for _ in order[:8]]
    with torch.cuda.graph(graph, stream=stream):
        for i, out, lse in zip(order, *again):
            mask.copy_(sets[i][0])
            table.copy_(sets[i][1])
            call(out, lse)
    for _ in range(20):
        graph.replay()
    torch.cuda.synchronize()
    cache.status()
    for i, out, lse in zip(order, *again):
        assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])

"""Captured calls of the cache, launched after other calls on the same cache have needed more scratch."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("new", [1, 40])
def test_a_masked_call_captured_before_a_larger_one(bits, new):
    """The list of the mask's tiles grows with n_seqs x table_stride; a graph writes and reads the one that it was captured
    with. What is allocated after the growth would lie where a freed one had been, so it has to stay as it was."""
    from paper_2609_03675_gb300 import KVCache
    h, kv, d, page = 8, 2, 64, 16
    g = torch.Generator(device="cuda").manual_seed(bits + new)
    normal = lambda n, heads: torch.randn((n, heads, d), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    cache = KVCache(64, page, h, kv, d, bits=bits)
    table = torch.arange(64, dtype=torch.int32, device="cuda").view(2, 32)
    lens = torch.tensor([500, 130], dtype=torch.int32, device="cuda")
    whole = torch.tensor([0, 500, 630], dtype=torch.int32, device="cuda")
    cache.append(normal(630, kv), normal(630, kv), table, lens, whole)
    offsets = torch.tensor([0, new, 2 * new], dtype=torch.int32, device="cuda")
    q = normal(2 * new, h)
    mask = (torch.rand((2, 512), generator=g, device="cuda") < 0.1).to(torch.uint8)
    mask[0, 64:300] = 0
    out, lse = torch.empty_like(q), torch.empty((2 * new, h), device="cuda")

    def call():
        cache.attend(q, table, lens, offsets, max_new=new, mask=mask, out=out, lse=lse)

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    others, kept = [], []
    for seqs in (40, 300, 2000):  # larger and larger masked batches over the same pages
        many = table[:1].expand(seqs, -1).contiguous()
        for _ in range(2):
            cache.attend(normal(seqs, h), many, lens[:1].expand(seqs).contiguous(), mask=mask[:1].expand(seqs, -1).contiguous())
        others.append(KVCache(4, page, h, kv, d))  # its flags and counters, zero between calls
        kept.append(torch.full((1 << 16,), 7, dtype=torch.int32, device="cuda"))
    for _ in range(3):
        mask.copy_(torch.rand((2, 512), generator=g, device="cuda") < 0.1)  # read anew at each launch
        out.fill_(9.0)
        lse.fill_(9.0)
        graph.replay()
        got = out.clone(), lse.clone()
        call()
        assert torch.equal(got[0], out) and torch.equal(got[1], lse)
        assert bool(torch.isfinite(out.float()).all())
    cache.status()
    for x in others:
        x.status()
    assert all(bool((x == 7).all()) for x in kept)

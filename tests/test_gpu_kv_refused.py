"""A call that is refused has launched nothing: neither into the stream nor into a graph that is being captured. A prefix
table with a page out of range tells: a kernel that had run would have reported it."""
import gc

import pytest
import torch

from tests.test_gpu_kv_shared import Shared

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


def _masked(new):
    """Room for the rows is there, and for the prefix's mask; that for the own tokens' mask is not."""
    x = Shared(16, torch.bfloat16, (4, 2, 64), [new, new], [new + 2, new], [300], [0, 2], 16)
    prefix_mask = torch.ones((2, 300), dtype=torch.uint8, device="cuda")
    own_mask = torch.ones((2, new + 2), dtype=torch.uint8, device="cuda")
    x.call(prefix_mask=prefix_mask)
    x.cache.status()
    bad = x.prefix_table.clone()
    bad[0, 2] = x.cache.n_pages
    out, lse = torch.full_like(x.q, 7.0), torch.full(x.q.shape[:2], 7.0, device="cuda")
    return x, dict(prefix_table=bad, prefix_mask=prefix_mask, mask=own_mask, out=out, lse=lse)


def _untouched(x, kw):
    torch.cuda.synchronize()
    x.cache.status()
    assert bool((kw["out"] == 7.0).all()) and bool((kw["lse"] == 7.0).all())
    kw = dict(kw, prefix_table=x.prefix_table)
    x.call(**kw)
    x.cache.status()
    x.compare(kw["out"], kw["lse"])


@pytest.mark.parametrize("new", [1, 40])
def test_no_memory_for_the_own_mask(new):
    from paper_2609_03675_gb300 import NGFFError, _abi
    x, kw = _masked(new)
    lib = _abi.load()
    lib.cofie_ngff_debug_fail_alloc(0)
    try:
        with pytest.raises(NGFFError) as e:
            x.call(**kw)
        assert e.value.code == _abi.ENOMEM
    finally:
        lib.cofie_ngff_debug_fail_alloc(-1)
    _untouched(x, kw)


@pytest.mark.parametrize("new", [1, 40])
def test_growth_for_the_own_mask_in_a_capture(new):
    from paper_2609_03675_gb300 import NGFFError
    x, kw = _masked(new)
    torch.cuda.synchronize()
    mark = torch.zeros(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mark += 1
        with pytest.raises(NGFFError, match="capture"):
            x.call(**kw)
    graph.replay()
    torch.cuda.synchronize()
    assert float(mark) == 1.0
    _untouched(x, kw)


@pytest.mark.parametrize("value", [-1, 1 << 32, 1.5, None])
def test_hints_that_are_no_counts(value):
    x = Shared(16, torch.bfloat16, (4, 2, 64), [1, 2], [3, 2], [40], [0, 2], 16)
    with pytest.raises(ValueError, match="max_shared"):
        x.call(max_shared=value)
    with pytest.raises(ValueError, match="max_new"):
        x.call(max_new=value)
    with pytest.raises(ValueError, match="max_new"):
        x.cache.attend(x.q, x.table, x.lens, x.offsets, max_new=value)
    x.check()

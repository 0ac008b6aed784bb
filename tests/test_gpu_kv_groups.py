"""Many groups, many sequences, and how far a NaN reaches."""
import math

import pytest
import torch

from tests import kv_bounds as B
from tests.test_gpu_kv_shared import BITS, Shared, _ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("new", [1, 6, 20])
def test_more_groups_than_are_kept_at_hand(bits, new):
    """300 groups of one or two sequences, some without a prefix, masked (one list of tiles each) and not."""
    g = torch.Generator().manual_seed(new)
    sizes = [1 + i % 2 for i in range(300)]
    ends = torch.tensor([0] + sizes).cumsum(0).tolist()
    S, prefixes = ends[-1], [(37 * i) % 200 if i % 7 else 0 for i in range(300)]
    own = [new + i % 5 for i in range(S)]
    pm = torch.rand((S, 200), generator=g) < 0.3
    pm[5] = False
    for mask in (None, pm):
        x = Shared(bits, torch.bfloat16, (8, 2, 64), [new] * S, own, prefixes, ends, 16, prefix_mask=mask)
        x.check()


@pytest.mark.parametrize("new", [1, 2])
def test_more_masked_sequences_than_a_grid_has_rows(new):
    """70000 sequences, each with evidence of its own."""
    from paper_2609_03675_gb300 import KVCache
    S, p, h, d, page = 70000, 130, 2, 64, 16
    g = torch.Generator(device="cuda").manual_seed(new)
    pages = -(-p // page)
    cache = KVCache(pages + 1, page, h, 1, d)
    k, v = (torch.randn((p, 1, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
    cache.append(k, v, table, _ints(p), _ints(0, p))
    own = torch.full((S, 1), pages, dtype=torch.int32, device="cuda")
    cache.append(k[:2], v[:2], own[:1], _ints(2), _ints(0, 2))
    q = torch.randn((S * new, h, d), generator=g, device="cuda").to(torch.bfloat16)
    mask = torch.rand((S, p), generator=g, device="cuda") < 0.1
    mask[65534:65540, 64:] = False
    offsets = torch.arange(0, S * new + 1, new, dtype=torch.int32, device="cuda")
    out, lse = cache.attend_shared(q, own, torch.full((S,), new, dtype=torch.int32, device="cuda"), offsets, prefix_table=table, prefix_lengths=_ints(p),
                                   prefix_mask=mask, max_new=new)
    cache.status()
    for s in (0, 1, 255, 65534, 65535, 65536, 65537, 69999):
        seen = torch.cat([mask[s][None].expand(new, -1).cpu(), torch.ones((new, new), dtype=torch.bool).tril()], 1)
        rows = slice(s * new, s * new + new)
        want = B.attend(q[rows], torch.cat([k, k[:new]]), torch.cat([v, v[:new]]), seen, d ** -0.5, torch.bfloat16)
        bad = B.exceeds(out[rows], lse[rows], want)
        assert not bool(bad[0].any()) and not bool(bad[1].any()), s


@pytest.mark.parametrize("new", [1, 3, 20])
@pytest.mark.parametrize("masked", [False, True])
def test_how_far_a_nan_reaches(new, masked):
    """A NaN among the values of a prefix that one of its sequences sees: rows of the group may have it, rows of other groups
    do not, and log-sum-exps are everybody's own. Where none of the group sees it, nobody has it. An infinity among the keys
    that nobody sees does not matter either."""
    S, groups, prefixes = 4, [0, 2, 4], [300, 300]
    mask = torch.ones((S, 300), dtype=torch.bool)
    mask[0, 100] = masked
    mask[1:, 100] = False
    x = Shared(16, torch.bfloat16, (8, 2, 64), [new] * S, [new + 2] * S, prefixes, groups, 64, prefix_mask=mask)
    clean = x.call()
    page = int(x.prefix_table[0, 1])
    x.cache.v_pages[page, :, 100 % 64] = math.nan
    if not masked:
        x.cache.k_pages[page, :, 100 % 64] = math.inf
        x.check()
        return
    out, lse = x.call()
    x.cache.status()
    of = torch.arange(S).repeat_interleave(new)
    assert bool(torch.isnan(out[of == 0]).all())
    assert torch.equal(out[of >= 2], clean[0][of >= 2]) and torch.equal(lse, clean[1])

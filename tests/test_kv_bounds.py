"""The bounds that the GPU tests of attention hold the kernels to are close enough to notice one token too few."""
import pytest
import torch

from tests import kv_bounds as B
from tests import kv_oracle as K


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("h,kv,d", [(8, 2, 128), (4, 2, 64)])
def test_a_missing_token_is_noticed(dtype, bits, h, kv, d):
    m = 1111
    g = torch.Generator().manual_seed(d + bits)
    k = (torch.randn((m, kv, d), generator=g) * torch.exp(0.3 * torch.randn((kv, d), generator=g))).to(dtype)
    v = torch.randn((m, kv, d), generator=g).to(dtype)
    q = (1.5 * torch.randn((1, h, d), generator=g)).to(dtype)
    if bits == 4:
        k, v = (K.unpack(*K.pack(*K.quantise(x)))[0] for x in (k, v))
    all_of = torch.ones((1, m), dtype=torch.bool)
    want = B.attend(q, k, v, all_of, d ** -0.5, dtype)
    assert not any(bool(x.any()) for x in B.exceeds(want[0], want[1], want))
    for gone in (slice(m - 1, m), slice(0, 1), slice(500, 501), slice(m - 32, m)):
        seen = all_of.clone()
        seen[0, gone] = False
        out, lse, _, _ = B.attend(q, k, v, seen, d ** -0.5, dtype)
        outs, sums = B.exceeds(out, lse, want)
        # a single token's share of a row may be under its bound by chance; not of every row
        assert bool(sums.any()), gone
        if gone == slice(m - 32, m):
            assert bool(sums.all()) and float(outs.float().mean()) > 0.3


def test_rows_that_see_nothing():
    q, k = torch.ones((1, 1, 64)), torch.ones((3, 1, 64))
    want = B.attend(q, k, k, torch.zeros((1, 3), dtype=torch.bool), 0.125, torch.bfloat16)
    zero, none = torch.zeros((1, 1, 64)), torch.full((1, 1), -float("inf"))
    assert not any(bool(x.any()) for x in B.exceeds(zero, none, want))
    assert bool(B.exceeds(zero + 1, none, want)[0].all()) and bool(B.exceeds(zero, none * 0, want)[1].all())

"""4-bit codes of rotated keys, which are fp32 numbers: the nearest code, where a quotient lies just under a half.

At position 0 a key is only multiplied, by yarn's m, and a product of two numbers is rounded once, here as there. With
m = 1.25 - 2^-23, 12 m is at most 15, so a group with that extreme has scale 1, and 2 m, 6 m, 10 m lie a few units in the
last place under 2.5, 7.5 and 12.5."""
import math

import pytest
import torch

from tests import kv_oracle as K

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


GROUPS = [[12.0, 2.0, 6.0, 10.0], [6.0, -6.0, 2.0, -2.0], [2.0, -10.0, -6.0, -2.0], [-12.0, -2.0, -6.0, -10.0], [12.0, 0.4, -0.0, 3.0],
          [10.0, -2.0, 6.0]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,rd,layout,start", [(128, 128, "half", 0), (128, 128, "interleaved", 0), (64, 64, "half", 0), (64, 64, "half", 1),
                                               (64, 32, "interleaved", 0), (128, 96, "half", 0)])
def test_quotients_just_under_a_half(dtype, d, rd, layout, start):
    from paper_2609_03675_gb300 import KVCache, Rotary
    m = 1.25 - 2.0 ** -23
    rotary = Rotary(d, rotary_dim=rd, layout=layout, scaling="yarn", factor=math.exp(10 * (m - 1)), original_len=4096)
    rows = []
    for p in range(-9, 10):  # the same at other scales
        for values in GROUPS:
            x = torch.zeros(d)
            for g in range(d // 64):  # an element every third, over both halves of the group
                for i, y in enumerate(values):
                    x[64 * g + (17 * i + 5 * g) % 64] = y * 2.0 ** p
            rows.append(x)
    flat = torch.zeros(len(rows) * d + 1, dtype=dtype)
    flat[start:start + len(rows) * d] = torch.cat(rows).to(dtype)
    k = flat.cuda()[start:start + len(rows) * d].view(-1, 1, d)  # from 1: rows that allow no wide loads
    n = k.shape[0]
    cache = KVCache(n, 16, 1, 1, d, dtype=dtype, bits=4, rotary=rotary)
    table = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous()
    ones = torch.ones(n, dtype=torch.int32, device="cuda")
    cache.append(k, k, table, ones, positions=torch.zeros(n, dtype=torch.int32, device="cuda"))
    cache.status()
    turned = k.cpu().float()
    turned[..., :rd] *= torch.tensor(m, dtype=torch.float32)
    for x, pages, scales in ((turned, cache.k_pages, cache.k_scales), (k.cpu().float(), cache.v_pages, cache.v_scales)):
        b, w = K.pack(*K.quantise(x))
        assert torch.equal(scales[:, :, 0].cpu(), w)
        assert torch.equal(pages[:, :, 0].cpu(), b)


def test_codes_of_rotated_keys_are_the_nearest():
    """Keys at every position: what is read back is within half a step of the rotated key, up to what fp32 costs it."""
    from paper_2609_03675_gb300 import KVCache, Rotary
    n, kv, d = 4096, 4, 128
    rotary = Rotary(d, base=1e6)
    g = torch.Generator().manual_seed(1)
    k = (torch.randn((n, kv, d), generator=g) * torch.exp(0.3 * torch.randn((kv, d), generator=g))).half().cuda()
    pos = torch.randint(0, 131072, (n,), generator=g).to(torch.int32).cuda()
    cache = KVCache(n // 64, 64, kv, kv, d, dtype=torch.float16, bits=4, rotary=rotary)
    table = torch.arange(n // 64, dtype=torch.int32, device="cuda").view(1, -1)
    lens, offsets = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    cache.append(k, k, table, lens, offsets, positions=pos)
    b, w = cache.k_pages.transpose(1, 2).reshape(n, kv, d // 2), cache.k_scales.transpose(1, 2).reshape(n, kv, d // 64)
    got, step = K.unpack(b, w)
    freq, m = K.frequencies(d, 1e6)
    want, slack = K.rotate(k, pos, freq, m, "half")
    # the codes' range covers the values to within half a step, the zero point being rounded: 15 s >= hi - lo
    assert bool(((got - want).abs() <= 0.5 * step + slack).all())

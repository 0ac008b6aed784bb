"""Bytes of keys that are rotated with an amplitude."""
import pytest
import torch

from tests import kv_oracle as K
from tests import test_gpu_kv_int8 as I

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("dtype", I.TYPES)
@pytest.mark.parametrize("factor", [6.5, 13.0])
@pytest.mark.parametrize("d,rd,layout", [(128, 128, "half"), (64, 48, "interleaved"), (128, 64, "half")])
def test_bytes_of_keys_with_an_amplitude_are_the_nearest(dtype, factor, d, rd, layout):
    """8 million keys, scaled by YARN with factors whose amplitudes 0.1 ln(factor) + 1 are far from fp32 numbers (2^-24 of
    their size and less): the bytes of the keys turned in 64 bits. (With the amplitude rounded to fp32, a byte of u steps is
    the neighbour with a probability of up to 5e-8 u: ten or so of these. The scale is that of fp32 numbers: groups whose largest
    is 1e-6 of its size or less from where it changes are left out.)"""
    from paper_2609_03675_gb300 import Rotary
    n, kv, page = 8192000 // d // 8, 8, 64
    g = torch.Generator().manual_seed(d + rd)
    k = (torch.randn((n, kv, d), generator=g) * torch.exp(0.3 * torch.randn((kv, d), generator=g))).to(dtype)
    pos = torch.randint(0, 131072, (n,), generator=g).to(torch.int32)
    rotary = Rotary(d, rotary_dim=rd, layout=layout, base=1e6, scaling="yarn", factor=factor, original_len=8192.0)
    cache = I.make(-(-n // page), page, kv, kv, d, dtype, rotary)
    table = torch.arange(-(-n // page), dtype=torch.int32, device="cuda").view(1, -1)
    dev = k.cuda()
    cache.append(dev, dev, table, I._ints(n), I._ints(0, n), positions=pos.cuda())
    got, _ = cache.read(table, I._ints(n), I._ints(0, n), n_tokens=n)
    cache.status()
    freq, m = K.frequencies(rd, 1e6, "yarn", factor, 8192.0)
    want, _ = K.rotate(k, pos, freq, m, layout)
    ratio = want.unflatten(-1, (-1, 64)).abs().amax(-1) / 127.0
    border = (torch.log2(ratio) - torch.round(torch.log2(ratio))).abs() < 2e-6
    wrong = (got.double().cpu() != I.numbers(*I.quantise(want, dtype))).unflatten(-1, (-1, 64)) & ~border[..., None]
    assert int(wrong.sum()) == 0, int(wrong.sum())

"""Where the count of rows decides how 4-bit numbers past fp16's range are seen, with a shared prefix and without."""
import pytest
import torch

from tests import kv_oracle as K

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("rows", [4, 16, 20, 32, 36])
@pytest.mark.parametrize("way", ["attend", "prefix", "own"])
def test_codes_past_fp16(rows, way):
    """Two tokens, whose weights are 2^-20 and nearly one; the light one's values are 15 2^13, infinite as fp16 numbers. Up to
    32 rows (16 with prefixes) the output has 2^-20 of them, else it is infinite; cofie_kv_read has them infinite."""
    from paper_2609_03675_gb300 import KVCache
    d, n = 64, rows // 4
    cache = KVCache(2, 16, 4, 1, d, dtype=torch.float16, bits=4)
    k, v = torch.zeros((2, 1, d)), torch.zeros((2, 1, d))
    k[1, 0, 0] = 15.0
    v[0], v[1] = 15.0 * 8192, 15.0 / 32  # codes hold both exactly
    for x, pages, scales in ((k, cache.k_pages, cache.k_scales), (v, cache.v_pages, cache.v_scales)):
        b, w = K.pack(*K.quantise(x))
        pages[0, 0, :2], scales[0, 0, :2] = b[:, 0].cuda(), w[:, 0].cuda()
    table = _ints(0).view(1, 1)
    q = torch.zeros((n, 4, d), dtype=torch.float16, device="cuda")
    q[..., 0] = 20.0 / 15.0
    scale, two, none = 0.6931471805599453, _ints(2), _ints(0)
    if way == "attend":
        out, _ = cache.attend(q, table, two, _ints(0, n), max_new=n, causal=False, scale=scale)
    elif way == "prefix":
        out, _ = cache.attend_shared(q, table, none, _ints(0, n), prefix_table=table, prefix_lengths=two, max_new=n, scale=scale)
    else:
        out, _ = cache.attend_shared(q, table, two, _ints(0, n), prefix_table=table, prefix_lengths=none, max_new=n, causal=False, scale=scale)
    held = cache.read(table, two, _ints(0, 2), n_tokens=2)[1]
    cache.status()
    assert bool(torch.isinf(held[0]).all()) and bool((held[1] == 15.0 / 32).all())
    if rows <= (32 if way == "attend" else 16):
        # to a rounding; the score is a rounding of q off, 20 2^-11 powers of two, and the light token's 0.1172 by 1 % with it
        want = (2.0 ** -20 * 122880.0 + 15.0 / 32) / (1 + 2.0 ** -20)
        assert bool(((out.double() - want).abs() <= 2.0 ** -11 * want + 0.1172 * 0.01).all())
    else:
        assert bool(torch.isinf(out).all())

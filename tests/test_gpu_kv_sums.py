"""Sums of very many light tokens behind one heavy one: the matrix units cut each product off at about 2^-24 of the sum that it
is added to, so no sum of fp16 outputs takes more than 8192 tokens, of few rows or many."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("bits", [16, "int8", 4])
@pytest.mark.parametrize("rows", [1, 8, 16, 20])
@pytest.mark.parametrize("shared", [False, True])
def test_light_tokens_are_not_cut_off(bits, rows, shared):
    """All values are one number, so that the output is it, whatever the weights: 524288 tokens 2^-23 to 2^-26 of the first.
    304 rows' blocks, so that a CTA has all tokens of one, and a warp of the kernel of few rows an eighth of them: 65536, which
    in one sum came out up to 2^-9 low. The bound: 8192 2^-24 of the number, and its rounding to fp16, 2^-11 of it."""
    from paper_2609_03675_gb300 import KVCache
    m, d, page, seqs = 524288, 64, 256, 304
    cache = KVCache(m // page, page, rows, 1, d, dtype=torch.float16, bits=bits)
    table = torch.arange(m // page, dtype=torch.int32, device="cuda").view(1, -1)
    lens, offsets = torch.tensor([m], dtype=torch.int32, device="cuda"), torch.tensor([0, m], dtype=torch.int32, device="cuda")
    v = torch.ones((m, 1, d), dtype=torch.float16, device="cuda")
    k = torch.zeros_like(v)
    k[0, 0, 0] = 15.0
    cache.append(k, v, table, lens, offsets)
    number = cache.read(table, lens, offsets, n_tokens=m)[1].double()
    assert bool((number == number[0, 0, 0]).all())
    number = float(number[0, 0, 0])
    worst = 0.0
    for below in (23.0, 24.0, 24.5, 25.0, 25.5, 26.0):
        q = torch.zeros((seqs, rows, d), dtype=torch.float16, device="cuda")
        q[..., 0] = below / 15.0
        every, length = table.expand(seqs, -1).contiguous(), lens.expand(seqs).contiguous()
        if shared:
            out, _ = cache.attend_shared(q, every[:, :1].contiguous(), torch.zeros_like(length), prefix_table=every, prefix_lengths=length,
                                         groups=torch.arange(seqs + 1, dtype=torch.int32, device="cuda"), max_shared=1, scale=0.6931471805599453)
        else:
            out, _ = cache.attend(q, every, length, scale=0.6931471805599453)
        cache.status()
        worst = max(worst, float((out.double() / number - 1.0).abs().max()))
    assert worst <= 8192 * 2.0 ** -24 + 2.0 ** -11, worst

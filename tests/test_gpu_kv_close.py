"""Attention over the cache held to bounds that notice one token too few or too many, with 4-bit pages as with 16-bit
ones; masks in every form that their rows' alignment gives; batches of more sequences than a CTA keeps."""
import pytest
import torch

from tests import kv_bounds as B
from tests.test_gpu_kv import BATCHES, HEADS, _cache, _fill, _offsets, _table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _check(cache, q, table, lengths, new, held, mask=None, causal=True, max_new=None, which=None):
    """which: the sequences that are compared."""
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out, lse = cache.attend(q, table, lens, _offsets(new), max_new=max(new) if max_new is None else max_new, mask=mask, causal=causal)
    cache.status()
    out, lse, t = out.cpu(), lse.cpu(), 0
    for s, (n, m) in enumerate(zip(new, lengths)):
        seen = torch.ones((n, m), dtype=torch.bool)
        if causal:
            seen = torch.arange(m)[None] <= (m - n + torch.arange(n))[:, None]
        if mask is not None:
            w = torch.zeros(m, dtype=torch.bool)
            w[:mask.shape[1]] = mask[s, :m].cpu() != 0
            seen = seen & w[None]
        if n and (which is None or s in which):
            bad = B.exceeds(out[t:t + n], lse[t:t + n], B.attend(q[t:t + n], held[s][0], held[s][1], seen, cache.head_dim ** -0.5, q.dtype))
            assert not bool(bad[0].any()), (s, "out")
            assert not bool(bad[1].any()), (s, "lse")
        t += n


@pytest.mark.parametrize("bits,dtype", [(4, torch.bfloat16), (4, torch.float16), (16, torch.float16)])
@pytest.mark.parametrize("new,lengths,page", BATCHES + [([1, 40], [3000, 2000], 64)])
def test_every_token_counts(bits, dtype, new, lengths, page):
    for i, (h, kv, d) in enumerate(HEADS):
        g = torch.Generator().manual_seed(7 * i + page)
        table, n_pages = _table(lengths, page, 1, g)
        cache = _cache(n_pages, page, h, kv, d, dtype, bits)
        held = _fill(cache, table, lengths, g)
        q = (1.5 * torch.randn((sum(new), h, d), generator=g)).to(dtype).cuda()
        _check(cache, q, table, lengths, new, held)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("new", [[1, 2, 1], [40, 3, 30]])
@pytest.mark.parametrize("width,shift", [(704, 0), (696, 0), (700, 0), (697, 0), (704, 4), (704, 1), (704, 2), (16, 0), (3, 0)])
def test_masks_of_every_alignment(bits, new, width, shift):
    """Rows of 16, 8, 4 and 1 bytes' alignment, from addresses of 16, 4 and 1; what is masked holds NaN."""
    h, kv, d, page, lengths = 8, 2, 64, 32, [701, 64, 333]
    g = torch.Generator().manual_seed(width + shift)
    table, n_pages = _table(lengths, page, 1, g)
    rows = torch.rand((3, width), generator=g) < 0.4
    rows[0, 128:640] = False
    rows[0, 511:512] = True  # the last place of a tile, alone
    rows[2, :width // 2] = False
    flat = torch.zeros(3 * width + shift, dtype=torch.uint8, device="cuda")
    mask = flat[shift:].view(3, width)
    mask.copy_(rows)
    seen = torch.zeros((3, 701), dtype=torch.bool)
    seen[:, :min(width, 701)] = rows[:, :701]
    cache = _cache(n_pages, page, h, kv, d, torch.bfloat16, bits)
    held = _fill(cache, table, lengths, g, seen)
    q = torch.randn((sum(new), h, d), generator=g).to(torch.bfloat16).cuda()
    for causal in (True, False):
        _check(cache, q, table, lengths, new, held, mask=mask, causal=causal)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("width", [140000, 140001])
def test_masks_past_a_thousand_tiles(bits, width):
    """1024 tiles of a mask are looked at at a time: frames kept in the first, the second and the third thousand."""
    h, kv, d, page, m = 4, 1, 64, 128, 140000
    g = torch.Generator().manual_seed(width)
    table, n_pages = _table([m], page, 1, g)
    mask = torch.zeros((1, width), dtype=torch.uint8)
    for first, last in ((0, 3), (65500, 65700), (100000, 100001), (131000, 131100), (139990, 140000)):
        mask[0, first:last] = 1
    cache = _cache(n_pages, page, h, kv, d, torch.bfloat16, bits)
    held = _fill(cache, table, [m], g, mask[:, :m] != 0)
    for n in (1, 20):
        q = torch.randn((n, h, d), generator=g).to(torch.bfloat16).cuda()
        _check(cache, q, table, [m], [n], held, mask=mask.cuda())


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("most", [2, 40])
@pytest.mark.parametrize("seqs", [300, 1500])
def test_more_sequences_than_are_kept(bits, most, seqs):
    """A CTA keeps 256 sequences' places (and 1024 sequences' offsets when it appends), its threads take several each."""
    from paper_2609_03675_gb300 import KVCache, Rotary
    h, kv, d, page = 2, 1, 64, 16
    g = torch.Generator().manual_seed(seqs + most)
    new = torch.randint(0, most + 1, (seqs,), generator=g).tolist()
    lengths = [a + b for a, b in zip(new, torch.randint(0, 60, (seqs,), generator=g).tolist())]
    table, n_pages = _table(lengths, page, 1, g)
    rotary = Rotary(d)
    cache, plain = (KVCache(n_pages, page, h, kv, d, bits=bits, rotary=rotary) for _ in range(2))
    n = sum(lengths)
    x = torch.randn((n, 2 * kv, d), generator=g).to(torch.bfloat16).cuda()
    pos = torch.randint(0, 5000, (n,), generator=g).to(torch.int32).cuda()
    lens, whole = torch.tensor(lengths, dtype=torch.int32, device="cuda"), _offsets(lengths)
    cache.append(x[:, :1], x[:, 1:], table, lens, whole, positions=pos)
    k, v = cache.read(table, lens, whole, n_tokens=n)
    # token by token into the places, by calls of up to 200 sequences each
    starts = whole.tolist()
    for a in range(0, seqs, 200):
        b = min(seqs, a + 200)
        i, j = starts[a], starts[b]
        plain.append(x[i:j, :1], x[i:j, 1:], table[a:b].contiguous(), lens[a:b].contiguous(), (whole[a:b + 1] - i).contiguous(), positions=pos[i:j].contiguous())
    for y, z in ((cache.k_pages, plain.k_pages), (cache.v_pages, plain.v_pages), (cache.k_scales, plain.k_scales), (cache.v_scales, plain.v_scales)):
        assert y is None or torch.equal(y, z)
    k, v = k.cpu(), v.cpu()
    held = [(k[i:j], v[i:j], None) for i, j in zip(starts, starts[1:])]
    q = torch.randn((sum(new), h, d), generator=g).to(torch.bfloat16).cuda()
    which = set(range(0, seqs, 7)) | {seqs - 1, 255, 256, 257} | {i for i, a in enumerate(new) if a == most}
    _check(cache, q, table, lengths, new, held, which=which)
    mask = torch.rand((seqs, max(lengths)), generator=g) < 0.5
    _check(cache, q, table, lengths, new, held, mask=mask.cuda(), which=which)

"""Rotary positions against their definition in 64 bits: layouts, parts of the
head, scalings, axes, types, strides, odd sizes, in place, and the gradient
against the formula and against differences."""
import math

import pytest
import torch

from tests import kv_oracle as K

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _inputs(n, h, d, dtype, seed, furthest=131072, axes=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, h, d), generator=g, device="cuda").to(dtype)
    pos = torch.randint(0, furthest, (axes, n), generator=g, device="cuda", dtype=torch.int32)
    return x, pos


def _check(y, x, pos, freq, m, layout, axes=None, back=False, label=""):
    want, slack = K.rotate(x, pos, freq, m, layout, axes, back)
    bound = slack + K.UNIT[y.dtype] * want.abs() + (2.0 ** -25 if y.dtype == torch.float16 else 0.0)
    # a value that passes through is the same
    bound = torch.where(slack == 0, torch.zeros_like(bound), bound)
    err = (y.double().cpu() - want).abs()
    assert bool((err <= bound).all()), (label, float((err - bound).max()))


CASES = [
    # tokens, heads, head_dim, rotary_dim, layout, dtype
    (1, 1, 2, 2, "half", torch.float32),
    (1, 32, 128, 128, "half", torch.bfloat16),
    (3, 5, 64, 64, "interleaved", torch.float16),
    (17, 3, 80, 24, "half", torch.bfloat16),
    (17, 3, 80, 24, "interleaved", torch.float32),
    (5, 7, 128, 96, "interleaved", torch.bfloat16),
    (9, 2, 74, 14, "half", torch.float16),
    (9, 2, 74, 6, "interleaved", torch.bfloat16),
    (33, 1, 256, 256, "half", torch.float32),
    (2500, 3, 64, 32, "half", torch.bfloat16),
    (2433, 4, 128, 128, "interleaved", torch.float16),
]


@pytest.mark.parametrize("n,h,d,rd,layout,dtype", CASES)
def test_rotation_and_gradient(n, h, d, rd, layout, dtype):
    from paper_2609_03675_gb300 import Rotary
    x, pos = _inputs(n, h, d, dtype, seed=n + d)
    r = Rotary(d, rotary_dim=rd, layout=layout, base=10000.0)
    freq, m = K.frequencies(rd, 10000.0)
    _check(r.apply(x, pos[0]), x, pos, freq, m, layout, label="forward")
    _check(r.backward(x, pos[0]), x, pos, freq, m, layout, back=True, label="gradient")


@pytest.mark.parametrize("scaling,factor", [("linear", 4.0), ("base", 8.0), ("yarn", 4.0), ("yarn", 1.0)])
def test_scalings_at_far_positions(scaling, factor):
    from paper_2609_03675_gb300 import Rotary
    x, _ = _inputs(64, 4, 128, torch.float32, seed=3)
    # up to 2^31 - 1, and negative ones; fp64 forms the oracle's angles to 2^31 2^-53 there
    pos = torch.tensor([0, 1, 2, 3, 1000, 131071, 10 ** 6, 2 ** 24 + 1, 2 ** 30, 2 ** 31 - 1, -1, -70000] + list(range(52)),
                       dtype=torch.int32, device="cuda")
    r = Rotary(128, base=1e6, scaling=scaling, factor=factor, original_len=32768)
    freq, m = K.frequencies(128, 1e6, scaling, factor, 32768)
    _check(r.apply(x, pos), x, pos, freq, m, "half")


def test_three_axes():
    from paper_2609_03675_gb300 import Rotary
    axes = [i % 3 for i in range(40)]
    x, pos = _inputs(300, 2, 128, torch.bfloat16, seed=4, axes=3)
    freq, m = K.frequencies(80, 1e4)
    for layout in ("half", "interleaved"):
        y = Rotary(128, rotary_dim=80, layout=layout, axes=axes).apply(x, pos)
        _check(y, x, pos, freq, m, layout, axes)


@pytest.mark.parametrize("offset", [0, 1, 2, 4])
def test_strided_views_unaligned_and_in_place(offset):
    """q and k as views of one projection whose start and row length allow narrower and narrower vectors."""
    from paper_2609_03675_gb300 import Rotary
    n, h, hk, d = 70, 6, 2, 64
    g = torch.Generator(device="cuda").manual_seed(offset)
    flat = torch.randn(n * ((h + 2 * hk) * d + offset) + offset, generator=g, device="cuda").to(torch.bfloat16)
    rows = flat[offset:].view(n, -1)
    q = rows[:, :h * d].unflatten(1, (h, d))
    k = rows[:, h * d:(h + hk) * d].unflatten(1, (hk, d))
    pos = torch.arange(n, device="cuda", dtype=torch.int32) * 91
    before = flat.clone()
    q0, k0 = q.clone(), k.clone()
    r = Rotary(d, rotary_dim=48)
    freq, m = K.frequencies(48, 1e4)
    yq, yk = r.apply((q, k), pos)
    assert torch.equal(flat, before)
    _check(yq, q0, pos, freq, m, "half")
    _check(yk, k0, pos, freq, m, "half")
    outs = r.apply((q, k), pos, out=(q, k))
    assert outs[0] is q and torch.equal(q, yq) and torch.equal(k, yk)
    rest = rows[:, (h + hk) * d:]
    assert torch.equal(rest, before[offset:].view(n, -1)[:, (h + hk) * d:]), "values between the views moved"


def test_transposed_heads_and_broadcast_input():
    """Token and head strides in the other order, and a head stride of zero."""
    from paper_2609_03675_gb300 import Rotary
    x, pos = _inputs(37, 8, 64, torch.float16, seed=6)
    t = x.transpose(0, 1).contiguous().transpose(0, 1)
    r = Rotary(64)
    assert torch.equal(r.apply(t, pos[0]), r.apply(x, pos[0]))
    one = x[:, :1].expand(-1, 8, -1)
    assert torch.equal(r.apply(one, pos[0]), r.apply(one.contiguous(), pos[0]))


def test_gradient_against_differences():
    """d/dx of <w, apply(x)> along random directions: apply is linear, so a difference of two calls is exact up to fp32."""
    from paper_2609_03675_gb300 import Rotary
    x, pos = _inputs(19, 3, 80, torch.float32, seed=8)
    w, v = torch.randn_like(x), torch.randn_like(x)
    r = Rotary(80, rotary_dim=40, layout="interleaved", scaling="yarn", factor=2.0, original_len=4096)
    slope = ((r.apply(x + v, pos[0]).double() - r.apply(x - v, pos[0]).double()) / 2 * w.double()).sum()
    grad = (r.backward(w, pos[0]).double() * v.double()).sum()
    # each of the n terms is off by at most 2^-20 (|x| + |v|) |w| m 2: 4560 terms of mean size 1, at most 6 each
    assert abs(float(slope - grad)) <= 2.0 ** -20 * float(((x.abs() + v.abs()) * w.abs()).sum()) * 4
    # and the two directions are inverse to each other, up to m^2
    m2 = (0.1 * math.log(2.0) + 1) ** 2
    there_and_back = r.backward(r.apply(x, pos[0]), pos[0])[..., :40] / m2
    assert float((there_and_back - x[..., :40]).abs().max()) <= 2.0 ** -18 * float(x.abs().max()) * 2


def test_empty_and_streams():
    from paper_2609_03675_gb300 import Rotary
    r = Rotary(64)
    empty = torch.empty((0, 4, 64), device="cuda", dtype=torch.bfloat16)
    assert r.apply(empty, torch.empty(0, device="cuda", dtype=torch.int32)).shape == (0, 4, 64)
    x, pos = _inputs(500, 4, 64, torch.bfloat16, seed=9)
    want = r.apply(x, pos[0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = r.apply(x, pos[0], cuda_stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(x)
    r.apply(x, pos[0], out=out)
    out.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.apply(x, pos[0], out=out)
    x.copy_(x * 2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, r.apply(x, pos[0]))


def test_refusals():
    from paper_2609_03675_gb300 import NGFFError, Rotary
    for kw, msg in (({"rotary_dim": 3}, "rotary_dim"), ({"rotary_dim": 130}, "rotary_dim"), ({"base": 1.0}, "base"),
                    ({"factor": 2.0}, "needs a scaling"), ({"scaling": "yarn", "factor": 2.0}, "original_len"),
                    ({"axes": [4] * 32}, "n_axes"), ({"scaling": "linear", "factor": 0.5}, "factor")):
        with pytest.raises(NGFFError, match=msg):
            Rotary(64, **kw)
    with pytest.raises(ValueError, match="layout"):
        Rotary(64, layout="both")
    with pytest.raises(ValueError, match="axes"):
        Rotary(64, axes=[0, 1])
    r = Rotary(64)
    x, pos = _inputs(8, 2, 64, torch.bfloat16, seed=1)
    with pytest.raises(ValueError, match="positions"):
        r.apply(x, pos[0].long())
    with pytest.raises(ValueError, match="positions"):
        r.apply(x, pos[0][:7])
    with pytest.raises(ValueError, match="contiguous"):
        r.apply(x.transpose(1, 2).contiguous().transpose(1, 2), pos[0])
    with pytest.raises(ValueError, match="bfloat16"):
        r.apply(x.double(), pos[0])
    with pytest.raises(ValueError):
        r.apply(x.cpu(), pos[0])
    with pytest.raises(ValueError, match="64"):
        r.apply(x[..., :32], pos[0])

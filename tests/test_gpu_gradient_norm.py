"""The norm over many tensors and their clipping against 64 bits.

The squares' sum is formed in 64 bits: the norm is off by its one rounding, u = 2^-24 (n 2^-53 beside it).  The scale max / norm carries that and its own
rounding, the product one more in fp32 and half a step of its type."""
import pytest
import torch

import paper_2006_16668_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def make(sizes, g, scale=1.0):
    return [(scale * torch.randn(n, generator=g, device=DEV)).to(torch.float32 if i % 3 == 0 else torch.bfloat16) for i, n in enumerate(sizes)]


def norm_of(lst):
    norm = torch.full((1,), float("nan"), device=DEV)
    ws = torch.full((moe.moe_gradient_norm_workspace_bytes(lst),), 255, dtype=torch.uint8, device=DEV)
    moe.moe_gradient_norm(lst, norm, ws)
    return norm


def exact(tensors):
    return float(sum((t.double() ** 2).sum() for t in tensors).sqrt()) if tensors else 0.0


SIZES = [[1], [3, 5], [8191, 8192, 8193], [0, 17, 0], [1, 2, 3, 4, 5, 6, 7, 8, 9, 15, 16, 17, 31, 33], [4096 * 4, 1, 4096 * 8 + 1],
         [100] * 99, [101] * 100, [77] * 165, [33] * 166, [33] * 500, [30_000_001, 5, 12_345_678]]


@pytest.mark.parametrize("ratio", [0.25, 2.0, 0.0])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_norm_and_clip(sizes, ratio):
    g = torch.Generator(device=DEV).manual_seed(len(sizes) + max(sizes))
    ts = make(sizes, g)
    outs = [torch.full_like(t, float("nan")) for t in ts]
    lst = moe.GradientList(ts, outs)
    norm = norm_of(lst)
    want = exact(ts)
    assert abs(float(norm) - want) <= 1.01 * U * want
    assert torch.equal(norm, norm_of(lst))
    keep = [t.clone() for t in ts]
    limit = ratio * want
    moe.moe_clip_gradients(lst, norm, limit)
    scale = min(1.0, limit / want)
    for t, k, o in zip(ts, keep, outs):
        assert torch.equal(t, k)
        if scale == 1.0:
            assert torch.equal(o, t)
        else:
            w = t.double() * scale
            assert ((o.double() - w).abs() <= (HALF[t.dtype] * 1.01 + 3 * U) * w.abs() + 1e-38).all()
    here = moe.GradientList(ts)
    moe.moe_clip_gradients(here, norm, limit)
    for t, o in zip(ts, outs):
        assert torch.equal(t, o)


def test_no_tensor_at_all():
    lst = moe.GradientList([])
    assert float(norm_of(lst)) == 0
    moe.moe_clip_gradients(lst, torch.ones(1, device=DEV), 1.0)


@pytest.mark.parametrize("value", [3e38, 1e-38, 2.0 ** -140, 1e-45])
def test_values_whose_squares_leave_fp32(value):
    t = torch.full((1000,), value, device=DEV)
    want = float(t[0].double()) * 1000 ** 0.5
    got = float(norm_of(moe.GradientList([t])).double())
    assert got == float("inf") if want > 3.4028235e38 else abs(got - want) <= U * want + 2.0 ** -150


@pytest.mark.parametrize("norm, limit", [(1e20, 1e-25), (1e30, 1e-12), (3e38, 1e-5), (3e38, 1e-40), (1e20, 1e-18)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_scales_below_the_normal_numbers(norm, limit, dtype):
    """limit / norm may be below 2^-126 (or the least number of fp32) where the clipped gradients are not: they keep their digits.  The
    mantissa's rounding, the product's and the result's, U each or half a step; below 2^-126 half of the least step, twice."""
    t = torch.tensor([1.0, -0.75, 0.3, 1e-3, 0.0], device=DEV).repeat(500) * (norm / 4)
    t = t.to(dtype)
    out = torch.full_like(t, float("nan"))
    n = torch.tensor([norm], device=DEV)
    moe.moe_clip_gradients(moe.GradientList([t], [out]), n, limit)
    want = t.double() * (limit / float(n))
    least = 2.0 ** -149 if dtype == torch.float32 else 2.0 ** -133
    assert ((out.double() - want).abs() <= (HALF[dtype] * 1.01 + 3 * U) * want.abs() + 1.01 * least).all()


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -float("inf")])
def test_a_norm_that_is_no_number_changes_nothing(bad):
    g = torch.Generator(device=DEV).manual_seed(1)
    ts = make([1000, 50000, 31], g)
    ts[1][777] = bad
    outs = [torch.zeros_like(t) for t in ts]
    lst = moe.GradientList(ts, outs)
    norm = norm_of(lst)
    assert not torch.isfinite(norm).any()
    keep = [t.clone() for t in ts]
    moe.moe_clip_gradients(lst, norm, 0.1)
    moe.moe_clip_gradients(moe.GradientList(ts), norm, 0.1)
    bits = lambda t: t.view(torch.int32 if t.dtype == torch.float32 else torch.int16)
    for t, k, o in zip(ts, keep, outs):
        assert torch.equal(bits(t), bits(k)) and torch.equal(bits(o), bits(k))


def test_at_the_limit_and_infinite_limit():
    t = torch.tensor([3.0, 4.0], device=DEV)
    lst = moe.GradientList([t])
    norm = norm_of(lst)
    assert float(norm) == 5.0
    for limit in (5.0, float("inf"), 6.0):
        moe.moe_clip_gradients(lst, norm, limit)
        assert t.tolist() == [3.0, 4.0]
    moe.moe_clip_gradients(lst, norm, 2.5)
    assert t.tolist() == [1.5, 2.0]


def test_refusals():
    a, b = torch.zeros(100, device=DEV), torch.zeros(100, device=DEV)
    for tensors, out in (([a, a], None), ([a], [a[:50]]), ([a[4:8], a[:8]], None), ([a, b], [b, a]), ([a[:96], b], [a[4:].contiguous(), b[:0]]),
                         ([a.view(10, 10).t()], None), ([b, a[:8]], [b, a[4:12]]), ([a], [])):
        with pytest.raises((ValueError, TypeError)):
            moe.GradientList(tensors, out)
    for bad in (a.half(), a.cpu(), None):
        with pytest.raises(TypeError):
            moe.GradientList([bad])
    moe.GradientList([a, a], [b, torch.zeros_like(a)])           # read twice: counts twice
    with pytest.raises(moe.MoEError):                            # not on a whole 16 bytes
        norm_of(moe.GradientList([a[1:]]))
    lst, norm = moe.GradientList([a]), torch.ones(1, device=DEV)
    for limit in (-1.0, float("nan")):
        with pytest.raises(moe.MoEError):
            moe.moe_clip_gradients(lst, norm, limit)
    with pytest.raises(moe.MoEError):
        moe.moe_gradient_norm(lst, norm, torch.empty(0, dtype=torch.uint8, device=DEV))


def test_a_tensor_of_more_than_2_gb():
    """Two launches' worth of pieces of one tensor, offsets past 2^31 bytes; the last elements are found and scaled."""
    n = (1 << 30) + (1 << 29) + 12345
    t = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    for at in (0, (1 << 30) - 1, 1 << 30, n - 1):
        t[at] = 3.0
    lst = moe.GradientList([t])
    norm = norm_of(lst)
    assert float(norm) == 6.0
    moe.moe_clip_gradients(lst, norm, 2.0)
    for at in (0, (1 << 30) - 1, 1 << 30, n - 1):
        assert float(t[at]) == 1.0
    assert float(t[1]) == 0 and float(t[(1 << 30) + 1]) == 0

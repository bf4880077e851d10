"""dbl_grad_norm and dbl_clip_grads on the GPU against binary64.

The norm is a binary64 sum rounded to fp32 once: within 2^-24 of the exact norm plus binary64's own
n 2^-53. The scale is max_norm / (norm + 1e-6) in fp32: three roundings of 2^-24 (the norm, the sum, the
quotient); the product rounds once more in fp32 and once to the tensor's type (bf16 2^-8)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def _tensors(sizes, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * scale).to(dt).cuda() for n, dt in sizes]


def _norm64(ts):
    return math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in ts))


def _check(ts, max_norm, out=None):
    from paper_2608_05448_amd import dblast as D
    before = [t.clone() for t in ts]
    want = _norm64(before)
    norm = D.dbl_grad_norm(ts)
    assert norm.shape == () and norm.dtype == F
    assert abs(norm.item() - want) <= (2.0 ** -24 + 2.0 ** -40) * want + 1e-45
    got = D.dbl_clip_grads(ts, norm, max_norm, out=out)
    scale = min(1.0, max_norm / (want + 1e-6))
    for t, b in zip(got, before):
        w = b.double() * scale
        half = 2.0 ** -8 if t.dtype == BF else 2.0 ** -24
        bound = (half + 6 * 2.0 ** -24) * w.abs() + 1e-40
        assert t.dtype == b.dtype and ((t.double() - w).abs() <= bound).all(), t.shape
    if out is not None:
        for t, b in zip(ts, before):
            assert torch.equal(t, b)
    if scale == 1.0:
        for t, b in zip(got, before):
            assert torch.equal(t, b)
    return norm


SETS = {
    "one-value": [(1, F)],
    "one-bf16": [(1, BF)],
    "small": [(3, BF), (5, F), (7, BF), (1, F), (0, BF), (9, F)],
    "chunk-edges": [(n, dt) for n in (2047, 2048, 2049, 16383, 16384, 16385, 32768) for dt in (BF, F)],
    "long": [(5_000_011, BF), (3_000_007, F)],
    "many": [(1 + (i * 37) % 300, (BF, F)[i % 2]) for i in range(500)],
    "launch-edge-130": [(11, F)] * 130, "launch-edge-131": [(11, BF)] * 131,
    "launch-edge-180": [(11, F)] * 180, "launch-edge-181": [(11, BF)] * 181,
    "empty-ones": [(0, F)] * 200 + [(4, F)],
}


@pytest.mark.parametrize("name", SETS)
@pytest.mark.parametrize("limit", [0.25, 4.0])
def test_norm_and_clip(name, limit):
    print(f"[clip] {name} limit={limit}", flush=True)
    ts = _tensors(SETS[name], 61)
    limit *= max(_norm64(ts), 1e-3)
    out = [torch.full_like(t, 7) for t in ts]
    _check(ts, limit, out=out)
    _check(ts, limit)


def test_views_into_a_bucket():
    """Views that start at any element, the outputs at other ones; what lies between is left alone."""
    from paper_2608_05448_amd import dblast as D
    for dt in (BF, F):
        flat = _tensors([(200_000, dt)], 62)[0]
        to = torch.full_like(flat, 3)
        cuts = [(1, 18), (20, 20), (33, 17_000), (17_007, 50_001), (70_003, 199_999)]
        ts = [flat[a:b] for a, b in cuts]
        outs = [to[a + 1:b + 1] for a, b in cuts]
        _check(ts, 1.0, out=outs)
        rest = torch.ones(len(to), dtype=torch.bool)
        for a, b in cuts:
            rest[a + 1:b + 1] = False
        assert (to.cpu()[rest] == 3).all()
        keep = flat.clone()
        D.dbl_clip_grads(ts, D.dbl_grad_norm(ts), 1.0)
        rest = torch.ones(len(to), dtype=torch.bool)
        for a, b in cuts:
            rest[a:b] = False
        assert torch.equal(flat.cpu()[rest], keep.cpu()[rest])


def test_huge_and_tiny_values():
    """Squares that leave fp32's range either way."""
    from paper_2608_05448_amd import dblast as D
    for dt in (BF, F):
        for v in (1e30, 1e-30, 3e38 / 64):
            t = torch.full((1000,), v, dtype=dt, device="cuda")
            want = _norm64([t])
            assert abs(D.dbl_grad_norm([t]).item() - want) <= 2.0 ** -23 * want
    t = torch.full((1000,), 3e38, device="cuda")
    assert math.isinf(D.dbl_grad_norm([t]).item())   # the norm itself is past fp32


def test_infinities_and_nan_are_not_hidden():
    from paper_2608_05448_amd import dblast as D
    a, b = _tensors([(1000, F), (77, BF)], 63)
    a[5] = float("inf")
    norm = D.dbl_grad_norm([a, b])
    assert math.isinf(norm.item())
    D.dbl_clip_grads([a, b], norm, 1.0)
    assert torch.isnan(a[5]) and (b == 0).all() and (a[6:] == 0).all()
    a, b = _tensors([(1000, F), (77, BF)], 63)
    b[3] = float("nan")
    norm = D.dbl_grad_norm([a, b])
    assert math.isnan(norm.item())
    D.dbl_clip_grads([a, b], norm, 1.0)
    assert torch.isnan(a).all() and torch.isnan(b).all()


def test_limits():
    from paper_2608_05448_amd import dblast as D
    a = _tensors([(1000, F)], 64)[0]
    keep = a.clone()
    norm = D.dbl_grad_norm([a])
    D.dbl_clip_grads([a], norm, float("inf"))
    assert torch.equal(a, keep)
    D.dbl_clip_grads([a], norm, 0.0)
    assert (a == 0).all()
    z = torch.zeros(10, device="cuda")
    n = D.dbl_grad_norm([z])
    assert n.item() == 0.0
    D.dbl_clip_grads([z], n, 1.0)
    assert (z == 0).all()
    assert D.dbl_clip_grads([], n, 1.0) == []


def test_norm_does_not_change_from_run_to_run():
    from paper_2608_05448_amd import dblast as D
    ts = _tensors([(3_000_001, BF), (70_000, F)], 65)
    first = D.dbl_grad_norm(ts)
    for _ in range(5):
        assert torch.equal(D.dbl_grad_norm(ts), first)


def test_refusals():
    from paper_2608_05448_amd import dblast as D
    a = torch.ones(100, device="cuda")
    n = D.dbl_grad_norm([a])
    with pytest.raises(D.DblastError):
        D.dbl_clip_grads([a, a], n, 1.0)                     # the same tensor twice
    with pytest.raises(D.DblastError):
        D.dbl_clip_grads([a[:60], a[50:]], n, 1.0)           # overlapping views
    with pytest.raises(D.DblastError):
        D.dbl_clip_grads([a[:50]], n, 1.0, out=[a[25:75]])   # an output over its input
    with pytest.raises(D.DblastError):
        D.dbl_clip_grads([a], n, -1.0)
    with pytest.raises(D.DblastError):
        D.dbl_clip_grads([a], n, float("nan"))
    with pytest.raises(TypeError):
        D.dbl_grad_norm([a.half()])
    with pytest.raises(ValueError):
        D.dbl_grad_norm([torch.ones((8, 8), device="cuda").t()])
    with pytest.raises(ValueError):
        D.dbl_grad_norm([a, torch.ones(4)])
    with pytest.raises(ValueError):
        D.dbl_grad_norm([])
    with pytest.raises(ValueError):
        D.dbl_clip_grads([a], n, 1.0, out=[a.bfloat16()])
    assert abs(D.dbl_grad_norm([a, a]).item() - 200 ** 0.5) < 1e-5   # reading twice is no fault

"""The training operators at shapes whose kernels the other tests' sizes do not take: the head's 256 x 256,
256 x 128 and 256 x 64 tiles with whole and partial last stages, hidden sizes whose sums start further on, a
vocabulary in several pieces for every product kernel, rows against the same rows in smaller calls, and a
norm of more than 512 MB.

Bounds as in test_gpu_train, with the length of a sum's longest chain in place of its number of terms: an
MFMA adds at least four bf16 products at a time, so a part of n terms is a chain of n / 4 additions at most
(fp32: n); its parts and the pieces of the vocabulary are added one after the other."""
import math

import pytest
import torch

from test_gpu_train import (DT, HALF, _check, _close, _expand_check, _expand_inputs, _nll_bounds,
                            _plain)

pytestmark = pytest.mark.gpu

CASES = [
    # dtype, B, K, R, d, V, mask: the head's kernel for the logits and their gradient
    ("bf16", 6, 50, 1, 136, 21000, "some"),      # 256 x 256 tiles, a partial last stage
    ("bf16", 6, 50, 1, 8, 21000, "but-last"),    # a hidden size of less than a stage
    ("bf16", 6, 50, 1, 2048, 21000, "some"),     # 256 x 256 tiles, sums that start at unit 0 or 1024
    ("bf16", 2, 30, 1, 136, 42001, "some"),      # 256 x 64 tiles, a partial last stage
    ("bf16", 2, 30, 1, 2048, 42001, "first"),    # whole stages, sums that start further on
    ("bf16", 2, 50, 1, 64, 50001, "some"),       # 256 x 128 tiles, whole stages
    ("bf16", 2, 60, 1, 4096, 41000, "some"),     # and sums that start at one of four units
    ("bf16", 2, 50, 1, 1000, 50257, "none"),     # 256 x 128 tiles, a partial last stage
]


@pytest.mark.parametrize("case", CASES, ids=["-".join(map(str, c)) for c in CASES])
def test_head_kernels(case):
    dtype, B, K, R, d, V, mask = case
    _check(dtype, B, K, R, d, V, mask)


@pytest.mark.parametrize("case", [("bf16", 136, 21000), ("bf16", 2048, 21000), ("bf16", 64, 50001),
                                  ("fp32", 40, 5000)], ids=str)
def test_a_row_is_the_same_in_calls_of_every_size(case):
    """300 rows on the 256 x 256 tiles of the head (fp32: 64-row tiles), parts of them on all others."""
    from paper_2608_05448_amd import dblast as D
    dtype, d, V = case
    g = torch.Generator(device="cuda").manual_seed(91)
    h = torch.randn((300, 1, 1, d), generator=g, device="cuda").to(DT[dtype])
    w = (torch.randn((V, d), generator=g, device="cuda") * (1.5 / d ** 0.5)).to(DT[dtype])
    x = torch.randint(0, V, (300, 1), generator=g, device="cuda", dtype=torch.int32)
    nll, lse = D.dbl_head_nll(h, w, x)
    for b, n in ((0, 1), (17, 33), (100, 100), (40, 129), (299, 1)):
        a, c = D.dbl_head_nll(h[b:b + n].clone(), w, x[b:b + n].clone())
        assert torch.equal(a, nll[b:b + n]) and torch.equal(c, lse[b:b + n]), (case, b, n)
    keep = x.clone()
    x[torch.arange(300, device="cuda") % 7 != 0] = -1  # 43 of them count
    a, c = D.dbl_head_nll(h, w, x)
    on = x >= 0
    assert torch.equal(a[on], nll[on]) and torch.equal(c[on], lse[on]) and (keep[on] == x[on]).all()


PIECES = [
    # dtype, rows, d, V: pieces and the kernels of dh
    ("bf16", 4096, 2048, 151936),    # two pieces of 77,824 ids (an odd number of 4096): 256 x 256 tiles
    ("bf16", 44000, 200, 16484),     # three of 8192, 8192 and 100 ids: 256 x 256 tiles, then 128 x 128
    ("bf16", 120, 136, 4500000),     # two: 256 x 128 tiles
    ("bf16", 60, 136, 9000000),      # two: 256 x 64 tiles
    ("bf16", 60, 72, 9000000),       # two: 128 x 64 tiles
    ("fp32", 22000, 131, 16484),     # three of 8192, 8192 and 100 ids
    ("fp32", 30, 17, 9000000),       # two: 32-row tiles
]


@pytest.mark.parametrize("case", PIECES, ids=["-".join(map(str, c)) for c in PIECES])
def test_gradient_over_pieces_of_the_vocabulary(case):
    """Logits' gradients of more than 1 GiB. Tokens lie in all pieces, so that a row whose sum lost an
    earlier piece, or its last one, is off by about all of its gradient."""
    from paper_2608_05448_amd import dblast as D
    dtype, M, d, V = case
    assert M * V * (2 if dtype == "bf16" else 4) > 1 << 30
    print(f"[pieces] {case}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(92)
    h = torch.randn((M, 1, 1, d), generator=g, device="cuda").to(DT[dtype])
    w = torch.empty((V, d), dtype=DT[dtype], device="cuda")
    for part in w.split(1 << 20):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * (2.0 / d ** 0.5))
    x = torch.randint(0, V, (M, 1), generator=g, device="cuda", dtype=torch.int32)
    x[:3, 0] = torch.tensor([0, V - 1, V // 2])
    x[5::11] = -1
    grad = torch.randn((M, 1, 1), generator=g, device="cuda") / M
    nll, lse = D.dbl_head_nll(h, w, x)
    dh, dw = D.dbl_head_nll_backward(h, w, x, nll, lse, grad)
    o = _plain(h, w, x, grad)
    le, ne = _nll_bounds(o)
    _close(lse, o["lse"].reshape(lse.shape), le.reshape(lse.shape), "lse")
    _close(nll, o["nll"].reshape(nll.shape), ne.reshape(nll.shape), "nll")
    half = HALF[dtype]
    deep = 4 if dtype == "bf16" else 1
    chain = (V / deep + 70) * 2.0 ** -24              # at most 64 parts and 3 pieces
    if M <= 128:                                      # few rows: 256 to 768 parts of a piece
        chain = (V / 256 / deep + 800) * 2.0 ** -24
    rel = 2 * o["e"] + 2.0 ** -20 + (half if dtype == "bf16" else 0.0)
    ga, q = o["g"].abs(), -torch.expm1(-o["nll"])
    tok = ga * torch.exp(-o["nll"]) * ne + ga * (half * torch.where(q < 2.0 ** -23, q, 0.0) + 2.0 ** -22 * q)
    wt = o["w"][o["t"]].abs()
    e = o["rest"].mul_(ga[:, None])
    sum_w = e @ o["w"].abs()
    eh = (rel + chain)[:, None] * sum_w + (tok + ga * q * chain)[:, None] * wt
    eh = 1.01 * (eh + half * o["dh"].abs()) + 1e-37
    assert eh.norm() < 0.1 * o["dh"].norm()           # far less than what a piece holds
    _close(dh.reshape(M, d), o["dh"], eh, "dh")
    rows = (M / deep + 70) * 2.0 ** -24
    e.mul_((rel + 2 * half + rows)[:, None])
    e[torch.arange(M, device="cuda"), o["t"]] = tok + ga * q * (2 * half + rows)
    ew = e.T @ o["h"].abs()
    _close(dw, o["dw"], 1.01 * (ew + half * o["dw"].abs()) + 1e-37, "dw")


@pytest.mark.parametrize("sizes", [[(150_000_011, "fp32")],
                                   [(200_000_003, "bf16"), (1, "fp32"), (60_000_001, "fp32"), (7, "bf16")]],
                         ids=["fp32", "mixed"])
def test_norm_of_more_than_512_megabytes(sizes):
    """The norm's streaming form; one element more or less in any chunk would show."""
    from paper_2608_05448_amd import dblast as D
    assert sum(n * (2 if t == "bf16" else 4) for n, t in sizes) > 512 << 20
    g = torch.Generator(device="cuda").manual_seed(93)
    ts = [torch.randn(n, generator=g, device="cuda").to(DT[t]) for n, t in sizes]
    want = math.sqrt(math.fsum(float(p.double().square().sum()) for t in ts for p in t.split(1 << 24)))
    got = D.dbl_grad_norm(ts).item()
    assert abs(got - want) <= (2.0 ** -24 + 2.0 ** -40) * want
    # The last element of each tensor alone, 1e6 times the rest: exact to the norm's rounding.
    for t in ts:
        t.zero_()
        t[-1] = 3.0
    assert abs(D.dbl_grad_norm(ts).item() - 3.0 * math.sqrt(len(ts))) <= 2.0 ** -23 * 3.0 * math.sqrt(len(ts))


@pytest.mark.parametrize("case", [(1, 201, 8, 4096), (1, 100, 9, 4064)], ids=str)
def test_weight_gradients_past_the_infinity_cache(case):
    """Outputs of 256 MB or more from 65 to 256 rows: the streaming kernel with non-temporal stores."""
    from paper_2608_05448_amd import dblast as D
    B, K, R, d = case
    assert 2 * R * d * d >= 256 << 20
    h, W, dout = _expand_inputs(*case)
    got = D.dbl_expand_branches_backward(h.cuda(), W.cuda(), dout.cuda())
    _expand_check(h, W, dout, got)

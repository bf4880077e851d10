"""The training operators with NaN and infinities in what counts: they show in the results that are made
of them, and in no others. All comparisons are exact: a value is NaN, or it is the bits of the clean call."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
NAN, INF = float("nan"), float("inf")

# dtype, rows, d, V: vocabularies of less than a tile of log-masses (128 ids in bf16, 32 in fp32), of one, of
# several, of more than a wave joins at once (262,144 ids in bf16, 65,536 in fp32)
CASES = [
    ("fp32", 5, 33, 20), ("fp32", 50, 70, 32), ("fp32", 50, 33, 300), ("fp32", 3, 16, 70000),
    ("bf16", 1, 8, 100), ("bf16", 5, 64, 100), ("bf16", 100, 72, 128), ("bf16", 300, 64, 90),
    ("bf16", 5, 64, 300), ("bf16", 100, 200, 900), ("bf16", 60, 64, 50001), ("bf16", 300, 64, 21000),
    ("bf16", 5, 64, 270000),
]
IDS = ["-".join(map(str, c)) for c in CASES]


def _inputs(dtype, M, d, V, seed=71):
    g = torch.Generator().manual_seed(seed)
    h = torch.randn((M, 1, 1, d), generator=g)
    w = torch.randn((V, d), generator=g) * (1.5 / d ** 0.5)
    h, w = (torch.where(t == 0, 1.0, t).to(DT[dtype]).cuda() for t in (h, w))
    x = torch.randint(0, V, (M, 1), generator=g, dtype=torch.int32).cuda()
    grad = (torch.randn((M, 1, 1), generator=g) / M).cuda()
    return h, w, x, grad


@pytest.mark.parametrize("case", CASES, ids=IDS)
@pytest.mark.parametrize("bad", [NAN, INF], ids=["nan", "inf"])
def test_a_state_that_is_not_finite_shows_in_its_row_only(case, bad):
    """One unit of one row. NaN: every logit of the row is NaN. Infinity: every logit is one, of either
    sign, and logits of plus infinity have no finite log-sum-exp."""
    from paper_2608_05448_amd import dblast as D
    print(f"[nonfinite] state {bad} {case}", flush=True)
    h, w, x, _ = _inputs(*case)
    M, d = h.shape[0], h.shape[3]
    w[0, d - 1], w[1, d - 1] = w[0, d - 1].abs(), -w[1, d - 1].abs()
    nll, lse = D.dbl_head_nll(h, w, x)
    assert torch.isfinite(nll).all() and torch.isfinite(lse).all()
    row = M // 2
    for token in (0, 1):  # logits of plus and of minus infinity
        x[row] = token
        clean, cleanlse = D.dbl_head_nll(h, w, x)
        hb = h.clone()
        hb[row, 0, 0, d - 1] = bad
        nll, lse = D.dbl_head_nll(hb, w, x)
        others = torch.arange(M, device="cuda") != row
        assert torch.equal(nll[others], clean[others]) and torch.equal(lse[others], cleanlse[others])
        assert torch.isnan(lse[row]).all(), lse[row]
        assert torch.isnan(nll[row]).all(), nll[row]


@pytest.mark.parametrize("case", CASES, ids=IDS)
@pytest.mark.parametrize("bad", [NAN, INF], ids=["nan", "inf"])
def test_one_logit_of_another_id(case, bad):
    """One id's weight: its logit is NaN, or plus infinity where the state's unit is positive (minus infinity,
    a probability of 0, where it is negative). The token's own logit is finite."""
    from paper_2608_05448_amd import dblast as D
    print(f"[nonfinite] weight {bad} {case}", flush=True)
    h, w, x, _ = _inputs(*case)
    M, d = h.shape[0], h.shape[3]
    V = w.shape[0]
    at = V // 2
    x[x == at] = at + 1
    h[0, 0, 0, 3] = h[0, 0, 0, 3].abs()
    w[at, 3] = bad
    nll, lse = D.dbl_head_nll(h, w, x)
    spoilt = (h[..., 3] > 0) if bad == INF else torch.ones_like(h[..., 3], dtype=torch.bool)
    assert torch.isnan(lse[spoilt]).all() and torch.isnan(nll[spoilt]).all()
    assert torch.isfinite(lse[~spoilt]).all() and torch.isfinite(nll[~spoilt]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_of_minus_infinity_and_certain_rows_are_as_they_were(dtype):
    """A token of logit minus infinity costs plus infinity; a vocabulary of one id costs 0."""
    from paper_2608_05448_amd import dblast as D
    h, w, x, _ = _inputs(dtype, 6, 64, 40)
    h[..., 3] = h[..., 3].abs()
    w[7, 3] = -INF
    x[2] = 7
    nll, lse = D.dbl_head_nll(h, w, x)
    assert torch.isfinite(lse).all()
    assert torch.isposinf(nll[2]).all() and torch.isfinite(nll[[0, 1, 3, 4, 5]]).all()
    w1 = w[:1].contiguous()
    x.zero_()
    nll, lse = D.dbl_head_nll(h, w1, x)
    assert (nll == 0).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_gradients_of_a_row_that_is_not_a_number(case):
    """Its states' gradient is NaN in every unit, and so is every weight's, the token's own among them (each
    is a sum over the rows that count); the other rows' gradients are those of the clean call."""
    from paper_2608_05448_amd import dblast as D
    print(f"[nonfinite] gradient {case}", flush=True)
    h, w, x, g = _inputs(*case)
    M, d = h.shape[0], h.shape[3]
    nll, lse = D.dbl_head_nll(h, w, x)
    clean, _ = D.dbl_head_nll_backward(h, w, x, nll, lse, g)
    row = M // 2
    h[row, 0, 0, d - 1] = NAN
    nll, lse = D.dbl_head_nll(h, w, x)
    dh, dw = D.dbl_head_nll_backward(h, w, x, nll, lse, g)
    others = torch.arange(M, device="cuda") != row
    assert torch.equal(dh[others], clean[others])
    assert torch.isnan(dh[row]).all()
    assert torch.isnan(dw).all(), torch.nonzero(~torch.isnan(dw).all(1))[:4]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradients_of_a_vocabulary_of_one_id(dtype):
    """The token is the only id: its entry is all there is to show a NaN in."""
    from paper_2608_05448_amd import dblast as D
    h, w, x, g = _inputs(dtype, 3, 64, 1)
    h[1, 0, 0, 9] = NAN
    nll, lse = D.dbl_head_nll(h, w, x)
    assert torch.isnan(nll[1]).all() and (nll[[0, 2]] == 0).all()
    dh, dw = D.dbl_head_nll_backward(h, w, x, nll, lse, g)
    assert torch.isnan(dh[1]).all() and torch.isnan(dw).all()
    assert (dh[[0, 2]] == 0).all()

"""The training operators on the GPU against plain binary64 forms: dbl_head_nll, its gradient, the
expander's backward pass, and a training step made of them.

Bounds, from the roundings that the operators make (half a step: bf16 2^-8, fp32 2^-24, relative):
 logits   a sum of d products: d 2^-24 sum_j |h_j w_j| =: e (the largest over the row's ids)
 lse      e, and the exponentials', sum's and logarithm's own few 2^-22 of 1 + |lse|; nll as lse + e
 dh       with p the probabilities without the token's, q their sum: every p_v has relative error
          2 e + 2^-20 (logit and lse, exponential) and, in bf16, 2^-8 more; q has absolute error
          (1 - q) times nll's; a sum of n terms adds n 2^-24 of its absolute terms; one last rounding
 dw       the same with h g rounded once more (2^-8 in bf16, 2^-24 in fp32)
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _inputs(dtype, B, K, R, d, V, seed=1, scale=1.5, mask="none"):
    g = _gen(seed)
    h = torch.randn((B, K, R, d), generator=g).to(DT[dtype])
    w = (torch.randn((V, d), generator=g) * (scale / d ** 0.5)).to(DT[dtype])
    x = torch.randint(0, V, (B, K), generator=g, dtype=torch.int32)
    drop = {"none": torch.zeros(B, K, dtype=torch.bool), "all": torch.ones(B, K, dtype=torch.bool),
            "some": torch.rand((B, K), generator=g) < 0.4,
            "first": torch.arange(B * K).reshape(B, K) < 1,
            "but-last": torch.arange(B * K).reshape(B, K) < B * K - 1}[mask]
    bad = torch.tensor([-1, V, -2 ** 31, 2 ** 31 - 1, -100])[torch.arange(B * K) % 5].reshape(B, K)
    x = torch.where(drop, bad, x.long()).to(torch.int32)
    grad = torch.randn((B, K, R), generator=g) / (B * K)
    return h, w, x, grad


def _plain(h, w, x, g, device="cuda"):
    """Everything in binary64, with what the bounds need."""
    B, K, R, d = h.shape
    V = w.shape[0]
    hd = h.reshape(-1, d).to(device).double()
    wd = w.to(device).double()
    t = x.long().to(device)[:, :, None].expand(B, K, R).reshape(-1)
    on = (t >= 0) & (t < V)
    t = torch.where(on, t, 0)
    hd = torch.where(on[:, None], hd, 0.0)
    gd = torch.where(on, g.reshape(-1).to(device).double(), 0.0)
    z = hd @ wd.T
    lse = torch.logsumexp(z, 1)
    nll = lse - z.gather(1, t[:, None])[:, 0]
    e = d * 2.0 ** -24 * (hd.abs() @ wd.abs().T).amax(1)
    p = torch.exp(z - lse[:, None])
    u = p.clone()
    u[torch.arange(len(t)), t] = torch.expm1(-nll)
    rest = p
    rest[torch.arange(len(t)), t] = 0.0
    G = u * gd[:, None]
    return dict(on=on, t=t, h=hd, w=wd, g=gd, lse=torch.where(on, lse, 0.0), nll=torch.where(on, nll, 0.0),
                e=e, rest=rest, G=G, dh=G @ wd, dw=G.T @ hd)


def _nll_bounds(o):
    le = o["e"] + 2.0 ** -20 * (1 + o["lse"].abs())
    return le, le + o["e"] + 2.0 ** -22 * (1 + o["nll"].abs())


def _grad_bounds(o, dtype):
    half, V, M = HALF[dtype], o["w"].shape[0], len(o["t"])
    _, ne = _nll_bounds(o)
    rel = 2 * o["e"] + 2.0 ** -20 + (half if dtype == "bf16" else 0.0)      # [M], of every p_v
    big = o["rest"] * o["g"].abs()[:, None]                                  # g p without the token
    tok = (o["g"].abs() * torch.exp(-o["nll"]) * ne)                        # error of g q at the token
    # and where q is kept from below by 2^-24 its rounding in bf16 is a half step of it
    q = -torch.expm1(-o["nll"])
    tok = tok + o["g"].abs() * (half * torch.where(q < 2.0 ** -23, q, 0.0) + 2.0 ** -22 * q)
    wt, at = o["w"].abs()[o["t"]], torch.arange(M)
    dh = (big * (rel + V * 2.0 ** -24)[:, None]) @ o["w"].abs() + tok[:, None] * wt + \
        (o["g"].abs() * q * V * 2.0 ** -24)[:, None] * wt
    E = big * (rel + 2 * half + M * 2.0 ** -24)[:, None]
    E[at, o["t"]] = tok + o["g"].abs() * q * (2 * half + M * 2.0 ** -24)
    dw = E.T @ o["h"].abs()
    last = 1.01 * half
    return dh * 1.01 + last * o["dh"].abs() + 1e-37, dw * 1.01 + last * o["dw"].abs() + 1e-37


def _close(got, want, bound, what):
    got = got.double().reshape(want.shape)
    off = (got - want).abs() - bound
    assert torch.isfinite(got).all(), what
    worst = off.max().item() if off.numel() else 0.0
    i = int(off.argmax()) if off.numel() else 0
    assert worst <= 0, (what, i, got.flatten()[i].item(), want.flatten()[i].item(),
                        bound.expand(want.shape).flatten()[i].item())


def _check(dtype, B, K, R, d, V, mask="none", scale=1.5, dw=True, seed=1, poison=True):
    from paper_2608_05448_amd import dblast as D
    print(f"[train] {dtype} B={B} K={K} R={R} d={d} V={V} mask={mask} scale={scale} dw={dw}", flush=True)
    h, w, x, g = _inputs(dtype, B, K, R, d, V, seed, scale, mask)
    o = _plain(h, w, x, g)
    off = ~o["on"].reshape(B, K, R).cpu()
    if poison:  # rows that do not count may hold anything
        h = torch.where(off[..., None], torch.tensor(float("nan"), dtype=h.dtype), h)
        g = torch.where(off, float("inf"), g)
    hc, wc, xc, gc = h.cuda(), w.cuda(), x.cuda(), g.cuda()
    nll, lse = D.dbl_head_nll(hc, wc, xc)
    le, ne = _nll_bounds(o)
    _close(lse, o["lse"].reshape(B, K, R), le.reshape(B, K, R), "lse")
    _close(nll, o["nll"].reshape(B, K, R), ne.reshape(B, K, R), "nll")
    assert (nll.cpu()[off] == 0).all() and (lse.cpu()[off] == 0).all()
    dh, dwt = D.dbl_head_nll_backward(hc, wc, xc, nll, lse, gc, want_dw=dw)
    eh, ew = _grad_bounds(o, dtype)
    _close(dh.reshape(-1, d), o["dh"], eh, "dh")
    assert (dh.cpu()[off] == 0).all()
    if dw:
        _close(dwt, o["dw"], ew, "dw")
    else:
        assert dwt is None
    return hc, wc, xc, gc, nll, lse, dh, dwt


HEAD_CASES = [
    # dtype, B, K, R, d, V, mask
    ("fp32", 1, 1, 1, 1, 1, "none"),
    ("fp32", 1, 1, 1, 5, 2, "none"),
    ("fp32", 1, 4, 2, 64, 256, "none"),
    ("fp32", 2, 3, 5, 33, 777, "some"),
    ("fp32", 3, 50, 1, 130, 129, "some"),
    ("fp32", 2, 9, 8, 100, 5000, "first"),
    ("fp32", 1, 2, 2, 17, 300, "all"),
    ("bf16", 1, 1, 1, 8, 1, "none"),
    ("bf16", 1, 1, 1, 64, 2, "none"),
    ("bf16", 1, 1, 1, 64, 127, "none"),
    ("bf16", 1, 1, 4, 128, 1000, "none"),       # few rows, 64-row tiles
    ("bf16", 2, 15, 4, 192, 2000, "some"),      # 120 rows, 128-row tiles
    ("bf16", 1, 15, 4, 64, 50001, "first"),     # 60 rows, tiles of 256 ids
    ("bf16", 2, 16, 8, 128, 1500, "some"),      # 256 rows, too few ids for the larger tiles: 128 x 128
    ("bf16", 3, 11, 9, 64, 1031, "some"),       # 297 rows, ragged in every direction
    ("bf16", 2, 5, 3, 96, 700, "some"),         # d % 64 = 32: half a last stage
    ("bf16", 2, 5, 3, 200, 700, "but-last"),    # d % 64 = 8: one chunk of a last stage
    ("bf16", 5, 13, 5, 72, 1153, "some"),
    ("bf16", 2, 4, 2, 64, 300, "all"),
    ("bf16", 1, 70, 1, 2048, 9000, "some"),     # sums that start further on
    ("bf16", 1, 33, 1, 104, 513, "some"),       # a partial last stage: 64-row tiles, 128-row tiles, two
    ("bf16", 2, 40, 1, 1000, 901, "some"),      # of them, and a hidden size below one stage
    ("bf16", 6, 40, 1, 136, 901, "some"),
    ("bf16", 2, 70, 2, 8, 2100, "some"),
    ("bf16", 3, 100, 1, 192, 600, "some"),      # 300 rows: the products' 256 x 256 tiles, short sums
    ("bf16", 11, 50, 1, 264, 3000, "some"),     # both products on 256 x 256 tiles, partial last stages
    ("bf16", 5, 100, 1, 72, 2500, "none"),      # a narrow hidden size: 128-column tiles
    ("bf16", 3, 67, 1, 1672, 40189, "some"),    # 2^26 weights: dw's stream kernel
    ("bf16", 1, 40, 2, 1672, 40189, "all"),
    ("bf16", 6, 50, 1, 128, 45000, "some"),     # 300 rows by tile of the head: 256 x 256, 256 x 128 and
    ("bf16", 6, 50, 1, 136, 15000, "some"),     # 128 x 128 (the smaller vocabularies above), 100 rows
    ("bf16", 2, 50, 1, 136, 42000, "some"),
    ("fp32", 1, 31, 1, 63, 95, "none"), ("fp32", 1, 33, 1, 65, 97, "none"),
    ("fp32", 2, 64, 3, 250, 3001, "some"),      # sums in several parts
    ("bf16", 64, 16, 1, 200, 300, "some"),      # many rows and a small head: dw in parts as well, of 256 x 256
    ("bf16", 64, 16, 2, 264, 700, "first"),     # tiles (most of them and all but one of the rows gone),
    ("bf16", 64, 16, 1, 256, 256, "but-last"),
    ("bf16", 64, 16, 1, 256, 257, "all"),
    ("bf16", 37, 15, 2, 64, 1000, "some"),      # of 128 x 128 tiles,
    ("bf16", 41, 13, 3, 520, 77, "some"),
    ("fp32", 37, 11, 2, 33, 77, "some"),        # and in fp32, also where a part's length is odd
    ("fp32", 64, 16, 1, 131, 259, "some"),
    ("fp32", 64, 16, 1, 5, 3, "but-last"),
]


@pytest.mark.parametrize("case", HEAD_CASES, ids=["-".join(map(str, c)) for c in HEAD_CASES])
def test_head_nll_and_gradient(case):
    dtype, B, K, R, d, V, mask = case
    _check(dtype, B, K, R, d, V, mask)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_frozen_head(dtype):
    a = _check(dtype, 2, 6, 3, 64, 500, "some", dw=False)
    b = _check(dtype, 2, 6, 3, 64, 500, "some", dw=True)
    assert torch.equal(a[6], b[6])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("scale", [0.0, 6.0, 40.0])
def test_flat_and_confident_rows(dtype, scale):
    """Flat logits; rows that are nearly sure of their token, or sure of another one."""
    _check(dtype, 3, 7, 2, 64, 300, "some", scale=scale, seed=3)


def test_a_row_that_is_sure_of_its_token():
    """nll rounds to 0 (and may come out a little below): the gradient is 0 to fp32's own error."""
    from paper_2608_05448_amd import dblast as D
    for dtype in ("bf16", "fp32"):
        d, V = 64, 200
        w = torch.zeros((V, d), dtype=DT[dtype])
        w[torch.arange(64), torch.arange(64)] = 8.0
        h = torch.zeros((1, 1, 4, d), dtype=DT[dtype])
        for r, v in enumerate((10.0, 2.5, 2.0, 0.0)):
            h[0, 0, r, 7] = v
        x = torch.tensor([[7]], dtype=torch.int32)
        g = torch.ones((1, 1, 4))
        o = _plain(h, w, x, g)
        nll, lse = D.dbl_head_nll(h.cuda(), w.cuda(), x.cuda())
        dh, dw = D.dbl_head_nll_backward(h.cuda(), w.cuda(), x.cuda(), nll, lse, g.cuda())
        eh, ew = _grad_bounds(o, dtype)
        _close(dh.reshape(4, d), o["dh"], eh, "dh")
        _close(dw, o["dw"], ew, "dw")


@pytest.mark.parametrize("case", [("bf16", 3, 72, 300), ("bf16", 50, 200, 3000), ("bf16", 100, 8, 40000),
                                  ("bf16", 100, 200, 1000), ("bf16", 300, 72, 20500), ("fp32", 5, 70, 300),
                                  ("fp32", 50, 33, 700)], ids=lambda c: "-".join(map(str, c)))
def test_an_id_that_an_infinite_weight_rules_out(case):
    """A logit of minus infinity is a probability of 0 and spoils no other id, wherever the weight stands
    (also in the first units of a last, partial stage, whose copies are repeated past the end) and however
    many there are (128 ids in a row are a whole tile)."""
    from paper_2608_05448_amd import dblast as D
    dtype, M, d, V = case
    h, w, x, g = _inputs(dtype, M, 1, 1, d, V, seed=11)
    unit = (d - 1) // 64 * 64
    h[..., unit] = h[..., unit].abs() + 0.5
    keep = torch.ones(V, dtype=torch.bool)
    keep[3] = keep[128:256] = False
    x = torch.where(keep[x.long()], x, 4).to(torch.int32)
    o = _plain(h, w[keep], (keep.cumsum(0) - 1)[x.long()].to(torch.int32), g)
    w[~keep, unit] = float("-inf")
    nll, lse = D.dbl_head_nll(h.cuda(), w.cuda(), x.cuda())
    le, ne = _nll_bounds(o)
    _close(lse, o["lse"].reshape(lse.shape), le.reshape(lse.shape), "lse")
    _close(nll, o["nll"].reshape(nll.shape), ne.reshape(nll.shape), "nll")


def test_gradient_matches_differences():
    """fp32: central differences of the binary64 loss along random directions."""
    B, K, R, d, V = 2, 3, 2, 24, 90
    h, w, x, g, nll, lse, dh, dw = [t.cpu() if t is not None else None
                                    for t in _check("fp32", B, K, R, d, V, "some", poison=False)]
    gen = _gen(8)
    on = ((x >= 0) & (x < V))[:, :, None].expand(B, K, R)
    t = x.long().clamp(0, V - 1)

    def loss(hh, ww):
        z = hh @ ww.T
        n = torch.logsumexp(z, -1) - z.gather(-1, t[:, :, None, None].expand(B, K, R, 1))[..., 0]
        return (torch.where(on, n, 0.0) * g.double()).sum()

    step = 1e-5
    for _ in range(5):
        a = torch.randn(h.shape, generator=gen, dtype=torch.float64)
        b = torch.randn(w.shape, generator=gen, dtype=torch.float64)
        hd, wd = h.double(), w.double()
        diff = (loss(hd + step * a, wd + step * b) - loss(hd - step * a, wd - step * b)) / (2 * step)
        got = (dh.double() * a).sum() + (dw.double() * b).sum()
        # step^2 of a third derivative of order |a|^3, and fp32's error of either gradient
        size = (dh.double() * a).abs().sum() + (dw.double() * b).abs().sum()
        assert abs(diff - got) <= 1e-4 * size, (diff, got, size)


def test_pieces_of_the_vocabulary():
    """More than 1 GiB of logits' gradient: two pieces in bf16."""
    from paper_2608_05448_amd import dblast as D
    B, K, R, d, V = 128, 8, 4, 64, 151936
    assert B * K * R * V * 2 > 1 << 30
    _check("bf16", B, K, R, d, V, "some", scale=2.5, seed=5)
    assert D.dbl_workspace_bytes(D.DBL_OP_HEAD_NLL_BACKWARD, B, K, R, d, V) < 3 << 30


def test_rows_do_not_depend_on_the_batch():
    from paper_2608_05448_amd import dblast as D
    for dtype, d, R in (("bf16", 64, 3), ("bf16", 2048, 2), ("bf16", 200, 3), ("bf16", 96, 2),
                        ("fp32", 40, 3)):
        h, w, x, g = [t.cuda() for t in _inputs(dtype, 40, 5, R, d, 5000, seed=9, mask="some")]
        nll, lse = D.dbl_head_nll(h, w, x)
        for b, n in ((0, 1), (3, 8), (20, 20)):
            a, c = D.dbl_head_nll(h[b:b + n].clone(), w, x[b:b + n].clone())
            assert torch.equal(a, nll[b:b + n]) and torch.equal(c, lse[b:b + n]), (dtype, d, b, n)


def test_more_positions_than_are_counted_inline():
    """Above 4096 positions one workgroup counts those that count."""
    _check("bf16", 600, 7, 1, 64, 130, "some", seed=11)
    _check("fp32", 600, 7, 1, 8, 40, "some", seed=12)


def test_runs_are_identical():
    from paper_2608_05448_amd import dblast as D
    h, w, x, g = [t.cuda() for t in _inputs("bf16", 9, 7, 6, 256, 3001, seed=13, mask="some")]
    nll, lse = D.dbl_head_nll(h, w, x)
    first = D.dbl_head_nll_backward(h, w, x, nll, lse, g)
    for _ in range(3):
        again = D.dbl_head_nll_backward(h, w, x, nll, lse, g)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_no_rows():
    from paper_2608_05448_amd import dblast as D
    for dt in (torch.bfloat16, torch.float32):
        h = torch.empty((0, 4, 2, 64), dtype=dt, device="cuda")
        w = torch.randn((300, 64), device="cuda").to(dt)
        x = torch.empty((0, 4), dtype=torch.int32, device="cuda")
        nll, lse = D.dbl_head_nll(h, w, x)
        assert nll.shape == (0, 4, 2)
        dh, dw = D.dbl_head_nll_backward(h, w, x, nll, lse, torch.empty_like(nll))
        assert dh.shape == h.shape and (dw == 0).all()
    h = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    W = torch.randn((128, 64), device="cuda").to(torch.bfloat16)
    dh, dW, dc = D.dbl_expand_branches_backward(h, W, torch.empty((0, 4, 2, 64), dtype=torch.bfloat16,
                                                                  device="cuda"))
    assert dh.shape == h.shape and (dW == 0).all() and (dc == 0).all()


EXPAND_CASES = [
    # B, K, R, d
    (1, 1, 1, 32), (1, 1, 3, 64), (1, 15, 4, 96), (2, 7, 5, 160), (3, 50, 2, 128), (5, 13, 8, 256),
    (1, 63, 2, 64), (1, 64, 2, 64), (1, 65, 2, 64), (4, 16, 64, 32), (17, 16, 3, 288), (2, 200, 2, 512),
    (5, 129, 2, 320), (9, 100, 4, 544), (1, 128, 5, 256),
    (1, 1, 1, 288), (1, 16, 3, 288), (1, 17, 2, 512), (1, 64, 1, 544), (1, 129, 2, 288), (1, 255, 2, 320),
    # 2^26 weights: the weight gradient's stream kernel with 65, 128, 201 and 256 rows, whole and partial
    # panels of 512 columns
    (1, 65, 9, 2752), (1, 128, 16, 2080), (3, 67, 8, 2912), (1, 256, 4, 4096),
    (64, 16, 2, 256), (43, 13, 4, 512), (70, 15, 1, 96), (300, 7, 3, 32),  # small weights of many rows: in parts
]


def _expand_inputs(B, K, R, d, seed=21):
    g = _gen(seed)
    bf = torch.bfloat16
    return (torch.randn((B, K, d), generator=g).to(bf),
            (torch.randn((R * d, d), generator=g) * (0.5 / d ** 0.5)).to(bf),
            torch.randn((B, K, R, d), generator=g).to(bf))


def _expand_check(h, W, dout, got):
    B, K, R, d = dout.shape
    n = R * d
    do, hd, Wd = (t.cuda().double() for t in (dout.reshape(B * K, n), h.reshape(B * K, d), W))
    want = dict(dh=do.reshape(B * K, R, d).sum(1) + do @ Wd, dW=do.T @ hd, dc=do.sum(0))
    size = dict(dh=do.abs().reshape(B * K, R, d).sum(1) + do.abs() @ Wd.abs(),
                dW=do.abs().T @ hd.abs(), dc=do.abs().sum(0))
    terms = dict(dh=n + R, dW=B * K, dc=B * K)
    for k, t in zip(("dh", "dW", "dc"), got):
        _close(t, want[k], terms[k] * 2.0 ** -24 * size[k] + 1.01 * 2.0 ** -8 * want[k].abs() + 1e-37, k)


@pytest.mark.parametrize("case", EXPAND_CASES, ids=["-".join(map(str, c)) for c in EXPAND_CASES])
def test_expander_backward(case):
    from paper_2608_05448_amd import dblast as D
    print(f"[expander backward] {case}", flush=True)
    h, W, dout = _expand_inputs(*case)
    got = D.dbl_expand_branches_backward(h.cuda(), W.cuda(), dout.cuda())
    _expand_check(h, W, dout, got)
    # any of the outputs alone is the same
    for i, kw in enumerate((dict(want_dW=False, want_dc=False), dict(want_dh=False, want_dc=False),
                            dict(want_dh=False, want_dW=False))):
        alone = D.dbl_expand_branches_backward(h.cuda(), W.cuda(), dout.cuda(), **kw)
        assert torch.equal(alone[i], got[i]) and all(alone[j] is None for j in range(3) if j != i)


@pytest.mark.parametrize("case", [(1, 15, 4, 96), (5, 13, 8, 288), (3, 50, 2, 512), (3, 100, 2, 320),
                                  (9, 100, 4, 544), (3, 67, 8, 2912)], ids=str)
def test_expander_backward_infinities_stay_infinities(case):
    """An infinity in the last row, next to what the kernels pad the sums with: the results are infinite
    where the formula's are, and finite elsewhere."""
    from paper_2608_05448_amd import dblast as D
    B, K, R, d = case
    h, W, dout = _expand_inputs(*case)
    dout[-1, -1, -1, 5] = float("inf")
    dout[0, 0, 0, 0] = -float("inf")
    h, W = torch.where(h == 0, 1.0, h), torch.where(W == 0, 1.0, W)
    got = D.dbl_expand_branches_backward(h.cuda(), W.cuda(), dout.cuda())
    do, hd, Wd = (t.cuda().double() for t in (dout.reshape(B * K, R * d), h.reshape(B * K, d), W))
    dh = do.reshape(B * K, R, d).sum(1) + do @ Wd
    for t, want in zip(got, (dh.reshape(B, K, d), do.T @ hd, do.sum(0))):
        inf = torch.isinf(want)
        assert inf.any() and torch.equal(t.double()[inf], want[inf])
        assert torch.isfinite(t[torch.isfinite(want)]).all()


def test_expander_backward_matches_differences():
    """dh, dW and dc against differences of the forward call's own map in binary64 (it is linear in each
    argument, so that a difference of any step is exact)."""
    from paper_2608_05448_amd import dblast as D
    B, K, R, d = 1, 5, 3, 64
    h, W, dout = _expand_inputs(B, K, R, d, seed=22)
    dh, dW, dc = (t.cpu().double() for t in
                  D.dbl_expand_branches_backward(h.cuda(), W.cuda(), dout.cuda()))
    g = _gen(23)
    c = torch.zeros(R * d, dtype=torch.float64)

    def out(hh, WW, cc):
        return ((hh @ WW.T + cc).reshape(B, K, R, d) + hh[:, :, None]).double()

    hd, Wd, do = h.double(), W.double(), dout.double()
    base = (out(hd, Wd, c) * do).sum()
    for arg, grad in ((0, dh), (1, dW), (2, dc)):
        v = torch.randn(grad.shape, generator=g, dtype=torch.float64)
        args = [hd, Wd, c]
        args[arg] = args[arg] + v
        diff = (out(*args) * do).sum() - base
        assert abs(diff - (grad * v).sum()) <= 1.1 * 2.0 ** -8 * (grad * v).abs().sum()


def _step(D, s, want_dw=True, ws=None):
    """A fine-tuning step's gradients for the block NLL of the latent mixture (Eq. dependent-nll), and
    their clipping: the loss -log sum_z pi_z prod_k q_k(x_k | z), averaged over blocks."""
    h, W, c, w, x, ell = s
    R = ell.shape[1]
    branch = D.dbl_expand_branches(h, W, c, R)
    nll, lse = D.dbl_head_nll(branch, w, x)
    joint = torch.log_softmax(ell, -1) - nll.sum(1)
    loss = -torch.logsumexp(joint, -1).mean()
    resp = torch.softmax(joint, -1) / len(ell)
    g = resp[:, None].expand_as(nll).contiguous()
    dell = torch.softmax(ell, -1) / len(ell) - resp
    dbranch, dw = D.dbl_head_nll_backward(branch, w, x, nll, lse, g, want_dw=want_dw)
    dh, dW, dc = D.dbl_expand_branches_backward(h, W, dbranch)
    grads = [dW, dc, dell] + ([dw] if want_dw else [])
    norm = D.dbl_grad_norm(grads)
    D.dbl_clip_grads(grads, norm, 0.05)
    return [loss, norm, dh] + grads


def _step_inputs(B, K, R, d, V, seed):
    g = _gen(seed)
    bf = torch.bfloat16
    x = torch.randint(0, V, (B, K), generator=g, dtype=torch.int32)
    x[1::2, -2:] = -1
    return [torch.randn((B, K, d), generator=g).to(bf),
            (torch.randn((R * d, d), generator=g) * (0.5 / d ** 0.5)).to(bf),
            (torch.randn(R * d, generator=g) * 0.1).to(bf),
            (torch.randn((V, d), generator=g) * (1.5 / d ** 0.5)).to(bf), x,
            torch.randn((B, R), generator=g)]


def test_training_step_against_autograd():
    """The whole chain against binary64 autograd of the loss. The branch states, their gradient and the
    results are rounded to bf16 on the way, so the gradients agree to a few 2^-8 of their size."""
    from paper_2608_05448_amd import dblast as D
    B, K, R, d, V = 4, 6, 3, 128, 700
    cpu = _step_inputs(B, K, R, d, V, 31)
    got = _step(D, [t.cuda() for t in cpu])
    h, W, c, w, x, ell = [t.double().requires_grad_() if t.dtype != torch.int32 else t for t in cpu]
    branch = h[:, :, None] + (h @ W.T + c).reshape(B, K, R, d)
    z = branch @ w.T
    on = (x >= 0)[:, :, None]
    n = torch.logsumexp(z, -1) - z.gather(-1, x.long().clamp_min(0)[:, :, None, None].expand(B, K, R, 1))[..., 0]
    loss = -torch.logsumexp(torch.log_softmax(ell, -1) - torch.where(on, n, 0.0).sum(1), -1).mean()
    loss.backward()
    norm = torch.sqrt(sum((t.grad ** 2).sum() for t in (W, c, ell, w)))
    scale = min(1.0, 0.05 / (norm.item() + 1e-6))
    assert scale < 1.0
    # A branch state is off by 2^-8 of its size: each logit by about 2^-8 sqrt(sum (h w)^2) ~ 0.01, each
    # block's log-likelihoods by about sqrt(K) times that, and the responsibilities with them.
    assert abs(got[0].item() - loss.item()) < 0.05
    for name, t, want in (("norm", got[1], norm), ("dh", got[2], h.grad), ("dW", got[3], W.grad * scale),
                          ("dc", got[4], c.grad * scale), ("dell", got[5], ell.grad * scale),
                          ("dw", got[6], w.grad * scale)):
        err = (t.cpu().double() - want).norm() / want.norm()
        print(f"[step] {name}: relative error {err:.2e}", flush=True)
        assert err < 0.05, (name, err)


def test_captured_steps_share_a_workspace():
    """The step captured into two graphs, whose calls may share one workspace as they are replayed in
    turn; every replay equals the eager step, with eager work between the replays."""
    from paper_2608_05448_amd import dblast as D
    sets = [[t.cuda() for t in _step_inputs(4, 6, 3, 128, 1500, s)] for s in (41, 42)]
    ws = torch.empty(max(D.dbl_workspace_bytes(op, 4, 6, 3, 128, 1500)
                         for op in (D.DBL_OP_HEAD_NLL, D.DBL_OP_HEAD_NLL_BACKWARD,
                                    D.DBL_OP_EXPAND_BACKWARD)), dtype=torch.uint8, device="cuda")

    def step(s, o):
        h, W, c, w, x, ell = s
        D.dbl_expand_branches(h, W, c, 3, out=o["branch"])
        D.dbl_head_nll(o["branch"], w, x, nll=o["nll"], lse=o["lse"], ws=ws)
        D.dbl_head_nll_backward(o["branch"], w, x, o["nll"], o["lse"], o["g"], dh=o["dbranch"],
                                dw=o["dw"], ws=ws)
        D.dbl_expand_branches_backward(h, W, o["dbranch"], dh=o["dh"], dW=o["dW"], dc=o["dc"], ws=ws)
        grads = [o["dw"], o["dW"], o["dc"]]
        D.dbl_grad_norm(grads, norm=o["norm"], ws=o["nws"])
        D.dbl_clip_grads(grads, o["norm"], 0.05)

    def buffers(s):
        h, W, c, w, x, ell = s
        B, K, d = h.shape
        e = lambda *n: torch.empty(n, dtype=torch.bfloat16, device="cuda")
        return dict(branch=e(B, K, 3, d), dbranch=e(B, K, 3, d), dh=e(B, K, d), dW=torch.empty_like(W),
                    dc=torch.empty_like(c), dw=torch.empty_like(w),
                    nll=torch.empty((B, K, 3), device="cuda"), lse=torch.empty((B, K, 3), device="cuda"),
                    norm=torch.empty((), device="cuda"),
                    nws=torch.empty(1 << 14, dtype=torch.uint8, device="cuda"),
                    g=torch.full((B, K, 3), 0.01, device="cuda"))

    outs, eager, graphs = [], [], []
    for s in sets:
        o = buffers(s)
        step(s, o)
        torch.cuda.synchronize()
        outs.append(o)
        eager.append({k: v.clone() for k, v in o.items() if k != "nws"})
    for s, o in zip(sets, outs):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(s, o)
        graphs.append(gr)
    for rep in range(3):
        for o, want, gr in zip(outs, eager, graphs):
            for k, v in o.items():
                if k not in ("g", "nws"):
                    v.fill_(-7)
            ws.fill_(255)
            torch.cuda.synchronize()
            gr.replay()
            torch.cuda.synchronize()
            for k, v in want.items():
                assert torch.equal(o[k], v), (rep, k)
        print(f"[graph] replay {rep} identical", flush=True)


def test_on_another_stream():
    from paper_2608_05448_amd import dblast as D
    s = [t.cuda() for t in _step_inputs(4, 6, 3, 128, 1500, 51)]
    want = _step(D, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _step(D, s)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)

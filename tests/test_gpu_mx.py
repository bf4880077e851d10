"""Microscaled rows on the GPU: quantisation and back, the norm, the products and the head, against plain
binary64 forms.

Bounds, from the roundings that the operators make (half a step: bf16 2^-8, fp32 2^-24, relative):
 quantise, dequantise   none: powers of two and one rounding that the format defines
 norm     the sum of d squares, at most 32 of them in a row in one register and then a tree of 8 levels
          (longer rows: d / 2048 in a row), half of its relative error after the root, a division, a root, an
          addition and two products: (d / 256 + 40) 2^-24 of y; codes and scales lie between those of y (1 - e) and y (1 + e)
 logits   the products are exact in fp32 and 64 of them are added at a time: dp 2^-24 sum |h w|; with
          8-bit states and bf16 logits each product is cut at 2^-13 of the largest exponent in its group of
          eight, 7 of them: 7 2^-13 sum over groups (max|h| max|w|); bf16 logits 2^-8 more of themselves
 head     logits as fp32's; a tile's log-mass the largest of its logits' bounds and 2^-21 (1 + |lmass|) for
          128 exponentials, their sum and a logarithm (__expf and __logf: 2^-21); tls both
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
DT = {"bf16": BF, "fp32": F32}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _table(bits):
    if bits == 4:
        return torch.tensor(E2M1, dtype=torch.float64)
    return torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()


def _nearest(a, bits):
    """Index of the code nearest to a >= 0, ties to the even index, saturating."""
    t = _table(bits)
    mid = (t[1:] + t[:-1]) / 2
    lo, hi = torch.searchsorted(mid, a), torch.searchsorted(mid, a, right=True)
    return torch.where(lo % 2 == 0, lo, hi)


def _blocks(x, dp):
    full = torch.zeros((*x.shape[:-1], dp), dtype=torch.float64)
    full[..., :x.shape[-1]] = x.double()
    return full.unflatten(-1, (dp // 32, 32))


def _scale_bytes(b, bits):
    """Scale byte of blocks b [..., n, 32] in binary64; 255 where one holds an infinity or NaN."""
    top = b.abs().amax(-1)
    bad = ~torch.isfinite(b).all(-1)
    _, e = torch.frexp(torch.where(bad, 1.0, top))
    e = torch.where(top > 0, e - 1, -1000) - (2 if bits == 4 else 8)
    return torch.where(bad, 255, e.clamp(min=-127) + 127)


def _quantize(x, bits):
    """(signed values over their scale [..., dp], scale bytes [..., dp / 32])."""
    dp = (x.shape[-1] + 127) // 128 * 128
    b = _blocks(x, dp)
    byte = _scale_bytes(b, bits)
    bad = byte == 255
    s = torch.ldexp(torch.ones((), dtype=torch.float64), byte - 127)[..., None]
    q = _table(bits)[_nearest(torch.where(bad[..., None], 0.0, (b / s).abs()), bits)]
    q = torch.where(torch.signbit(b), -q, q)
    return torch.where(bad[..., None], 0.0, q).flatten(-2), byte


def _unpack(codes):
    """Values over the scale from codes on the GPU."""
    if codes.dtype == torch.uint8:
        c = codes.cpu().long()
        t = torch.cat([_table(4), -_table(4)])
        return torch.stack([t[c & 15], t[c >> 4]], -1).flatten(-2)
    return codes.cpu().double()


def _values(codes, scales):
    byte = scales.cpu().view(torch.uint8).long()
    s = torch.ldexp(torch.ones((), dtype=torch.float64), byte - 127)
    s = torch.where(byte == 255, torch.nan, s)
    return (_unpack(codes).unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def _data(M, d, dtype, seed, scale=1.0):
    g = _gen(seed)
    x = torch.randn((M, d), generator=g) * torch.exp(2 * torch.randn((M, d), generator=g)) * scale
    return x.to(DT[dtype])


SIZES = [(1, 1), (1, 32), (3, 33), (2, 127), (5, 128), (7, 129), (4, 200), (300, 64), (9, 1000), (2, 2560),
         (1, 8200), (65, 4096), (257, 1001)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_quantisation_and_back_are_exact(dtype, bits):
    from paper_2608_05448_amd import dblast as D
    for M, d in SIZES:
        print(f"[quant] {dtype} {bits} {M}x{d}", flush=True)
        x = _data(M, d, dtype, M * 7 + d)
        codes, scales = D.dbl_mx_quantize(x.cuda(), bits=bits)
        q, byte = _quantize(x, bits)
        assert torch.equal(scales.cpu().view(torch.uint8).long(), byte), (M, d)
        assert torch.equal(_unpack(codes), q), (M, d)
        out = D.dbl_mx_dequantize(codes, scales, d, dtype=F32)
        want = _values(codes, scales)[:, :d]
        assert torch.equal(out.cpu().double(), want), (M, d)
        assert torch.equal(D.dbl_mx_dequantize(codes, scales, d).cpu().double(), want), (M, d)


@pytest.mark.parametrize("bits", [4, 8])
def test_quantisation_of_every_border(bits):
    """Halfway points, their neighbours, zeros of both signs, subnormals, the largest numbers, and blocks
    with infinities and NaN beside whole ones."""
    from paper_2608_05448_amd import dblast as D
    t = _table(bits)
    mid = torch.cat([(t[1:] + t[:-1]) / 2, t])
    f = mid.float()
    near = torch.cat([f, torch.nextafter(f, torch.tensor(1e9)), torch.nextafter(f, torch.tensor(0.0))])
    near = torch.cat([near, -near, torch.tensor([0.0, -0.0])])
    top = float(t[-1])
    near = near[torch.randperm(len(near), generator=_gen(1))]
    near = torch.cat([near, torch.zeros(-len(near) % 31)]).reshape(-1, 31)
    rows = torch.cat([torch.full((len(near), 1), top), near], 1)  # a block each, its scale 1
    x = torch.cat([rows.flatten(), torch.zeros(-rows.numel() % 128)]).reshape(-1, 128)
    big = torch.finfo(torch.float32).max
    special = torch.zeros((6, 128))
    special[0, :4] = torch.tensor([1e-45, -1e-44, 1e-40, 3e-39])
    special[1, 0], special[1, 40], special[1, 70] = float("nan"), float("inf"), 1.0
    special[2, 0], special[2, 1] = -float("inf"), 5.0
    special[3, :3] = torch.tensor([big, -big, 1e30])
    special[4, :] = -0.0
    special[5, :2] = torch.tensor([2.0 ** -126, 2.0 ** -149])
    for scale in (1.0, 2.0 ** 90, 2.0 ** -100):
        y = torch.cat([x * scale, special])
        codes, scales = D.dbl_mx_quantize(y.cuda(), bits=bits)
        q, byte = _quantize(y, bits)
        assert torch.equal(scales.cpu().view(torch.uint8).long(), byte)
        assert torch.equal(_unpack(codes), q)
        out = D.dbl_mx_dequantize(codes, scales, 128, dtype=F32).cpu().double()
        want = _values(codes, scales)
        assert torch.equal(torch.isnan(out), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want.float().double()))


def _between(codes, scales, y, e, bits):
    """Whether codes and scales are those of values within a relative e of y."""
    dp = codes.shape[-1] * 8 // bits
    b = _blocks(y, dp)
    byte = scales.cpu().view(torch.uint8).long()
    lo, hi = _scale_bytes(b * (1 - e), bits), _scale_bytes(b * (1 + e), bits)
    assert bool(((byte >= lo) & (byte <= hi)).all())
    s = torch.ldexp(torch.ones((), dtype=torch.float64), byte - 127)[..., None]
    a = (b / s).abs().flatten(-2)
    got = _unpack(codes)
    t = _table(bits)
    assert bool((got.abs() >= t[_nearest(a * (1 - e), bits)]).all())
    assert bool((got.abs() <= t[_nearest(a * (1 + e), bits)]).all())
    assert bool((torch.signbit(got) == torch.signbit(b.flatten(-2)))[a > 0].all())


NORM_SIZES = [(1, 1), (3, 5), (5, 64), (4, 512), (3, 513), (2, 1000), (6, 1001), (3, 2560), (2, 4096), (2, 8192),
              (2, 8200), (1, 20001)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("residual", [True, False])
def test_norm(dtype, residual, bits):
    from paper_2608_05448_amd import dblast as D
    for M, d in NORM_SIZES:
        print(f"[norm] {dtype} {bits} residual={residual} {M}x{d}", flush=True)
        x = _data(M, d, dtype, d)
        r = _data(M, d, dtype, d + 1) if residual else None
        w = (1 + 0.3 * torch.randn(d, generator=_gen(d + 2))).to(DT[dtype])
        got = D.dbl_add_rmsnorm_mx(x.cuda(), r.cuda() if residual else None, w.cuda(), eps=1e-5, bits=bits,
                                   want_y=True)
        h = x
        if residual:
            h = (x.float() + r.float()).to(DT[dtype])
            assert torch.equal(got[0].cpu(), h)
        else:
            assert got[0] is None
        hd = h.double()
        y = hd / torch.sqrt((hd * hd).mean(-1, keepdim=True) + 1e-5) * w.double()
        e = (d / 256 + 40) * 2.0 ** -24
        _between(got[1], got[2], y, e, bits)
        half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        assert bool(((got[3].cpu().double() - y).abs() <= (half * (1 + e) + e) * y.abs() + 1e-40).all())
        # the same codes without y
        again = D.dbl_add_rmsnorm_mx(x.cuda(), r.cuda() if residual else None, w.cuda(), eps=1e-5, bits=bits)
        assert torch.equal(again[1].view(torch.uint8), got[1].view(torch.uint8))
        assert torch.equal(again[2].view(torch.uint8), got[2].view(torch.uint8))


@pytest.mark.parametrize("d", [200, 2560, 9000, 1001])
def test_norm_in_place(d):
    from paper_2608_05448_amd import dblast as D
    x, r, w = _data(3, d, "bf16", 5).cuda(), _data(3, d, "bf16", 6).cuda(), torch.ones(d, dtype=BF).cuda()
    want = D.dbl_add_rmsnorm_mx(x, r, w)
    for name in ("x", "residual"):
        a, b = x.clone(), r.clone()
        got = D.dbl_add_rmsnorm_mx(a, b, w, sum=a if name == "x" else b)
        assert got[0].data_ptr() == (a if name == "x" else b).data_ptr()
        for g, t in zip(got, want):
            assert torch.equal(g.view(torch.uint8), t.view(torch.uint8)), (d, name)


def test_norm_rows_with_nothing_or_nan():
    from paper_2608_05448_amd import dblast as D
    x = torch.randn((4, 100), generator=_gen(1))
    x[0] = 0.0
    x[1, 3] = float("nan")
    x[2, 50] = float("inf")
    _, codes, scales, y = D.dbl_add_rmsnorm_mx(x.cuda(), None, torch.ones(100).cuda(), want_y=True)
    v = _values(codes, scales)
    assert bool((v[0] == 0).all())
    assert bool(torch.isnan(v[1, :96]).all()) and bool(torch.isnan(y[1]).all())
    # an infinite value makes the root infinite: the others are 0, its own is NaN, and its block with it
    assert bool(torch.isnan(v[2, 32:64]).all()) and bool((v[2, :32] == 0).all())
    assert bool(torch.isfinite(v[3]).all())


def _operands(M, V, d, bits, seed=3):
    """Microscaled operands on the GPU, their values in binary64, and sums of absolute products."""
    from paper_2608_05448_amd import dblast as D
    g = _gen(seed)
    h = torch.randn((M, d), generator=g) * torch.exp(torch.randn((M, d), generator=g))
    h[:, 0] *= 20
    w = torch.randn((V, d), generator=g) * (1.5 / d ** 0.5)
    h, w = D.dbl_mx_quantize(h.to(BF).cuda(), bits=bits), D.dbl_mx_quantize(w.to(BF).cuda(), bits=4)
    hd, wd = _values(*h), _values(*w)
    return h, w, hd, wd


def _logit_bound(hd, wd, bits, dtype):
    e = hd.shape[1] * 2.0 ** -24 * (hd.abs() @ wd.abs().T)
    if dtype == BF:
        if bits == 8:
            top = [v.abs().unflatten(-1, (-1, 8)).amax(-1) for v in (hd, wd)]
            e = e + 7 * 2.0 ** -13 * 2 * (top[0] @ top[1].T)  # an exponent is up to half a value
        e = e * (1 + 2.0 ** -8) + 2.0 ** -8 * (hd @ wd.T).abs()
    return e


SHAPES = [(1, 1, 1), (1, 5, 64), (3, 127, 33), (17, 1000, 200), (32, 129, 128), (33, 256, 512), (64, 1001, 1000),
          (65, 640, 96), (128, 300, 256), (129, 2049, 384), (260, 515, 1024), (5, 50257, 64),
          (513, 33000, 512), (70, 400, 2560)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_matmul(dtype, bits):
    from paper_2608_05448_amd import dblast as D
    for M, V, d in SHAPES:
        print(f"[matmul] {dtype} {bits} {M}x{V}x{d}", flush=True)
        h, w, hd, wd = _operands(M, V, d, bits)
        out = torch.full((M * V + 64,), 7.0, dtype=DT[dtype], device="cuda")
        got = D.dbl_mx_matmul(*h, *w, dtype=DT[dtype], out=out[:M * V].view(M, V))
        assert bool((out[M * V:] == 7.0).all()), "written behind the logits"
        err = (got.cpu().double() - hd @ wd.T).abs()
        assert bool((err <= _logit_bound(hd, wd, bits, DT[dtype])).all()), (M, V, d, float(err.max()))


def test_products_of_all_codes():
    """Every e4m3 code against every e2m1 code beside the largest ones of both, in fp32: nothing is cut."""
    from paper_2608_05448_amd import dblast as D
    codes = torch.arange(256, dtype=torch.uint8)
    codes = codes[(codes & 127) != 127]
    M = len(codes)
    h = torch.zeros((M, 128), dtype=torch.uint8)
    h[:, 0], h[:, 1] = codes, 126              # 448 in the same group of eight
    w = torch.zeros((16, 64), dtype=torch.uint8)
    w[:, 0] = torch.arange(16, dtype=torch.uint8) + 16 * 7  # 6
    one = lambda n: torch.full((n, 4), 127, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    hq, hs, wq, ws = h.view(torch.float8_e4m3fn).cuda(), one(M).cuda(), w.cuda(), one(16).cuda()
    got = D.dbl_mx_matmul(hq, hs, wq, ws).cpu().double()
    want = _values(hq, hs) @ _values(wq, ws).T
    assert bool(((got - want).abs() <= 2.0 ** -23 * want.abs()).all())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("argmax", [False, True])
def test_head(bits, argmax):
    from paper_2608_05448_amd import dblast as D
    for (B, K, R), V, d in [((1, 1, 1), 1, 8), ((1, 4, 2), 256, 64), ((2, 5, 3), 1001, 200), ((1, 13, 5), 129, 1000),
                            ((3, 11, 4), 640, 128), ((2, 17, 8), 2000, 512)]:
        M = B * K * R
        print(f"[head] {bits} {M}x{V}x{d}", flush=True)
        h, w, hd, wd = _operands(M, V, d, bits)
        h = [t.reshape(B, K, R, -1) for t in h]
        got = D.dbl_mx_head_logprobs(*h, *w, argmax=argmax)
        z = hd @ wd.T
        e = _logit_bound(hd, wd, bits, F32)
        nT = (V + 127) // 128
        pad = torch.full((M, nT * 128), -np.inf, dtype=torch.float64)
        pad[:, :V] = z
        lm = torch.logsumexp(pad.unflatten(-1, (nT, 128)), -1)
        pe = torch.zeros((M, nT * 128), dtype=torch.float64)
        pe[:, :V] = e
        le = pe.unflatten(-1, (nT, 128)).amax(-1) + 2.0 ** -21 * (1 + lm.abs())
        tls = z - lm.repeat_interleave(128, 1)[:, :V]
        te = e + le.repeat_interleave(128, 1)[:, :V] + 2.0 ** -24 * tls.abs()
        lse = torch.logsumexp(lm, 1)
        assert bool(((got[0].cpu().double().reshape(M, V) - tls).abs() <= te).all()), (M, V, d)
        assert bool(((got[1].cpu().double().reshape(M, nT) - lm).abs() <= le).all()), (M, V, d)
        se = le.amax(1) + 2.0 ** -20 * (1 + lse.abs())
        assert bool(((got[2].cpu().double().reshape(M) - lse).abs() <= se).all()), (M, V, d)
        if argmax:
            pick = got[3].cpu().reshape(M).long()
            best = z.amax(1)
            assert bool((z.gather(1, pick[:, None])[:, 0] >= best - 2 * e.amax(1)).all())
            logits = D.dbl_mx_matmul(*h, *w).cpu().reshape(M, V)
            assert torch.equal(pick, logits.argmax(1))  # the same fp32 logits; the lowest id


@pytest.mark.parametrize("bits", [4, 8])
def test_rows_do_not_depend_on_the_batch(bits):
    from paper_2608_05448_amd import dblast as D
    h, w, _, _ = _operands(300, 1000, 384, bits)
    for dtype in (F32, BF):
        whole = D.dbl_mx_matmul(*h, *w, dtype=dtype)
        for a, b in [(0, 1), (5, 37), (100, 164), (170, 299), (299, 300)]:
            part = D.dbl_mx_matmul(h[0][a:b].clone(), h[1][a:b].clone(), *w, dtype=dtype)
            assert torch.equal(part, whole[a:b]), (a, b)


def test_nan_scale_reaches_its_rows_and_columns_only():
    from paper_2608_05448_amd import dblast as D
    for bits in (4, 8):
        h, w, hd, wd = _operands(40, 200, 256, bits)
        h[1].view(torch.uint8)[3, 2] = 255
        w[1].view(torch.uint8)[7, 5] = 255
        for dtype in (F32, BF):
            nan = torch.isnan(D.dbl_mx_matmul(*h, *w, dtype=dtype)).cpu()
            want = torch.zeros_like(nan)
            want[3], want[:, 7] = True, True
            assert torch.equal(nan, want)


def test_empty_batches():
    from paper_2608_05448_amd import dblast as D
    codes, scales = D.dbl_mx_quantize(torch.empty((0, 100), device="cuda"))
    assert codes.shape == (0, 64) and scales.shape == (0, 4)
    assert D.dbl_mx_dequantize(codes, scales, 100).shape == (0, 100)
    w = D.dbl_mx_quantize(torch.ones((7, 100), device="cuda"))
    assert D.dbl_mx_matmul(codes, scales, *w).shape == (0, 7)
    got = D.dbl_add_rmsnorm_mx(torch.empty((0, 100), device="cuda"), None, torch.ones(100, device="cuda"))
    assert got[1].shape == (0, 128)


def test_serving_chain_and_graph():
    """A step as a server makes it: norm, codes, 4-bit head, draw; and the drafter's: expander, codes, head,
    block draw, verification. Captured once; replays between eager work give the eager results."""
    from paper_2608_05448_amd import dblast as D
    B, K, R, d, V = 3, 5, 4, 256, 3001
    g = _gen(9)
    dev = "cuda"
    x, res = torch.randn((B, K + 1, d), generator=g).to(BF).to(dev), torch.randn((B, K + 1, d), generator=g).to(BF).to(dev)
    nw = torch.ones(d, dtype=BF, device=dev)
    wq, ws = D.dbl_mx_quantize((torch.randn((V, d), generator=g) * 0.15).to(BF).to(dev))
    W = (torch.randn((R * d, d), generator=g) * 0.02).to(BF).to(dev)
    c = torch.zeros(R * d, dtype=BF, device=dev)
    prior = torch.randn((B, R), generator=g).to(dev)
    words = torch.randint(-2 ** 31, 2 ** 31, (B, K + 1), generator=g).to(torch.int32).to(dev)
    temps = torch.tensor([0.7, 0.0, 1.2])[:, None].expand(B, K + 1).contiguous().to(dev)

    def step():
        total, q, s = D.dbl_add_rmsnorm_mx(x, res, nw)
        logits = D.dbl_mx_matmul(q, s, wq, ws)
        token, lp = D.dbl_sample_logits(logits, words, temperature=temps, top_p=0.9, min_p=0.01)
        logp = D.dbl_target_logprobs(logits, temperature=0.7)
        h = D.dbl_expand_branches(total[:, :K].contiguous(), W, c, R)
        hq, hs = D.dbl_mx_quantize(h, bits=8)
        tls, lmass, lse, best = D.dbl_mx_head_logprobs(hq, hs, wq, ws, argmax=True)
        z, xs = D.dbl_sample_block(tls, lmass, lse, prior, seed=4, step=1)
        out = D.dbl_verify_block(tls, lmass, lse, prior, xs, logp, seed=4, step=1)
        return [total, q.view(torch.uint8), s.view(torch.uint8), logits, token, lp, tls, lmass, lse, best, z, xs,
                out["n_accept"], out["next_token"]]

    eager = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for t, e in zip(other, eager):
        assert torch.equal(t, e)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for _ in range(3):
        for t in kept:
            t.fill_(3)
        step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, e in zip(kept, eager):
            assert torch.equal(t, e)
    # the drafted tokens' probabilities are those of the values that the codes stand for
    h = D.dbl_expand_branches(eager[0][:, :K].contiguous(), W, c, R)
    hq, hs = D.dbl_mx_quantize(h, bits=8)
    z = _values(hq, hs).reshape(-1, d) @ _values(wq, ws).T
    lq = torch.log_softmax(z, 1).reshape(B, K, R, V)
    nT = D.ntiles(V)
    got = (eager[6].cpu().double() + (eager[7].cpu().double() - eager[8].cpu().double()[..., None])
           .repeat_interleave(128, -1)[..., :V])
    assert nT == eager[7].shape[-1] and float((got - lq).abs().max()) < 1e-4

"""What the low-precision serving operators state of themselves, at the places where it is decided: the norm's
codes and y are those of the exact value and its padding is what quantising y gives, no product of 8-bit states
is cut where the result is binary32, a row does not depend on the batch for any tile, and the draw over more
than 64 segments and of rows that its list does not hold.

Bounds. The norm is computed in binary64 (half a step 2^-53): squares are exact (24 bits each), and are added
8 ceil(dp / 2048) at a time in a register and then by 8 levels; after the root half of that error is left, and a
division, an addition, a root, a division and two products follow, each within one step: y lies within
(dp / 512 + 24) 2^-53 of the exact one, which is formed here in 64-bit significands. Away from a border by more,
code and rounding are fixed. Products: see each test."""
import numpy as np
import pytest
import torch

from test_gpu_draw import check, rand_logits, rand_words
from test_gpu_mx import _operands, _table, _values

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
LD = np.longdouble


def _exact_norm(h, w, eps):
    """y of rows h and weight w (tensors) in 64-bit significands, and the kernel's relative bound."""
    h, w = h.double().numpy().astype(LD), w.double().numpy().astype(LD)
    d = h.shape[-1]
    y = h / np.sqrt((h * h).sum(-1, keepdims=True) / LD(d) + LD(np.float32(eps))) * w
    return y, ((d + 127) // 128 * 128 / 512 + 24) * 2.0 ** -53


def _coded(y, bits):
    """(magnitude index of the code, scale's byte) of y [M, d] in 64-bit significands, d a multiple of 128."""
    b = y.reshape(len(y), -1, 32)
    top = np.abs(b).max(-1)
    power = np.frexp(top)[1].astype(np.int64) - 1 - (2 if bits == 4 else 8)
    a = np.abs(b) / np.ldexp(LD(1), power)[..., None]
    t = _table(bits).numpy().astype(LD)
    mid = (t[1:] + t[:-1]) / 2
    lo, hi = np.searchsorted(mid, a), np.searchsorted(mid, a, side="right")
    return np.where(lo % 2 == 0, lo, hi).reshape(y.shape), power + 127


def _index(codes):
    """Magnitude index of codes on the GPU."""
    if codes.dtype == torch.uint8:
        c = codes.cpu().long()
        return torch.stack([c & 7, (c >> 4) & 7], -1).flatten(-2).numpy()
    return (codes.cpu().view(torch.uint8).long() & 127).numpy()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("d", [512, 4096, 9088])
def test_norm_codes_beside_a_border_are_on_their_own_side(bits, d):
    """Weights one step of binary32 below and above the number that would put y on a border between two
    codes: y lies within 2^-23 of the border, where a norm in binary32 takes the neighbour for many."""
    from paper_2608_05448_amd import dblast as D
    g = torch.Generator().manual_seed(d + bits)
    x = (torch.randn((1, d), generator=g).abs() + 0.3) * torch.where(torch.rand((1, d), generator=g) < 0.5, -1.0, 1.0)
    y1, e = _exact_norm(x, torch.ones(d), 1e-5)
    t = _table(bits).numpy().astype(LD)
    mid = ((t[1:] + t[:-1]) / 2)
    mid = mid[mid > t[-1] / 128]                 # borders of normal and the larger subnormal codes
    pick = torch.randint(0, len(mid), (d,), generator=g).numpy()
    want = np.where(np.arange(d) % 32 == 0, t[-1] * LD(0.999), mid[pick])
    w = (want / np.abs(y1[0])).astype(np.float32)
    below = torch.rand(d, generator=g).numpy() < 0.5
    over = w.astype(LD) * np.abs(y1[0]) > want
    w = np.where(below & over, np.nextafter(w, np.float32(0)), w)
    w = np.where(~below & ~over, np.nextafter(w, np.float32(1e30)), w).astype(np.float32)
    w = torch.from_numpy(w)
    y, e = _exact_norm(x, w, 1e-5)
    low, high = _coded(y * (1 - LD(e)), bits), _coded(y * (1 + LD(e)), bits)
    sure = low[0] == high[0]
    assert sure.mean() > 0.999 and np.array_equal(low[1], high[1])
    # the same through binary32 differs: the planted values do what they are for
    s = np.float32(1) / np.sqrt((x.numpy() ** 2).mean(dtype=np.float32) + np.float32(1e-5))
    y32 = (x.numpy() * s * w.numpy()).astype(LD)
    assert (_coded(y32, bits)[0] != low[0])[sure].sum() > d // 50
    _, codes, scales = D.dbl_add_rmsnorm_mx(x.cuda(), None, w.cuda(), eps=1e-5, bits=bits)
    assert np.array_equal(scales.cpu().view(torch.uint8).long().numpy(), low[1])
    assert np.array_equal(_index(codes)[sure], low[0][sure])


def _to_bf16(y):
    """Exact numbers rounded once to bf16 (normal ones), ties to even."""
    m, e = np.frexp(y)
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def test_norm_result_in_bf16_is_rounded_once():
    """Of 2^21 values some lie so near to the middle of two bf16 numbers that a rounding to binary32 on the
    way puts them on it, and a second one on the wrong side."""
    from paper_2608_05448_amd import dblast as D
    M, d = 512, 4096
    g = torch.Generator().manual_seed(3)
    x = torch.randn((M, d), generator=g).to(BF)
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(BF)
    y, e = _exact_norm(x, w, 1e-6)
    once = _to_bf16(y)
    sure = _to_bf16(y * (1 - LD(e))) == _to_bf16(y * (1 + LD(e)))
    twice = torch.from_numpy(y.astype(np.float32)).to(BF).double().numpy().astype(LD)
    assert (~sure).sum() < 10 and (twice != once)[sure].sum() >= 3
    got = D.dbl_add_rmsnorm_mx(x.cuda(), None, w.cuda(), eps=1e-6, want_y=True)[3]
    got = got.cpu().double().numpy().astype(LD)
    assert np.array_equal(got[sure], once[sure])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [1, 33, 100, 200, 1000, 1001, 4104, 9000])
def test_norm_padding_is_that_of_the_quantised_result(d, dtype, bits):
    """Rows of zeros without eps, with NaN and with infinities have their padding as any other: code 0 under
    the smallest scale, as quantising y gives it."""
    from paper_2608_05448_amd import dblast as D
    x = torch.randn((5, d), generator=torch.Generator().manual_seed(d))
    x[0] = 0.0
    x[1, d // 2] = float("nan")
    x[2, d - 1] = float("inf")
    x[3, 0] = -float("inf")
    x = x.to(dtype).cuda()
    w = torch.ones(d, dtype=dtype).cuda()
    _, codes, scales, y = D.dbl_add_rmsnorm_mx(x, None, w, eps=0.0, bits=bits, want_y=True)
    want = D.dbl_mx_quantize(y, bits=bits)
    dp, blocks = D.mx_row(d), (d + 31) // 32
    s = scales.view(torch.uint8).cpu()
    assert s.shape == (5, dp // 32)
    assert bool((s[:, blocks:] == 0).all()), "scale of a block of padding"
    broken = want[1].view(torch.uint8).cpu() == 255
    assert torch.equal(s == 255, broken)
    assert bool((codes.view(torch.uint8).cpu()[:, blocks * 4 * bits:] == 0).all()), "codes of padding"


@pytest.mark.parametrize("half", ["small", "large"])
@pytest.mark.parametrize("others", [1, 7])
def test_no_product_of_eight_bit_states_is_cut(half, others):
    """Every code of magnitude below 2 beside the largest one of these (1.875), and every other one beside 448, at
    every place of a group of eight, against every 4-bit code beside 6; with one and with seven such products
    beside it. Products are multiples of 2^-10 (2^-3) and their sums below 2^7 (2^15): exact in binary32."""
    from paper_2608_05448_amd import dblast as D
    codes = torch.arange(256, dtype=torch.uint8)
    mag = codes & 127
    codes, worst = (codes[mag < 0x40], 0x3f) if half == "small" else (codes[(mag >= 0x40) & (mag < 0x7f)], 0x7e)
    n = len(codes)
    h = torch.zeros((8 * n, 128), dtype=torch.uint8)
    w = torch.zeros((8 * 16, 128), dtype=torch.uint8)
    for at in range(8):
        beside = [(at + 1 + i) % 8 for i in range(others)]
        h[at * n:(at + 1) * n, at] = codes
        w[at * 16:(at + 1) * 16, at] = torch.arange(16, dtype=torch.uint8)
        for b in beside:
            h[at * n:(at + 1) * n, b] = worst
            w[at * 16:(at + 1) * 16, b] = 7
    w = w[:, 0::2] + 16 * w[:, 1::2]
    one = lambda m: torch.full((m, 4), 127, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    hq, hs, wq, ws = h.view(torch.float8_e4m3fn).cuda(), one(len(h)).cuda(), w.cuda(), one(len(w)).cuda()
    want = _values(hq, hs) @ _values(wq, ws).T
    # The same group at the other places of the row of 128 is the same instruction or the next one.
    for shift in (0, 8, 24, 32, 56, 64, 120):
        a = torch.roll(h, shift, 1).view(torch.float8_e4m3fn).cuda()
        b = torch.roll(w, shift // 2, 1).cuda()
        assert torch.equal(D.dbl_mx_matmul(a, hs, b, ws).cpu().double(), want), shift


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [512, 2560, 1000])
def test_rows_are_the_same_under_every_tile(d, bits):
    """Up to 64 rows, up to 128, more, and vocabularies under which the larger and the smaller tiles are taken."""
    from paper_2608_05448_amd import dblast as D
    for V in (1000, 33100):
        h, w, _, _ = _operands(300, V, d, bits)
        for dtype in (F32, BF):
            print(f"[tiles] {d} {bits} {V} {dtype}", flush=True)
            whole = D.dbl_mx_matmul(*h, *w, dtype=dtype)
            for a, b in [(0, 1), (7, 47), (100, 165), (172, 300), (1, 300), (299, 300)]:
                part = D.dbl_mx_matmul(h[0][a:b].clone(), h[1][a:b].clone(), *w, dtype=dtype)
                assert torch.equal(part, whole[a:b]), (a, b)
        tls, lmass, lse = D.dbl_mx_head_logprobs(*[t.reshape(1, 300, 1, -1) for t in h], *w)
        for a, b in [(0, 1), (100, 165), (1, 300)]:
            got = D.dbl_mx_head_logprobs(*[t[a:b].clone().reshape(1, b - a, 1, -1) for t in h], *w)
            for x, y in zip(got, (tls, lmass, lse)):
                assert torch.equal(x, y[:, a:b]), (a, b)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_draw_over_many_segments(dtype):
    """Vocabularies of 74 segments and the largest one, 2^24 - 1, of 4097."""
    for N, V, fs in [(3, 300001, [dict(), dict(top_k=50), dict(top_k=3000), dict(top_k=5000, top_p=0.9), dict(top_p=0.9),
                                  dict(min_p=0.01), dict(top_k=70, top_p=0.5, min_p=0.01), dict(temperature=0.0)]),
                     (1, (1 << 24) - 1, [dict(), dict(top_k=50), dict(top_p=0.9), dict(temperature=0.0)])]:
        x, words = rand_logits(N, V, V % 1000, dtype, slope=1.0), rand_words(N, 6)
        for f in fs:
            print(f"[draw] V={V} {dtype} {f}", flush=True)
            check(x, words, **f)


def test_draw_of_rows_that_the_list_does_not_hold():
    """bf16 logits under a nucleus, where one value in the tail has more ids than the list; ids in the order of their
    frequency, whose largest logits share their groups of 128; and a top-k near the most that the groups bound."""
    N, V = 6, 151936
    g = torch.Generator().manual_seed(12)
    slope = 0.6 + 1.4 * torch.rand((N, 1), generator=g)
    spread = 18.0 - slope * torch.log1p(torch.rand((N, V), generator=g) * V) + 0.5 * torch.randn((N, V), generator=g)
    ordered = 18.0 - 1.2 * torch.log1p(torch.arange(V)) + 0.5 * torch.randn((N, V), generator=g)
    words = rand_words(N, 13)
    for f in [dict(top_p=0.95), dict(temperature=0.7, top_p=0.95), dict(top_p=0.95, min_p=1e-4)]:
        print(f"[draw] bf16 {f}", flush=True)
        check(spread.to(BF), words, **f)
    for x in (ordered, ordered.to(BF), spread):
        for f in [dict(top_k=50), dict(top_k=400, top_p=0.9), dict(top_k=1187), dict(top_k=1188), dict(top_k=1150, min_p=1e-4)]:
            print(f"[draw] ordered {x.dtype} {f}", flush=True)
            check(x, words, **f)


def test_draw_takes_any_whole_number_as_top_k():
    """0, or the vocabulary's size and more: off, also past 64 bits."""
    from paper_2608_05448_amd import dblast as D
    x, words = rand_logits(8, 3000, 1).cuda(), rand_words(8, 2).cuda()
    want = D.dbl_sample_logits(x, words)
    for k in (3000, 1 << 31, (1 << 32) + 1, (1 << 63) - 1, 1 << 63, (1 << 64) + 1):
        got = D.dbl_sample_logits(x, words, top_k=k)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), k
    for k in (-1, -(1 << 63) - 1, -(1 << 64) + 5):
        with pytest.raises(D.DblastError):
            D.dbl_sample_logits(x, words, top_k=k)


@pytest.mark.parametrize("argmax", [False, True])
def test_head_of_more_rows_than_a_launch_of_a_wave_each_takes(argmax):
    """2^26 rows, a wave each, are 2^32 threads: more than one launch has. Rows around that place, the first and
    the last ones are what a small call gives."""
    from paper_2608_05448_amd import dblast as D
    M, V = (1 << 26) + 205, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.empty((M, 64), dtype=torch.uint8, device="cuda").random_(0, 256, generator=g)
    hs = torch.full((M, 4), 126, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    w, ws = D.dbl_mx_quantize(torch.randn((V, 128), generator=torch.Generator().manual_seed(2)).cuda())
    lse = torch.full((M, 1, 1), float("nan"), device="cuda")
    got = D.dbl_mx_head_logprobs(h.view(M, 1, 1, 64), hs.view(M, 1, 1, 4), w, ws, lse=lse, argmax=argmax)
    assert not bool(torch.isnan(lse).any())
    most = ((1 << 32) - 1) // 256 * 4
    for a in (0, most - 50, M - 100):
        want = D.dbl_mx_head_logprobs(h[a:a + 100].clone().view(100, 1, 1, 64), hs[a:a + 100].clone().view(100, 1, 1, 4),
                                      w, ws, argmax=argmax)
        for x, y in zip(got, want):
            assert torch.equal(x[a:a + 100], y), a

"""Host side of the low-precision serving operators and the token draw: what the binding and the C ABI
refuse, and the workspace's size. No GPU is touched: every call below fails before anything is launched."""
import ctypes
import math

import pytest
import torch

from paper_2608_05448_amd import dblast as D

BF = torch.bfloat16
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
NULL = ctypes.c_void_p(None)


@pytest.fixture(scope="module")
def lib():
    return D.load()


def _fake(n):
    """Addresses that are far apart and aligned; never read."""
    return [ctypes.c_void_p((i + 1) << 44) for i in range(n)]


def test_row_length(lib):
    for d, dp in [(1, 128), (127, 128), (128, 128), (129, 256), (2560, 2560), (1000, 1024), (1 << 20, 1 << 20)]:
        assert lib.dbl_mx_row(d) == dp == D.mx_row(d)
    assert lib.dbl_mx_row(0) == 0 and lib.dbl_mx_row(-5) == 0


def test_quantize_refuses(lib):
    x, c, s = _fake(3)
    q = lib.dbl_mx_quantize
    assert q(-1, 64, D.DBL_BF16, x, 4, c, s, NULL) == D.DBL_ESHAPE
    assert q(1, 0, D.DBL_BF16, x, 4, c, s, NULL) == D.DBL_ESHAPE
    assert q(1, (1 << 20) + 1, D.DBL_BF16, x, 4, c, s, NULL) == D.DBL_ESHAPE
    assert q(1 << 40, 64, D.DBL_BF16, x, 4, c, s, NULL) == D.DBL_ESHAPE
    assert q(1, 64, 2, x, 4, c, s, NULL) == D.DBL_EDTYPE
    assert q(1, 64, D.DBL_F32, x, 6, c, s, NULL) == D.DBL_EINVAL
    for args in ((NULL, c, s), (x, NULL, s), (x, c, NULL)):
        assert q(1, 64, D.DBL_F32, args[0], 4, args[1], args[2], NULL) == D.DBL_EINVAL
    assert q(1, 64, D.DBL_F32, ctypes.c_void_p((1 << 44) + 4), 4, c, s, NULL) == D.DBL_EINVAL
    assert q(4, 64, D.DBL_F32, x, 4, x, s, NULL) == D.DBL_EINVAL  # codes over x
    assert "overlaps" in lib.dbl_last_error().decode()
    # codes end where the scales begin: 4 rows of 64 bytes
    assert q(4, 64, D.DBL_F32, x, 4, c, ctypes.c_void_p(c.value + 240), NULL) == D.DBL_EINVAL
    d = lib.dbl_mx_dequantize
    assert d(1, 64, 5, c, s, D.DBL_F32, x, NULL) == D.DBL_EINVAL
    assert d(1, 64, 4, c, s, 9, x, NULL) == D.DBL_EDTYPE
    assert d(1, 64, 4, c, s, D.DBL_F32, c, NULL) == D.DBL_EINVAL
    assert q(0, 64, D.DBL_F32, NULL, 4, NULL, NULL, NULL) == D.DBL_OK  # no rows


def test_norm_refuses(lib):
    x, r, w, u, c, s, y = _fake(7)

    def norm(M=2, d=64, dt=D.DBL_BF16, x=x, r=r, w=w, eps=1e-6, u=u, bits=8, c=c, s=s, y=NULL):
        return lib.dbl_add_rmsnorm_mx(M, d, dt, x, r, w, eps, u, bits, c, s, y, NULL)

    for eps in (-1e-9, math.inf, math.nan):
        assert norm(eps=eps) == D.DBL_EINVAL
    assert norm(r=NULL) == D.DBL_EINVAL  # a sum without a residual
    assert norm(dt=5) == D.DBL_EDTYPE and norm(bits=3) == D.DBL_EINVAL and norm(d=0) == D.DBL_ESHAPE
    for name in ("x", "w", "c", "s"):
        assert norm(**{name: NULL}) == D.DBL_EINVAL, name
    assert norm(u=w) == D.DBL_EINVAL and norm(y=x) == D.DBL_EINVAL and norm(y=u) == D.DBL_EINVAL
    assert norm(c=r) == D.DBL_EINVAL and norm(s=c) == D.DBL_EINVAL
    assert norm(u=ctypes.c_void_p(x.value + 16)) == D.DBL_EINVAL  # in place, but not the same rows
    assert norm(y=ctypes.c_void_p(y.value + 8)) == D.DBL_EINVAL


def test_products_refuse(lib):
    h, hs, w, ws, o, lm, ls, am, mem = _fake(9)

    def matmul(M=2, V=10, d=64, bits=8, h=h, hs=hs, w=w, ws=ws, dt=D.DBL_F32, o=o):
        return lib.dbl_mx_matmul(M, V, d, bits, h, hs, w, ws, dt, o, NULL)

    assert matmul(V=0) == D.DBL_ESHAPE and matmul(V=1 << 24) == D.DBL_ESHAPE
    assert matmul(M=-1) == D.DBL_ESHAPE and matmul(d=0) == D.DBL_ESHAPE
    assert matmul(M=1 << 39, V=(1 << 24) - 1) == D.DBL_ESHAPE
    assert matmul(bits=16) == D.DBL_EINVAL and matmul(dt=3) == D.DBL_EDTYPE
    for name in ("h", "hs", "w", "ws", "o"):
        assert matmul(**{name: NULL}) == D.DBL_EINVAL, name
    assert matmul(o=w) == D.DBL_EINVAL and matmul(o=ctypes.c_void_p(o.value + 2)) == D.DBL_EINVAL

    def head(s=D.Shape(1, 2, 3, 64, 10), bits=4, tls=o, lmass=lm, lse=ls, argmax=NULL, mem=NULL, n=0):
        return lib.dbl_mx_head_logprobs(s, bits, h, hs, w, ws, tls, lmass, lse, argmax, mem, n, NULL)

    assert head(bits=2) == D.DBL_EINVAL and head(s=D.Shape(1, 2, 65, 64, 10)) == D.DBL_ESHAPE
    assert head(s=D.Shape(1, 2, 3, 0, 10)) == D.DBL_ESHAPE and head(lse=NULL) == D.DBL_EINVAL
    assert head(lmass=o) == D.DBL_EINVAL
    assert head(argmax=am) == D.DBL_EWORKSPACE  # NULL
    assert head(argmax=am, mem=mem, n=8) == D.DBL_EWORKSPACE  # too small
    assert head(argmax=am, mem=ctypes.c_void_p(mem.value + 16), n=1 << 20) == D.DBL_EWORKSPACE
    assert head(s=D.Shape(0, 2, 3, 64, 10)) == D.DBL_OK


def test_draw_refuses(lib):
    x, r, t, lp, ws, a = _fake(6)
    n = D.dbl_workspace_bytes(D.DBL_OP_SAMPLE_LOGITS, 3, 1, 1, 1, 100)

    def draw(N=3, V=100, dt=D.DBL_F32, x=x, r=r, t=t, lp=lp, ws=ws, n=n, temperature=1.0, top_p=1.0, min_p=0.0, top_k=0,
             temperatures=None, top_ks=None):
        p = D.Sampling(temperature, top_p, min_p, top_k, temperatures, None, None, top_ks)
        return lib.dbl_sample_logits(N, V, dt, x, r, p, t, lp, ws, n, NULL)

    for bad in (-0.5, math.inf, math.nan):
        assert draw(temperature=bad) == D.DBL_EINVAL
    for bad in (0.0, -1.0, 1.5, math.nan):
        assert draw(top_p=bad) == D.DBL_EINVAL
    for bad in (-0.1, 1.1, math.nan):
        assert draw(min_p=bad) == D.DBL_EINVAL
    assert draw(top_k=-1) == D.DBL_EINVAL
    assert draw(V=0) == D.DBL_ESHAPE and draw(V=1 << 24) == D.DBL_ESHAPE and draw(N=-1) == D.DBL_ESHAPE
    assert draw(dt=2) == D.DBL_EDTYPE
    for name in ("x", "r", "t", "lp"):
        assert draw(**{name: NULL}) == D.DBL_EINVAL, name
    assert draw(t=r) == D.DBL_EINVAL and draw(lp=x) == D.DBL_EINVAL and draw(lp=t) == D.DBL_EINVAL
    assert draw(t=a, temperatures=a.value) == D.DBL_EINVAL  # over a parameter array
    assert draw(top_ks=a.value + 2) == D.DBL_EINVAL
    assert draw(ws=NULL) == D.DBL_EWORKSPACE and draw(n=n - 1) == D.DBL_EWORKSPACE
    assert draw(ws=ctypes.c_void_p(ws.value + 128)) == D.DBL_EWORKSPACE
    assert draw(N=0) == D.DBL_OK


def test_workspace_of_the_draw():
    """A state, per 4096 ids a maximum, a sum and 32 group maxima, a list of 4096 and 4096 bins of 12 bytes."""
    one = D.dbl_workspace_bytes(D.DBL_OP_SAMPLE_LOGITS, 1, 1, 1, 1, 151936)
    G = -(-(151936 + 7) // 4096)
    assert one == -(-(64 + G * (8 + 8 + 4 * 32)) // 256) * 256 + 8 * 4096 + 12 * 4096
    assert D.dbl_workspace_bytes(D.DBL_OP_SAMPLE_LOGITS, 16, 17, 1, 1, 151936) == 272 * one
    assert D.dbl_workspace_bytes(D.DBL_OP_SAMPLE_LOGITS, 0, 1, 1, 1, 10) == 0
    assert D.dbl_workspace_bytes(D.DBL_OP_MX_HEAD, 16, 16, 8, 4096, 151936) == 2048 * 8


def test_binding_refuses_tensors():
    x = torch.zeros((3, 64), dtype=BF)
    with pytest.raises(ValueError, match="GPU tensor"):
        D.dbl_mx_quantize(x)
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        D.dbl_mx_quantize(x.half())
    with pytest.raises(TypeError):
        D.dbl_mx_quantize([1.0])
    with pytest.raises(ValueError, match="GPU tensor"):
        D.dbl_add_rmsnorm_mx(x, None, torch.ones(64, dtype=BF))
    with pytest.raises(ValueError, match="d"):
        D.dbl_mx_quantize(torch.zeros((3, 0)))
    codes = torch.zeros((3, 64), dtype=torch.uint8)
    with pytest.raises(TypeError, match="uint8"):
        D.dbl_mx_dequantize(codes.int(), torch.zeros((3, 4)).to(E8M0), 100)
    with pytest.raises(ValueError, match="64 n"):
        D.dbl_mx_dequantize(codes[:, :60], torch.zeros((3, 4)).to(E8M0), 100)
    with pytest.raises(ValueError, match="128 n"):
        D.dbl_mx_matmul(torch.zeros((3, 64)).to(E4M3), None, codes, None)
    with pytest.raises(TypeError):
        D.dbl_sample_logits([[1.0]], None)
    with pytest.raises(ValueError, match="GPU tensor"):
        D.dbl_sample_logits(torch.zeros((3, 5)), torch.zeros(3, dtype=torch.int32))

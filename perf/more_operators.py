"""The low-precision serving operators of the DBLast library on one GPU: what is timed, with which inputs,
their plain forms, what one pass has to move and compute at least, and the same in binary64.

With ``own`` false a pass computes an operator's plain form from elementary torch operations; with ``own``
true it makes the calls of the public binding that a serving program makes. Kinds, in the order in which a
step uses them:

  quant   rows in microscaled 4 or 8 bits (blocks of 32 values that share a power of two), and back
  norm    the residual's addition and the root-mean-square norm, with the result in microscaled 8 or 4 bits
  matmul  logits of microscaled states against a head in microscaled 4 bits
  head    branch log-probabilities of the same, in the head's two-level form
  sample  one token per row of logits by temperature, top-k, top-p and min-p, from given random words

A microscaled row of d values is padded with zeros to dp = 128 ceil(d / 128): dp codes (4 bits: the even
value in the low half of a byte) and dp / 32 scales, a byte b for 2^(b - 127). A block's scale is
2^(floor(log2 of its largest magnitude) - E), E = 2 for 4 bits (e2m1) and 8 for 8 bits (e4m3), and its
values over the scale are rounded to the nearest code, ties to even, up to the type's largest.

A token is drawn by the library's integer weights: with s = fl32(logit / T) and m the row's largest s, id v
weighs floor(detexp32(fl32(s - m)) 2^40), detexp32 being the library's exponential of separately rounded
binary32 operations. Top-k keeps every id whose s is at least the k-th largest; top-p then keeps, by
decreasing s and increasing id, each id before which less than ceil(p * total) is kept; min-p keeps the
ids that weigh at least min_p 2^40. The token is the first id at which the kept weights, summed by
increasing id, exceed floor(word * sum / 2^32). T = 0 takes the lowest-index maximum.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

QWEN_V = 151936
own = False


def listed():
    return [
        # The final norm of one sequence's single token: all latency.
        dict(name="norm_one", kind="norm", dtype="bf16", M=1, d=2560, bits=8, residual=True),
        # The final norm of a verification pass: 16 sequences, 16 drafted positions and the one before.
        dict(name="norm_272", kind="norm", dtype="bf16", M=272, d=4096, bits=8, residual=True),
        # The same over the tokens of a long prompt batch.
        dict(name="norm_16k", kind="norm", dtype="bf16", M=16384, d=4096, bits=8, residual=True),
        # Branch states of 16 blocks of 16 positions and 8 categories, 8 bits, before the head.
        dict(name="quant_states", kind="quant", dtype="bf16", M=2048, d=4096, bits=8),
        # The Qwen3-8B head laid out in 4 bits when a server starts.
        dict(name="quant_head", kind="quant", dtype="bf16", M=QWEN_V, d=4096, bits=4),
        # Target logits of one sequence's verification pass at the Qwen3-4B shape, states in 8 bits.
        dict(name="matmul_17", kind="matmul", M=17, d=2560, V=QWEN_V, bits=8, out="fp32"),
        # Target logits of 16 sequences' verification at the Qwen3-8B shape.
        dict(name="matmul_272", kind="matmul", M=272, d=4096, V=QWEN_V, bits=8, out="bf16"),
        # Short blocks of three categories, a hidden size and a vocabulary of no round number, with the
        # greedy branch tokens.
        dict(name="head_ragged", kind="head", M=168, d=1000, V=50257, bits=8, argmax=True),
        # The drafter's head for 16 blocks of 16 positions and 8 categories, states in 4 bits.
        dict(name="head_2048", kind="head", M=2048, d=4096, V=QWEN_V, bits=4, argmax=False),
        # One sequence's next token under a nucleus.
        dict(name="sample_one", kind="sample", dtype="fp32", N=1, V=QWEN_V, mode="nucleus"),
        # The rows of 16 sequences' verification pass, each request with parameters of its own.
        dict(name="sample_272", kind="sample", dtype="fp32", N=272, V=QWEN_V, mode="mixed"),
        # Trajectories for training drawn at a temperature alone, a smaller vocabulary, bf16 logits.
        dict(name="sample_1024", kind="sample", dtype="bf16", N=1024, V=50257, mode="temperature"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HIDDEN = [64, 96, 200, 512, 1000, 1024, 1440, 2048, 2560, 4096]


def draw(rng):
    kind = rng.choice(["norm", "norm", "quant", "matmul", "matmul", "head", "head", "sample", "sample"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if kind == "norm":
        c = dict(kind=kind, dtype=dtype, d=rng.choice(_HIDDEN + [_log_int(rng, 33, 5000)]),
                 bits=rng.choice([8, 8, 4]), residual=rng.random() < 0.7)
        return dict(c, M=_log_int(rng, 1, 8192 if dtype == "fp32" else 16384))
    if kind == "quant":
        return dict(kind=kind, dtype=dtype, d=rng.choice(_HIDDEN + [_log_int(rng, 33, 5000)]),
                    bits=rng.choice([8, 4]), M=_log_int(rng, 1, 60000))
    V = rng.choice([QWEN_V, _log_int(rng, 1000, 150000)])
    if kind == "sample":
        n = _log_int(rng, 1, min(1024, 60000000 // V))
        return dict(kind=kind, dtype=rng.choice(["fp32", "bf16"]), N=n, V=V,
                    mode=rng.choice(["temperature", "topk", "nucleus", "mixed", "mixed"]))
    c = dict(kind=kind, M=_log_int(rng, 1, 2048), d=rng.choice(_HIDDEN), V=V, bits=rng.choice([8, 4]))
    if kind == "matmul":
        c["out"] = rng.choice(["fp32", "bf16"])
    else:
        c["argmax"] = rng.random() < 0.3
    return c


# --- inputs --------------------------------------------------------------------------------

_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 64 + stream)
    return g


def _randn(shape, g, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale


def _rand(shape, g):
    return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)


def _outliers(d, g):
    """Factor by hidden unit: a few units of transformer states are many times the others."""
    return torch.where(_rand((d,), g) < 0.01, 20.0, 1.0) * torch.exp(_randn((d,), g, 0.3))


def _row(d):
    return (d + 127) // 128 * 128


def _quantized(x, bits):
    """Codes and scales of rows x [M, d] as a serving program holds them, a piece at a time."""
    parts = [_plain_quantize(p.float(), bits) for p in x.split(16384)]
    return tuple(torch.cat([p[i].view(torch.uint8) for p in parts]).view(parts[0][i].dtype)
                 for i in range(2))


def _head_inputs(c, seed):
    """Microscaled states [1, M, 1, d] and head. The logits have a Zipf-like bias (hidden unit 0), noise,
    and each row knows one token to another degree, so that its rows are from flat to sure."""
    M, d, V = c["M"], c["d"], c["V"]
    g = _gen(seed, 1)
    w = _randn((V, d), g, 1.3 / math.sqrt(d))
    rank = torch.randperm(V, generator=g, device="cuda")
    w[:, 0] = -0.275 * torch.log1p(rank.float())
    known = torch.randint(0, V, (M,), generator=g, device="cuda")
    h = _randn((M, d), g) + 12.0 * _rand((M, 1), g) / 1.69 * w[known]
    h[:, 0] = 4.0
    hq, hs = _quantized(h.to(torch.bfloat16), c["bits"])
    wq, ws = _quantized(w.to(torch.bfloat16), 4)
    return dict(h=hq.reshape(1, M, 1, -1), hs=hs.reshape(1, M, 1, -1), w=wq, ws=ws)


def _sample_inputs(c, seed):
    """Logits that fall with the rank like Zipf's law, to another exponent in every row, random words, and
    the parameters: numbers where the whole batch shares them, a value per row in mixed batches."""
    N, V, mode = c["N"], c["V"], c["mode"]
    g = _gen(seed, 4)
    slope = 0.6 + 1.4 * _rand((N, 1), g)
    x = 18.0 - slope * torch.log1p(torch.rand((N, V), generator=g, device="cuda") * V)
    x += _randn((N, V), g, 0.5)
    s = dict(logits=x.to(_DTYPES[c["dtype"]]),
             words=torch.randint(-2 ** 31, 2 ** 31, (N,), generator=g, device="cuda").to(torch.int32),
             temperature=0.8, top_k=0, top_p=1.0, min_p=0.0)
    if mode == "topk":
        s.update(top_k=50)
    elif mode == "nucleus":
        s.update(temperature=0.7, top_p=0.95)
    elif mode == "mixed":
        def pick(values, dtype=torch.float32):
            at = torch.randint(0, len(values), (N,), generator=g, device="cuda")
            return torch.tensor(values, device="cuda", dtype=dtype)[at]
        s.update(temperature=pick([0.0, 0.6, 0.8, 1.0, 1.0, 1.3]),
                 top_k=pick([0, 0, 20, 50, 400], torch.int32),
                 top_p=pick([1.0, 1.0, 0.8, 0.95, 0.99]), min_p=pick([0.0, 0.0, 0.02, 0.1]))
    return s


def prepare(case, seed):
    c, kind = case, case["kind"]
    if kind in ("matmul", "head"):
        return dict(_head_inputs(c, seed), kind=kind, argmax=c.get("argmax", False),
                    out=_DTYPES[c.get("out", "fp32")])
    if kind == "sample":
        return dict(_sample_inputs(c, seed), kind=kind)
    g = _gen(seed, 2)
    M, d, dt = c["M"], c["d"], _DTYPES[c["dtype"]]
    unit = _outliers(d, g)
    if kind == "quant":
        return dict(kind=kind, x=(_randn((M, d), g, 0.02) * unit).to(dt), bits=c["bits"])
    return dict(kind=kind, x=(_randn((M, d), g) * unit).to(dt), bits=c["bits"], eps=1e-6,
                residual=(_randn((M, d), g, 4.0) * unit).to(dt) if c["residual"] else None,
                weight=(1.0 + _randn((d,), g, 0.2)).to(dt))


# --- one pass ------------------------------------------------------------------------------

def _two_to(n, dtype):
    """2^n, exactly, for whole numbers -1022 <= n <= 1023."""
    return ((n.long() + 1023) << 52).view(torch.float64).to(dtype)


def _plain_quantize(x, bits):
    """Codes and scales of x [..., d] of 32 or 64 bits. Dividing by a power of two and rounding to a
    multiple of one are exact operations."""
    d = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, _row(d) - d)).unflatten(-1, (-1, 32))
    largest = x.abs().amax(-1, keepdim=True)
    power = (torch.frexp(largest).exponent - 1 - (2 if bits == 4 else 8)).clamp(min=-127)
    power = torch.where(largest > 0, power, -127)
    scaled = x * _two_to(-power, x.dtype)
    mant, least, most = (1, 0, 6.0) if bits == 4 else (3, -6, 448.0)
    scaled = scaled.clamp(-most, most)
    step = (torch.frexp(scaled).exponent - 1).clamp(min=least) - mant
    step = _two_to(step, x.dtype)
    value = (torch.round(scaled / step) * step).flatten(-2)
    scales = (power + 127)[..., 0].to(torch.uint8).view(torch.float8_e8m0fnu)
    if bits == 8:
        return value.float().to(torch.float8_e4m3fn), scales
    a = value.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code += 8 * torch.signbit(value).to(torch.uint8)
    return code[..., 0::2] + 16 * code[..., 1::2], scales


def _plain_values(codes, scales):
    """The binary32 values [..., dp] of microscaled rows."""
    if codes.dtype == torch.uint8:
        table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
        v = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], -1).flatten(-2)
    else:
        v = codes.float()
    return (v.unflatten(-1, (-1, 32)) * scales.float()[..., None]).flatten(-2)


def _plain_quant(s):
    codes, scales = _plain_quantize(s["x"].float(), s["bits"])
    d = s["x"].shape[-1]
    return dict(values=_plain_values(codes, scales)[..., :d].to(s["x"].dtype))


def _plain_norm(s):
    h, out = s["x"], {}
    if s["residual"] is not None:
        h = out["sum"] = (h.float() + s["residual"].float()).to(h.dtype)
    h = h.double()
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + s["eps"]) * s["weight"].double()
    codes, scales = _plain_quantize(y, s["bits"])
    if s["bits"] == 4:
        return dict(out, values=_plain_values(codes, scales)[..., :h.shape[-1]].to(torch.bfloat16))
    return dict(out, codes=codes, scales=scales)


def _plain_logits(s):
    h = _plain_values(s["h"], s["hs"]).flatten(0, -2)
    return h @ _plain_values(s["w"], s["ws"]).T


def _plain_head(s):
    logits = _plain_logits(s)
    M, V = logits.shape
    tiles = (V + 127) // 128
    x = torch.nn.functional.pad(logits, (0, tiles * 128 - V), value=-math.inf).unflatten(-1, (tiles, 128))
    top = x.amax(-1, keepdim=True)
    lmass = torch.log(torch.exp(x - top).sum(-1, keepdim=True)) + top
    tls = (x - lmass).flatten(-2)[:, :V]
    lmass = lmass[..., 0]
    top = lmass.amax(-1, keepdim=True)
    lse = (torch.log(torch.exp(lmass - top).sum(-1, keepdim=True)) + top)[:, 0]
    shape = s["h"].shape[:3]
    out = dict(tls=tls.reshape(*shape, V), lmass=lmass.reshape(*shape, tiles), lse=lse.reshape(shape))
    if s["argmax"]:
        at = torch.where(logits == logits.amax(-1, keepdim=True), torch.arange(V, device=logits.device), V)
        out["argmax"] = at.amin(-1).to(torch.int32).reshape(shape)
    return out


def _plain_weights(x):
    """floor(detexp32(x) 2^40) for x <= 0 in binary32: every operation rounded on its own."""
    c = x.clamp(min=-100.0)
    n = torch.round(c * 1.44269502162933349609375)
    r = c - n * 0.693145751953125
    r = r - n * 1.42860676533018704503775e-06
    p = torch.full_like(r, 1.0 / 5040.0)
    p = p * r + torch.full_like(r, 1.0 / 720.0)
    p = p * r + torch.full_like(r, 1.0 / 120.0)
    p = p * r + torch.full_like(r, 1.0 / 24.0)
    p = p * r + torch.full_like(r, 1.0 / 6.0)
    p = p * r + 0.5
    p = p * r + 1.0
    p = p * r + 1.0
    return torch.floor(p.double() * _two_to(n + 40.0, torch.float64)).long()


def _plain_sample(s):
    x = s["logits"].float()
    N, V = x.shape
    dev = x.device

    def per_row(v, dtype):
        return torch.as_tensor(v, dtype=dtype, device=dev).expand(N)[:, None]

    T, p, least = (per_row(s[k], torch.float32).double() for k in ("temperature", "top_p", "min_p"))
    k = per_row(s["top_k"], torch.int64)
    greedy = T == 0
    z = (x.double() / torch.where(greedy, 1.0, T)).float()
    z, ids = torch.sort(z, dim=-1, descending=True, stable=True)
    w = _plain_weights(z - z[:, :1])
    kth = z.gather(1, torch.where(k == 0, V, k.clamp(max=V)) - 1)
    w = torch.where(z >= kth, w, 0)
    total = w.sum(-1, keepdim=True)
    before = torch.cumsum(w, -1) - w
    limit = torch.where(p < 1, torch.ceil(p * total.double()).long(), total)
    keep = (before < limit) & (w.double() >= least * 2.0 ** 40)
    keep = torch.where(greedy, torch.arange(V, device=dev) == 0, keep)
    w = torch.zeros_like(w).scatter_(1, ids, torch.where(keep, w, 0))
    cum = torch.cumsum(w, -1)
    total = cum[:, -1:]
    word = s["words"].long()[:, None] & 0xFFFFFFFF
    high, low = total >> 32, total & 0xFFFFFFFF
    at = word * high + ((word * (low >> 16) + ((word * (low & 0xFFFF)) >> 16)) >> 16)
    token = (cum <= at).sum(-1, keepdim=True)
    mass, total = w.gather(1, token).double(), total.double()
    logprob = torch.where(2 * mass > total, torch.log1p(-(total - mass) / total), torch.log(mass / total))
    return dict(token=token[:, 0].to(torch.int32), logprob=logprob[:, 0].float())


def run(state):
    s, kind = state, state["kind"]
    if not own:
        if kind == "matmul":
            return dict(logits=_plain_logits(s).to(s["out"]).reshape(*s["h"].shape[:-1], -1))
        return {"quant": _plain_quant, "norm": _plain_norm, "head": _plain_head,
                "sample": _plain_sample}[kind](s)
    from paper_2608_05448_amd import dblast as D
    if kind == "quant":
        codes, scales = D.dbl_mx_quantize(s["x"], bits=s["bits"])
        return dict(values=D.dbl_mx_dequantize(codes, scales, s["x"].shape[-1], dtype=s["x"].dtype))
    if kind == "norm":
        total, codes, scales = D.dbl_add_rmsnorm_mx(s["x"], s["residual"], s["weight"], eps=s["eps"],
                                                    bits=s["bits"])
        out = {} if total is None else dict(sum=total)
        if s["bits"] == 4:
            return dict(out, values=D.dbl_mx_dequantize(codes, scales, s["x"].shape[-1],
                                                        dtype=torch.bfloat16))
        return dict(out, codes=codes, scales=scales)
    if kind == "matmul":
        return dict(logits=D.dbl_mx_matmul(s["h"], s["hs"], s["w"], s["ws"], dtype=s["out"]))
    if kind == "head":
        got = D.dbl_mx_head_logprobs(s["h"], s["hs"], s["w"], s["ws"], argmax=s["argmax"])
        return dict(zip(("tls", "lmass", "lse", "argmax"), got))
    token, logprob = D.dbl_sample_logits(s["logits"], s["words"], temperature=s["temperature"],
                                         top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return dict(token=token, logprob=logprob)


def work(case):
    """Each input read once and each output written once; two operations per multiply-add of the
    products, a few per value of the others (no floor of theirs is set by arithmetic)."""
    c, kind = case, case["kind"]
    if kind == "sample":
        n = c["N"] * c["V"]
        return dict(bytes=n * (2.0 if c["dtype"] == "bf16" else 4.0) + 12.0 * c["N"], flops=20.0 * n)
    d, e = c["d"], 2.0 if c.get("dtype", "bf16") == "bf16" else 4.0
    coded = _row(d) * (c["bits"] / 8 + 1 / 32)
    if kind == "quant":  # read, and the coded rows written; those read, and the values written
        return dict(bytes=c["M"] * (2 * e * d + 2 * coded), flops=8.0 * c["M"] * d)
    if kind == "norm":
        moved = c["M"] * (e * d * (3 if c["residual"] else 1) + coded) + e * d
        if c["bits"] == 4:
            moved += c["M"] * (coded + 2.0 * d)
        return dict(bytes=moved, flops=10.0 * c["M"] * d)
    V, M = c["V"], c["M"]
    moved = M * coded + V * _row(d) * (0.5 + 1 / 32) + M * V * (2.0 if c.get("out") == "bf16" else 4.0)
    if kind == "head":
        moved += 4.0 * M * ((V + 127) // 128 + 1 + c["argmax"])
    return dict(bytes=moved, flops=2.0 * M * V * d)


# --- the same in binary64 ------------------------------------------------------------------

def _powers(device):
    """2^k at place 300 + k, for -300 <= k < 300."""
    return torch.tensor([2.0 ** k for k in range(-300, 300)], dtype=torch.float64, device=device)


def _exact_blocks(x, bits):
    """Values over their scale and scales of x [M, d] in binary64, from a table of the type's values."""
    M, d = x.shape
    codes = torch.arange(8 if bits == 4 else 127, device=x.device)
    two = _powers(x.device)
    man = 1 if bits == 4 else 3
    exp, frac = codes >> man, (codes & (2 ** man - 1)).double() / 2 ** man
    bias = 1 if bits == 4 else 7
    table = torch.where(exp == 0, frac * 2.0 ** (1 - bias), (1 + frac) * two[300 + exp - bias])
    full = torch.zeros((M, _row(d)), dtype=torch.float64, device=x.device)
    full[:, :d] = x
    blocks = full.reshape(M, -1, 32)
    top = blocks.abs().max(-1).values
    scale = two[torch.searchsorted(two, top, right=True).sub(1).clamp(min=200) - (2 if bits == 4 else 8)]
    scale = torch.clamp(scale, min=2.0 ** -127)[..., None]
    a = (blocks / scale).abs()
    # Halfway points between neighbours; at one, the even code (its index's last bit is 0) is taken.
    mid = (table[1:] + table[:-1]) / 2
    below, above = torch.searchsorted(mid, a), torch.searchsorted(mid, a, right=True)
    value = table[torch.where(below % 2 == 0, below, above)] * torch.sign(blocks)
    return value, scale


def _exact_norm(s):
    x = s["x"].double()
    out = {}
    if s["residual"] is not None:
        out["sum"] = x + s["residual"].double()
        x = (s["x"].float() + s["residual"].float()).to(s["x"].dtype).double()
    y = x * torch.rsqrt(torch.square(x).sum(1, keepdim=True) / x.shape[1] + s["eps"]) * s["weight"].double()
    value, scale = _exact_blocks(y, s["bits"])
    if s["bits"] == 4:
        return dict(out, values=(value * scale).reshape(len(x), -1)[:, :x.shape[1]])
    return dict(out, codes=value.reshape(len(x), -1), scales=scale[..., 0])


def _exact_values(codes, scales):
    b = codes.view(torch.uint8).reshape(-1, codes.shape[-1]).long()
    if codes.dtype == torch.uint8:
        b = torch.stack((b % 16, b // 16), 2).reshape(len(b), -1)
        man, bias, width = 1, 1, 4
    else:
        man, bias, width = 3, 7, 8
    mag = b % 2 ** (width - 1)
    exp, frac = mag // 2 ** man, (mag % 2 ** man).double() / 2 ** man
    two = _powers(b.device)
    v = torch.where(exp == 0, frac * 2.0 ** (1 - bias), (1 + frac) * two[300 + exp - bias])
    v = torch.where(b >= 2 ** (width - 1), -v, v)
    power = two[scales.view(torch.uint8).reshape(len(b), -1).long() + (300 - 127)]
    return v * power.repeat_interleave(32, dim=1)


def _exact_head(c, s):
    if 2.0 * c["M"] * c["V"] * c["d"] > 3e13:
        return None
    h, V = _exact_values(s["h"], s["hs"]), s["w"].shape[0]
    z = torch.empty((len(h), V), dtype=torch.float64, device=h.device)
    for v in range(0, V, 8192):
        z[:, v:v + 8192] = h @ _exact_values(s["w"][v:v + 8192], s["ws"][v:v + 8192]).T
    rows = s["h"].shape[:3]
    if c["kind"] == "matmul":
        return dict(logits=z.reshape(*rows, V))
    tiles = z.split(128, dim=1)
    lmass = torch.stack([torch.logsumexp(t, 1) for t in tiles], 1)
    out = dict(lmass=lmass.reshape(*rows, len(tiles)), lse=torch.logsumexp(z, 1).reshape(rows))
    if c["argmax"]:
        out["argmax"] = z.argmax(1).to(torch.int32).reshape(rows)
    z -= lmass.repeat_interleave(128, dim=1)[:, :V]
    return dict(out, tls=z.reshape(*rows, V))


def _exact_weight(x):
    """The integer weights of binary32 differences x <= 0."""
    f = np.float32
    x = np.maximum(x, f(-100))
    n = np.rint(x * f(float.fromhex("0x1.715476p+0")))
    r = (x - n * f(float.fromhex("0x1.62e4p-1"))) - n * f(float.fromhex("0x1.7f7d1cp-20"))
    p = np.full_like(r, f(1 / 5040))
    for c in (1 / 720, 1 / 120, 1 / 24, 1 / 6, 0.5, 1, 1):
        p = p * r + f(c)
    return np.floor(p.astype(np.float64) * 2.0 ** (n.astype(np.float64) + 40)).astype(np.int64)


def _exact_sample(s):
    x = s["logits"].float().cpu().numpy()
    N, V = x.shape
    words = s["words"].cpu().numpy().astype(np.int64) % 2 ** 32

    def rows(v):
        return np.broadcast_to(v.cpu().numpy() if isinstance(v, torch.Tensor) else v, (N,))

    par = list(zip(*(rows(s[k]) for k in ("temperature", "top_k", "top_p", "min_p"))))
    token, logprob = [], []
    for i, (T, k, p, least) in enumerate(par):
        if T == 0:
            token.append(int(np.argmax(x[i])))
            logprob.append(0.0)
            continue
        z = x[i] / np.float32(T)
        w = _exact_weight(z - z.max())
        if 0 < k < V:
            w[z < np.partition(z, V - k)[V - k]] = 0
        if p < 1:
            order = np.argsort(-z, kind="stable")
            total = int(w.sum())
            run = np.cumsum(w[order])
            n = int(np.searchsorted(run, int(np.ceil(np.float64(np.float32(p)) * total)))) + 1
            w[order[n:]] = 0
        w[w < np.float64(np.float32(least)) * 2.0 ** 40] = 0
        run = np.cumsum(w)
        total = int(run[-1])
        v = int(np.searchsorted(run, int(words[i]) * total >> 32, side="right"))
        token.append(v)
        mass = int(w[v])
        logprob.append(math.log1p((mass - total) / total) if 2 * mass > total else math.log(mass / total))
    return dict(token=torch.tensor(token, dtype=torch.int32),
                logprob=torch.tensor(logprob, dtype=torch.float64))


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("matmul", "head"):
        return _exact_head(case, s)
    if kind == "sample":
        return _exact_sample(s)
    if kind == "norm":
        return _exact_norm(s)
    parts = []
    for x in s["x"].split(16384):
        value, scale = _exact_blocks(x.double(), s["bits"])
        parts.append((value * scale).reshape(len(x), -1)[:, :x.shape[1]].to(s["x"].dtype))
    return dict(values=torch.cat(parts))

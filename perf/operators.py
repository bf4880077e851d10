"""The training operators of the DBLast library on one GPU: what is timed, with which inputs, their
plain forms, what one pass has to move and compute at least, and the same in binary64.

With ``own`` false a pass computes an operator's plain form from elementary torch operations in
binary32; with ``own`` true it makes the calls of the public binding that a fine-tuning program makes.
Kinds:

  nll     negative log-likelihood of given tokens under the LM head, and each row's log-sum-exp
  grad    the same and its gradient with respect to the branch states, and to the head with ``dw``
  expand  backward pass of the branch expander: trunk states, weight and bias
  clip    global norm of a set of gradients, and the gradients scaled to a largest norm

Rows of the head are (block, position, category) as everywhere in the library; a position whose token
is -1 is padding behind the end of its sequence and counts for nothing (the last ``b % (pad + 1)``
positions of block b).
"""
from __future__ import annotations

import math
import random

import torch

QWEN_V = 151936
own = False

# Cost of the largest listed gradient, in rows x hidden size x vocabulary.
_MOST = 8192 * 4096 * QWEN_V


def listed():
    return [
        # The smallest training pass there is, in binary32: a handful of launches, all latency.
        dict(name="grad_fp32_tiny", kind="grad", dtype="fp32", B=1, K=4, R=2, d=64, V=256, pad=0,
             dw=True),
        # Scoring one sequence's block of 15 tokens under 4 categories at the Qwen3-4B shape.
        dict(name="nll_one", kind="nll", dtype="bf16", B=1, K=15, R=4, d=2560, V=QWEN_V, pad=0),
        # Scoring the blocks of 16 sequences at the Qwen3-8B shape.
        dict(name="nll_16", kind="nll", dtype="bf16", B=16, K=16, R=8, d=4096, V=QWEN_V, pad=0),
        # Gradient of one sequence's block with the head frozen.
        dict(name="grad_one", kind="grad", dtype="bf16", B=1, K=15, R=4, d=2560, V=QWEN_V, pad=0,
             dw=False),
        # The paper's fine-tuning step, 16 blocks: the target's head is reused and frozen, some
        # sequences end inside their block.
        dict(name="grad_16", kind="grad", dtype="bf16", B=16, K=16, R=8, d=4096, V=QWEN_V, pad=6,
             dw=False),
        # Short blocks, three categories, a hidden size and a vocabulary of no round number, the head
        # trained too.
        dict(name="grad_ragged", kind="grad", dtype="bf16", B=8, K=7, R=3, d=1000, V=50257, pad=4,
             dw=True),
        # A large batch with the head trained too.
        dict(name="grad_64", kind="grad", dtype="bf16", B=64, K=16, R=8, d=4096, V=QWEN_V, pad=3,
             dw=True),
        # Expander of one sequence's block, Qwen3-4B shape.
        dict(name="expand_one", kind="expand", B=1, K=15, R=4, d=2560),
        # Expander of 16 sequences, Qwen3-8B shape.
        dict(name="expand_16", kind="expand", B=16, K=16, R=8, d=4096),
        # The gradients of the added parameters (expander and prior head) at the Qwen3-4B shape.
        dict(name="clip_adapter", kind="clip", dtype="bf16", d=2560, R=4, V=0, small=0, over=3.0),
        # A drafter's many small parameters, odd sizes, both types; the norm is below the limit.
        dict(name="clip_small", kind="clip", dtype="mixed", d=128, R=2, V=0, small=240, over=0.6),
        # Added parameters and a trained head at the Qwen3-8B shape, gradients in binary32.
        dict(name="clip_head", kind="clip", dtype="fp32", d=4096, R=8, V=QWEN_V, small=20, over=3.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _vocabulary(rng):
    u = rng.random()
    if u < 0.4:
        return QWEN_V
    v = _log_int(rng, 1000, 150000)
    return v // 128 * 128 if u < 0.6 else v


def draw(rng):
    kind = rng.choice(["nll", "grad", "grad", "grad", "expand", "expand", "clip"])
    if kind == "clip":
        d = rng.choice([64, 200, 512, 1000, 1024, 2048, 2560, 4096])
        return dict(kind=kind, dtype=rng.choice(["bf16", "fp32", "mixed"]), d=d,
                    R=rng.randint(1, 8), V=rng.choice([0, 0, _log_int(rng, 1000, 150000)]),
                    small=_log_int(rng, 1, 300), over=rng.choice([0.3, 0.9, 2.0, 10.0]))
    K = rng.randint(1, 16)
    R = rng.choice([1, 2, 3, 4, 4, 5, 8, 8, 16])
    if kind == "expand":
        d = rng.choice([96, 256, 512, 1024, 1440, 2048, 2560, 4096])
        return dict(kind=kind, B=_log_int(rng, 1, 96), K=K, R=min(R, 8), d=d)
    c = dict(kind=kind, dtype="bf16", K=K, R=R, d=rng.choice([64, 200, 512, 1000, 1024, 1056, 2048,
                                                              2560, 4096]),
             V=_vocabulary(rng), pad=rng.choice([0, 0, 2, K]))
    if rng.random() < 0.2:
        c.update(dtype="fp32", d=rng.choice([33, 64, 100, 256, 500]), V=_log_int(rng, 50, 20000))
    most = max(1, min(512 if c["dtype"] == "bf16" else 8, _MOST // (K * R * c["d"] * c["V"])))
    c["B"] = _log_int(rng, 1, most)
    if kind == "grad":
        c["dw"] = rng.random() < 0.5
    return c


# --- inputs --------------------------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 64 + stream)
    return g


def _randn(shape, g, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale


def _rand(shape, g):
    return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)


_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _kept(c):
    """Positions of each block that are trained on."""
    return [c["K"] - min(c["K"], b % (c["pad"] + 1)) for b in range(c["B"])]


def _head_inputs(c, seed):
    """Branch states, head, tokens and the loss's gradient by row. The logits have a Zipf-like bias
    (hidden unit 0), noise, and each row knows its token to another degree, so that the tokens'
    probabilities run from 1e-6 to nearly 1. A row's gradient is its category's responsibility over
    the number of positions."""
    B, K, R, d, V = c["B"], c["K"], c["R"], c["d"], c["V"]
    g = _gen(seed, 1)
    dt = _DTYPES[c["dtype"]]
    w = _randn((V, d), g, 1.3 / math.sqrt(d))
    rank = torch.randperm(V, generator=g, device="cuda")
    w[:, 0] = -0.275 * torch.log1p(rank.float())
    by_rank = torch.empty_like(rank)
    by_rank[rank] = torch.arange(V, device="cuda")
    x = by_rank[torch.exp(_rand((B, K), g) * math.log(V)).long().sub_(1).clamp_(0, V - 1)]
    h = _randn((B, K, 1, d), g, math.sqrt(0.7)) + _randn((B, K, R, d), g, math.sqrt(0.3))
    known = 12.0 * _rand((B, K, R, 1), g) / 1.69
    h += known * w[x][:, :, None]
    h[..., 0] = 4.0
    kept = torch.tensor(_kept(c), device="cuda")[:, None]
    x = torch.where(torch.arange(K, device="cuda") < kept, x, -1).to(torch.int32)
    grad = torch.softmax(_randn((B, 1, R), g), dim=-1).expand(B, K, R) / float(B * K)
    return dict(h=h.to(dt), w=w.to(dt), x=x, g=grad.contiguous())


def _clip_sizes(c):
    """Numbers of elements: weight, bias and prior head of the expander, the head if it is trained, and
    small parameters of all sizes (norms, biases, little projections)."""
    d, R = c["d"], c["R"]
    sizes = [R * d * d, R * d, R * d, R]
    if c["V"]:
        sizes.append(c["V"] * d)
    rng = random.Random(c["small"])
    return sizes + [_log_int(rng, 1, 40000) for _ in range(c["small"])]


def _clip_dtype(c, i):
    return c["dtype"] if c["dtype"] != "mixed" else ("bf16", "fp32")[i % 2]


def prepare(case, seed):
    c, kind = case, case["kind"]
    if kind in ("nll", "grad"):
        return dict(_head_inputs(c, seed), kind=kind, dw=c.get("dw", False))
    if kind == "expand":
        B, K, R, d = c["B"], c["K"], c["R"], c["d"]
        g = _gen(seed, 2)
        bf = torch.bfloat16
        return dict(kind=kind, h=_randn((B, K, d), g).to(bf),
                    W=_randn((R * d, d), g, 0.5 / math.sqrt(d)).to(bf),
                    dout=_randn((B, K, R, d), g, 1e-3).to(bf))
    g = _gen(seed, 3)
    sizes = _clip_sizes(c)
    scale = c["over"] / math.sqrt(sum(sizes))  # the limit is a norm of 1
    grads, out, buckets = [], [], []
    for name, dt in _DTYPES.items():
        mine = [n for i, n in enumerate(sizes) if _clip_dtype(c, i) == name]
        if mine:
            # Gradients live in one bucket per type, as a data-parallel program keeps them. The clipped
            # ones go to buckets of their own (the raw ones stay for the log), so that a pass can be
            # made again.
            flat = _randn((sum(mine),), g, scale).to(dt)
            buckets.append(torch.empty_like(flat))
            grads += flat.split(mine)
            out += buckets[-1].split(mine)
    return dict(kind=kind, grads=grads, out=out, buckets=buckets, max_norm=1.0)


# --- one pass ------------------------------------------------------------------------------

def _plain_head(s):
    h, w, x = s["h"], s["w"], s["x"]
    B, K, R, d = h.shape
    hf, wf = h.reshape(-1, d).float(), w.float()
    t = x[:, :, None].expand(B, K, R).reshape(-1).long()
    kept = t >= 0
    logits = hf @ wf.T
    top = logits.max(-1, keepdim=True).values
    total = torch.exp(logits - top).sum(-1, keepdim=True)
    lse = torch.log(total) + top
    picked = logits.gather(1, t.clamp_min(0)[:, None])
    zero = torch.zeros((), device=h.device)
    out = dict(nll=torch.where(kept, (lse - picked)[:, 0], zero).reshape(B, K, R),
               lse=torch.where(kept, lse[:, 0], zero).reshape(B, K, R))
    if s["kind"] == "nll":
        return out
    g = torch.where(kept, s["g"].reshape(-1), zero)[:, None]
    logits.sub_(lse).exp_().mul_(g)
    logits.scatter_add_(1, t.clamp_min(0)[:, None], -g)
    out["dh"] = (logits @ wf).reshape(h.shape).to(h.dtype)
    if s["dw"]:
        out["dw"] = (logits.T @ torch.where(kept[:, None], hf, zero)).to(w.dtype)
    return out


def _plain_expand(s):
    h, W, dout = s["h"], s["W"], s["dout"]
    B, K, R, d = dout.shape
    do = dout.reshape(B * K, R * d).float()
    dh = do.reshape(B * K, R, d).sum(1) + do @ W.float()
    return dict(dh=dh.reshape(B, K, d).to(h.dtype),
                dW=(do.T @ h.reshape(-1, d).float()).to(W.dtype), dc=do.sum(0).to(W.dtype))


def _plain_clip(s):
    norm = torch.sqrt(sum((t.double() * t.double()).sum() for t in s["grads"]))
    scale = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0).float()
    for t, o in zip(s["grads"], s["out"]):
        o.copy_(t.float() * scale)
    return [norm.float()] + s["buckets"]


def run(state):
    s, kind = state, state["kind"]
    if not own:
        return {"expand": _plain_expand, "clip": _plain_clip}.get(kind, _plain_head)(s)
    from paper_2608_05448_amd import dblast as D
    if kind == "expand":
        dh, dW, dc = D.dbl_expand_branches_backward(s["h"], s["W"], s["dout"])
        return dict(dh=dh, dW=dW, dc=dc)
    if kind == "clip":
        norm = D.dbl_grad_norm(s["grads"])
        D.dbl_clip_grads(s["grads"], norm, s["max_norm"], out=s["out"])
        return [norm] + s["buckets"]
    nll, lse = D.dbl_head_nll(s["h"], s["w"], s["x"])
    if kind == "nll":
        return dict(nll=nll, lse=lse)
    dh, dw = D.dbl_head_nll_backward(s["h"], s["w"], s["x"], nll, lse, s["g"], want_dw=s["dw"])
    return dict(nll=nll, lse=lse, dh=dh, dw=dw) if s["dw"] else dict(nll=nll, lse=lse, dh=dh)


def work(case):
    """Each input read once and each output written once; two operations per multiply-add of the rows
    that count (logits, and one product per gradient), none for the element-wise parts. Gradients are
    read for their norm and, where they are scaled, once more."""
    c, kind = case, case["kind"]
    if kind == "clip":
        sizes = _clip_sizes(c)
        total = sum(n * (2 if _clip_dtype(c, i) == "bf16" else 4) for i, n in enumerate(sizes))
        return dict(bytes=3.0 * total + 4, flops=3.0 * sum(sizes))
    B, K, R, d = c["B"], c["K"], c["R"], c["d"]
    if kind == "expand":
        n = B * K
        return dict(bytes=2.0 * (2 * n * d + 2 * R * d * d + n * R * d + R * d),
                    flops=4.0 * n * R * d * d)
    rows, kept, e = B * K * R, R * sum(_kept(c)), 2 if c["dtype"] == "bf16" else 4
    moved = e * (kept * d + c["V"] * d) + 4.0 * B * K + 8.0 * rows
    flops = 2.0 * kept * c["V"] * d
    if kind == "grad":
        moved += e * rows * d + 4.0 * rows + (e * c["V"] * d if c["dw"] else 0)
        flops *= 3 if c["dw"] else 2
    return dict(bytes=moved, flops=flops)


# --- the same in binary64 ------------------------------------------------------------------

def _exact_head(c, s):
    B, K, R, d = s["h"].shape
    V = s["w"].shape[0]
    dev = s["h"].device
    h = s["h"].reshape(-1, d).double()
    token = s["x"].long().repeat_interleave(R, dim=1).reshape(-1)
    rows = torch.nonzero(token >= 0)[:, 0]
    w = s["w"].double()
    nll = torch.zeros(B * K * R, dtype=torch.float64, device=dev)
    lse = torch.zeros_like(nll)
    dh, dw = torch.zeros_like(h), torch.zeros_like(w) if s["dw"] else None
    weight = s["g"].reshape(-1).double()
    for part in rows.split(1024):
        hp, tp = h[part], token[part]
        z = hp @ w.T
        total = torch.logsumexp(z, dim=1)
        at = torch.arange(len(part), device=dev)
        nll[part], lse[part] = total - z[at, tp], total
        if s["kind"] == "nll":
            continue
        p = torch.softmax(z, dim=1)
        p[at, tp] -= 1.0
        p *= weight[part][:, None]
        dh[part] = p @ w
        if dw is not None:
            dw += p.T @ hp
    out = dict(nll=nll.reshape(B, K, R), lse=lse.reshape(B, K, R))
    if s["kind"] == "grad":
        out["dh"] = dh.reshape(B, K, R, d)
        if dw is not None:
            out["dw"] = dw
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("nll", "grad"):
        return _exact_head(case, s)
    if case["kind"] == "clip":
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(t, dtype=torch.float64)) ** 2
                                   for t in s["grads"]))
        scale = min(1.0, s["max_norm"] / (norm + 1e-6))
        return [torch.tensor(norm, dtype=torch.float64, device="cuda")] + \
            [torch.cat([t for t in s["grads"] if t.dtype == b.dtype]).double() * scale
             for b in s["buckets"]]
    R = case["R"]
    h, W = s["h"].flatten(0, 1).double(), s["W"].double()
    d = h.shape[1]
    dh = torch.zeros_like(h)
    dW, dc = [], []
    for z in range(R):
        do = s["dout"][:, :, z].flatten(0, 1).double()
        dh += do + do @ W[z * d:(z + 1) * d]
        dW.append(do.T @ h)
        dc.append(do.sum(0))
    return dict(dh=dh.reshape(s["h"].shape), dW=torch.cat(dW), dc=torch.cat(dc))

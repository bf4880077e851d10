"""dbl_sample_logits on the GPU against a plain NumPy form on the oracle's deterministic exponential. Tokens are
equal bit for bit: everything that decides is an integer. logprob is a binary64 logarithm rounded once to
fp32 (2^-24 relative; 2^-23 here)."""
import math

import numpy as np
import pytest
import torch

from oracle import contract as C

pytestmark = pytest.mark.gpu

SEG = 4096  # ids of a row that one workgroup takes at a time


def plain(x, T, k, p, least, word):
    """(token, logprob) of one row x (float32)."""
    V = len(x)
    none = (-1, math.nan)
    if not (0 <= T < math.inf and 0 < p <= 1 and 0 <= least <= 1 and k >= 0) or np.isnan(x).any():
        return none
    T = np.float32(T)
    with np.errstate(over="ignore", divide="ignore", invalid="ignore"):
        s = x / T if T > 0 else x
        if not np.isfinite(s.max()):
            return none
        if T == 0:
            return int(np.argmax(x)), 0.0
        w = np.asarray(C.quant40(C.detexp32((s - s.max()).astype(np.float32))), dtype=np.int64)
    if 0 < k < V:
        w = np.where(s >= np.sort(s)[V - k], w, 0)
    if p < 1:
        total = int(w.sum())
        limit = math.ceil(float(np.float32(p)) * float(total))
        order = np.argsort(-s, kind="stable")
        cum = np.cumsum(w[order])
        w[order[(cum - w[order]) >= limit]] = 0
    w = np.where(w >= float(np.float32(least)) * 2.0 ** 40, w, 0)
    total = int(w.sum())
    v = int(np.searchsorted(np.cumsum(w), (int(word) & 0xFFFFFFFF) * total >> 32, side="right"))
    m = int(w[v])
    return v, math.log1p((m - total) / total) if 2 * m > total else math.log(m / total)


def check(logits, words, **par):
    from paper_2608_05448_amd import dblast as D
    N, V = logits.shape
    dev = {k: (v.cuda() if isinstance(v, torch.Tensor) else v) for k, v in par.items()}
    token, logprob = D.dbl_sample_logits(logits.cuda(), words.cuda(), **dev)
    x = logits.float().numpy()

    def rows(name, default):
        v = par.get(name, default)
        return v.numpy() if isinstance(v, torch.Tensor) else np.full(N, v)

    T, k, p, m = rows("temperature", 1.0), rows("top_k", 0), rows("top_p", 1.0), rows("min_p", 0.0)
    want = [plain(x[i], T[i], int(k[i]), p[i], m[i], int(words[i])) for i in range(N)]
    t, lp = token.cpu().tolist(), logprob.cpu().tolist()
    for i in range(N):
        assert t[i] == want[i][0], (i, V, t[i], want[i], T[i], k[i], p[i], m[i])
        if math.isnan(want[i][1]):
            assert math.isnan(lp[i]), i
        else:
            assert abs(lp[i] - want[i][1]) <= 2.0 ** -23 * abs(want[i][1]), (i, lp[i], want[i])


def rand_words(n, seed):
    return torch.randint(-2 ** 31, 2 ** 31, (n,), generator=torch.Generator().manual_seed(seed)).to(torch.int32)


def rand_logits(n, V, seed, dtype=torch.float32, slope=1.2):
    g = torch.Generator().manual_seed(seed)
    x = 15.0 - slope * torch.log1p(torch.rand((n, V), generator=g) * V) + 0.5 * torch.randn((n, V), generator=g)
    return x.to(dtype)


FILTERS = [dict(), dict(temperature=0.7), dict(temperature=0.0), dict(top_k=1), dict(top_k=5), dict(top_k=50),
           dict(top_p=0.9), dict(top_p=1e-6), dict(temperature=1.5, top_p=0.999), dict(min_p=0.1), dict(min_p=1.0),
           dict(min_p=1e-7), dict(top_k=40, top_p=0.8), dict(top_k=300, top_p=0.95, min_p=0.001),
           dict(top_p=0.99, min_p=0.02), dict(top_k=10 ** 9), dict(top_k=100, min_p=0.3)]
SIZES = [1, 2, 5, 127, 1000, SEG - 1, SEG, SEG + 1, 2 * SEG, 50257]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", SIZES)
def test_filters(V, dtype):
    x, words = rand_logits(4, V, V, dtype), rand_words(4, V)
    for f in FILTERS:
        print(f"[draw] V={V} {dtype} {f}", flush=True)
        check(x, words, **f)


@pytest.mark.parametrize("V", [20000, 151936])
def test_lists_sums_and_radix(V):
    """Kept sets that a list holds, that only sums by segment hold, and that neither does: flat rows with many ids
    in a bin of the maximum's distance, large top-k with top-p, many equal values."""
    g = torch.Generator().manual_seed(1)
    rows = torch.stack([rand_logits(1, V, 2, slope=0.3)[0], torch.randn(V, generator=g) * 0.01,
                        torch.zeros(V), torch.round(torch.randn(V, generator=g) * 2),
                        torch.where(torch.rand(V, generator=g) < 0.5, 1.0, 0.0),
                        torch.randn(V, generator=g) * 6])
    for f in [dict(top_p=0.9), dict(top_p=0.5), dict(top_k=6000), dict(top_k=6000, top_p=0.9),
              dict(top_k=V - 1, top_p=0.999), dict(min_p=0.9), dict(min_p=0.3), dict(top_p=0.9, min_p=0.2),
              dict(top_k=5000, min_p=0.4), dict(top_k=50), dict(top_k=7000, top_p=0.7, min_p=0.1)]:
        print(f"[draw] V={V} {f}", flush=True)
        check(rows, rand_words(len(rows), 5), **f)


def test_words_reach_every_kept_id_and_no_other():
    """The smallest and the largest words take the first and the last kept id."""
    x = rand_logits(2, 3000, 3).repeat(4, 1)
    words = torch.tensor([0, 0, -1, -1, 1, 1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    for f in FILTERS:
        check(x, words, **f)


def test_parameters_by_row():
    N, V = 60, 9001
    g = torch.Generator().manual_seed(4)
    pick = lambda v, dt=torch.float32: torch.tensor(v, dtype=dt)[torch.randint(0, len(v), (N,), generator=g)]
    for dtype in (torch.float32, torch.bfloat16):
        x, words = rand_logits(N, V, 8, dtype), rand_words(N, 9)
        check(x, words, temperature=pick([0.0, 0.5, 1.0, 1.7]), top_k=pick([0, 1, 30, 5000, 9000], torch.int32),
              top_p=pick([1.0, 0.3, 0.9, 0.999]), min_p=pick([0.0, 0.01, 0.5]))
        # values out of range make a row without a token, whatever the others are
        check(x, words, temperature=pick([-1.0, float("nan"), float("inf"), 1.0, -0.0]),
              top_k=pick([-1, 0, 3], torch.int32), top_p=pick([0.0, 1.5, 1.0, 0.5, float("nan")]),
              min_p=pick([-0.5, 0.0, 1.5, 0.1]))


@pytest.mark.parametrize("V", [7, 5000, 17000])
def test_masked_and_broken_rows(V):
    inf, nan = float("inf"), float("nan")
    x = rand_logits(12, V, 11)
    x[0] = -inf
    x[1, :] = -inf
    x[1, V - 1] = 2.0
    x[2, 3] = nan
    x[3, 4] = inf
    x[4, ::2] = -inf
    x[5] = torch.finfo(torch.float32).min
    x[6, 1:] = torch.finfo(torch.float32).min
    x[7, V // 2] = -nan
    x[8] = -0.0
    x[8, ::3] = 0.0
    x[9, 2] = 3e38
    x[10] = -1e30
    for f in [dict(), dict(top_k=3), dict(top_p=0.7), dict(min_p=0.2), dict(temperature=0.0),
              dict(temperature=1e-30), dict(temperature=1e30, top_k=2, top_p=0.5)]:
        print(f"[draw] masked V={V} {f}", flush=True)
        check(x, rand_words(12, 12), **f)


def test_rows_do_not_depend_on_the_batch_or_the_split():
    from paper_2608_05448_amd import dblast as D
    x, words = rand_logits(33, 30001, 21, torch.bfloat16).cuda(), rand_words(33, 22).cuda()
    for f in FILTERS:
        t, lp = D.dbl_sample_logits(x, words, **f)
        for i in (0, 7, 32):
            a, b = D.dbl_sample_logits(x[i:i + 1].clone(), words[i:i + 1].clone(), **f)
            assert int(a) == int(t[i]) and float(b) == float(lp[i])


def test_agrees_with_the_target_transform():
    """Tokens have positive probability under dbl_target_logprobs and logprob is theirs (both to 2^-20)."""
    from paper_2608_05448_amd import dblast as D
    x, words = rand_logits(40, 20000, 31).cuda(), rand_words(40, 32).cuda()
    for f in [dict(), dict(top_k=20), dict(top_p=0.9), dict(top_k=100, top_p=0.7), dict(temperature=0.6, top_p=0.95)]:
        t, lp = D.dbl_sample_logits(x, words, **f)
        want = D.dbl_target_logprobs(x, **f).gather(1, t.long()[:, None])[:, 0]
        assert bool(torch.isfinite(want).all())
        assert float((lp - want).abs().max()) <= 2.0 ** -20 * float(1 + want.abs().max())


def test_graphs_that_share_a_workspace():
    from paper_2608_05448_amd import dblast as D
    N, V = 9, 20000
    ws = torch.empty(D.dbl_workspace_bytes(D.DBL_OP_SAMPLE_LOGITS, N, 1, 1, 1, V), dtype=torch.uint8, device="cuda")
    xs = [rand_logits(N, V, s).cuda() for s in (1, 2)]
    words = rand_words(N, 3).cuda()
    pars = [dict(top_p=0.9), dict(top_k=40, min_p=0.01)]
    outs = [(torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, device="cuda")) for _ in xs]

    def step(i):
        D.dbl_sample_logits(xs[i], words, **pars[i], token=outs[i][0], logprob=outs[i][1], ws=ws)

    eager, graphs = [], []
    for i in (0, 1):
        step(i)
        eager.append([t.clone() for t in outs[i]])
    torch.cuda.synchronize()
    for i in (0, 1):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(i)
        graphs.append(g)
    for rep in range(3):
        ws.fill_(255)
        for i in (0, 1, 1, 0):
            for t in outs[i]:
                t.fill_(-5)
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i][0], eager[i][0]) and torch.equal(outs[i][1], eager[i][1]), (rep, i)
            step(i)

"""Calls whose launch would need 2^32 threads, which the device drops without an error: refused as DBL_EHIP before
anything is launched, at the first size that does not fit; the largest that does is computed whole."""
import pytest
import torch

pytestmark = pytest.mark.gpu

N = 1 << 24  # workgroups of 256 threads


def _refused(call):
    from paper_2608_05448_amd import dblast as D
    with pytest.raises(D.DblastError) as e:
        call()
    assert e.value.status == D.DBL_EHIP, str(e.value)


def _blocks(B):
    """Branch log-probabilities of blocks of one position, one category and one id, drafted 0."""
    z = torch.zeros((B, 1, 1, 1), device="cuda")
    return z, z.clone(), torch.zeros((B, 1, 1), device="cuda"), torch.zeros((B, 1), device="cuda")


def test_sample_block():
    from paper_2608_05448_amd import dblast as D
    args = _blocks(N)
    _refused(lambda: D.dbl_sample_block(*args))
    z, x = (torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((N - 1,), (N - 1, 1)))
    D.dbl_sample_block(*[t[:-1].contiguous() for t in args], z_out=z, x_out=x)
    assert bool((z == 0).all()) and bool((x == 0).all())


def test_verify_expected_len_and_objective():
    from paper_2608_05448_amd import dblast as D
    args = _blocks(N)
    x = torch.zeros((N, 1), dtype=torch.int32, device="cuda")
    logp = torch.zeros((N, 1, 1), device="cuda")
    _refused(lambda: D.dbl_verify_block(*args, x, logp))
    _refused(lambda: D.dbl_verify_block(*args, x, logp, want_beta=False, want_exp_len=False))
    _refused(lambda: D.dbl_expected_len(*args, x, logp))
    _refused(lambda: D.dbl_acceptance_objective(*args, x, logp))
    xh = torch.zeros((N, 1, 1), dtype=torch.int32, device="cuda")
    _refused(lambda: D.dbl_verify_greedy(xh, args[3], x, logp))
    _refused(lambda: D.dbl_expected_len_greedy(xh, args[3], x, logp))
    less = [t[:-1].contiguous() for t in (*args, x, logp)]
    out = D.dbl_verify_block(*less)
    assert bool((out["n_accept"] == 1).all()) and bool((out["accept_mass"] == 1).all())


def test_sample_greedy():
    from paper_2608_05448_amd import dblast as D
    B = 1 << 26  # of 64 threads
    xh, prior = torch.zeros((B, 1, 1), dtype=torch.int32, device="cuda"), torch.zeros((B, 1), device="cuda")
    _refused(lambda: D.dbl_sample_greedy(xh, prior))


def test_target_rows():
    from paper_2608_05448_amd import dblast as D
    lib = D.load()

    def run(n, k):
        x, y = torch.zeros((n, 2), device="cuda"), torch.full((n, 2), 7.0, device="cuda")
        status = lib.dbl_target_logprobs(n, 2, x.data_ptr(), 1.0, k, 1.0, y.data_ptr(), None, 0,
                                         torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return status, y

    for n, k in ((1 << 22, 1), (N, 0)):  # 1024 threads a row under filters, 256 without
        status, y = run(n, k)
        assert status == D.DBL_EHIP and bool((y == 7.0).all())
        status, y = run(n - 1, k)
        assert status == D.DBL_OK and bool(((y - torch.log(torch.tensor(0.5))).abs() < 1e-6).all())


def test_prior_head():
    from paper_2608_05448_amd import dblast as D
    h = torch.ones((N, 8), dtype=torch.bfloat16, device="cuda")
    U, e = torch.ones((1, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.bfloat16, device="cuda")
    _refused(lambda: D.dbl_prior_head(h, U, e))
    assert bool((D.dbl_prior_head(h[:-1], U, e) == 8).all())

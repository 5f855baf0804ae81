"""bf16 results of long sums, all products of one sign.

The tensor core cuts low bits off its running sum at every instruction (16 products), towards zero and never coarser than 2^-23 of it.  The library
takes a running sum over at most 1024 products, 64 instructions: half of them on average, 2^-18 of the result, and adds such sums up in fp32 registers
(256 additions at the longest here, of independent roundings: sqrt(256) u = 2^-20).  Rows and columns have factors of their own, so that results lie anywhere
between two bf16 values and their roundings, at most 2^-8 and uniform, cancel in the mean of 80 000 results or more: 2^-8 / sqrt(3) / sqrt(80 000) = 8e-6,
three times that allowed.  So the mean relative error is 2^-18 + 2^-20 + 2.4e-5 < 3e-5 at most; one running sum over 2^18 products is off by 1e-3.
"""
import pytest

from tests.operators_util import U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2402_14139_b200 import nf
    nf.lib()
    nf.nf_set_stream(None)
    return nf, torch


@pytest.mark.parametrize("P,Q,R", [(2048, 2048, 1 << 18), (2048, 2040, (1 << 18) - 8), (256, 320, 1 << 21), (2056, 2048, 1032)])
def test_bf16_results_of_long_sums(env, P, Q, R):
    nf, torch = env
    g = torch.Generator(device="cuda").manual_seed(9)
    some = lambda n: torch.rand((n, R), generator=g, device="cuda", dtype=torch.bfloat16) * (1 + torch.rand((n, 1), generator=g, device="cuda")).to(torch.bfloat16)
    x, w = some(P), some(Q)

    def off(got, b):              # b [R, Q]: relative errors against fp64, in pieces along the sum
        want = torch.zeros((P, b.shape[1]), dtype=torch.float64, device="cuda")
        for k in range(0, R, 1 << 15):
            want += x[:, k:k + (1 << 15)].double() @ b[k:k + (1 << 15)].double()
        e = got.double() / want - 1
        assert float(e.abs().max()) <= 2.0 ** -8 + 2.0 ** -16
        return abs(float(e.mean()))

    # forward: K = R; the input gradient: the sum runs over N = R
    y = torch.empty((P, Q), dtype=torch.bfloat16, device="cuda")
    scratch = torch.full((nf.nf_linear_scratch_bytes(1, P, R, Q),), 0xFF, dtype=torch.uint8, device="cuda")
    nf.nf_linear_forward(1, x, w, None, None, "none", scratch, None, y)
    assert off(y, w.t()) <= 3e-5
    v = w.t().contiguous()
    del w
    scratch = torch.full((nf.nf_linear_scratch_bytes(1, P, Q, R),), 0xFF, dtype=torch.uint8, device="cuda")
    y.fill_(float("nan"))
    nf.nf_linear_dgrad(1, x, v, scratch, y)
    assert off(y, v) <= 3e-5
    assert nf.nf_op_status() == 0


@pytest.mark.parametrize("M,K,N", [(2100, 1100, 2048), (2048, 2500, 2050), (300, 5000, 260)])
def test_epilogue_behind_sums_in_pieces(env, M, K, N):
    """Bias, shortcut, kept sum and activation behind sums longer than 1024, large tiles and small, rows that TMA stores and rows it cannot."""
    nf, torch = env
    g = torch.Generator(device="cuda").manual_seed(10)
    x = torch.randn((M, K), generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn((N, K), generator=g, device="cuda") * K ** -0.5).to(torch.bfloat16)
    b, r = torch.randn(N, generator=g, device="cuda"), torch.randn((M, N), generator=g, device="cuda").to(torch.bfloat16)
    pre, y = (torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    scratch = torch.full((nf.nf_linear_scratch_bytes(1, M, K, N),), 0xFF, dtype=torch.uint8, device="cuda")
    nf.nf_linear_forward(1, x, w, b, r, "relu", scratch, pre, y)
    z = x.double() @ w.double().t() + b.double() + r.double()
    mag = x.double().abs() @ w.double().abs().t()
    slack = K * U * mag + 3 * U * (z.abs() + b.double().abs() + r.double().abs())
    allowed = slack + 2.0 ** -8 * (z.abs() + slack)
    assert bool(((pre.double() - z).abs() <= allowed).all()) and bool(((y.double() - z.clamp(min=0)).abs() <= allowed).all())
    assert nf.nf_op_status() == 0

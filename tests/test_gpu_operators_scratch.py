"""Scratch allocated once for the largest batch serves every smaller one with the same bits, and no call writes behind what it asked for."""
import pytest

from tests.operators_util import storage

pytestmark = pytest.mark.gpu
GUARD = 1 << 20


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2402_14139_b200 import nf
    nf.lib()
    nf.nf_set_stream(None)
    return nf, torch


def _buffer(torch, n):
    whole = torch.full((n + GUARD,), 0xFF, dtype=torch.uint8, device="cuda")
    return whole[:n], whole[n:]


def _same(torch, a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("K,N,rows", [(1024, 512, (2100, 512, 129, 128, 64, 24, 7, 1)), (4096, 1000, (1777, 300, 64, 25, 3, 1)), (200, 72, (9000, 129, 3)),
                                      (1003, 517, (700, 128, 5)), (8192, 4096, (1024, 128, 64, 1))])
def test_linear_layers_at_smaller_batches(env, K, N, rows, dtype):
    nf, torch = env
    td, need = storage(torch, dtype), nf.nf_linear_scratch_bytes(dtype, rows[0], K, N)
    g = torch.Generator(device="cuda").manual_seed(21)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda").to(td)
    w, shared = randn(N, K), _buffer(torch, need)
    for M in rows:
        x, d = randn(M, K), randn(M, N)
        results = []
        for scratch, guard in (shared, _buffer(torch, nf.nf_linear_scratch_bytes(dtype, M, K, N))):
            y, dx, dw, db = (torch.full(s, float("nan"), dtype=t, device="cuda") for s, t in
                             (((M, N), td), ((M, K), td), ((N, K), torch.float32), ((N,), torch.float32)))
            for call in (lambda: nf.nf_linear_forward(dtype, x, w, None, None, "relu", scratch, None, y), lambda: nf.nf_linear_dgrad(dtype, d, w, scratch, dx),
                         lambda: nf.nf_linear_wgrad(dtype, x, d, scratch, dw, db)):
                scratch.fill_(0xFF)
                call()
            results.append((y, dx, dw, db))
            assert bool((guard == 0xFF).all()) and all(bool(t.isfinite().all()) for t in results[-1])
        assert _same(torch, *results), M
        with pytest.raises(nf.NfError):
            nf.nf_linear_dgrad(dtype, d, w, scratch[:-1], dx)
    assert nf.nf_op_status() == 0


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("P,C,G,images", [(49, 64, 8, (2000, 300, 17, 1)), (3136, 64, 8, (600, 40, 3, 1)), (300, 48, 4, (1300, 64, 1)), (16, 512, 32, (8602, 150, 2)),
                                          (1, 30, 3, (2500, 7))])
def test_group_norm_at_smaller_batches(env, P, C, G, images, dtype):
    nf, torch = env
    td = storage(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(22)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")
    ga, be, shared = 1 + 0.1 * randn(C), randn(C), _buffer(torch, nf.nf_group_norm_scratch_bytes(dtype, images[0], P, C, G))
    for N in images:
        x, dy = randn(N, P, C).to(td), randn(N, P, C).to(td)
        mean, rstd = 0.1 * randn(N, G), 1 + 0.1 * randn(N, G).abs()
        results = []
        for scratch, guard in (shared, _buffer(torch, nf.nf_group_norm_scratch_bytes(dtype, N, P, C, G))):
            scratch.fill_(0xFF)
            dx, dga, dbe = torch.full_like(x, float("nan")), torch.full((C,), float("nan"), device="cuda"), torch.full((C,), float("nan"), device="cuda")
            nf.nf_group_norm_backward(dtype, x, dy, ga, be, mean, rstd, "silu", scratch, dx, dga, dbe)
            results.append((dx, dga, dbe))
            assert bool((guard == 0xFF).all()) and all(bool(t.isfinite().all()) for t in results[-1])
        assert _same(torch, *results), N
    assert nf.nf_op_status() == 0

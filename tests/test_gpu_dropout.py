"""Dropout against the oracle's generator: the same bits for every element, storage type and offset."""
import numpy as np
import pytest

from oracle import nfo_ops as oo
from tests.operators_util import storage

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2402_14139_b200 import nf
    nf.lib()
    nf.nf_set_stream(None)
    return nf, torch


def _want(torch, x, p, seed, offset):
    v = oo.dropout(x.float().cpu().numpy(), p, seed, offset)
    return torch.from_numpy(v).to(x.dtype)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 31, 255, 2048, 2049, 4100, 20003])
def test_bits(env, n, dtype):
    nf, torch = env
    x = torch.from_numpy(np.random.default_rng(n).standard_normal(n).astype(np.float32)).cuda().to(storage(torch, dtype))
    for p, seed, offset in ((0.0, 1, 2), (0.1, 0xFEDCBA9876543210, 0), (0.5, 3, (1 << 63) + 5), (0.999999, 1 << 40, 77)):
        y = torch.full((n + 16,), 7.0, dtype=x.dtype, device="cuda")
        nf.nf_dropout(dtype, x, p, seed, offset, y[:n])
        assert torch.equal(y[:n].cpu(), _want(torch, x, p, seed, offset))
        assert (y[n:] == 7).all()


def test_in_place_and_as_its_own_gradient(env):
    nf, torch = env
    x = torch.ones(5000, device="cuda")
    y = torch.empty_like(x)
    nf.nf_dropout(0, x, 0.3, 11, 12, y)
    nf.nf_dropout(0, x, 0.3, 11, 12, x)       # the gradient of a vector of ones, in place
    assert torch.equal(x, y) and 0.25 < float((y == 0).float().mean()) < 0.35


def test_dropped_nonfinite_values_are_zero(env):
    nf, torch = env
    x = torch.full((4096,), float("inf"), device="cuda")
    x[1::2] = float("nan")
    y = torch.empty_like(x)
    nf.nf_dropout(0, x, 0.5, 5, 6, y)
    kept = torch.from_numpy(oo.dropout(np.ones(4096, dtype=np.float32), 0.5, 5, 6)).cuda() != 0
    assert (y[~kept] == 0).all() and not torch.isfinite(y[kept]).any()


def test_recorded_step_draws_anew_with_its_counter(env):
    """The device counter is added to the offset, past 32 bits too; a graph that advances it never repeats a mask."""
    nf, torch = env
    x = torch.ones(3000, device="cuda")
    y = torch.empty_like(x)
    step = torch.tensor([(1 << 33) + 1], dtype=torch.int64, device="cuda")
    nf.nf_dropout(0, x, 0.5, 9, 4, y, offset_dev=step)
    assert torch.equal(y.cpu(), _want(torch, x, 0.5, 9, (1 << 33) + 5))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nf.nf_set_stream(torch.cuda.current_stream())
        nf.nf_dropout(0, x, 0.5, 9, 4, y, offset_dev=step)
        step.add_(1)
    nf.nf_set_stream(None)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.cpu(), _want(torch, x, 0.5, 9, (1 << 33) + 5 + k))


def test_elements_beyond_32_bits(env):
    """Element 2^32 + 40 uses block 2^30 + 10 of the generator."""
    nf, torch = env
    n = (1 << 32) + 64
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    nf.nf_dropout(1, x, 0.5, 21, 22, x)
    words = np.empty((16, 4), dtype=np.uint32)
    for i in range(16):
        b = (1 << 30) + i
        c, k = [b & 0xFFFFFFFF, b >> 32, 22, 0], [21, 0]
        for _ in range(10):
            p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        words[i] = c
    want = np.where(words.reshape(-1) >= (1 << 31), 2.0, 0.0)
    assert np.array_equal(x[1 << 32:].float().cpu().numpy(), want)

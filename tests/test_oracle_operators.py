"""Pins of the operators' fp64 oracle: against autograd in double precision, finite differences, published test vectors and hand values."""
import numpy as np
import pytest
import torch

from oracle import nfo_ops as oo


def _data(seed, N, P, C):
    r = np.random.default_rng(seed)
    return (r.standard_normal((N, P, C)) + 0.5 * r.standard_normal(C), r.standard_normal((N, P, C)), 1 + 0.3 * r.standard_normal(C),
            0.3 * r.standard_normal(C))


@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("shape", [(2, 5, 12, 3), (3, 1, 8, 2), (1, 7, 6, 6), (2, 4, 5, 1)])
def test_group_norm_against_autograd(kind, shape):
    N, P, C, G = shape
    x, dy, ga, be = _data(1, N, P, C)
    t = torch.from_numpy(x).transpose(1, 2).contiguous().requires_grad_()
    tg, tb = torch.from_numpy(ga).requires_grad_(), torch.from_numpy(be).requires_grad_()
    z = torch.nn.functional.group_norm(t, G, tg, tb, 1e-5)
    y = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[kind](z)
    y.backward(torch.from_numpy(dy).transpose(1, 2))
    got, mean, rstd, _ = oo.group_norm(x, ga, be, G, 1e-5, kind)
    np.testing.assert_allclose(got, y.detach().transpose(1, 2).numpy(), rtol=1e-10, atol=1e-12)
    dx, dga, dbe, _, _ = oo.group_norm_grad(x, dy, ga, be, mean, rstd, kind)
    np.testing.assert_allclose(dx, t.grad.transpose(1, 2).numpy(), rtol=1e-8, atol=1e-10)
    np.testing.assert_allclose(dga, tg.grad.numpy(), rtol=1e-9, atol=1e-11)
    np.testing.assert_allclose(dbe, tb.grad.numpy(), rtol=1e-9, atol=1e-11)


def test_group_norm_gradient_against_differences():
    x, dy, ga, be = _data(2, 2, 3, 4)
    f = lambda v: float((oo.group_norm(v, ga, be, 2, 1e-3, "silu")[0] * dy).sum())
    mean, rstd = oo.group_stats(x, 2, 1e-3)
    dx = oo.group_norm_grad(x, dy, ga, be, mean, rstd, "silu")[0]
    for i in np.ndindex(x.shape):
        h = np.zeros_like(x)
        h[i] = 1e-5
        assert abs((f(x + h) - f(x - h)) / 2e-5 - dx[i]) <= 1e-8


@pytest.mark.parametrize("kind", ["relu", "silu", "gelu"])
def test_activation_gradients_against_differences(kind):
    z = np.linspace(-6, 6, 97) + 0.013
    d = (oo.act(z + 1e-6, kind) - oo.act(z - 1e-6, kind)) / 2e-6
    np.testing.assert_allclose(oo.act_grad(z, kind), d, atol=1e-8)


def test_linear_against_autograd():
    r = np.random.default_rng(3)
    x, w, b, s = r.standard_normal((4, 6)), r.standard_normal((5, 6)), r.standard_normal(5), r.standard_normal((4, 5))
    y, z = oo.linear(x, w, b, s, "gelu")
    want = torch.nn.functional.gelu(torch.nn.functional.linear(torch.from_numpy(x), torch.from_numpy(w), torch.from_numpy(b)) + torch.from_numpy(s))
    np.testing.assert_allclose(y, want.numpy(), rtol=1e-12, atol=1e-14)


def test_philox_against_its_published_vectors():
    """Known answers of philox4x32-10 that its authors distribute, for counters that a (block, offset) pair can take."""
    assert [hex(v) for v in oo.philox(0, 0, 1)[0]] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    # counter 243f6a88 85a308d3 13198a2e 03707344, key a4093822 299f31d0: one round trip through the same rounds, block number given
    c, k = [0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    assert [hex(v) for v in c] == ["0xd16cfe09", "0x94fdcceb", "0x5001e420", "0x24126ea1"]


def test_dropout_keeps_the_mean_and_the_rate():
    y = oo.dropout(np.ones(20000, dtype=np.float32), 0.25, 7, 1 << 40)
    assert abs((y == 0).mean() - 0.25) < 5 * np.sqrt(0.25 * 0.75 / 20000) and set(np.unique(y)) == {np.float32(0), np.float32(1 / 0.75)}


def test_e4m3_codes_against_the_library_type():
    v = oo.e4m3_values()
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    np.testing.assert_array_equal(np.isnan(v), np.isnan(t))
    np.testing.assert_array_equal(v[~np.isnan(v)], t[~np.isnan(t)])
    q = np.random.default_rng(4).standard_normal(4000).astype(np.float32) * np.float32(60)
    q = np.concatenate([q, (v[:126] + v[1:127])[:126].astype(np.float32) / 2, np.float32([448.0, -448.0, 0.0, 1e-9])])   # ties too
    want = torch.from_numpy(q).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(oo._e4m3_code(q), want)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_quantiser_error_is_half_a_step(fmt):
    x = np.random.default_rng(5).standard_normal((7, 150)).astype(np.float32)
    x[2] = 0
    codes, scales = oo.quantize(x, fmt, 64)
    back = oo.dequantize(codes, scales, fmt, 64).astype(np.float64)
    s = np.repeat(scales, 64, axis=1)[:, :150]
    # half a step of the code, and the fp32 roundings of the reciprocal, product, scale and product (2^-24 each)
    step = 0.5 * s if fmt == "int8" else np.maximum(2.0 ** -4 * np.abs(x), s * 2.0 ** -10)
    assert (np.abs(back - x) <= step + 4 * 2.0 ** -24 * 448 * s).all()
    assert (codes[2] == 0).all() and (back[2] == 0).all()

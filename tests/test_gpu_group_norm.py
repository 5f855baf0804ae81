"""Group normalisation with its activation, forward and backward, against the fp64 oracle.

Tolerances.  u = 2^-24.  A thread adds in fp32 what it sees of a group, at most 8 channels of the image's P pixels, then come a tree of 5 levels
over lanes, up to 16 warps and the blocks' means: T = 8 P + 32 roundings at most.  What is added are distances from a value of the group
itself, so at most its range D: a mean is off by T u D and u |mean| for its own rounding, a variance by (T + 4) u D^2; xh and z add one
rounding per operation.  In units of the normalised value: |xh| error <= E = u ((T + 8) (1 + |xh|) (1 + D / sigma)^2 + |mean| / sigma).  The
activations have slopes of at most 1.13.
"""
import numpy as np
import pytest

from oracle import nfo_ops as oo
from tests.operators_util import U, check, host, put, put_f32, storage

pytestmark = pytest.mark.gpu

SHAPES = [  # N, P, C, groups
    (1, 1, 1, 1), (3, 1, 8, 4), (2, 1, 30, 1), (1, 5, 7, 7), (2, 9, 15, 5), (4, 16, 512, 32), (5, 4, 24, 3), (2, 49, 64, 32), (3, 100, 36, 9),
    (2, 63, 8, 8), (1, 784, 16, 2), (1, 1024, 64, 16), (300, 4, 64, 8), (1300, 1, 16, 4), (1, 333, 520, 13), (2, 7, 2056, 1), (1, 30, 4096, 1),
    (1, 6, 8192, 4), (1, 5, 4099, 4099), (2, 3000, 32, 32), (1, 20000, 16, 4), (3, 50000, 64, 16),
    (2, 41000, 64, 32), (5, 169, 20, 4), (3, 50, 6, 3), (2, 90, 30, 10),
]


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2402_14139_b200 import nf
    nf.lib()
    nf.nf_set_stream(None)
    return nf, torch


def _inputs(seed, N, P, C, shift):
    r = np.random.default_rng(seed)
    return (r.standard_normal((N, P, C)) + shift * r.standard_normal((N, 1, C)), r.standard_normal((N, P, C)), 1 + 0.3 * r.standard_normal(C),
            0.3 * r.standard_normal(C))


def _spread(x, mean, rstd, G):
    """Per group, over its sigma: the range of its values, and the magnitude of its mean."""
    N, P, C = x.shape
    v = x.reshape(N, P, G, C // G)
    d = (v.max(axis=(1, 3)) - v.min(axis=(1, 3))) * rstd
    return np.repeat(d, C // G, axis=1)[:, None, :], np.repeat(np.abs(mean) * rstd, C // G, axis=1)[:, None, :]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("si", range(len(SHAPES)))
def test_forward_and_backward(env, si, dtype):
    nf, torch = env
    N, P, C, G = SHAPES[si]
    kind = ["relu", "silu", "none", "gelu"][si % 4]
    a = _inputs(100 + si, N, P, C, 0.5)
    (x, xv), (dy, dyv), (ga, gv), (be, bv) = put(torch, a[0], dtype), put(torch, a[1], dtype), put_f32(torch, a[2]), put_f32(torch, a[3])
    eps = 1e-5
    y, mean, rstd = torch.full_like(x, float("nan")), torch.full((N, G), float("nan"), device="cuda"), torch.full((N, G), float("nan"), device="cuda")
    nf.nf_group_norm_forward(dtype, x, ga, be, G, eps, kind, y, mean, rstd)
    wy, wm, wr, wz = oo.group_norm(xv, gv, bv, G, eps, kind)
    T = 8 * P + 32
    spread, offset = _spread(xv, wm, wr, G)
    xh = np.abs((wz - bv) / np.where(gv == 0, 1, gv))
    E = U * ((T + 8) * (1 + xh) * (1 + spread) ** 2 + offset)
    fast = 2.0 ** -20 * (1 + np.abs(wz)) * np.abs(wy) if dtype == 1 and kind == "silu" else 8 * U * (np.abs(wy) + np.abs(wz) * 1e-3)
    check(y, wy, dtype, 1.13 * (np.abs(gv) * E + 3 * U * (np.abs(wz) + np.abs(bv))) + fast, "y")
    sp = spread[:, 0, ::C // G]
    check(mean, wm, 0, (T + 2) * U * sp / wr, "mean")
    check(rstd, wr, 0, wr * (T + 4) * U * (1 + sp) ** 2, "rstd")
    # backward at the statistics the library left
    sb = nf.nf_group_norm_scratch_bytes(dtype, N, P, C, G)
    scratch = torch.full((sb,), 0xFF, dtype=torch.uint8, device="cuda")
    dx, dga, dbe = torch.full_like(x, float("nan")), torch.full((C,), float("nan"), device="cuda"), torch.full((C,), float("nan"), device="cuda")
    nf.nf_group_norm_backward(dtype, x, dy, ga, be, mean, rstd, kind, scratch, dx, dga, dbe)
    mv, rv = host(mean), host(rstd)
    wdx, wdga, wdbe, sa, sb_ = oo.group_norm_grad(xv, dyv, gv, bv, mv, rv, kind)
    # dz: act' has slope <= 1.1 and the error of z is a few u of its parts; the fast sigmoid of bf16 is 2^-20 off
    rs = np.repeat(rv, C // G, axis=1)[:, None, :]
    xh = np.abs(xv - np.repeat(mv, C // G, axis=1)[:, None, :]) * rs
    ez = 0 if kind in ("relu", "none") else 8 * U * (1 + np.abs(gv) * xh + np.abs(bv)) + (2.0 ** -19 * (1 + np.abs(wz)) if dtype == 1 else 0)
    edz = np.abs(dyv) * (ez + 4 * U)
    adz = np.abs(dyv) * 1.13
    mean_of = lambda t: np.repeat(t.reshape(N, P, G, C // G).mean(axis=(1, 3)), C // G, axis=1)[:, None, :]
    e1, e2 = mean_of(np.abs(gv) * (edz + (T + 4) * U * adz)), mean_of(np.abs(gv) * (edz + (T + 4) * U * adz) * (xh + 1))
    m2 = mean_of(np.abs(gv) * adz * xh)
    check(dx, wdx, dtype, rs * (np.abs(gv) * edz + e1 + xh * e2 + 6 * U * (np.abs(gv) * adz + mean_of(np.abs(gv) * adz) + xh * m2)), "dx")
    check(dbe, wdbe, 0, edz.sum(axis=(0, 1)) + (T * min(N, 64) + 4) * U * sb_, "dbeta")
    check(dga, wdga, 0, (edz * (xh + 1)).sum(axis=(0, 1)) + (T * min(N, 64) + 8) * U * sa, "dgamma")
    assert nf.nf_op_status() == 0


def test_mean_far_from_zero_keeps_the_variance(env):
    """Values around 3000 with a deviation of 1: one-pass sums of squares would lose it, sums about the first pixel do not."""
    nf, torch = env
    N, P, C, G = 2, 256, 32, 4
    r = np.random.default_rng(7)
    x, xv = put_f32(torch, 3000 + r.standard_normal((N, P, C)))
    ga, be = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty((N, G), device="cuda"), torch.empty((N, G), device="cuda")
    nf.nf_group_norm_forward(0, x, ga, be, G, 1e-5, "none", y, mean, rstd)
    wm, wr = oo.group_stats(xv, G, 1e-5)
    # range 8 sigma, at most 8 P = 2048 additions a thread: T u D = 2080 * 8 u and the mean's own rounding, 3000 u.  Errors of additions are
    # independent: the variance, a sum of squares below 64, is off by far less than its bound of T u D^2 = 8e-3; sqrt(T) u D^2 = 1.7e-4
    assert np.abs(host(mean) - wm).max() <= (3000 + 2080 * 8) * U
    assert np.abs(host(rstd) / wr - 1).max() <= 0.5 * 1.7e-4


@pytest.mark.parametrize("dtype", [0, 1])
def test_constant_and_nonfinite_images_stay_to_themselves(env, dtype):
    """An image of one value has rstd = 1 / sqrt(eps) and y = act(beta); a NaN in one group of one image reaches that group alone."""
    nf, torch = env
    N, P, C, G = 3, 20, 16, 4
    r = np.random.default_rng(8)
    a = r.standard_normal((N, P, C))
    a[1] = 2.0
    x, xv = put(torch, a, dtype)
    x[2, 7, 5] = float("nan")
    ga, be = torch.ones(C, device="cuda"), torch.full((C,), 0.5, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty((N, G), device="cuda"), torch.empty((N, G), device="cuda")
    nf.nf_group_norm_forward(dtype, x, ga, be, G, 1e-4, "relu", y, mean, rstd)
    assert torch.equal(y[1], torch.full_like(y[1], 0.5)) and float((rstd[1] - 100).abs().max()) <= 1e-4
    bad = torch.isnan(y)
    assert bad[2, :, 4:8].all() and int(bad.sum()) == P * 4


def test_repeatable_in_place_of_other_work_and_on_a_side_stream(env):
    """Same bits on every call, on another stream, and from a replayed graph whose inputs change between replays."""
    nf, torch = env
    N, P, C, G = 70, 196, 128, 32
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn((N, P, C), generator=g, device="cuda").to(torch.bfloat16)
    dy = torch.randn((N, P, C), generator=g, device="cuda").to(torch.bfloat16)
    ga, be = torch.randn(C, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda")
    scratch = torch.empty(nf.nf_group_norm_scratch_bytes(1, N, P, C, G), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(x), torch.empty((N, G), device="cuda"), torch.empty((N, G), device="cuda"), torch.empty_like(x), torch.empty(C, device="cuda"),
           torch.empty(C, device="cuda")]

    def both():
        nf.nf_group_norm_forward(1, x, ga, be, G, 1e-5, "silu", out[0], out[1], out[2])
        nf.nf_group_norm_backward(1, x, dy, ga, be, out[1], out[2], "silu", scratch, out[3], out[4], out[5])

    both()
    first = [t.clone() for t in out]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    nf.nf_set_stream(s)
    for t in out:
        t.record_stream(s)
    both()
    nf.nf_set_stream(None)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, out))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nf.nf_set_stream(torch.cuda.current_stream())
        both()
    nf.nf_set_stream(None)
    keep = x.clone()
    x.copy_(torch.randn((N, P, C), generator=g, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(out[0], first[0])
    x.copy_(keep)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, out))


def test_offsets_beyond_32_bits(env):
    """2.2e9 elements: the last image is as right as the first."""
    nf, torch = env
    N, P, C, G = 33, 512 * 512, 256, 32
    x = torch.zeros((N, P, C), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x[0] = torch.randn((P, C), generator=g, device="cuda").to(torch.bfloat16)
    x[-1] = x[0]
    ga, be = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty((N, G), device="cuda"), torch.empty((N, G), device="cuda")
    nf.nf_group_norm_forward(1, x, ga, be, G, 1e-5, "none", y, mean, rstd)
    assert torch.equal(y[0], y[-1]) and torch.equal(mean[0], mean[-1]) and float(y[0].float().std()) > 0.99 and float(y[1].abs().max()) == 0


def test_an_image_of_more_than_2_to_31_elements(env):
    """Offsets beyond 32 bits, in the held form's last block as well.  A thread adds P / 16 pixels' pieces of 8 over 256 threads of 8 to a pixel: its
    chain is n = P / 512 steps per channel pair and T = n + 40 roundings with the joins, each of them independent and at most u of a running sum: a sum is
    off by less than e = 8 sqrt(T) u of what its terms' magnitudes come to.  Distances from a pivot below 6 sigma have a mean magnitude below 7 and a mean
    square below 37: a mean is off by 7 e, a second moment by 37 e."""
    nf, torch = env
    P, C, G = 37_000_001, 64, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.empty((1, P, C), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    dy = torch.empty((1, P, C), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    ga, be = torch.linspace(0.5, 1.5, C, device="cuda"), torch.linspace(-1, 1, C, device="cuda")
    y, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    mean, rstd = (torch.full((1, G), float("nan"), device="cuda") for _ in range(2))
    nf.nf_group_norm_forward(1, x, ga, be, G, 1e-5, "none", y, mean, rstd)
    scratch = torch.empty(nf.nf_group_norm_scratch_bytes(1, 1, P, C, G), dtype=torch.uint8, device="cuda")
    dga, dbe = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    nf.nf_group_norm_backward(1, x, dy, ga, be, mean, rstd, "none", scratch, dx, dga, dbe)
    s = [torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(4)]          # sums of x, x^2, dy, dy x
    for p in range(0, P, 1 << 20):
        v, d = x[0, p:p + (1 << 20)].double(), dy[0, p:p + (1 << 20)].double()
        for t, w in zip(s, (v, v * v, d, d * v)):
            t += w.sum(0)
        assert bool(y[0, p:p + (1 << 20)].isfinite().all()) and bool(dx[0, p:p + (1 << 20)].isfinite().all())
    M, grp, e = P * (C // G), lambda t: t.reshape(G, C // G).sum(1), 8 * np.sqrt(P / 512 + 40) * U
    wm = grp(s[0]) / M
    wr = 1 / (grp(s[1]) / M - wm * wm + 1e-5).sqrt()
    assert float((mean[0] - wm).abs().max()) <= 7 * e and float((rstd[0] - wr).abs().max()) <= 0.51 * (37 + 2 * 49) * e
    m, r = (t.repeat_interleave(C // G) for t in (wm, wr))
    gd, bd = ga.double(), be.double()
    wdb, wdg = s[2], (s[3] - m * s[2]) * r
    m1, m2 = (grp(gd * t).repeat_interleave(C // G) / M for t in (wdb, wdg))
    off = 0.51 * (37 + 2 * 49) * e                                                       # of xh, for each of 1 + |xh|
    for p in (0, P // 2, 34_700_000, P - 2000):
        xh = (x[0, p:p + 2000].double() - m) * r
        d = dy[0, p:p + 2000].double()
        wy, wdx = xh * gd + bd, r * (gd * d - m1 - xh * m2)
        assert bool(((y[0, p:p + 2000] - wy).abs() <= wy.abs() * 2.0 ** -8 + 1.5 * off * (1 + xh.abs())).all())
        assert bool(((dx[0, p:p + 2000] - wdx).abs() <= wdx.abs() * 2.0 ** -8 + 3 * off * (1 + xh.abs() + d.abs())).all())
    assert nf.nf_op_status() == 0

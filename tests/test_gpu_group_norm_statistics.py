"""Statistics of group normalisation where single values or whole pixels are not like the others, and every form of the kernels at tolerances that
a wrong statistic, an output that ignores x or an empty gradient cannot meet.

Tolerances, u = 2^-24.  A thread takes runs of n <= 40 pixels of up to V = 8 channels, subtracts p from each value and joins (mean, squared deviations)
of the runs.  p is the mean of its first m pixels (n / m <= 10) or of all it has seen.
  - Squares added in a run, q = M2 + n (mean - p)^2: the first run's M2 is at least m (p - mean)^2, so q <= 11 M2; a later run that finds N pixels seen
    adds M2 + D^2 n N / (n + N) to the deviations, D its mean's distance from p, and q = M2 + n D^2 is at most (1 + n / N) times that, n / N < 2.  So
    all that is ever added is at most 11 times the deviations that come out.
  - q is rounded n + V + 2 <= 50 times and s^2 / n, at most q, twice that relative to q: independent roundings of at most u of a running sum, together about
    u sqrt(50 / 3) (1 + 2) q <= 12 u q <= 135 u M2.  Joins of lanes, warps and blocks are a few roundings of positive numbers each: 10 u.
  - A mean is held as two numbers until it is stored, so distances between means are rounded relative to themselves: they count among the joins.
  - rstd has half the relative error of the variance and a rounding or two of its own: 75 u.  Allowed: 128 u = 2^-17.
  - A mean is off by u sqrt(50 / 3) times the root of q / n in a run, 3 sigma at most: 12 u sigma, and by u |mean| where it is rounded: at every join,
    independently, at most 64 of them: 8 u |mean|.  Allowed: 32 u sigma + 16 u |mean|.
  - xh = (x - mean) rstd follows: E = u (128 |xh| + 32 + 16 |mean| rstd), and a few roundings of xh, z and the activation.
Gradients: chains of c terms of a thread, rounded independently, are off by sqrt(c) u of the 2-norm at most (sqrt(c / 6) on average); the joins after them
are shorter than that.
"""
import numpy as np
import pytest

from tests.operators_util import HALF, U, storage

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2402_14139_b200 import nf
    nf.lib()
    nf.nf_set_stream(None)
    return nf, torch


def _act(torch, z, kind):
    """(value, derivative) in fp64"""
    if kind == "relu":
        return z.clamp(min=0), (z > 0).double()
    if kind == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    if kind == "gelu":
        c = 0.5 * torch.erfc(-z / np.sqrt(2.0))
        return z * c, c + z * torch.exp(-0.5 * z * z) / np.sqrt(2 * np.pi)
    return z, torch.ones_like(z)


class _Case:
    """Inputs, the library's forward pass and the definition in fp64 on the device."""

    def __init__(self, env, x, G, kind, dtype, seed=1, eps=1e-5):
        self.nf, self.torch = nf, torch = env
        self.dtype, self.kind, self.G = dtype, kind, G
        self.N, self.P, self.C = N, P, C = x.shape
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.gen = g
        self.x = x.to(storage(torch, dtype))
        self.ga = 1 + 0.3 * torch.randn(C, generator=g, device="cuda")
        self.be = 0.3 * torch.randn(C, generator=g, device="cuda")
        self.y = torch.full_like(self.x, float("nan"))
        self.mean, self.rstd = (torch.full((N, G), float("nan"), device="cuda") for _ in range(2))
        nf.nf_group_norm_forward(dtype, self.x, self.ga, self.be, G, eps, kind, self.y, self.mean, self.rstd)
        v = self.x.double().view(N, P, G, C // G)
        self.wm = v.mean(dim=(1, 3))
        self.wr = 1 / (((v - self.wm[:, None, :, None]) ** 2).mean(dim=(1, 3)) + eps).sqrt()

    def per_channel(self, t):
        return t.double().repeat_interleave(self.C // self.G, dim=1)[:, None, :]

    def check_forward(self, statistics_only=False):
        torch = self.torch
        dev = self.mean.double() - self.wm
        assert bool((dev.abs() <= U * (32 / self.wr + 16 * self.wm.abs())).all()), float((dev.abs() / (U * (32 / self.wr + 16 * self.wm.abs()))).max())
        off = (self.rstd.double() / self.wr - 1).abs().max()
        assert float(off) <= 128 * U, float(off)
        if statistics_only:
            return
        xh = (self.x.double() - self.per_channel(self.wm)) * self.per_channel(self.wr)
        ga, be = self.ga.double(), self.be.double()
        z = xh * ga + be
        want, _ = _act(torch, z, self.kind)
        e = ga.abs() * U * (128 * xh.abs() + 32 + 16 * self.per_channel(self.wm.abs() * self.wr)) + 4 * U * (z.abs() + be.abs())
        fast = (2.0 ** -20 * (1 + z.abs()) * want.abs() if self.dtype == 1 else 8 * U * (want.abs() + 1e-3 * z.abs())) if self.kind in ("silu", "gelu") else 0
        slack = 1.13 * e + fast
        allowed = slack + HALF[self.dtype] * (want.abs() + slack) + 1e-37
        off = (self.y.double() - want).abs() / allowed
        assert float(off.max()) <= 1.0, (float(off.max()), int(off.argmax()))
        # what ignores x, or half of it, is far outside
        for wrong in (_act(torch, be.expand_as(z), self.kind)[0], _act(torch, 0.5 * z, self.kind)[0]):
            assert float(((wrong - want).abs() > allowed).double().mean()) > 0.3

    def check_backward(self, chain):
        """chain: terms of dgamma that one thread adds"""
        nf, torch = self.nf, self.torch
        N, P, C, G = self.N, self.P, self.C, self.G
        dy = torch.randn((N, P, C), generator=self.gen, device="cuda").to(self.x.dtype)
        scratch = torch.full((nf.nf_group_norm_scratch_bytes(self.dtype, N, P, C, G),), 0xFF, dtype=torch.uint8, device="cuda")
        dx = torch.full_like(self.x, float("nan"))
        dga, dbe = (torch.full((C,), float("nan"), device="cuda") for _ in range(2))
        nf.nf_group_norm_backward(self.dtype, self.x, dy, self.ga, self.be, self.mean, self.rstd, self.kind, scratch, dx, dga, dbe)
        ga, be, rs = self.ga.double(), self.be.double(), self.per_channel(self.rstd)
        xh = (self.x.double() - self.per_channel(self.mean)) * rs
        if self.kind == "relu":          # the mask as the operator defines it: every operation rounded to fp32
            f = lambda t: t.float()[:, None, :].repeat_interleave(C // G, dim=2)
            h = (self.x.float() - f(self.mean)) * f(self.rstd)
            dz = dy.double() * (h * self.ga + self.be > 0)
        else:
            dz = dy.double() * _act(torch, xh * ga + be, self.kind)[1]
        e = dz * ga
        m = lambda t: self.per_channel(t.view(N, P, G, C // G).mean(dim=(1, 3)))
        wdx = rs * (e - m(e) - xh * m(e * xh))
        rel = lambda got, want: float((got.double() - want).norm() / want.norm())
        fast = 2.0 ** -19 if self.dtype == 1 and self.kind in ("silu", "gelu") else 0
        few = U * (16 + np.sqrt(chain)) + fast
        assert rel(dbe, dz.sum(dim=(0, 1))) <= few and rel(dga, (dz * xh).sum(dim=(0, 1))) <= few
        assert rel(dx, wdx) <= 16 * U + fast + (HALF[1] if self.dtype == 1 else 0)
        assert nf.nf_op_status() == 0


def _randn(torch, shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda") * scale


SHAPES = [  # N, P, C, groups: a warp, several warps, a block, clusters; held whole and in part; groups within a piece; shapes no piece fits
    (1300, 16, 64, 8), (300, 4, 64, 8), (4, 16, 512, 32), (160, 300, 128, 32), (2, 2304, 64, 1), (3, 9000, 64, 1), (3, 2000, 64, 64), (160, 1000, 64, 16),
    (330, 1500, 32, 8), (9, 12544, 64, 1), (2, 50000, 64, 4), (7, 700, 64, 32), (2, 784, 48, 4), (2, 9000, 24, 2), (2, 600, 30, 3), (2, 9000, 5, 1),
    (3, 3000, 20, 2), (300, 3000, 12, 1), (1, 1, 64, 2), (5, 3, 64, 2), (40, 1, 2048, 1),
]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("si", range(len(SHAPES)))
def test_a_first_value_far_from_the_others(env, si, dtype):
    """The first value of every group of every image is 1000 sigma out; then the whole first pixel and the last one are 0 among values around 1000."""
    _, torch = env
    N, P, C, G = SHAPES[si]
    x = _randn(torch, (N, P, C), 10 + si)
    x[:, 0, ::C // G] = 1000.0
    _Case(env, x, G, "none", dtype).check_forward(statistics_only=True)
    x = _randn(torch, (N, P, C), 20 + si) + 1000
    x[:, 0] = 0
    x[:, -1] = 0
    if P > 3:
        _Case(env, x, G, "none", dtype).check_forward(statistics_only=True)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("si", range(len(SHAPES)))
def test_a_mean_far_from_zero(env, si, dtype):
    """Values around 1000 with a deviation of 1: a mean of a few pixels that was rounded to fp32 would be off by 1000 u, and the squares of distances
    between such means by twice that."""
    _, torch = env
    N, P, C, G = SHAPES[si]
    for P in {P, 3, 6, 40}:
        x = _randn(torch, (min(N, 400), P, C), 50 + si) + 1000
        _Case(env, x, G, "none", dtype).check_forward(statistics_only=True)


def test_a_mean_far_from_zero_in_small_blocks(env):
    """Clusters whose blocks have 36 values of a group, means of up to 4000 sigma."""
    _, torch = env
    x = _randn(torch, (10, 283, 64), 51) + 1000 * _randn(torch, (10, 1, 64), 52)
    _Case(env, x, 64, "none", 0).check_forward(statistics_only=True)


@pytest.mark.parametrize("size", [100.0, 1e4])
def test_dark_borders_and_single_values_of_any_size(env, size):
    """A frame of zeros around values far from zero, and one value in the middle, in the three forms of the kernel."""
    _, torch = env
    for N, H, C, G in ((2, 48, 64, 1), (150, 28, 64, 16), (2, 120, 24, 2)):
        x = _randn(torch, (N, H, H, C), 31) + size
        x[:, :3], x[:, -3:], x[:, :, :3], x[:, :, -3:] = 0, 0, 0, 0
        x[:, H // 2, H // 2, C // 2] = -100 * size
        _Case(env, x.view(N, H * H, C), G, "none", 0).check_forward(statistics_only=True)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("si", range(len(SHAPES)))
def test_every_form_at_tight_tolerances(env, si, dtype):
    _, torch = env
    N, P, C, G = SHAPES[si]
    if P * (C // G) < 12:        # a handful of values: nothing that ignores x would be told apart
        P = 12
    kind = ["relu", "silu", "gelu", "none"][si % 4]
    x = _randn(torch, (N, P, C), 40 + si) + 0.5 * _randn(torch, (N, 1, C), 41 + si)
    c = _Case(env, x, G, kind, dtype)
    c.check_forward()
    # a thread has its channels of every pixel that is its, over all images of its team: at most those of all images on one team of 148 or of N
    c.check_backward(-(-N // 148) * max(1, P * C // 64 // 32))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("kind", ["relu", "silu", "gelu", "none"])
def test_the_ring_from_one_image_to_the_next(env, kind, dtype):
    """More images than there are teams, each larger than what is held and each with a mean and a deviation of its own."""
    _, torch = env
    N, P, C, G = 330, 1500, 64, 8
    x = _randn(torch, (N, P, C), 60) * (0.5 + _randn(torch, (N, 1, 1), 61).abs()) + 3 * _randn(torch, (N, 1, C), 62)
    c = _Case(env, x, G, kind, dtype)
    c.check_forward()
    c.check_backward(3 * P * C // 64 // 32)


def test_an_infinity_gives_its_group_an_infinite_mean(env):
    nf, torch = env
    for N, P, C, G in ((3, 300, 64, 8), (2, 300, 24, 2), (3, 4, 64, 8)):
        for at in (0, P // 2, P - 1):
            x = _randn(torch, (N, P, C), 70)
            x[1, at, 5] = float("inf")
            c = _Case(env, x, G, "none", 0)
            assert float(c.mean[1, 0]) == float("inf") and bool(torch.isnan(c.rstd[1, 0])) and bool(torch.isnan(c.y[1, :, :C // G]).all())
            ok = torch.ones_like(c.y, dtype=torch.bool)
            ok[1, :, :C // G] = False
            assert bool(torch.isfinite(c.y[ok]).all())

"""Linear layers and their gradients against the fp64 oracle.

Tolerances.  A sum of K products whose running value is rounded to fp32 (or cut off, in the tensor cores, at most once per 16 products and
never coarser than 2^-23) is off by at most K u times the sum of the products' magnitudes, u = 2^-24, in whatever order it is taken; bias,
residual and activation add a rounding each.  That bound is loose for long sums, so fp32 results also have to be within
2^-20 of the exact ones in the 2-norm: errors of single roundings are independent, so a chain of n of them is off by about
sqrt(n / 6) u, and no chain of the library is longer than 512 steps before its sum moves on to a higher precision or a shorter chain.
"""
import numpy as np
import pytest

from oracle import nfo_ops as oo
from tests.operators_util import U, check, host, put, put_f32, rel, storage

pytestmark = pytest.mark.gpu

SHAPES = [  # M, K, N
    (1, 1, 1), (1, 8, 8), (1, 4096, 1000), (2, 2048, 10), (3, 64, 200), (5, 33, 7), (7, 512, 129), (8, 1024, 512), (16, 72, 64), (17, 520, 264), (33, 8, 1000),
    (64, 2048, 100), (100, 27, 64), (127, 129, 130), (128, 128, 128), (129, 256, 256), (200, 64, 8), (256, 1000, 96), (300, 264, 520), (511, 511, 511),
    (640, 2056, 264), (1000, 16, 1000), (1777, 256, 72), (2050, 40, 300), (4097, 64, 64), (9000, 24, 10),
    (3600, 72, 1030), (1800, 2000, 2056), (1801, 2009, 2051), (20000, 128, 136),
]

SHAPES += [  # few rows forwards and backwards (whole and odd widths, sums cut into ranges and not), few terms, a thin side of many rows
    (1, 4, 1), (2, 264, 63), (3, 1000, 65), (4, 516, 700), (6, 4096, 4100), (9, 260, 5000), (15, 1001, 130), (23, 72, 2056), (24, 2048, 1000), (25, 128, 640),
    (16, 1028, 68), (17, 1028, 68), (12, 63, 77), (20000, 512, 10), (20000, 10, 512), (30000, 3, 600), (5, 20000, 36), (4, 36, 20000),
]

SHAPES += [  # short products of any number of rows, on either side of what the kernels for few rows take
    (30, 700, 701), (64, 256, 256), (64, 512, 512), (65, 1023, 40), (128, 1000, 100), (256, 256, 256), (1000, 512, 10), (5000, 128, 10), (100, 129, 1000),
    (131072, 4, 68), (131073, 68, 2), (3, 3261, 1941), (8, 2001, 300), (9, 2001, 4097),
]


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2402_14139_b200 import nf
    nf.lib()
    nf.nf_set_stream(None)
    return nf, torch


def _scratch(nf, torch, dtype, M, K, N):
    n = nf.nf_linear_scratch_bytes(dtype, M, K, N)
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")       # NaN whatever type it is read as


def _nan(torch, shape, t):
    return torch.full(shape, float("nan"), dtype=t, device="cuda")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("si", range(len(SHAPES)))
def test_forward(env, si, dtype):
    nf, torch = env
    M, K, N = SHAPES[si]
    r = np.random.default_rng(200 + si)
    td = storage(torch, dtype)
    (x, xv), (w, wv) = put(torch, r.standard_normal((M, K)), dtype), put(torch, r.standard_normal((N, K)) * np.sqrt(2 / K), dtype)
    (b, bv), (s, sv) = put_f32(torch, r.standard_normal(N)), put(torch, r.standard_normal((M, N)), dtype)
    scratch = _scratch(nf, torch, dtype, M, K, N)
    mag = np.abs(xv) @ np.abs(wv).T
    for kind, bias, res, keep in (("none", False, False, False), ("relu", True, True, False), ("silu", True, False, True), ("gelu", False, True, True)):
        y, pre = _nan(torch, (M, N), td), (_nan(torch, (M, N), td) if keep else None)
        nf.nf_linear_forward(dtype, x, w, b if bias else None, s if res else None, kind, scratch, pre, y)
        wy, wz = oo.linear(xv, wv, bv if bias else None, sv if res else None, kind)
        ez = K * U * mag + 3 * U * (np.abs(wz) + (np.abs(bv) if bias else 0) + (np.abs(sv) if res else 0))
        act = 2.0 ** -20 * (1 + np.abs(wz)) * np.abs(wy) if dtype == 1 else 8 * U * (np.abs(wy) + 1e-3 * np.abs(wz))
        check(y, wy, dtype, 1.13 * ez + (act if kind not in ("none", "relu") else 0), kind)
        if keep:
            check(pre, wz, dtype, ez, "pre")
        if dtype == 0:
            assert rel(y, wy) <= 2.0 ** -20
    assert nf.nf_op_status() == 0


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("si", range(len(SHAPES)))
def test_gradients(env, si, dtype):
    nf, torch = env
    M, K, N = SHAPES[si]
    r = np.random.default_rng(300 + si)
    td = storage(torch, dtype)
    (x, xv), (w, wv) = put(torch, r.standard_normal((M, K)), dtype), put(torch, r.standard_normal((N, K)) * np.sqrt(2 / K), dtype)
    (g, gv) = put(torch, r.standard_normal((M, N)), dtype)
    scratch = _scratch(nf, torch, dtype, M, K, N)
    dx, dw, db = _nan(torch, (M, K), td), _nan(torch, (N, K), torch.float32), _nan(torch, (N,), torch.float32)
    nf.nf_linear_dgrad(dtype, g, w, scratch, dx)
    wdx = gv @ wv
    check(dx, wdx, dtype, N * U * (np.abs(gv) @ np.abs(wv)), "dx")
    scratch.fill_(0xFF)
    nf.nf_linear_wgrad(dtype, x, g, scratch, dw, db)
    wdw = gv.T @ xv
    check(dw, wdw, 0, M * U * (np.abs(gv).T @ np.abs(xv)), "dw")
    check(db, gv.sum(axis=0), 0, M * U * np.abs(gv).sum(axis=0), "db")
    assert rel(dw, wdw) <= 2.0 ** -20 and (dtype == 1 or rel(dx, wdx) <= 2.0 ** -20)
    dw2 = _nan(torch, (N, K), torch.float32)
    scratch.fill_(0xFF)
    nf.nf_linear_wgrad(dtype, x, g, scratch, dw2)             # without db; the same bits
    assert torch.equal(dw, dw2) and nf.nf_op_status() == 0


def test_gradients_against_differences(env):
    """f(x, w, b) = sum of dy * silu(x w^T + b + r): the chain of calls against central differences of the oracle."""
    nf, torch = env
    M, K, N = 5, 12, 6
    r = np.random.default_rng(9)
    vals = [r.standard_normal(s) for s in ((M, K), (N, K), (N,), (M, N), (M, N))]
    (x, xv), (w, wv), (b, bv), (s, sv), (dy, dyv) = (put_f32(torch, v) for v in vals)
    scratch = _scratch(nf, torch, 0, M, K, N)
    y, pre, g = (torch.empty((M, N), device="cuda") for _ in range(3))
    dx, dw, db = torch.empty((M, K), device="cuda"), torch.empty((N, K), device="cuda"), torch.empty(N, device="cuda")
    nf.nf_linear_forward(0, x, w, b, s, "silu", scratch, pre, y)
    nf.nf_act_backward(0, "silu", pre, dy, g)
    nf.nf_linear_dgrad(0, g, w, scratch, dx)
    nf.nf_linear_wgrad(0, x, g, scratch, dw, db)
    f = lambda *p: float((oo.linear(*p, "silu")[0] * dyv).sum())
    for got, k in ((dx, 0), (dw, 1), (db, 2), (g, 3)):
        args = [xv, wv, bv, sv]
        for i in np.ndindex(args[k].shape):
            hi, lo = [a.copy() for a in args], [a.copy() for a in args]
            hi[k][i] += 1e-4
            lo[k][i] -= 1e-4
            assert abs((f(*hi) - f(*lo)) / 2e-4 - float(got[i])) <= 2e-5     # third derivative times 1e-8, and fp32 sums of 12


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n", [1, 7, 8, 2049, 10001])
def test_activation_gradient(env, n, dtype):
    nf, torch = env
    r = np.random.default_rng(n)
    (z, zv), (dy, dyv) = put(torch, 3 * r.standard_normal(n), dtype), put(torch, r.standard_normal(n), dtype)
    for kind in ("none", "relu", "silu", "gelu"):
        g = torch.full((n + 8,), 3.0, dtype=z.dtype, device="cuda")
        nf.nf_act_backward(dtype, kind, z, dy, g[:n])
        d = oo.act_grad(zv, kind)
        # act' itself: a few fp32 roundings of its parts (each at most 1 + |z| in size); the fast sigmoid of bf16 as stated beside it
        e = (2.0 ** -19 * (1 + np.abs(zv)) if dtype == 1 else 16 * U) * (1 + np.abs(zv)) if kind in ("silu", "gelu") else 0
        check(g[:n], dyv * d, dtype, np.abs(dyv) * e, kind)
        assert (g[n:] == 3).all()
        h = dy.clone()
        nf.nf_act_backward(dtype, kind, z, h, h)               # in place of dy
        assert torch.equal(h, g[:n])


@pytest.mark.parametrize("dtype", [0, 1])
def test_relu_from_the_output_and_from_the_sum(env, dtype):
    nf, torch = env
    z = torch.randn(3000, device="cuda").to(storage(torch, dtype))
    dy = torch.randn(3000, device="cuda").to(z.dtype)
    a, b = torch.empty_like(z), torch.empty_like(z)
    nf.nf_act_backward(dtype, "relu", z, dy, a)
    nf.nf_act_backward(dtype, "relu", z.clamp(min=0), dy, b)
    assert torch.equal(a, b) and torch.equal(a != 0, (z > 0) & (dy != 0))


def test_nonfinite_rows_stay_to_themselves(env):
    """A NaN in one row of x reaches that row of y alone, in whatever tile the row lies (bf16: an infinity too)."""
    nf, torch = env
    for M, K, N in ((3, 64, 40), (300, 512, 264)):
        for dtype in (0, 1):
            x = torch.randn((M, K), device="cuda").to(storage(torch, dtype))
            w = torch.randn((N, K), device="cuda").to(x.dtype)
            x[1, 5] = float("nan")
            y = torch.empty((M, N), dtype=x.dtype, device="cuda")
            nf.nf_linear_forward(dtype, x, w, None, None, "none", _scratch(nf, torch, dtype, M, K, N), None, y)
            assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2:]).all()


def test_long_sums_keep_fp32_accuracy(env):
    """dw and db over 60 000 rows, all products of one sign: a running sum that drops low bits would show at once."""
    nf, torch = env
    M, K, N = 60000, 64, 72
    for dtype in (0, 1):
        g = torch.Generator(device="cuda")
        g.manual_seed(5)
        x = torch.rand((M, K), generator=g, device="cuda").to(storage(torch, dtype))
        d = torch.rand((M, N), generator=g, device="cuda").to(x.dtype)
        dw, db = torch.empty((N, K), device="cuda"), torch.empty(N, device="cuda")
        nf.nf_linear_wgrad(dtype, x, d, _scratch(nf, torch, dtype, M, K, N), dw, db)
        assert rel(dw, host(d.double().t() @ x.double())) <= 2.0 ** -20 and rel(db, host(d.double().sum(0))) <= 2.0 ** -20


def test_recorded_calls_and_two_of_them(env):
    """Two graphs with scratch of their own replay side by side on two streams and give the eager bits."""
    nf, torch = env
    jobs = []
    for M, K, N, dtype in ((96, 1024, 200, 1), (2100, 264, 328, 0)):
        x, w = torch.randn((M, K), device="cuda").to(storage(torch, dtype)), torch.randn((N, K), device="cuda").to(storage(torch, dtype))
        g = torch.randn((M, N), device="cuda").to(x.dtype)
        out = [torch.empty((M, N), dtype=x.dtype, device="cuda"), torch.empty((M, K), dtype=x.dtype, device="cuda"),
               torch.empty((N, K), device="cuda"), torch.empty(N, device="cuda")]
        sc = _scratch(nf, torch, dtype, M, K, N)

        def run(dtype=dtype, x=x, w=w, g=g, out=out, sc=sc):
            nf.nf_linear_forward(dtype, x, w, None, None, "relu", sc, None, out[0])
            nf.nf_linear_dgrad(dtype, g, w, sc, out[1])
            nf.nf_linear_wgrad(dtype, x, g, sc, out[2], out[3])
        run()
        want = [t.clone() for t in out]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            nf.nf_set_stream(torch.cuda.current_stream())
            run()
        nf.nf_set_stream(None)
        for t in out:
            t.zero_()
        jobs.append((graph, out, want, run))     # run keeps the tensors that the graph reads
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(3):
        for (graph, _, _, _), s in zip(jobs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for _, out, want, _ in jobs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert nf.nf_op_status() == 0

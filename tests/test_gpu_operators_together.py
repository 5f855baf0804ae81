"""The operators as they are used together: a classifier behind a cached block (8-bit cache -> batch -> convolution -> group norm + ReLU ->
linear + SiLU -> dropout -> linear) forward and backward, eager and as a recorded step; and the block-wise driver with its cache in 8 bits."""
import numpy as np
import pytest

from oracle import nfo_ops as oo
from paper_2402_14139_b200 import pipeline, synth
from tests.operators_util import U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2402_14139_b200 import nf
    nf.lib()
    nf.nf_set_stream(None)
    return nf, torch


class _Step:
    """One training step of the classifier on a batch drawn from an 8-bit cache; fp32 activations."""
    N, H, C, Co, G, Hid, K = 6, 8, 16, 24, 6, 40, 10

    def __init__(self, nf, torch, seed):
        self.nf, self.torch = nf, torch
        r = np.random.default_rng(seed)
        f = lambda *s: torch.from_numpy(r.standard_normal(s).astype(np.float32)).cuda()
        e = lambda *s: torch.full(s, float("nan"), device="cuda")
        N, H, C, Co, G, Hid, K = self.N, self.H, self.C, self.Co, self.G, self.Hid, self.K
        D = H * H * Co
        acts = f(20, H, H, C).clamp_(min=0)
        self.codes, self.scales = torch.empty(acts.shape, dtype=torch.uint8, device="cuda"), e(20, H * H * C // 32)
        nf.nf_cache_quantize("e4m3", 0, acts, 32, self.codes, self.scales)
        self.idx = torch.from_numpy(r.permutation(20)[:N].astype(np.int32)).cuda()
        self.labels, self.y = torch.arange(20, dtype=torch.int32, device="cuda") % K, torch.empty(N, dtype=torch.int32, device="cuda")
        self.wc, self.ga, self.be = f(9, Co, C) / np.sqrt(4.5 * C), 1 + 0.2 * f(Co), 0.2 * f(Co)
        self.w1, self.b1, self.w2, self.b2 = f(Hid, D) / np.sqrt(D / 2), 0.1 * f(Hid), f(K, Hid) / np.sqrt(Hid / 2), 0.1 * f(K)
        self.x, self.u, self.a, self.mean, self.rstd = e(N, H, H, C), e(N, H, H, Co), e(N, H, H, Co), e(N, G), e(N, G)
        self.pre, self.h, self.hd, self.z = e(N, Hid), e(N, Hid), e(N, Hid), e(N, K)
        self.dz = f(N, K)                                       # the gradient of whatever loss stands behind the logits
        self.gw2, self.gb2, self.dhd, self.dh, self.g1, self.gw1, self.gb1 = e(K, Hid), e(K), e(N, Hid), e(N, Hid), e(N, Hid), e(Hid, D), e(Hid)
        self.da, self.du, self.dga, self.dbe, self.gwc = e(N, D), e(N, H, H, Co), e(Co), e(Co), e(9, Co, C)
        nb = max(nf.nf_linear_scratch_bytes(0, N, D, Hid), nf.nf_linear_scratch_bytes(0, N, Hid, K), nf.nf_group_norm_scratch_bytes(0, N, H * H, Co, G),
                 nf.nf_conv3x3_wgrad_scratch_bytes(N, H, H, C, Co, 1))
        self.scratch = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def run(self):
        nf, s = self.nf, self.scratch
        N, flat = self.N, self.a.view(self.N, -1)
        nf.nf_cache_gather_quantized("e4m3", self.codes, self.scales, self.labels, self.idx, 32, 0, self.x, self.y)
        nf.nf_conv3x3_forward(0, self.x, self.wc, 1, self.u)
        nf.nf_group_norm_forward(0, self.u, self.ga, self.be, self.G, 1e-5, "relu", self.a, self.mean, self.rstd)
        nf.nf_linear_forward(0, flat, self.w1, self.b1, None, "silu", s, self.pre, self.h)
        nf.nf_dropout(0, self.h, 0.25, 1234, 7, self.hd, offset_dev=self.step)
        nf.nf_linear_forward(0, self.hd, self.w2, self.b2, None, "none", s, None, self.z)
        nf.nf_linear_wgrad(0, self.hd, self.dz, s, self.gw2, self.gb2)
        nf.nf_linear_dgrad(0, self.dz, self.w2, s, self.dhd)
        nf.nf_dropout(0, self.dhd, 0.25, 1234, 7, self.dh, offset_dev=self.step)
        nf.nf_act_backward(0, "silu", self.pre, self.dh, self.g1)
        nf.nf_linear_wgrad(0, flat, self.g1, s, self.gw1, self.gb1)
        nf.nf_linear_dgrad(0, self.g1, self.w1, s, self.da)
        nf.nf_group_norm_backward(0, self.u, self.da.view_as(self.u), self.ga, self.be, self.mean, self.rstd, "relu", s, self.du, self.dga, self.dbe)
        nf.nf_conv3x3_wgrad(0, self.x, self.du, 1, s, self.gwc)
        self.step.add_(1)

    OUT = ("z", "gw2", "gb2", "gw1", "gb1", "dga", "dbe", "gwc")

    def out(self):
        return {k: getattr(self, k).clone() for k in self.OUT}

    def want(self, step):
        """The same in fp64 by autograd; the dropout mask and the cache's values from the oracle."""
        torch, F = self.torch, self.torch.nn.functional
        rows = oo.dequantize(self.codes.cpu().numpy().reshape(20, -1), self.scales.cpu().numpy(), "e4m3", 32)
        x = torch.from_numpy(rows.astype(np.float64)).view(20, self.H, self.H, self.C)[self.idx.cpu().long()].permute(0, 3, 1, 2)
        p = {k: getattr(self, k).double().cpu().requires_grad_() for k in ("wc", "ga", "be", "w1", "b1", "w2", "b2")}
        w = p["wc"].view(3, 3, self.Co, self.C).permute(2, 3, 0, 1)
        a = F.relu(F.group_norm(F.conv2d(x, w, padding=1), self.G, p["ga"], p["be"], 1e-5)).permute(0, 2, 3, 1).reshape(self.N, -1)
        h = F.silu(F.linear(a, p["w1"], p["b1"]))
        mask = torch.from_numpy(oo.dropout(np.ones((self.N, self.Hid), dtype=np.float32), 0.25, 1234, 7 + step)).double()
        z = F.linear(h * mask, p["w2"], p["b2"])
        z.backward(self.dz.double().cpu())
        return dict(z=z.detach(), gw2=p["w2"].grad, gb2=p["b2"].grad, gw1=p["w1"].grad, gb1=p["b1"].grad, dga=p["ga"].grad, dbe=p["be"].grad,
                    gwc=p["wc"].grad)


def _close(torch, got, want):
    # fourteen calls, each off by a few u of its terms, its sums (up to 1536 terms) by up to sqrt(1536) u: 256 u of the whole tensor
    for k in want:
        err = float((got[k].double().cpu() - want[k]).norm() / want[k].norm())
        assert err <= 256 * U, (k, err)


def test_training_step_eager_and_recorded(env):
    nf, torch = env
    s = _Step(nf, torch, 31)
    s.run()
    first = s.out()
    _close(torch, first, s.want(0))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nf.nf_set_stream(torch.cuda.current_stream())
        s.run()
    nf.nf_set_stream(None)
    s.step.zero_()
    for k in range(3):                         # the recorded step draws another mask each time
        s.scratch.fill_(0xFF)
        graph.replay()
        got = s.out()
        _close(torch, got, s.want(k))
        assert torch.equal(got["z"], first["z"]) == (k == 0)
    assert nf.nf_op_status() == 0


def test_two_steps_side_by_side_keep_to_themselves(env):
    """Two recorded steps with buffers of their own replay on two streams at once and give their own results."""
    nf, torch = env
    steps, graphs, want = [_Step(nf, torch, 41), _Step(nf, torch, 42)], [], []
    for s in steps:
        s.run()
        s.step.zero_()
        want.append(s.out())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            nf.nf_set_stream(torch.cuda.current_stream())
            s.run()
        nf.nf_set_stream(None)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in steps]
    for s in steps:
        s.step.zero_()
    torch.cuda.synchronize()
    for g, st in zip(graphs, streams):
        with torch.cuda.stream(st):
            g.replay()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        got = s.out()
        assert all(torch.equal(got[k], w[k]) for k in w)


def _wl(blocks):
    l = lambda Cin, Cout, H, F, pool=False: dict(Cin=Cin, Cout=Cout, H=H, W=H, F=F, stride=1, pool=pool)
    return dict(name="mini", dtype="bf16", classes=4, in_shape=(3, 16, 16),
                blocks=[(6, [l(3, 64, 16, 8), l(64, 64, 16, 8, pool=True)]), (8, [l(64, 128, 8, 16)])][:blocks])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_blockwise_pass_with_its_cache_in_8_bits(env, fmt):
    """The cache of a block is the quantiser's image of what the exact pass caches; the tiers agree bit for bit; the next block trains from it."""
    nf, torch = env
    K = 22                                     # no multiple of either batch size: ragged chunks
    data = torch.from_numpy(synth.round_bf16(synth.normal(6, 1, (K, 16, 16, 3)))).cuda().to(torch.bfloat16)
    labels = torch.from_numpy(synth.labels(6, 2, K, 4)).cuda()
    _, exact = pipeline.train_blockwise(nf, torch, _wl(1), data, labels, epochs=2, lr=0.05, seed=3)
    _, q = pipeline.train_blockwise(nf, torch, _wl(1), data, labels, epochs=2, lr=0.05, seed=3, cache_format=fmt, cache_group=32)
    wc, ws = oo.quantize(exact.float().cpu().numpy().reshape(K, -1), fmt, 32)
    assert q.shape == tuple(exact.shape)
    np.testing.assert_array_equal(q.codes.cpu().numpy().reshape(K, -1), wc)
    np.testing.assert_array_equal(q.scales.cpu().numpy(), ws)
    r0, _ = pipeline.train_blockwise(nf, torch, _wl(2), data, labels, epochs=2, lr=0.05, seed=3)
    r1, q1 = pipeline.train_blockwise(nf, torch, _wl(2), data, labels, epochs=2, lr=0.05, seed=3, cache_format=fmt)
    r2, q2 = pipeline.train_blockwise(nf, torch, _wl(2), data, labels, epochs=2, lr=0.05, seed=3, cache="host", cache_format=fmt)
    assert r0[0]["losses"] == r1[0]["losses"] == r2[0]["losses"] and r1[1]["losses"] == r2[1]["losses"]
    assert q1.is_cuda and not q2.is_cuda and q2.codes.is_pinned()
    assert torch.equal(q1.codes, q2.codes.cuda()) and torch.equal(q1.scales, q2.scales.cuda()) and np.isfinite(r1[1]["losses"]).all()
    with pytest.raises(ValueError):
        pipeline.train_blockwise(nf, torch, _wl(1), data, labels, cache="disk", cache_format=fmt)
    nf.nf_set_stream(None)

"""The activation cache in 8 bits: codes, scales and read-back rows bit for bit against the oracle."""
import numpy as np
import pytest

from oracle import nfo_ops as oo
from tests.operators_util import storage

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 16), (3, 31), (2, 32), (5, 48), (4, 64), (3, 80), (7, 127), (2, 128), (6, 130), (3, 144), (2, 1000), (9, 2048), (3, 4112), (70, 512)]


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2402_14139_b200 import nf
    nf.lib()
    nf.nf_set_stream(None)
    return nf, torch


def _rows(torch, seed, rows, E, dtype):
    r = np.random.default_rng(seed)
    x = r.standard_normal((rows, E)) * np.exp(r.uniform(-30, 30, (rows, 1)))
    x[r.random((rows, E)) < 0.4] = 0
    if rows > 2:
        x[1] = 0
        x[2] *= 1e-36 / np.abs(x[2]).max() if np.abs(x[2]).max() else 1      # below the floor of the scale
    return torch.from_numpy(x.astype(np.float32)).cuda().to(storage(torch, dtype))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("si", range(len(SHAPES)))
def test_codes_scales_and_rows(env, si, fmt, dtype):
    nf, torch = env
    rows, E = SHAPES[si]
    for group in (32, 64, 128):
        x = _rows(torch, 50 + si, rows, E, dtype)
        n = -(-E // group)
        codes = torch.full((rows + 1, E), 0xAA, dtype=torch.uint8, device="cuda")
        scales = torch.full((rows + 1, n), -1.0, device="cuda")
        nf.nf_cache_quantize(fmt, dtype, x, group, codes[:rows], scales[:rows])
        wc, ws = oo.quantize(x.float().cpu().numpy(), fmt, group)
        np.testing.assert_array_equal(scales[:rows].cpu().numpy(), ws)
        np.testing.assert_array_equal(codes[:rows].cpu().numpy(), wc)
        assert (codes[rows:] == 0xAA).all() and (scales[rows:] == -1).all()
        idx = torch.tensor([rows - 1, 0, rows // 2, 0], dtype=torch.int32, device="cuda")      # a row twice
        labels = torch.arange(rows, dtype=torch.int32, device="cuda") + 100
        for out_dtype in (0, 1):
            out = torch.full((5, E), 9.0, dtype=storage(torch, out_dtype), device="cuda")
            ol = torch.zeros(5, dtype=torch.int32, device="cuda")
            nf.nf_cache_gather_quantized(fmt, codes[:rows], scales[:rows], labels, idx, group, out_dtype, out[:4], ol[:4])
            back = torch.from_numpy(oo.dequantize(wc, ws, fmt, group)).to(out.dtype)[idx.cpu().long()]
            assert torch.equal(out[:4].cpu(), back) and (out[4] == 9).all()
            assert ol.tolist() == [100 + rows - 1, 100, 100 + rows // 2, 100, 0]
            nf.nf_cache_gather_quantized(fmt, codes[:rows], scales[:rows], None, idx, group, out_dtype, out[:4], None)
    assert nf.nf_op_status() == 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("E", [96, 97])
def test_every_halfway_point(env, fmt, E):
    """Products that fall exactly between two codes go to the even one: scale 1 (a = top), values on all midpoints."""
    nf, torch = env
    top = 127.0 if fmt == "int8" else 448.0
    if fmt == "int8":
        mid = np.arange(-127, 127) + 0.5
    else:
        v = oo.e4m3_values()[:127]
        mid = np.concatenate([(v[1:] + v[:-1]) / 2, -(v[1:] + v[:-1]) / 2])
    vals = np.zeros((len(mid) // 30 + 1, E))
    vals[:, 0] = top
    vals[:, 32] = -top
    flat = np.resize(mid, vals.shape[0] * 30)
    vals[:, 1:31] = flat.reshape(-1, 30)
    x = torch.from_numpy(vals.astype(np.float32)).cuda()
    codes, scales = torch.empty((x.shape[0], E), dtype=torch.uint8, device="cuda"), torch.empty((x.shape[0], -(-E // 32)), device="cuda")
    nf.nf_cache_quantize(fmt, 0, x, 32, codes, scales)
    wc, ws = oo.quantize(vals.astype(np.float32), fmt, 32)
    assert float(scales[0, 0]) == 1.0
    np.testing.assert_array_equal(codes.cpu().numpy(), wc)


@pytest.mark.parametrize("E", [128, 130])
def test_nonfinite_groups_and_bad_indices(env, E):
    nf, torch = env
    x = torch.ones((4, E), device="cuda")
    x[1, 40] = float("nan")
    x[3, 70] = -float("inf")
    for fmt in ("int8", "e4m3"):
        codes, scales = torch.empty((4, E), dtype=torch.uint8, device="cuda"), torch.empty((4, -(-E // 32)), device="cuda")
        assert nf.nf_op_status() == 0
        nf.nf_cache_quantize(fmt, 0, x, 32, codes, scales)
        assert nf.nf_op_status() == nf.NF_ENONFINITE
        idx = torch.tensor([0, 1, 3, -1, 4, 2**31 - 1, 2], dtype=torch.int32, device="cuda")
        labels, ol = torch.arange(4, dtype=torch.int32, device="cuda"), torch.empty(7, dtype=torch.int32, device="cuda")
        out = torch.full((7, E), 5.0, device="cuda")
        nf.nf_cache_gather_quantized(fmt, codes, scales, labels, idx, 32, 0, out, ol)
        assert nf.nf_op_status() == nf.NF_EINDEX
        assert ol.tolist() == [0, 1, 3, -1, -1, -1, 2]
        nan = torch.isnan(out)
        assert nan[1, 32:64].all() and nan[2, 64:96].all() and int(nan.sum()) == 64
        assert (out[3:6] == 0).all() and (out[0] == 1).all() and (out[6] == 1).all()


def test_cache_in_pinned_host_memory(env):
    """Rows read straight from pinned memory are those of the device-resident cache."""
    nf, torch = env
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((100, 8, 8, 32), generator=g, device="cuda").clamp_(min=0).to(torch.bfloat16)
    codes, scales = torch.empty(x.shape, dtype=torch.uint8, device="cuda"), torch.empty((100, 64), device="cuda")
    nf.nf_cache_quantize("e4m3", 1, x, 32, codes, scales)
    hc, hs = codes.cpu().pin_memory(), scales.cpu().pin_memory()
    idx = torch.randperm(100, generator=g, device="cuda")[:37].to(torch.int32)
    a, b = torch.empty((37, 8, 8, 32), dtype=torch.bfloat16, device="cuda"), torch.empty((37, 8, 8, 32), dtype=torch.bfloat16, device="cuda")
    nf.nf_cache_gather_quantized("e4m3", codes, scales, None, idx, 32, 1, a, None)
    nf.nf_cache_gather_quantized("e4m3", hc, hs, None, idx, 32, 1, b, None)
    assert torch.equal(a, b) and float((a.float() - x[idx.long()].float()).abs().max()) < 0.2


def test_rows_beyond_32_bits(env):
    """A cache of 4.4e9 codes: its last rows are read and written like the first."""
    nf, torch = env
    rows, E = 66, 1 << 26
    codes = torch.empty((rows, E), dtype=torch.uint8, device="cuda")
    scales = torch.empty((rows, E // 128), device="cuda")
    x = torch.zeros((rows, E), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x[0] = torch.randn(E, generator=g, device="cuda").to(torch.bfloat16)
    x[-1] = x[0]
    nf.nf_cache_quantize("int8", 1, x, 128, codes, scales)
    assert torch.equal(codes[0], codes[-1]) and torch.equal(scales[0], scales[-1])
    del x
    out = torch.empty((2, E), dtype=torch.bfloat16, device="cuda")
    nf.nf_cache_gather_quantized("int8", codes, scales, None, torch.tensor([65, 0], dtype=torch.int32, device="cuda"), 128, 1, out, None)
    assert torch.equal(out[0], out[1]) and float(out[0].abs().max()) > 3

"""The block-wise driver with its cache in 8 bits where a chunk of a block's outputs starts at any byte of the cache."""
import numpy as np
import pytest

from oracle import nfo_ops as oo
from paper_2402_14139_b200 import pipeline, synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2402_14139_b200 import nf
    nf.lib()
    nf.nf_set_stream(None)
    return nf, torch


@pytest.mark.parametrize("H,Cout,N,group", [
    (14, 64, 6, 64),     # 7 x 7 x 64: 49 scales a row, the second chunk's scales start at byte 1176
    (14, 64, 5, 128),    # 25 scales a row
    (4, 64, 7, 128),     # 2 x 2 x 64: two scales a row
    (14, 10, 6, 32),     # 490 codes a row: the second chunk's codes start at byte 2940
    (16, 64, 6, 64),     # as a control: every chunk starts at a multiple of 16 bytes
])
def test_chunks_that_start_at_any_byte(env, H, Cout, N, group):
    nf, torch = env
    K = 22
    layers = [dict(Cin=16, Cout=Cout, H=H, W=H, F=8, stride=1, pool=True)]
    wl = dict(name="mini", dtype="bf16", classes=4, in_shape=(16, H, H), blocks=[(N, layers)])
    data = torch.from_numpy(synth.round_bf16(synth.normal(6, 1, (K, H, H, 16)))).cuda().to(torch.bfloat16)
    labels = torch.from_numpy(synth.labels(6, 2, K, 4)).cuda()
    run = lambda **k: pipeline.train_blockwise(nf, torch, wl, data, labels, epochs=1, lr=0.05, seed=3, **k)[1]
    exact = run(cache="host")      # which has buffers of its own for every chunk
    for tier in ("hbm", "host"):
        for fmt in ("int8", "e4m3"):
            q = run(cache=tier, cache_format=fmt, cache_group=group)
            wc, ws = oo.quantize(exact.float().cpu().numpy().reshape(K, -1), fmt, group)
            np.testing.assert_array_equal(q.codes.cpu().numpy().reshape(K, -1), wc)
            np.testing.assert_array_equal(q.scales.cpu().numpy(), ws)
            assert q.is_cuda == (tier == "hbm")
    nf.nf_set_stream(None)

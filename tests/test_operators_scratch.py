"""Scratch sizes: what covers a batch covers every smaller one (no GPU)."""
import random

import pytest


@pytest.fixture(scope="module")
def nf():
    from paper_2402_14139_b200 import build
    build.build()
    from paper_2402_14139_b200 import nf as mod
    return mod


def _sizes(rng, top):
    return max(1, int(2 ** rng.uniform(0, top)))


@pytest.mark.parametrize("dtype", [0, 1])
def test_linear_scratch_grows_with_the_rows(nf, dtype):
    rng = random.Random(3)
    layers = [(8192, 4096), (25088, 4096), (512, 10), (64, 64), (256, 256)]
    layers += [(_sizes(rng, 14), _sizes(rng, 14)) for _ in range(200)] + [(8 * _sizes(rng, 11), 8 * _sizes(rng, 11)) for _ in range(200)]
    for K, N in layers:
        rows = sorted({1, 2, 3, 4, 8, 9, 24, 25, 64, 128, 129, 512, 1777, 8602, 200704} | {_sizes(rng, 17) for _ in range(30)})
        need = [nf.nf_linear_scratch_bytes(dtype, M, K, N) for M in rows]
        assert need == sorted(need) and need[0] > 0, (K, N)
        splits = 148 * 128 * 128 * 4 + 296 * 64 * 64 * 4 + 592 * 8 * 512 * 4         # partial sums are bounded whatever the layer ...
        copies = (3 if dtype == 0 else 1) * 2 * (2 * rows[-1] * (max(K, N) + 8) + (K + 8) * (N + 8) + 4096)
        forced = ((max(K, N) - 1) // 4096 + 1) * 24 * max(K, N) * 4                  # ... but for ranges of very long sums over few rows
        assert need[-1] <= splits + copies + forced + 300 * N * 4 + (1 << 20), (K, N)


@pytest.mark.parametrize("dtype", [0, 1])
def test_group_norm_scratch_grows_with_the_images(nf, dtype):
    rng = random.Random(4)
    for _ in range(300):
        G = rng.choice([1, 2, 3, 4, 5, 8, 16, 32, 64])
        C, P = G * rng.choice([1, 2, 3, 4, 5, 8, 12, 16, 32, 64]), _sizes(rng, 16)
        images = sorted({1, 2, 3, 8, 100, 300, 8602} | {_sizes(rng, 13) for _ in range(20)})
        need = [nf.nf_group_norm_scratch_bytes(dtype, N, P, C, G) for N in images]
        assert need == sorted(need) and 0 < need[-1] <= 2400 * 2 * 4 * max(C, 256), (P, C, G)

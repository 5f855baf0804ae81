"""Every output that shares memory with an input, with scratch or with another output is refused, through the C ABI without a GPU: the refusal comes
before any device work, so the addresses are never used."""
import ctypes as C

import pytest

A = [C.c_void_p(0x100000 * (i + 1)) for i in range(14)]


@pytest.fixture(scope="module")
def nf():
    from paper_2402_14139_b200 import build
    build.build()
    from paper_2402_14139_b200 import nf as mod
    return mod


def _all_refused(nf, f, args, written, read, both_ways=()):
    """Each tensor of `written` (argument positions) laid over each other tensor's first and last bytes.  read, written: {position: bytes}."""
    n = 0
    for w, nw in written.items():
        for o, no in {**read, **written}.items():
            if o == w or args[o] is None or (w, o) in both_ways:
                continue
            for at in (args[o].value, args[o].value + (no - 1) // 16 * 16, args[o].value - (nw - 1) // 16 * 16):
                bad = list(args)
                bad[w] = C.c_void_p(at)
                assert f(*bad) == nf.NF_EINVAL, (f.__name__, w, o, at - args[o].value)
                n += 1
    return n


def test_group_norm(nf):
    L, N, P, C_, G = nf.lib(), 2, 40, 64, 4
    x, c, s = N * P * C_ * 2, C_ * 4, N * G * 4
    assert _all_refused(nf, L.nf_group_norm_forward, [1, A[0], A[1], A[2], N, P, C_, G, 1e-5, 1, A[3], A[4], A[5]],
                        {10: x, 11: s, 12: s}, {1: x, 2: c, 3: c}) == 45
    sb = L.nf_group_norm_scratch_bytes(1, N, P, C_, G)
    assert _all_refused(nf, L.nf_group_norm_backward, [1, A[0], A[1], A[2], A[3], A[4], A[5], N, P, C_, G, 1, A[6], sb, A[7], A[8], A[9]],
                        {12: sb, 14: x, 15: c, 16: c}, {1: x, 2: x, 3: c, 4: c, 5: s, 6: s}) == 108


def test_dropout(nf):
    """The offset on the device may not lie in y: blocks read it while others write."""
    L, n = nf.lib(), 1000
    for at in (0, 8, n * 2 - 8):
        assert L.nf_dropout(1, A[0], n, 0.5, 1, 2, C.c_void_p(A[1].value + at), A[1]) == nf.NF_EINVAL
        assert L.nf_dropout(1, A[1], n, 0.5, 1, 2, C.c_void_p(A[1].value + at), A[1]) == nf.NF_EINVAL


def test_gather_from_the_quantised_cache(nf):
    L, rows, count, E, group = nf.lib(), 50, 40, 1000, 64
    args = [0, A[0], A[1], A[2], rows, A[3], count, E, group, 1, A[4], A[5]]
    read = {1: rows * E, 2: rows * 16 * 4, 3: rows * 4, 5: count * 4}
    assert _all_refused(nf, L.nf_cache_gather_quantized, args, {10: count * E * 2, 11: count * 4}, read) == 30


def test_linear_and_cache_write(nf):
    """As before: these calls compared every pair already."""
    L, M, K, N = nf.lib(), 40, 64, 48
    x, w, y, b = M * K * 2, N * K * 2, M * N * 2, N * 4
    sb = L.nf_linear_scratch_bytes(1, M, K, N)
    assert _all_refused(nf, L.nf_linear_forward, [1, A[0], A[1], A[2], A[3], M, K, N, 1, A[4], sb, A[5], A[6]], {9: sb, 11: y, 12: y},
                        {1: x, 2: w, 3: b, 4: y}) == 54
    assert _all_refused(nf, L.nf_linear_dgrad, [1, A[0], A[1], M, K, N, A[2], sb, A[3]], {6: sb, 8: x}, {1: y, 2: w}) == 18
    assert _all_refused(nf, L.nf_linear_wgrad, [1, A[0], A[1], M, K, N, A[2], sb, A[3], A[4]], {6: sb, 8: 2 * w, 9: b}, {1: x, 2: y}) == 36
    assert _all_refused(nf, L.nf_cache_quantize, [0, 1, A[0], 4, 1000, 64, A[1], A[2]], {6: 4000, 7: 4 * 16 * 4}, {2: 8000}) == 12

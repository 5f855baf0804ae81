"""What the operators refuse, through the C ABI without a GPU: every refusal comes before any device work, so the addresses are never used."""
import ctypes as C

import pytest

A = [C.c_void_p(0x100000 * (i + 1)) for i in range(12)]      # aligned, far apart, never read
ODD = C.c_void_p(0x100008)


@pytest.fixture(scope="module")
def nf():
    from paper_2402_14139_b200 import build
    build.build()
    from paper_2402_14139_b200 import nf as mod
    return mod


def _calls(nf):
    """Per entry point: the function, valid arguments, and for each refusal {position: value} with its code."""
    L = nf.lib()
    E, S = nf.NF_EINVAL, nf.NF_EALIGN
    gsb = L.nf_group_norm_scratch_bytes(1, 2, 4, 16, 4)
    lsb = L.nf_linear_scratch_bytes(1, 4, 16, 8)
    yield L.nf_group_norm_forward, [1, A[0], A[1], A[2], 2, 4, 16, 4, 1e-5, 1, A[3], A[4], A[5]], [
        ({0: 2}, E), ({1: None}, E), ({2: None}, E), ({3: None}, E), ({4: 0}, E), ({5: 0}, E), ({6: 0}, E), ({7: 0}, E), ({7: 5}, E), ({8: 0.0}, E),
        ({8: float("nan")}, E), ({9: 4}, E), ({9: -1}, E), ({10: None}, E), ({11: None}, E), ({12: None}, E), ({1: ODD}, S), ({12: ODD}, S),
        ({10: A[0]}, E), ({10: C.c_void_p(A[0].value + 64)}, E), ({6: 8194, 7: 2}, nf.NF_EUNSUPPORTED)]
    yield L.nf_group_norm_backward, [1, A[0], A[1], A[2], A[3], A[4], A[5], 2, 4, 16, 4, 1, A[6], gsb, A[7], A[8], A[9]], [
        ({0: -1}, E), ({2: None}, E), ({5: None}, E), ({7: 0}, E), ({10: 3}, E), ({11: 9}, E), ({12: None}, E), ({13: gsb - 1}, nf.NF_ENOWS),
        ({14: A[0]}, E), ({14: A[1]}, E), ({15: None}, E), ({16: ODD}, S), ({9: 8194, 10: 2}, nf.NF_EUNSUPPORTED)]
    yield L.nf_linear_forward, [1, A[0], A[1], A[2], A[3], 4, 16, 8, 1, A[4], lsb, A[5], A[6]], [
        ({0: 3}, E), ({1: None}, E), ({2: None}, E), ({5: 0}, E), ({6: 0}, E), ({7: -8}, E), ({8: 7}, E), ({9: None}, E), ({10: lsb - 1}, nf.NF_ENOWS),
        ({12: None}, E), ({3: ODD}, S), ({4: ODD}, S), ({11: ODD}, S), ({12: A[0]}, E), ({12: A[1]}, E), ({12: A[3]}, E), ({11: A[6]}, E)]
    yield L.nf_linear_dgrad, [1, A[0], A[1], 4, 16, 8, A[2], lsb, A[3]], [
        ({0: 3}, E), ({1: None}, E), ({2: None}, E), ({3: 0}, E), ({6: None}, E), ({7: 0}, nf.NF_ENOWS), ({8: None}, E), ({8: ODD}, S), ({8: A[0]}, E),
        ({8: A[1]}, E)]
    yield L.nf_linear_wgrad, [1, A[0], A[1], 4, 16, 8, A[2], lsb, A[3], A[4]], [
        ({0: 3}, E), ({1: None}, E), ({2: None}, E), ({5: 0}, E), ({6: None}, E), ({7: 0}, nf.NF_ENOWS), ({8: None}, E), ({9: ODD}, S), ({8: A[0]}, E),
        ({9: A[3]}, E)]
    yield L.nf_act_backward, [1, 2, A[0], A[1], 100, A[2]], [
        ({0: 3}, E), ({1: 4}, E), ({2: None}, E), ({3: None}, E), ({4: 0}, E), ({5: None}, E), ({5: ODD}, S), ({5: C.c_void_p(A[1].value + 16)}, E)]
    yield L.nf_dropout, [1, A[0], 100, 0.5, 1, 2, A[1], A[2]], [
        ({0: 3}, E), ({1: None}, E), ({2: 0}, E), ({3: 1.0}, E), ({3: -0.1}, E), ({3: float("nan")}, E), ({6: C.c_void_p(0x100004)}, S), ({7: None}, E),
        ({7: C.c_void_p(A[0].value + 16)}, E), ({1: ODD}, S)]
    yield L.nf_cache_quantize, [0, 1, A[0], 4, 100, 64, A[1], A[2]], [
        ({0: 2}, E), ({1: 2}, E), ({2: None}, E), ({3: 0}, E), ({4: 0}, E), ({4: 1 << 31}, E), ({5: 16}, E), ({5: 96}, E), ({6: None}, E), ({7: None}, E),
        ({6: A[0]}, E), ({7: A[1]}, E), ({6: ODD}, S)]
    yield L.nf_cache_gather_quantized, [1, A[0], A[1], A[2], 10, A[3], 4, 100, 64, 1, A[4], A[5]], [
        ({0: -1}, E), ({1: None}, E), ({2: None}, E), ({3: None}, E), ({4: 0}, E), ({5: None}, E), ({6: 0}, E), ({7: 0}, E), ({8: 0}, E), ({9: 2}, E),
        ({10: None}, E), ({11: None}, E), ({10: ODD}, S), ({5: C.c_void_p(0x100002)}, S), ({10: A[0]}, E)]


def test_refusals(nf):
    n = 0
    for f, good, bad in _calls(nf):
        for change, code in bad:
            args = list(good)
            for k, v in change.items():
                args[k] = v
            assert f(*args) == code, (f.__name__, change)
            n += 1
    assert n > 100


def test_refusals_of_sizes_and_of_scratch_in_use(nf):
    """Sizes whose counters would pass 32 bits, and scratch that lies in a tensor of the call."""
    L, E, U = nf.lib(), nf.NF_EINVAL, nf.NF_EUNSUPPORTED
    big = (1 << 30) + 1
    far = [C.c_void_p(a.value << 24) for a in A]       # 2^44 apart: the sizes below do not make them overlap
    for n, p, c, g in ((big, 1, 1, 1), (1, big, 1, 1), (0x7fffffff, 1, 1, 1), (1, 0x7fffffff, 1, 1), (1, 1, 1 << 25, 1 << 25)):
        assert L.nf_group_norm_forward(1, far[0], far[1], far[2], n, p, c, g, 1e-5, 1, far[3], far[4], far[5]) == U
        assert L.nf_group_norm_backward(1, far[0], far[1], far[2], far[3], far[4], far[5], n, p, c, g, 1, far[6], 1 << 40, far[7], far[8], far[9]) == U
        assert L.nf_group_norm_scratch_bytes(1, n, p, c, g) == 0
    for m, k, n in ((big, 1, 1), (1, big, 1), (1, 1, big)):
        assert L.nf_linear_forward(1, far[0], far[1], None, None, m, k, n, 0, far[2], 1 << 40, None, far[3]) == U
        assert L.nf_linear_dgrad(1, far[0], far[1], m, k, n, far[2], 1 << 40, far[3]) == U
        assert L.nf_linear_wgrad(1, far[0], far[1], m, k, n, far[2], 1 << 40, far[3], None) == U
        assert L.nf_linear_scratch_bytes(1, m, k, n) == 0
    for n in ((1 << 21) - 31, 1 << 23):                # bias gradients of more columns than a launch covers
        assert L.nf_linear_wgrad(1, far[0], far[1], 4, 16, n, far[2], 1 << 40, far[3], far[4]) == U
    gsb, lsb = L.nf_group_norm_scratch_bytes(1, 2, 4, 16, 4), L.nf_linear_scratch_bytes(1, 4, 16, 8)
    for k in (0, 1, 2, 3, 7, 8, 9):
        assert L.nf_group_norm_backward(1, *A[:6], 2, 4, 16, 4, 1, A[k], gsb, *A[7:10]) == E, k
    for k in (0, 1, 2, 3, 5, 6):
        assert L.nf_linear_forward(1, *A[:4], 4, 16, 8, 1, A[k], lsb, A[5], A[6]) == E, k
    for k in (0, 1, 3):
        assert L.nf_linear_dgrad(1, A[0], A[1], 4, 16, 8, A[k], lsb, A[3]) == E, k
    for k in (0, 1, 3, 4):
        assert L.nf_linear_wgrad(1, A[0], A[1], 4, 16, 8, A[k], lsb, A[3], A[4]) == E, k


def test_scratch_sizes_are_host_only(nf):
    L = nf.lib()
    assert L.nf_linear_scratch_bytes(1, 0, 16, 8) == 0 and L.nf_linear_scratch_bytes(5, 4, 16, 8) == 0
    assert L.nf_group_norm_scratch_bytes(1, 2, 4, 16, 5) == 0 and L.nf_group_norm_scratch_bytes(1, 2, 4, 8194, 2) == 0
    assert L.nf_linear_scratch_bytes(1, 128, 512, 256) > 0 and L.nf_group_norm_scratch_bytes(0, 128, 1024, 64, 32) > 0


def test_binding_refuses_wrong_tensors(nf):
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(nf.NfError, match="CUDA device"):
        nf.nf_dropout(nf.NF_F32, x, 0.5, 1, 2, torch.zeros(4, 8))
    with pytest.raises(nf.NfError, match="want torch.bfloat16"):
        nf.nf_dropout(nf.NF_BF16, x, 0.5, 1, 2, x)
    with pytest.raises(nf.NfError, match="dense"):
        nf.nf_dropout(nf.NF_F32, x.t(), 0.5, 1, 2, x.t())
    with pytest.raises(nf.NfError, match="dtype"):
        nf.nf_dropout(7, x, 0.5, 1, 2, x)
    with pytest.raises(nf.NfError, match="act"):
        nf.nf_act_backward(nf.NF_F32, "tanh", x, x, x)
    with pytest.raises(nf.NfError, match="two dimensions"):
        nf.nf_linear_dgrad(nf.NF_F32, x, x[None], x, x)
    with pytest.raises(nf.NfError, match="N, ..., C"):
        nf.nf_group_norm_forward(nf.NF_F32, x[0], x[0], x[0], 1, 1e-5, "none", x[0], x[0], x[0])
    with pytest.raises(nf.NfError, match="2\\^31"):
        nf.nf_cache_quantize("int8", nf.NF_F32, torch.zeros(1).expand(1 << 31), 64, x, x)
    with pytest.raises(nf.NfError, match="format"):
        nf.nf_cache_quantize("int4", nf.NF_F32, x, 64, x, x)

"""What the binding of the operators refuses before the library sees it, without a GPU: the library stands in by a recorder that must not be called."""
import pytest


@pytest.fixture
def nf(monkeypatch):
    import torch
    from paper_2402_14139_b200 import nf as mod

    class Recorder:
        def __getattr__(self, name):
            def call(*args):
                raise AssertionError(f"{name} reached the library")
            return call
    # host tensors pass for device ones, so that the check in question is the one that answers
    monkeypatch.setattr(mod, "lib", lambda: Recorder())
    monkeypatch.setattr(mod, "_TYPES", {mod.NF_F32: torch.float32, mod.NF_BF16: torch.bfloat16, "i32": torch.int32, "i64": torch.int64,
                                        "u8": torch.uint8, "device": lambda: -1})
    return mod


@pytest.mark.parametrize("group", [(1 << 32) + 64, (1 << 32) + 32, -64, 0, 1, 48, 256, 64.5])
def test_group_of_a_quantised_cache(nf, group):
    """A C int keeps the low 32 bits of what it is given: 2^32 + 64 would be 64 there, with scales for one group of each row."""
    import torch
    x, codes = torch.zeros(4, 1000), torch.zeros(4, 1000, dtype=torch.uint8)
    scales = torch.zeros(4, max(1, -int(-1000 // (group or 1))))
    idx, labels = torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(nf.NfError, match="group"):
        nf.nf_cache_quantize("int8", nf.NF_F32, x, group, codes, scales)
    with pytest.raises(nf.NfError, match="group"):
        nf.nf_cache_gather_quantized("int8", codes, scales, labels, idx, group, nf.NF_F32, torch.zeros(2, 1000), torch.zeros(2, dtype=torch.int32))


def test_groups_beyond_a_c_int(nf):
    import torch
    x, c = torch.zeros(1, 3, 8), torch.zeros(8)
    wide = torch.zeros(1, 1).expand(1, (1 << 32) + 4)
    with pytest.raises(nf.NfError, match="2\\^31"):
        nf.nf_group_norm_forward(nf.NF_F32, x, c, c, (1 << 32) + 4, 1e-5, "none", x.clone(), wide, wide)
    with pytest.raises(nf.NfError, match="2\\^31"):
        nf.nf_group_norm_backward(nf.NF_F32, x, x, c, c, wide, wide, "none", c, x.clone(), c, c)

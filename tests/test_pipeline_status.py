"""What the block-wise driver makes of the stand-alone operations' status word, and the cache arguments it refuses before a block is trained; no GPU."""
import pytest

from paper_2402_14139_b200 import nf as real
from paper_2402_14139_b200 import pipeline


class _Nf:
    NF_ELABEL, NF_ENONFINITE, NF_ETIMEOUT, NF_EINDEX = real.NF_ELABEL, real.NF_ENONFINITE, real.NF_ETIMEOUT, real.NF_EINDEX
    CACHE_FORMATS = real.CACHE_FORMATS

    def __init__(self, status=0):
        self.status, self.looks = status, 0

    def nf_op_status(self):
        self.looks += 1
        status, self.status = self.status, 0
        return status


def test_each_bit_under_its_own_name():
    pipeline._check_operators(_Nf(0), "block 0")
    with pytest.raises(RuntimeError, match="block 0: activations that are not finite"):
        pipeline._check_operators(_Nf(real.NF_ENONFINITE), "block 0")
    with pytest.raises(RuntimeError, match="block 1: .*NF_EINDEX") as e:
        pipeline._check_operators(_Nf(real.NF_EINDEX), "block 1")
    assert "finite" not in str(e.value)
    with pytest.raises(RuntimeError, match="NF_ENONFINITE \\| NF_ETIMEOUT"):
        pipeline._check_operators(_Nf(real.NF_ETIMEOUT | real.NF_ENONFINITE), "block 1")


class _Stop(Exception):
    pass


def test_bits_of_earlier_calls_are_cleared_on_entry():
    class Data:
        shape = (4, 8, 8, 3)

    class Wl(dict):
        def __getitem__(self, k):
            raise _Stop
    nf = _Nf(real.NF_EINDEX)
    with pytest.raises(_Stop):
        pipeline.train_blockwise(nf, None, Wl(), Data(), None, cache_format="int8")
    assert nf.looks == 1 and nf.status == 0
    nf = _Nf(real.NF_EINDEX)
    with pytest.raises(_Stop):          # without an 8-bit cache the word is the caller's
        pipeline.train_blockwise(nf, None, Wl(), Data(), None)
    assert nf.looks == 0


@pytest.mark.parametrize("bad", [dict(cache_format="int4"), dict(cache_format="int8", cache_group=48), dict(cache_format="e4m3", cache_group=0),
                                 dict(cache_format="e4m3", cache="disk")])
def test_cache_arguments(bad):
    class Data:
        shape = (4, 8, 8, 3)
    with pytest.raises(ValueError):
        pipeline.train_blockwise(_Nf(), None, None, Data(), None, **bad)

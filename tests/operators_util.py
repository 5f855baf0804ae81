"""Shared by the GPU tests of the operators: tensors on both sides and the tolerance rule."""
import numpy as np

U = 2.0 ** -24                       # half a step of fp32, relative
HALF = {0: 2.0 ** -24, 1: 2.0 ** -8}  # half a step of the storage type (nf_dtype), relative


def storage(torch, dtype):
    return torch.float32 if dtype == 0 else torch.bfloat16


def put(torch, a, dtype):
    """numpy -> (device tensor of the type, the float64 values it holds)."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(storage(torch, dtype))
    return t, t.double().cpu().numpy()


def put_f32(torch, a):
    return put(torch, a, 0)


def host(t):
    return t.double().cpu().numpy()


def check(got, want, dtype, slack, what=""):
    """|got - want| <= what the arithmetic before the last rounding may be off by (slack), and half a step of the storage type."""
    got = host(got) if hasattr(got, "cpu") else np.asarray(got, dtype=np.float64)
    assert np.isfinite(got).all(), what
    slack = np.broadcast_to(slack, want.shape)
    allowed = slack + HALF[dtype] * (np.abs(want) + slack) + 1e-37
    off = np.abs(got - want) / allowed
    assert off.max() <= 1.0, (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))


def rel(got, want):
    got = host(got) if hasattr(got, "cpu") else got
    off, size = float(np.linalg.norm(got - want)), float(np.linalg.norm(want))
    return off / size if size else off

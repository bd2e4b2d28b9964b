"""Shared helpers of the operators' GPU tests."""
import torch

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": U}     # one rounding, relative


def close(name, got, want, bound):
    """|got - want| <= bound everywhere (NaN nowhere)."""
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), (name, int(bad.sum()), float(off.max()), float((off / bound).max()))


def rounded(want, bound, dtype):
    """The bound of a value that is off by `bound` before it is rounded to dtype."""
    return bound + HALF[dtype] * (want.abs() + bound) + 1e-38


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def spread(t, columns, offset=0):
    """t with `columns` more elements between its rows, at an odd place."""
    wide = torch.full((t.shape[0], t.shape[1] + columns), 7.0, dtype=t.dtype, device=t.device)
    wide[:, offset:offset + t.shape[1]] = t
    return wide[:, offset:offset + t.shape[1]]


def far(t, stride):
    """t with rows `stride` elements apart: offsets past 32 bits."""
    store = torch.empty(stride * (t.shape[0] - 1) + t.shape[1], dtype=t.dtype, device=t.device)
    out = store.as_strided(t.shape, (stride, 1))
    out.copy_(t)
    return out

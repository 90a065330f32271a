"""What the tests of the attention block share: tensors in the framework's layout and the bounds of its roundings."""
import numpy as np

from paper_1702_02181_amd import gen

U = 2.0 ** -24                        # fp32's half step
HALF = {"f32": U, "bf16": 2.0 ** -8}  # half a step of a type, relative to the value


def ld(n):
    return (n + 63) // 64 * 64


def rounded(a, dtype):
    a = np.asarray(a, np.float32)
    return a if dtype == "f32" else gen.round_bf16(a)


def torch_type(dtype):
    import torch
    return torch.float32 if dtype == "f32" else torch.bfloat16


def dev(a, dtype="f32", fill=0.0):
    """[rows, ld(width)] on the GPU; `fill` in the pad columns."""
    import torch
    a = np.asarray(a, np.float32)
    out = torch.full((a.shape[0], ld(a.shape[1])), fill, dtype=torch.float32)
    out[:, :a.shape[1]] = torch.from_numpy(a)
    return out.to(torch_type(dtype)).cuda()


def vec(a, kind=np.float32):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, kind)).cuda()


def host(t, width=None):
    a = t.float().cpu().numpy().astype(np.float64)
    return a if width is None else a[:, :width]


def within(got, want, bound, what):
    """Elementwise; infinities and NaN have to be the same ones."""
    got, want = np.asarray(got), np.asarray(want)
    bound = np.broadcast_to(bound, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
    off = np.abs(got[fine] - want[fine]) - bound[fine]
    assert not (off > 0).any(), (what, float(off.max()), int((off > 0).sum()), off.size)


def pads_are_zero(t, width):
    assert not t[:, width:].float().any().item()

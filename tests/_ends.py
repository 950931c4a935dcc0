"""What the tests of a model's two ends share: tensors of a type with their exact values, and roundings."""
import numpy as np
import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# A rounding to the type is off by at most this, relative to the value ...
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
# ... or by half the smallest subnormal.
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}
U32 = 2.0 ** -24
NEAR = 1.0 + 2.0 ** -6  # for the products of these bounds that they leave out


def put(a, dt):
    """(device tensor, its exact values in float64) of an array in a type."""
    t = torch.from_numpy(np.ascontiguousarray(a, np.float64)).to(DT[dt])
    return t.cuda(), t.double().numpy()


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def within(got, want, tol, what=""):
    """|got - want| <= tol elementwise; NaN and infinities where and as wanted."""
    got, want, tol = np.broadcast_arrays(np.asarray(got, np.float64), np.asarray(want, np.float64), np.asarray(tol, np.float64))
    fine = np.isfinite(want)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=f"{what}: NaN")
    np.testing.assert_array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)], err_msg=f"{what}: infinities")
    off = np.abs(got[fine] - want[fine]) - tol[fine]
    if off.size and off.max() > 0:
        k = int(off.argmax())
        raise AssertionError(f"{what}: {got[fine][k]!r} for {want[fine][k]!r}, off {abs(got[fine][k] - want[fine][k]):.3g}, "
                             f"bound {tol[fine][k]:.3g} ({int((off > 0).sum())} of {off.size})")


def bits(t):
    t = t.detach().contiguous()
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32, 8: torch.int64}[t.element_size()]).cpu().numpy()

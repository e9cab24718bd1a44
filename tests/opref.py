"""Sequence operators in fp64 from their formulas, on the CPU, one row and one
step at a time where that is plainest; and what the tests of them share.

U is the unit roundoff of fp32 (half a step).  A sum of n terms in any order
that adds at most c of them one after another is off by at most about
c U sum|terms|; CHAIN is a bound on c for the kernels' sums over columns: 64
elements a lane at most, then the lanes and wavefronts, with room for the
handful of operations that follow."""
import torch

F64 = torch.float64
U = 2.0 ** -24
CHAIN = 160
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# the smallest step of a type: below its normal range a rounding is off by half of it
STEP = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24,
        torch.float8_e4m3fn: 2.0 ** -9}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rounded(ref, dtype):
    """What one rounding to dtype may be off by."""
    return half_step(dtype) * ref.abs() + STEP[dtype] / 2


def check(name, got, ref, tol):
    """|got - ref| <= tol where ref is finite; the same infinities and NaN elsewhere."""
    got = got.detach().to("cpu", F64)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{name}: NaN at other places"
    inf = ~fine & ~torch.isnan(ref)
    assert torch.equal(got[inf], ref[inf]), f"{name}: infinities differ"
    off = (got - ref).abs()[fine] - tol.expand_as(ref)[fine]
    if off.numel():
        k = int(off.argmax())
        assert float(off[k]) <= 0, (f"{name}: {float(got[fine][k])} against "
                                    f"{float(ref[fine][k])}, {float(off[k]):.3g} past the tolerance")


def cpu64(*ts):
    return [None if t is None else t.detach().to("cpu", F64) for t in ts]


# ------------------------------------------------------------------- norm
def norm(x, w, eps, res=None):
    x, w, res = cpu64(x, w, res)
    t = x if res is None else x + res
    q = (t.square().mean(1, keepdim=True) + eps) ** -0.5
    return t, t * q * w


def norm_grads(t, w, dy, eps, dtotal=None):
    """(dx, dw, scale of dx's error, scale of dw's)."""
    t, w, dy, dtotal = cpu64(t, w, dy, dtotal)
    q = (t.square().mean(1, keepdim=True) + eps) ** -0.5
    g = w * dy
    dx = q * (g - t * q ** 2 * (g * t).mean(1, keepdim=True))
    sx = q * (g.abs() + t.abs() * q ** 2 * (g * t).abs().mean(1, keepdim=True))
    if dtotal is not None:
        dx, sx = dx + dtotal, sx + dtotal.abs()
    return dx, (dy * t * q).sum(0), sx, (dy * t * q).abs().sum(0)

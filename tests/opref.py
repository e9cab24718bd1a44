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


# ------------------------------------------------------------------- scan
def scan(g, x, begin, end, h0=None, reverse=False, dy=None, dh_last=None):
    """Row by row.  ``begin``, ``end``: the rows of each sequence.  Returns a
    dict of results, and under "err_" the fp32 error that they may have: every
    step's own roundings (GATE for each gate, one for each operation), carried
    along by the gates as the states are."""
    g, x, h0, dy, dh_last = cpu64(g, x, h0, dy, dh_last)
    S, (R, D) = len(begin), g.shape
    h0 = torch.zeros(S, D, dtype=F64) if h0 is None else h0
    a = torch.sigmoid(g)
    i = torch.sigmoid(-g)
    # a gate's error in units of U: exp's argument (|g| log2 e) rounded, exp, 1 + e, the
    # reciprocal (1 step), a product
    gate = U * (g.abs().nan_to_num(0, 0, 0).clamp(max=90) + 8)
    out = {k: torch.full((R, D), float("nan"), dtype=F64) for k in ("y", "dg", "dx")}
    err = {k: torch.zeros(R, D, dtype=F64) for k in ("y", "dg", "dx")}
    out["h_last"], err["h_last"] = h0.clone(), torch.zeros(S, D, dtype=F64)
    before = torch.zeros(R, D, dtype=F64)
    err_before = torch.zeros(R, D, dtype=F64)
    inside = torch.zeros(R, dtype=torch.bool)
    for s in range(S):
        rows = list(range(begin[s], end[s]))
        rows = rows[::-1] if reverse else rows
        h, e = h0[s], torch.zeros(D, dtype=F64)
        for t in rows:
            inside[t] = True
            before[t], err_before[t] = h, e
            # the state may also come by the tile's map (P, Q): as many roundings again
            e = a[t] * e + (gate[t] + 6 * U) * ((a[t] * h).abs() + (i[t] * x[t]).abs())
            h = a[t] * h + i[t] * x[t]
            out["y"][t], err["y"][t] = h, 2 * e
        out["h_last"][s], err["h_last"][s] = h, 2 * e
    out["inside"] = inside
    if dy is None:
        return out, err
    dh_last = torch.zeros(S, D, dtype=F64) if dh_last is None else dh_last
    out["dh0"], err["dh0"] = dh_last.clone(), torch.zeros(S, D, dtype=F64)
    for s in range(S):
        rows = list(range(begin[s], end[s]))
        rows = rows if reverse else rows[::-1]
        c, e = dh_last[s], torch.zeros(D, dtype=F64)
        for t in rows:
            v = dy[t] + c
            e = e + 2 * U * (dy[t].abs() + c.abs())
            out["dx"][t] = i[t] * v
            err["dx"][t] = 2 * (i[t] * e + gate[t] * (i[t] * v).abs())
            d = before[t] - x[t]
            out["dg"][t] = v * a[t] * i[t] * d
            err["dg"][t] = 2 * a[t] * i[t] * (
                e * d.abs() + v.abs() * (2 * err_before[t] + (2 * gate[t] + 4 * U) *
                                         (before[t].abs() + x[t].abs())))
            c = a[t] * v
            e = a[t] * e + (gate[t] + 4 * U) * c.abs()
        out["dh0"][s], err["dh0"][s] = c, 2 * e
    return out, err

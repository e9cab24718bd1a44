"""Infinite states, inputs and gradients through tgm_scan and tgm_scan_backward: they
stay infinite however often the gates multiply, over tiles, workgroups and the blocks
of the chain, until a gate that is zero makes NaN of them.  Against fp64; tolerances as
in test_gpu_seq_scan."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from opref import F64, TYPES, U, scan  # noqa: E402
from test_gpu_seq_scan import Batch  # noqa: E402

INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def tgm():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2402_15113_amd import tgm as t
    t.lib()
    return t


def may_cancel(b, out, err):
    """Rows whose h_(t-1) - x_t is no larger than what rounding h_(t-1) and the
    difference to fp32 may be off by: dg is an infinite e times a difference that may come
    out as zero, NaN then."""
    before, off = torch.zeros(b.rows, b.D, dtype=F64), torch.zeros(b.rows, b.D, dtype=F64)
    for s in range(b.S):
        rows = list(range(b.begin[s], b.end[s]))[::-1 if b.reverse else 1]
        if rows:
            before[rows[0]] = b.h0[s].cpu().to(F64)
            before[rows[1:]], off[rows[1:]] = out["y"][rows[:-1]], err["y"][rows[:-1]]
    x = b.x.cpu().to(F64)
    off = off + 2 * U * (before.abs() + x.abs())
    return torch.isfinite(before) & torch.isfinite(x) & ((before - x).abs() <= off)


LAYOUTS = [dict(lengths=[700, 40, 0, 5000]), dict(lengths=[20, 700, 40], front=7, extra=50),
           dict(S=3, L=700), dict(S=40, L=20), dict(S=2, L=333, length=[333, 290])]


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_infinities_go_on(tgm, layout, dtype, reverse):
    D = 130
    b = Batch(tgm, D, TYPES[dtype], reverse=reverse, **LAYOUTS[layout])
    s = max(range(b.S), key=lambda k: b.end[k] - b.begin[k])   # the longest sequence
    lo, hi = b.begin[s], b.end[s]
    first, last = (hi - 1, lo) if reverse else (lo, hi - 1)
    mid = (lo + hi) // 2
    # gates whose product over a tile, or over two rows, is below every number
    b.g[:, 0:3], b.g[:, 3], b.g[:, 64:67] = -5.0, -80.0, -60.0
    # an infinite state from the start, an infinite input, and one that goes in the middle
    b.h0[s, 0], b.h0[s, 64], b.h0[s, 3], b.h0[s, 5] = INF, -INF, INF, INF
    b.x[mid, 1], b.x[first, 65] = -INF, INF
    b.h0[s, 2] = INF
    b.g[mid, 2] = -INF
    # gradients that come in infinite, at the end and in a row
    b.dh_last[s, 7], b.dh_last[s, 66] = INF, -INF
    b.g[:, 7] = -5.0
    b.dy[last, 8], b.dy[mid, 9] = INF, -INF
    b.g[:, 8:10] = -20.0
    ref, _ = scan(b.g, b.x, b.begin, b.end, b.h0, reverse)
    assert (ref["y"][lo:hi, 0] == INF).all() and torch.isnan(ref["y"][mid, 2])
    b.forward()
    b.backward()
    inside = ref["inside"].cuda()
    want, err = scan(b.g, b.x, b.begin, b.end, b.h0, reverse, b.dy, b.dh_last)
    either = may_cancel(b, want, err)[ref["inside"]]
    for name in ("y", "dx", "dg"):
        got, r = getattr(b, name)[inside].cpu().double(), want[name][ref["inside"]]
        if name == "dg":
            got = torch.where(either & torch.isnan(got) & torch.isinf(r), r, got)
        if TYPES[dtype] == torch.float16:   # past its largest value a result is infinite
            r = torch.where(r.abs() >= 65520, INF * r.sign(), r)
        assert torch.equal(torch.isnan(got), torch.isnan(r)), name
        assert torch.equal(torch.isinf(got), torch.isinf(r)), name
        m = torch.isinf(r)
        assert torch.equal(got[m], r[m]), name
    for name in ("h_last", "dh0"):
        got, r = getattr(b, name).cpu().double(), want[name]
        assert torch.equal(torch.isnan(got), torch.isnan(r)), name
        m = torch.isinf(r)
        assert torch.equal(torch.isinf(got), m) and torch.equal(got[m], r[m]), name
    # the channels without an infinity are as they were
    plain = [c for c in range(D) if c not in (0, 1, 2, 3, 5, 7, 8, 9, 64, 65, 66)]
    y, dx, dg = (getattr(b, n)[inside][:, plain].clone() for n in ("y", "dx", "dg"))
    for v in (b.h0, b.dh_last, b.x, b.dy):
        v[~torch.isfinite(v)] = 0
    b.g[mid, 2] = -5.0
    b.forward()
    b.backward()
    for n, was in (("y", y), ("dx", dx), ("dg", dg)):
        assert torch.equal(getattr(b, n)[inside][:, plain], was), n

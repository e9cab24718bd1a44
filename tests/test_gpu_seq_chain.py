"""The scan's chain of workgroups: more channels than runners fit the chip, histories of
hundreds of workgroups and of more than one look of a runner, odd widths over several
workgroups, rows past 32-bit offsets.

Tolerances as in test_gpu_seq_scan (opref.scan), the running error carried along with
the states in the same way, all rows at once."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from opref import F64, TYPES, U, check, rounded  # noqa: E402
from test_gpu_seq_scan import Batch  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def tgm():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2402_15113_amd import tgm as t
    t.lib()
    return t


@pytest.mark.parametrize("dtype,D", [("f32", 700), ("bf16", 1101), ("f32", 33000),
                                     ("f16", 65536)])
def test_wide_rows(tgm, dtype, D):
    """Up to 32 slices of channel blocks, each with chains of two or three workgroups
    forward and five back, in both directions."""
    for reverse in (False, True):
        Batch(tgm, D, TYPES[dtype], lengths=[330, 0, 200], extra=2, reverse=reverse).run()


def test_wide_rows_on_two_streams(tgm):
    """Two such calls at once, each with its own work space."""
    D = 33000
    batches = [Batch(tgm, D, torch.float32, lengths=[330, 0, 200], seed=s) for s in (0, 9)]
    want = []
    for b in batches:
        b.forward()
        b.backward()
        want.append([v.clone() for v in (b.y, b.h_last, b.dg, b.dx, b.dh0)])
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    for _ in range(3):
        for b, s in zip(batches, streams):
            with torch.cuda.stream(s):
                b.forward()
                b.backward()
    torch.cuda.synchronize()
    for b, w in zip(batches, want):
        for u, v in zip(w, (b.y, b.h_last, b.dg, b.dx, b.dh0)):
            assert torch.equal(u, v)


# ------------------------------------------------------------------- long histories
def recurrence(a, b):
    """h_t = a_t h_(t-1) + b_t from h = 0, for pieces of about the square root of the rows side
    by side, then from piece to piece."""
    rows, D = a.shape
    C = max(1, math.isqrt(rows))
    P = -(-rows // C)
    a, h = (torch.cat([v, v.new_zeros(P * C - rows, D)]).view(P, C, D).clone() for v in (a, b))
    gain = a.clone()
    for t in range(1, C):
        h[:, t] += a[:, t] * h[:, t - 1]
        gain[:, t] *= gain[:, t - 1]
    before = torch.zeros(P, D, dtype=h.dtype, device=h.device)
    for p in range(1, P):
        before[p] = h[p - 1, -1] + gain[p - 1, -1] * before[p - 1]
    return (h + gain * before[:, None]).view(P * C, D)[:rows]


def reference(b):
    """opref.scan's results and errors for the sequences of a Batch, on the GPU."""
    g, x, dy = (v.to(F64) for v in (b.g, b.x, b.dy))
    dev = g.device
    at = lambda v: torch.tensor(v, dtype=torch.int64, device=dev)
    some = [k for k in range(b.S) if b.end[k] > b.begin[k]]
    seqs, lo, hi = at(some), at([b.begin[k] for k in some]), at([b.end[k] - 1 for k in some])
    head, tail = (hi, lo) if b.reverse else (lo, hi)
    mark = torch.zeros(b.rows + 1, dtype=torch.int64, device=dev)
    mark[lo] += 1
    mark[hi + 1] -= 1
    inside = mark.cumsum(0)[:b.rows] > 0
    m = inside[:, None].to(F64)
    h0 = torch.zeros(b.S, b.D, dtype=F64, device=dev) if b.h0 is None else b.h0.to(F64)
    dl = torch.zeros_like(h0) if b.dh_last is None else b.dh_last.to(F64)
    a, i = torch.sigmoid(g), torch.sigmoid(-g)
    gate = U * (g.abs().clamp(max=90) + 8)
    turn = (lambda v: v.flip(0)) if b.reverse else (lambda v: v)
    back = (lambda v: v) if b.reverse else (lambda v: v.flip(0))

    def shift(v, step):   # the row before (step 1) or after in the scan's order, 0 at the ends
        step = -step if b.reverse else step
        out = torch.zeros_like(v)
        if step == 1:
            out[1:] = v[:-1]
        else:
            out[:-1] = v[1:]
        return out

    keep = a * m
    keep[head] = 0
    add = i * x * m
    add[head] += a[head] * h0[seqs]
    y = turn(recurrence(turn(keep), turn(add)))
    before = shift(y, 1)
    before[head] = h0[seqs]
    ey = turn(recurrence(turn(keep), turn((gate + 6 * U) * ((a * before).abs() +
                                                            (i * x).abs()) * m)))
    eb = shift(ey, 1)
    eb[head] = 0
    follows = shift(a * m, -1)
    follows[tail] = 0
    add = dy * m
    add[tail] += dl[seqs]
    v = back(recurrence(back(follows * m), back(add)))
    came = shift(a * v * m, -1)
    came[tail] = dl[seqs]
    lost = shift((gate + 4 * U) * (a * v).abs() * m, -1)
    lost[tail] = 0
    ev = back(recurrence(back(follows * m), back((lost + 2 * U * (dy.abs() + came.abs())) * m)))
    d = before - x
    out = dict(y=y, dx=i * v, dg=v * a * i * d, h_last=h0.clone(), dh0=dl.clone())
    err = dict(y=2 * ey, dx=2 * (i * ev + gate * (i * v).abs()),
               dg=2 * a * i * (ev * d.abs() + v.abs() * (2 * eb + (2 * gate + 4 * U) *
                                                         (before.abs() + x.abs()))),
               h_last=torch.zeros_like(h0), dh0=torch.zeros_like(h0))
    out["h_last"][seqs], err["h_last"][seqs] = y[tail], 2 * ey[tail]
    out["dh0"][seqs] = (a * v)[head]
    err["dh0"][seqs] = 2 * (a * ev + (gate + 4 * U) * (a * v).abs())[head]
    return out, err, inside


def check_all(b):
    out, err, m = reference(b)
    for name in ("y", "dx", "dg"):
        got, r, e = getattr(b, name), out[name][m].cpu(), err[name][m].cpu()
        check(name, got[m], r, e + rounded(r.abs() + e, b.dt))
        assert (got[~m] == 7).all(), f"{name}: rows of no sequence were written"
    for name in ("h_last", "dh0"):
        r, e = out[name].cpu(), err[name].cpu()
        check(name, getattr(b, name), r, e + rounded(r.abs() + e, torch.float32))


def drifting(b):
    """Gates that hold several workgroups' rows (a of 0.9975 to 0.9997), inputs and incoming
    gradients whose mean drifts, so that states that lie rows apart differ."""
    r = torch.arange(b.rows, device="cuda")[:, None]
    c = torch.arange(b.D, device="cuda")[None]
    b.g.copy_(6 + 2 * torch.rand(b.rows, b.D, device="cuda",
                                 generator=torch.Generator(device="cuda").manual_seed(1)))
    b.x.add_(2 * torch.sin(r / 900 + c))
    b.dy.mul_(0.1).add_(0.05 * torch.cos(r / 700 + 2 * c))
    return b


LONG = [dict(lengths=[100003, 0, 7, 30000], extra=5), dict(lengths=[5, 120001], front=3),
        dict(S=2, L=60001), dict(S=3, L=40000, length=[40000, 33333, -1])]


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("D,dtype", [(20, "f32"), (129, "bf16"), (131, "f16"), (131, "f32")])
@pytest.mark.parametrize("layout", range(len(LONG)))
def test_long_histories(tgm, layout, D, dtype, reverse):
    """Over 100,000 rows: some 470 workgroups forward and 940 back, four and fifteen times
    what a runner looks at at once."""
    b = drifting(Batch(tgm, D, TYPES[dtype], reverse=reverse, **LONG[layout]))
    b.forward()
    b.backward()
    check_all(b)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("D,dtype", [(600, "f32"), (1100, "bf16")])
def test_long_and_wide(tgm, D, dtype, reverse):
    """Runners of one wavefront each."""
    b = drifting(Batch(tgm, D, TYPES[dtype], lengths=[30000, 9, 0, 12000], reverse=reverse))
    b.forward()
    b.backward()
    check_all(b)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D", [1, 2, 3, 63, 65, 66, 127, 129, 130, 131, 257, 385, 513])
def test_widths_over_several_workgroups(tgm, D, dtype):
    for rev, pad in ((False, 3), (True, 0)):
        Batch(tgm, D, TYPES[dtype], lengths=[700, 0, 400], extra=2, reverse=rev, pad=pad).run()


def test_a_long_history_past_32_bit_offsets(tgm):
    """The last rows of a matrix of more than 2^31 elements and 2^32 bytes, inside one
    history of all its rows."""
    n, cols, D = 700_000, 4096, 20
    whole = torch.zeros(n, cols, device="cuda", dtype=torch.bfloat16)
    r = torch.arange(n, device="cuda")[:, None]
    g, x, y = whole[:, :D], whole[:, 64:64 + D], whole[:, 128:128 + D]
    g.copy_(6 + 2 * torch.rand(n, D, device="cuda"))
    x.copy_(torch.randn(n, D, device="cuda") + 2 * torch.sin(r / 900))
    off = torch.tensor([0, n], device="cuda")
    work = torch.empty(tgm.tgm_scan_work_bytes(n, D, 1), dtype=torch.uint8, device="cuda")
    tgm.tgm_scan(g, x, y, 1, work, offsets=off)
    G, X = g.to(F64), x.to(F64)
    a, i = torch.sigmoid(G), torch.sigmoid(-G)
    ref = recurrence(a, i * X)
    gate = U * (G.abs() + 8)
    e = 2 * recurrence(a, (gate + 6 * U) * ((a * ref.roll(1, 0)).abs() + (i * X).abs()))
    k = 3000
    check("y", y[-k:], ref[-k:].cpu(), (e + rounded(ref.abs() + e, y.dtype))[-k:].cpu())


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype,D", [("f32", 600), ("f16", 1030)])
def test_wide_padded(tgm, dtype, D, reverse):
    """Long padded sequences with lengths, short ones that share a tile, and ones without
    rows, more channels than one counter a block serves."""
    for kw in (dict(S=3, L=700, length=[700, 0, 431]), dict(S=40, L=10, length=[7] * 39 + [0]),
               dict(S=5, L=33), dict(lengths=[0] * 30 + [600] + [0] * 30)):
        Batch(tgm, D, TYPES[dtype], reverse=reverse, **kw).run()


def test_wide_calls_captured(tgm):
    """A wide call and its gradient in a graph, replayed on new inputs with eager calls
    between the replays."""
    kw = dict(lengths=[1500, 0, 900], extra=3)
    b, eager = (Batch(tgm, 1100, torch.bfloat16, **kw) for _ in range(2))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        b.forward()
        b.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.forward()
        b.backward()
    for k in range(4):
        for v, e in ((b.x, eager.x), (b.dy, eager.dy), (b.h0, eager.h0)):
            v.copy_(torch.randn(v.shape, generator=torch.Generator().manual_seed(k)))
            e.copy_(v)
        eager.forward()
        eager.backward()
        if k % 2:
            torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in ("y", "h_last", "dg", "dx", "dh0"):
            assert torch.equal(getattr(b, n), getattr(eager, n)), (k, n)

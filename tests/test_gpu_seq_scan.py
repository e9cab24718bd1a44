"""tgm_scan, tgm_scan_backward and tgm_scan_step against fp64, row by row: packed
and padded sequences of lengths around a tile, empty ones, rows of no sequence,
both directions, odd widths and strides, in place, infinite and NaN inputs.

Tolerances: one rounding of the output's type, plus the running fp32 error
that opref.scan carries along with the states."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from opref import F64, TYPES, check, rounded, scan  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def tgm():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2402_15113_amd import tgm as t
    t.lib()
    return t


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def strided(v, dtype, pad):
    """v on the GPU in rows that are `pad` wider."""
    w = torch.full((v.shape[0], v.shape[1] + pad), 7.0, dtype=dtype, device="cuda")
    w[:, :v.shape[1]] = v.to(dtype)
    return w[:, :v.shape[1]]


class Batch:
    """Inputs, sequences and outputs of one call."""

    def __init__(self, tgm, D, dtype, *, lengths=None, L=None, S=None, extra=0, front=0, h0=True,
                 reverse=False, pad=0, seed=0, length=None):
        self.tgm, self.D, self.dt, self.reverse = tgm, D, dtype, reverse
        if lengths is not None:
            self.S = len(lengths)
            off = front + torch.cat([torch.zeros(1, dtype=torch.int64),
                                     torch.tensor(lengths, dtype=torch.int64).cumsum(0)])
            self.begin, self.end = off[:-1].tolist(), off[1:].tolist()
            self.rows = int(off[-1]) + extra
            self.offsets = off.cuda()
        else:
            self.S, self.rows, self.offsets = S, S * L, None
            self.begin = [s * L for s in range(S)]
            self.end = [b + L for b in self.begin]
        self.length = None
        if length is not None:
            self.length = torch.tensor(length, dtype=torch.int32, device="cuda")
            self.end = [max(b, min(e, b + n)) for b, e, n in zip(self.begin, self.end, length)]
        R, S = self.rows, self.S
        # gates around open and closed, and wide of both
        self.g = strided(randn(seed, R, D) * 2 + torch.linspace(-2, 5, D), dtype, pad)
        self.x = strided(randn(seed + 1, R, D), dtype, 2 * pad)
        self.dy = strided(randn(seed + 2, R, D), dtype, pad)
        self.h0 = randn(seed + 3, S, D).cuda() if h0 else None
        self.dh_last = randn(seed + 4, S, D).cuda() if h0 else None
        self.y, self.dg, self.dx = (strided(torch.full((R, D), 7.0), dtype, pad)
                                    for _ in range(3))
        self.h_last = torch.full((S, D), 7.0, device="cuda")
        self.dh0 = torch.full((S, D), 7.0, device="cuda")
        n = tgm.tgm_scan_carry_rows(R, S, self.offsets is not None)
        self.carry = torch.full((n, D), 7.0, device="cuda")
        self.work = torch.empty(tgm.tgm_scan_work_bytes(R, D, S), dtype=torch.uint8,
                                device="cuda")
        self.seq = dict(offsets=self.offsets, length=self.length, h0=self.h0, reverse=reverse)

    def forward(self, **kw):
        a = dict(y=self.y, h_last=self.h_last, carry=self.carry)
        a.update(kw)
        self.tgm.tgm_scan(self.g, self.x, a.pop("y"), self.S, self.work, **a, **self.seq)

    def backward(self, **kw):
        a = dict(dy=self.dy, dg=self.dg, dx=self.dx)
        a.update(kw)
        self.tgm.tgm_scan_backward(self.g, self.x, a["dy"], self.carry, a["dg"], a["dx"], self.S,
                                   self.work, dh_last=self.dh_last, dh0=self.dh0, **self.seq)

    def check(self, backward=True):
        ref, err = scan(self.g, self.x, self.begin, self.end, self.h0, self.reverse, self.dy,
                        self.dh_last)
        m = ref["inside"]
        for name in ("y",) + (("dg", "dx") if backward else ()):
            got = getattr(self, name)
            check(name, got[m.cuda()], ref[name][m],
                  err[name][m] + rounded(ref[name][m] if name == "y" else
                                         ref[name][m].abs() + err[name][m], self.dt))
            assert (got[~m.cuda()] == 7).all(), f"{name}: rows of no sequence were written"
            whole = got._base if got._base is not None else got
            assert (whole[:, self.D:] == 7).all(), f"{name}: columns past the row were written"
        for name in ("h_last",) + (("dh0",) if backward else ()):
            check(name, getattr(self, name), ref[name],
                  err[name] + rounded(ref[name], torch.float32))

    def run(self):
        self.forward()
        self.backward()
        self.check()
        return self


PACKED = [
    dict(lengths=[1]), dict(lengths=[2, 0, 1]), dict(lengths=[31, 1, 33, 32, 0, 0, 64]),
    dict(lengths=[0, 0, 5, 0], extra=40), dict(lengths=[700], extra=3),
    dict(lengths=[3] * 50, front=35, extra=70), dict(lengths=[257, 1, 1, 300, 0, 129]),
    dict(lengths=[0] * 100 + [40] + [0] * 100), dict(lengths=[1] * 150),
    dict(lengths=[2000, 5, 1100]),
]


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("case", range(len(PACKED)))
def test_packed(tgm, case, dtype, reverse):
    Batch(tgm, 20, TYPES[dtype], reverse=reverse, h0=case % 2 == 0, seed=case, **PACKED[case]).run()


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("S,L", [(1, 1), (7, 1), (70, 10), (5, 16), (4, 32), (3, 33), (9, 31),
                                 (2, 64), (3, 100), (2, 700), (300, 3)])
def test_padded(tgm, S, L, reverse):
    Batch(tgm, 33, torch.float32, S=S, L=L, reverse=reverse, pad=1).run()
    length = [(3 * s * s + s) % (L + 3) - 1 for s in range(S)]   # -1, 0, ..., L + 1
    Batch(tgm, 33, torch.bfloat16, S=S, L=L, reverse=reverse, length=length, h0=False).run()


def test_packed_with_lengths(tgm):
    for rev in (False, True):
        Batch(tgm, 8, torch.float32, lengths=[40, 3, 100, 0, 7], extra=9, reverse=rev,
              length=[33, 5, 0, 2, -4]).run()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D", [1, 2, 3, 63, 64, 65, 66, 100, 127, 128, 129, 130, 131, 255, 257,
                               385, 513])
def test_widths(tgm, D, dtype):
    for rev, pad in ((False, 0), (True, 3)):
        Batch(tgm, D, TYPES[dtype], lengths=[50, 0, 90], extra=2, reverse=rev, pad=pad).run()


@pytest.mark.parametrize("D", [20, 129])
def test_in_place(tgm, D):
    for dt in (torch.float32, torch.bfloat16):
        for kw in (dict(lengths=[5, 300, 0, 40], extra=3), dict(S=20, L=10)):
            b = Batch(tgm, D, dt, **kw)
            b.forward()
            b.backward()
            g, x, dy = b.g.clone(), b.x.clone(), b.dy.clone()
            m = scan(g, x, b.begin, b.end)[0]["inside"].cuda()
            for name in ("g", "x"):
                v = getattr(b, name)
                b.forward(y=v)
                assert torch.equal(v[m], b.y[m])
                v.copy_(dict(g=g, x=x)[name])
            b.forward()
            b.backward(dg=b.dy, dx=b.x)
            assert torch.equal(b.dy[m], b.dg[m]) and torch.equal(b.x[m], b.dx[m])
            b.x.copy_(x), b.dy.copy_(dy)
            b.backward(dg=b.g, dx=b.dy)
            assert torch.equal(b.g[m], b.dg[m]) and torch.equal(b.dy[m], b.dx[m])


def test_optional_outputs(tgm):
    b = Batch(tgm, 40, torch.float32, lengths=[70, 0, 200]).run()
    y, dg = b.y.clone(), b.dg.clone()
    b.forward(h_last=None, carry=None)
    assert torch.equal(b.y, y)
    b.forward()
    b.dh0 = None
    b.backward()
    assert torch.equal(b.dg, dg)


def test_nothing_to_do(tgm):
    b = Batch(tgm, 5, torch.float32, lengths=[0, 0])
    b.forward()
    b.backward()
    assert torch.equal(b.h_last, b.h0) and torch.equal(b.dh0, b.dh_last)
    e = torch.empty(0, 5, device="cuda")
    tgm.tgm_scan(e, e, e, 0, None)
    tgm.tgm_scan(e, e, e, 3, None, h_last=b.h_last[:1].repeat(3, 1).contiguous())


def test_gates_at_their_ends_and_bad_inputs(tgm):
    """Infinite gates hold or replace the state exactly; a NaN or an infinity
    stays in its channel and its sequence."""
    inf, nan = float("inf"), float("nan")
    b = Batch(tgm, 6, torch.float32, lengths=[100, 40, 60])
    b.g[10:20, 0], b.g[70, 1], b.g[30, 2] = inf, -inf, nan
    b.x[50, 3], b.x[130, 4] = inf, nan
    b.g[:, 5] = 200.0
    b.forward()
    b.check(backward=False)
    assert torch.equal(b.y[9:19, 0], b.y[9:10, 0].expand(10)) and float(b.y[70, 1]) == float(
        b.x[70, 1])
    assert torch.isfinite(b.y[100:, :4]).all() and torch.isnan(b.y[30:100, 2]).all()
    assert (b.y[50:100, 3] == inf).all() and torch.isfinite(b.y[140:, 4]).all()


def test_reproducible(tgm):
    b = Batch(tgm, 128, torch.bfloat16, lengths=[1000, 3, 5000, 0, 900]).run()
    first = [v.clone() for v in (b.y, b.h_last, b.dg, b.dx, b.dh0)]
    for _ in range(3):
        b.work.fill_(255)
        b.forward()
        b.backward()
        for u, v in zip(first, (b.y, b.h_last, b.dg, b.dx, b.dh0)):
            assert torch.equal(u, v)


def test_disordered_offsets_stay_in_range(tgm):
    """Offsets that decrease or leave the rows give some values, and no access
    out of range: the guard rows around the tensors keep theirs."""
    b = Batch(tgm, 16, torch.float32, lengths=[30, 40, 50])
    for off in ([0, 90, 20, 500], [-7, -3, 4, 60], [200, 100, 50, 0], [0, 2 ** 40, -2 ** 40, 120]):
        b.offsets.copy_(torch.tensor(off))
        whole = torch.full((b.rows + 200, 16), 7.0, device="cuda")
        b.forward(y=whole[100:-100])
        b.backward()
        assert (whole[:100] == 7).all() and (whole[-100:] == 7).all()


def test_against_differences(tgm):
    b = Batch(tgm, 3, torch.float32, lengths=[4, 40], seed=3).run()

    def f(g, x, h0):
        ref, _ = scan(g, x, b.begin, b.end, h0)
        return float((ref["y"] * b.dy.cpu().to(F64)).sum() +
                     (ref["h_last"] * b.dh_last.cpu().to(F64)).sum())

    ins = [v.cpu().to(F64) for v in (b.g, b.x, b.h0)]
    h = 1e-6
    for k, grad, at in ((0, b.dg, (2, 1)), (0, b.dg, (30, 2)), (1, b.dx, (0, 0)),
                        (1, b.dx, (43, 1)), (2, b.dh0, (0, 1)), (2, b.dh0, (1, 2))):
        lo, hi = [v.clone() for v in ins], [v.clone() for v in ins]
        lo[k][at] -= h
        hi[k][at] += h
        n = (f(*hi) - f(*lo)) / (2 * h)
        # the differences' own error (rounding 2^-53 |f| / h, truncation h^2) and fp32's
        assert abs(float(grad[at]) - n) <= 1e-5 * (1 + abs(n))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D", [1, 3, 4, 5, 100, 257])
def test_step(tgm, D, dtype):
    dt, S = TYPES[dtype], 50
    for n, count in ((1, None), (40, None), (40, 17), (40, 0)):
        g, x = strided(randn(1, n, D) * 3, dt, 1), strided(randn(2, n, D), dt, 2)
        slots = torch.randperm(S, generator=torch.Generator().manual_seed(3))[:n].to(
            torch.int32).cuda()
        if n > 3:
            slots[1], slots[3] = -1, S   # not kept
        state, y = randn(4, S, D).cuda(), strided(torch.full((n, D), 7.0), dt, 3)
        want, used = state.clone(), n if count is None else count
        nr = None if count is None else torch.tensor([count], dtype=torch.int32, device="cuda")
        tgm.tgm_scan_step(g, x, state, y, slots=slots, n_rows=nr)
        h0 = torch.zeros(n, D)
        for p in range(n):
            if 0 <= int(slots[p]) < S:
                h0[p] = want[int(slots[p])].cpu()
        ref, err = scan(g, x, list(range(n)), list(range(1, n + 1)), h0)
        check("y", y[:used], ref["y"][:used],
              err["y"][:used] + rounded(ref["y"][:used], dt))
        assert (y[used:] == 7).all()
        for p in range(used):
            s = int(slots[p])
            if 0 <= s < S:
                check("state", state[s], ref["y"][p], err["y"][p] +
                      rounded(ref["y"][p], torch.float32))
                want[s] = state[s]
        assert torch.equal(state, want), "other slots changed"


def test_step_continues_a_scan(tgm):
    """Row by row through the step, against the whole sequence at once."""
    b = Batch(tgm, 100, torch.float32, S=6, L=9)
    b.forward()
    state, y = b.h0.clone(), torch.empty(6, 100, device="cuda")
    for t in range(9):
        g, x = b.g[t::9], b.x[t::9]
        tgm.tgm_scan_step(g, x, state, y)
        assert torch.equal(y, b.y[t::9])   # the same operations on the same numbers
    assert torch.equal(state, b.h_last)

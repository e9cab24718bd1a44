"""tgm_decay_attn and tgm_decay_attn_backward against fp64, row by row: types, shared heads,
odd widths and strides, sequences of no row, one row and many, packed and padded, both
directions, states, row by row continuation, what does not belong to a sequence, values that
are not finite, far decays, captured graphs and streams.  Tolerances: decayref."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import decayref  # noqa: E402
from opref import F64, TYPES, U, check, rounded  # noqa: E402


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
    w = torch.full((v.shape[0], v.shape[1] + pad), 7.0, device="cuda").to(dtype)
    w[:, :v.shape[1]] = v.to(dtype)
    return w[:, :v.shape[1]]


def work(tgm, rows, S, H, dk, dv, dtype, G, backward):
    n = tgm.tgm_decay_attn_work_bytes(rows, S, H, dk, dv, dtype, kv_heads=G, backward=backward)
    return torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)


def packed(lengths, before=0, behind=0, cut=None):
    """offsets, length, and the rows of each sequence; ``before`` and ``behind``: rows of none."""
    off = torch.tensor([before] + list(lengths), dtype=torch.int64).cumsum(0)
    begin, end = off[:-1].tolist(), off[1:].tolist()
    length = None
    if cut is not None:
        length = torch.tensor(cut, dtype=torch.int32).cuda()
        end = [min(e, b + max(0, c)) for b, e, c in zip(begin, end, cut)]
    return dict(offsets=off.cuda(), length=length), begin, end, int(off[-1]) + behind


def padded(lengths, L):
    begin = [s * L for s in range(len(lengths))]
    end = [b + min(L, max(0, n)) for b, n in zip(begin, lengths)]
    return dict(offsets=None, length=torch.tensor(lengths, dtype=torch.int32).cuda()), begin, end, \
        len(lengths) * L


def make(seqs, H, G, dk, dv, dtype, seed=0, pad=0, state=True, decay=None, size=1.0):
    kw, begin, end, rows = seqs
    S = len(begin)
    m = lambda k, w, p: strided(size * randn(seed + k, rows, w), dtype, p)
    d = dict(q=m(0, H * dk, pad), k=m(1, G * dk, 2 * pad), v=m(2, G * dv, 3 * pad),
             do=m(3, H * dv, pad))
    d["decay"] = (torch.log1p(-torch.exp2(-torch.linspace(1.0, 8.0, H))) if decay is None
                  else torch.as_tensor(decay, dtype=torch.float32)).cuda()
    d["state"] = size * randn(seed + 4, S, H, dk, dv).cuda() if state else None
    d["dlast"] = size * randn(seed + 5, S, H, dk, dv).cuda() if state else None
    return d


def both(tgm, seqs, H, G, dk, dv, dtype, reverse=False, pad=0, d=None, what=None, scale=None,
         **kw):
    """Runs forward and backward; returns inputs and outputs, of which nothing outside the
    sequences has been written."""
    how, begin, end, rows = seqs
    S = len(begin)
    d = d or make(seqs, H, G, dk, dv, dtype, pad=pad, **kw)
    scale = dk ** -0.5 if scale is None else scale
    new = lambda w, p: strided(torch.full((rows, w), 7.0), dtype, p)
    st = lambda: torch.full((S, H, dk, dv), 7.0, device="cuda")
    out = dict(o=new(H * dv, pad), state_last=st(), dq=new(H * dk, pad), dk=new(G * dk, pad),
               dv=new(G * dv, pad), dstate=st())
    common = dict(scale=scale, kv_heads=G, state=d["state"], reverse=reverse, **how)
    tgm.tgm_decay_attn(d["q"], d["k"], d["v"], d["decay"], out["o"], S,
                       work(tgm, rows, S, H, dk, dv, dtype, G, False),
                       state_last=out["state_last"], **common)
    give = {n: out[n] if what is None or n in what else None for n in ("dq", "dk", "dv", "dstate")}
    tgm.tgm_decay_attn_backward(d["q"], d["k"], d["v"], d["decay"], d["do"], give["dq"],
                                give["dk"], give["dv"], S,
                                work(tgm, rows, S, H, dk, dv, dtype, G, True),
                                dstate_last=d["dlast"], dstate=give["dstate"], **common)
    return d, out, scale


def go(tgm, seqs, H, G, dk, dv, dtype, reverse=False, what=None, **kw):
    d, out, scale = both(tgm, seqs, H, G, dk, dv, dtype, reverse=reverse, what=what, **kw)
    how, begin, end, rows = seqs
    rows_of = decayref.chains(begin, end, reverse)
    ref = decayref.run(d["q"], d["k"], d["v"], d["decay"], scale, H, G, rows_of, d["state"],
                       d["do"], d["dlast"])
    inside = torch.zeros(rows, dtype=torch.bool)
    for r in rows_of:
        inside[r] = True
    for n, got in out.items():
        if what is not None and n not in ("o", "state_last") and n not in what:
            assert (got.float() == 7).all(), f"{n} was not asked for"
            continue
        tol = decayref.tolerance(n, ref, dtype)
        if n in ("state_last", "dstate"):
            check(n, got, ref[n], tol + rounded(ref[n].abs() + tol, torch.float32))
            continue
        in_range(n, got[inside], ref[n][inside],
                 (tol + rounded(ref[n].abs() + tol, dtype))[inside], dtype)
        assert (got[~inside].float() == 7).all(), f"{n}: rows of no sequence were written"
        if got._base is not None:
            assert (got._base[:, got.shape[1]:].float() == 7).all(), f"{n}: past the row"
    return d, out, ref


def in_range(name, got, ref, tol, dtype):
    """check() for what the type can hold: past (2 - 2^-11) 2^15 = 65,520 fp16's rounding is
    to infinity, and so has to be what lies past it by more than the tolerance."""
    if dtype == torch.float16:
        got, most = got.detach().cpu(), 65520.0
        over, near = ref.abs() - tol >= most, ref.abs() + tol >= most
        assert torch.equal(got.double()[over], ref[over].sign() * math.inf), name
        got, ref, tol = got[~near], ref[~near], tol[~near]
    check(name, got, ref, tol)


MIX = [5, 0, 64, 1, 33, 130, 63, 65, 0, 2]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("H,G,dk,dv", [(1, 1, 1, 1), (2, 2, 50, 50), (4, 2, 32, 16), (3, 1, 17, 33),
                                       (2, 2, 64, 128), (2, 1, 128, 64), (1, 1, 128, 128),
                                       (1, 1, 97, 5), (2, 2, 8, 100)])
def test_heads(tgm, H, G, dk, dv, dtype):
    go(tgm, packed(MIX), H, G, dk, dv, TYPES[dtype])
    go(tgm, packed(MIX, before=3, behind=9), H, G, dk, dv, TYPES[dtype], reverse=True, pad=3,
       state=False)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("L", [1, 2, 10, 31, 64, 100])
def test_padded(tgm, L, dtype):
    n = [0, L, L // 2, 1, L + 5, -3, L - 1, L]
    go(tgm, padded(n, L), 2, 2, 50, 50, TYPES[dtype], reverse=L % 2 == 0)
    go(tgm, padded(n, L), 2, 1, 64, 64, TYPES[dtype], reverse=L % 2 == 1, state=False)


@pytest.mark.parametrize("n", list(range(1, 20)) + [31, 32, 33, 47, 48, 127, 128, 129])
def test_lengths(tgm, n):
    go(tgm, packed([n]), 1, 1, 32, 32, torch.bfloat16)
    go(tgm, packed([n]), 1, 1, 20, 36, torch.float32, reverse=True)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("reverse", [False, True])
def test_long(tgm, dtype, reverse):
    """Sequences over many chunks and pieces of rows, next to short ones."""
    go(tgm, packed([3, 1100, 700, 0, 40], behind=5), 2, 1, 40, 24, TYPES[dtype], reverse=reverse)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_longer(tgm, dtype, reverse):
    """A sequence over several cells of rows, with states handed along them."""
    go(tgm, packed([700, 4500, 2], before=100), 1, 1, 16, 20, TYPES[dtype], reverse=reverse)
    go(tgm, padded([3000, 2047, 1, 2300], 3000), 1, 1, 12, 16, TYPES[dtype], reverse=reverse)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_shortened(tgm, dtype):
    go(tgm, packed([30, 200, 5, 70], cut=[0, 130, 9, -1]), 2, 2, 48, 48, TYPES[dtype])


@pytest.mark.parametrize("what", [(), ("dq",), ("dk",), ("dv",), ("dstate",), ("dk", "dstate")])
def test_some_gradients(tgm, what):
    go(tgm, packed([40, 100]), 4, 2, 24, 40, torch.bfloat16, what=what)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_decays(tgm, dtype):
    """None at all, all at once, far below what fp32 holds after a few rows, and growth."""
    g = [0.0, -math.inf, -60.0, -3.0, 0.02, -1e-6]
    go(tgm, packed([150, 64, 3]), 6, 6, 16, 16, TYPES[dtype], decay=g)
    go(tgm, packed([150, 64, 3]), 6, 2, 16, 16, TYPES[dtype], decay=g, reverse=True)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", [2.0 ** -10, 30.0])
def test_small_and_large(tgm, dtype, size):
    """Products past fp16's range, and below it."""
    go(tgm, packed([200, 20]), 2, 2, 64, 64, TYPES[dtype], size=size, scale=1.0 / size)


def test_no_rows(tgm):
    d, out, _ = both(tgm, packed([0, 0, 0]), 2, 2, 8, 16, torch.float32)
    assert torch.equal(out["state_last"], d["state"]) and torch.equal(out["dstate"], d["dlast"])
    both(tgm, packed([]), 2, 2, 8, 16, torch.bfloat16, state=False)
    d, out, _ = both(tgm, packed([0, 0], behind=4), 1, 1, 8, 8, torch.float16, state=False)
    assert (out["state_last"] == 0).all() and (out["dstate"] == 0).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_of_no_sequence_may_hold_anything(tgm, dtype):
    seqs = padded([7, 0, 64, 30], 70)
    d = make(seqs, 2, 2, 32, 32, TYPES[dtype])
    _, a, _ = both(tgm, seqs, 2, 2, 32, 32, TYPES[dtype], d=d)
    for s, n in enumerate([7, 0, 64, 30]):
        for name in ("q", "k", "v", "do"):
            d[name][s * 70 + n:(s + 1) * 70] = math.nan if s % 2 else math.inf
    _, b, _ = both(tgm, seqs, 2, 2, 32, 32, TYPES[dtype], d=d)
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_not_finite(tgm, name, bad, dtype):
    """What is not finite in row 37 reaches no earlier row, no other sequence and no other
    head, and of a column of v no other one."""
    seqs = packed([20, 150, 30])
    d = make(seqs, 2, 2, 40, 40, TYPES[dtype])
    _, a, _ = both(tgm, seqs, 2, 2, 40, 40, TYPES[dtype], d=d)
    d[name][37, 40 + 3] = bad
    _, b, _ = both(tgm, seqs, 2, 2, 40, 40, TYPES[dtype], d=d)
    far = torch.ones(200, 80, dtype=torch.bool)
    if name == "q":
        far[37, 40:] = False
    elif name == "k":
        far[37:170, 40:] = False
    else:
        far[37:170, 43] = False
    assert torch.equal(a["o"].cpu()[far], b["o"].cpu()[far])
    assert not torch.isfinite(b["o"].cpu()[~far]).any()
    # backwards: dq as o; k and v reach their own row's gradients, q and do earlier rows
    for n in ("dq", "dk", "dv"):
        same = torch.ones(200, dtype=torch.bool)
        if n == "dq":
            same[37:170] = name == "q"
        elif name == "q":
            same[20:38] = False
        else:
            same[37] = False
        x, y = a[n].cpu(), b[n].cpu()
        assert torch.equal(x[:, :40], y[:, :40]), n
        assert torch.equal(x[same], y[same]), n


@pytest.mark.parametrize("dtype", list(TYPES))
def test_continued(tgm, dtype):
    """A prompt in two calls, and then row by row, from the state that each leaves."""
    dt, H, dk, dv, n = TYPES[dtype], 2, 64, 48, 150
    seqs = packed([n])
    d = make(seqs, H, H, dk, dv, dt)
    rows_of = [list(range(n))]
    ref = decayref.run(d["q"], d["k"], d["v"], d["decay"], 0.125, H, H, rows_of, d["state"])
    o = torch.zeros(n, H * dv, device="cuda", dtype=dt)
    state, cut = d["state"].clone(), 70
    part = lambda lo, hi: [d[x][lo:hi] for x in ("q", "k", "v")]
    for lo, hi in ((0, cut), (cut, 140)):
        last = torch.empty_like(state)
        off = torch.tensor([0, hi - lo], device="cuda")
        tgm.tgm_decay_attn(*part(lo, hi), d["decay"], o[lo:hi], 1,
                           work(tgm, hi - lo, 1, H, dk, dv, dt, H, False), scale=0.125,
                           offsets=off, state=state, state_last=last)
        state = last
    for r in range(140, n):
        tgm.tgm_decay_attn_step(*part(r, r + 1), d["decay"], state, o[r:r + 1], scale=0.125)
    for name, got, t in (("o", o, dt), ("state_last", state, torch.float32)):
        # three calls' roundings of the state
        tol = 3 * decayref.tolerance(name, ref, dt)
        check(name, got, ref[name], tol + rounded(ref[name].abs() + tol, t))


def test_differences(tgm):
    """The gradient against central differences in fp32: the operator is linear in each of
    q, k, v and the state, so that only roundings (of sums of absolute values) are off."""
    H, G, dk, dv = 4, 2, 12, 20
    seqs = packed([9, 70, 0, 33])
    d, out, scale = both(tgm, seqs, H, G, dk, dv, torch.float32)
    how, begin, end, rows = seqs
    ref = decayref.run(d["q"], d["k"], d["v"], d["decay"], scale, H, G,
                       decayref.chains(begin, end, False), d["state"], d["do"], d["dlast"])
    size = float((ref["abs_o"] * d["do"].cpu().abs().to(F64)).sum() +
                 (ref["abs_state_last"] * d["dlast"].cpu().abs().to(F64)).sum())

    def total(e):
        o, last = torch.zeros(rows, H * dv, device="cuda"), torch.zeros_like(d["state"])
        tgm.tgm_decay_attn(e["q"], e["k"], e["v"], d["decay"], o, 4,
                           work(tgm, rows, 4, H, dk, dv, torch.float32, G, False), scale=scale,
                           kv_heads=G, state=e["state"], state_last=last, **how)
        return float((o.double() * d["do"].double()).sum() +
                     (last.double() * d["dlast"].double()).sum())

    for i, name in enumerate(("q", "k", "v", "state")):
        v = randn(60 + i, *d[name].shape).cuda()
        up, down = dict(d), dict(d)
        up[name], down[name] = d[name] + v, d[name] - v
        slope = (total(up) - total(down)) / 2
        mine = float((out["d" + name].double() * v.double()).sum())
        # |d| + |v| moves the sums of absolute values by some factor below 8
        assert abs(slope - mine) <= 8 * decayref.SUMS * size, name


def test_same_bits_and_other_sequences(tgm):
    """Twice the same, and each sequence as if it were alone."""
    dt = torch.bfloat16
    seqs = packed([64, 90, 10])
    d = make(seqs, 2, 1, 64, 64, dt)
    _, a, _ = both(tgm, seqs, 2, 1, 64, 64, dt, d=d)
    _, b, _ = both(tgm, seqs, 2, 1, 64, 64, dt, d=d)
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_offsets_that_make_no_sense(tgm):
    """Decreasing or outside the rows: values are unspecified, other memory is not touched."""
    dt, rows = torch.bfloat16, 100
    for off in ([50, 20, 80, 10], [-40, 30, 500, 900], [90, 90, -1, 2 ** 62]):
        seqs = (dict(offsets=torch.tensor(off).cuda(), length=None), [0] * 3, [0] * 3, rows)
        d, out, _ = both(tgm, seqs, 2, 1, 32, 48, dt, pad=8)
        torch.cuda.synchronize()
        for n in ("o", "dq", "dk", "dv"):
            assert (out[n]._base[:, out[n].shape[1]:].float() == 7).all()


def test_many_sequences(tgm):
    """More of them than a search looks at in one step, and than rows."""
    lengths = [(7 * i) % 4 for i in range(5000)]
    go(tgm, packed(lengths), 1, 1, 4, 4, torch.float32)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_short_sequences(tgm, dtype, reverse):
    """Few rows each for the most part, packed and padded, and a sequence of many among them."""
    few = [(5 * i) % 9 for i in range(120)]
    go(tgm, packed(few + [230, 16, 17] + few[::-1]), 2, 1, 50, 50, TYPES[dtype], reverse=reverse)
    go(tgm, packed(few, before=2, behind=3), 3, 3, 17, 31, TYPES[dtype], reverse=reverse, pad=1)
    go(tgm, padded([16, 0, 3, 20, 9, 1], 16), 2, 2, 64, 40, TYPES[dtype], reverse=reverse)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_uneven_lengths(tgm, dtype, reverse):
    """Many heads and sequences of many rows, taken in the order of their lengths: more pieces
    than workgroups of a CU each, some without rows, some of part of a cell."""
    go(tgm, packed([40, 0, 900, 310, 1, 700, 33], before=5, behind=60), 32, 8, 8, 12,
       TYPES[dtype], reverse=reverse)
    go(tgm, padded([200, 0, 64, 17, 199, -5, 300, 1, 150, 33], 200), 32, 32, 12, 8, TYPES[dtype],
       reverse=reverse, state=False)


def test_uneven_offsets_that_make_no_sense(tgm):
    """As above: other memory is not touched."""
    dt, rows = torch.bfloat16, 1100
    for off in ([500, 20, 800, 10], [-40, 300, 5000, 900], [900, 900, -1, 2 ** 62]):
        seqs = (dict(offsets=torch.tensor(off).cuda(), length=None), [0] * 3, [0] * 3, rows)
        d, out, _ = both(tgm, seqs, 64, 16, 32, 48, dt, pad=8)
        torch.cuda.synchronize()
        for n in ("o", "dq", "dk", "dv"):
            assert (out[n]._base[:, out[n].shape[1]:].float() == 7).all()


def test_captured_and_two_streams(tgm):
    dt, H, G, dk, dv = torch.bfloat16, 4, 2, 64, 64
    seqs = packed([700, 0, 90, 300], behind=6)
    how, begin, end, rows = seqs
    S = 4
    d = make(seqs, H, G, dk, dv, dt)
    n = max(tgm.tgm_decay_attn_work_bytes(rows, S, H, dk, dv, dt, kv_heads=G, backward=b)
            for b in (False, True))
    ks = [torch.empty(max(n, 1), dtype=torch.uint8, device="cuda") for _ in range(3)]
    new = lambda w: torch.zeros(rows, w, device="cuda", dtype=dt)
    st = lambda: torch.zeros(S, H, dk, dv, device="cuda")
    outs = [dict(o=new(H * dv), last=st(), dq=new(H * dk), dk=new(G * dk), dv=new(G * dv),
                 ds=st()) for _ in range(3)]

    def call(k, o, stream=None):
        kw = dict(kv_heads=G, state=d["state"], stream=stream, **how)
        tgm.tgm_decay_attn(d["q"], d["k"], d["v"], d["decay"], o["o"], S, k, state_last=o["last"],
                           **kw)
        tgm.tgm_decay_attn_backward(d["q"], d["k"], d["v"], d["decay"], d["do"], o["dq"], o["dk"],
                                    o["dv"], S, k, dstate_last=d["dlast"], dstate=o["ds"], **kw)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(ks[0], outs[0])
    for i in range(4):
        d["q"].copy_(randn(50 + i, rows, H * dk))
        how["offsets"].copy_(torch.tensor([0, 100 * i, 700, 700 + 50 * i, 1090]))
        for o in outs:
            for t in o.values():
                t.zero_()
        torch.cuda.synchronize()
        g.replay()
        side = torch.cuda.Stream()
        call(ks[1], outs[1], side)
        call(ks[2], outs[2])
        torch.cuda.synchronize()
        for name in outs[0]:
            assert torch.equal(outs[0][name], outs[1][name]), name
            assert torch.equal(outs[0][name], outs[2][name]), name


def test_captured_uneven_lengths(tgm):
    """The order of the pieces is made anew in every replay."""
    dt, H, G, d = torch.bfloat16, 32, 8, 16
    seqs = packed([40, 0, 900, 310, 1, 700, 33], before=5, behind=60)
    how, begin, end, rows = seqs
    S = len(begin)
    m = make(seqs, H, G, d, d, dt, state=False)
    ks = [work(tgm, rows, S, H, d, d, dt, G, False) for _ in range(2)]
    outs = [torch.zeros(rows, H * d, device="cuda", dtype=dt) for _ in range(2)]
    call = lambda i: tgm.tgm_decay_attn(m["q"], m["k"], m["v"], m["decay"], outs[i], S, ks[i],
                                        kv_heads=G, **how)
    call(0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(0)
    for i in range(4):
        ends = [0, 400 * i, 400 * i, 1300, 1301 + 100 * i, 1800, 1801, rows - i]
        how["offsets"].copy_(torch.tensor(ends))
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        g.replay()
        call(1)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1])
        ref = decayref.run(m["q"], m["k"], m["v"], m["decay"], 1.0, H, G,
                           decayref.chains(ends[:-1], ends[1:], False))
        tol = decayref.tolerance("o", ref, dt)
        check("o", outs[0], ref["o"], tol + rounded(ref["o"].abs() + tol, dt))


# ------------------------------------------------------------------- single rows
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("H,G,dk,dv", [(1, 1, 1, 1), (2, 2, 50, 50), (4, 1, 128, 128), (3, 3, 7, 33),
                                       (8, 2, 64, 96), (2, 1, 128, 130 - 2)])
def test_step(tgm, H, G, dk, dv, dtype):
    dt, rows, S = TYPES[dtype], 13, 20
    q, k, v = (strided(randn(i, rows, w), dt, 5) for i, w in enumerate((H * dk, G * dk, G * dv)))
    decay = torch.linspace(-2.0, -0.01, H).cuda()
    g = torch.Generator().manual_seed(8)
    slots = torch.randperm(S, generator=g)[:rows].to(torch.int32)
    slots[3], slots[7] = -1, S
    state = randn(9, S, H, dk, dv).cuda()
    before = state.clone()
    o = strided(torch.full((rows, H * dv), 7.0), dt, 2)
    nr = torch.tensor([11], dtype=torch.int32, device="cuda")
    tgm.tgm_decay_attn_step(q, k, v, decay, state, o, scale=0.5, kv_heads=G, slots=slots.cuda(),
                            n_rows=nr)
    first = torch.zeros(11, H, dk, dv)
    for p in range(11):
        if 0 <= slots[p] < S:
            first[p] = before[slots[p]].cpu()
    ref = decayref.run(q[:11], k[:11], v[:11], decay, 0.5, H, G, [[p] for p in range(11)], first)
    tol = decayref.SUMS * ref["abs_o"]
    check("o", o[:11], ref["o"], tol + rounded(ref["o"].abs() + tol, dt))
    assert (o[11:].float() == 7).all() and (o._base[:, H * dv:].float() == 7).all()
    want = before.cpu().to(F64)
    err = torch.zeros_like(want)
    for p in range(11):
        if 0 <= slots[p] < S:
            want[slots[p]] = ref["state_last"][p]
            err[slots[p]] = decayref.SUMS * ref["abs_state_last"][p]
    check("state", state, want, err)
    # without o, and without slots
    s2 = before.clone()
    tgm.tgm_decay_attn_step(q, k, v, decay, s2, None, kv_heads=G)
    ref = decayref.run(q, k, v, decay, 1.0, H, G, [[p] for p in range(rows)], before[:rows])
    check("state", s2[:rows], ref["state_last"], decayref.SUMS * ref["abs_state_last"])
    assert torch.equal(s2[rows:], before[rows:])


def test_step_not_finite(tgm):
    """A state that is not finite stays in its slot and head."""
    H, d = 2, 16
    q, k, v = (randn(i, 3, H * d).cuda() for i in range(3))
    state = randn(4, 3, H, d, d).cuda()
    state[1, 1, 2, 5] = math.nan
    o = torch.zeros(3, H * d, device="cuda")
    tgm.tgm_decay_attn_step(q, k, v, torch.tensor([-0.1, -0.2]).cuda(), state, o)
    bad = torch.isnan(o)
    assert bad[1, d + 5] and int(bad.sum()) == 1 and int(torch.isnan(state).sum()) == 1


# ---- sizes that differ by columns and rows
def sized(t, heads, exponents):
    """Columns of each head times powers of two."""
    R = t.shape[0]
    f = torch.exp2(torch.tensor(exponents, dtype=torch.float32))
    v = t.view(R, heads, -1)
    return (v * f[torch.arange(v.shape[2]) % len(exponents)]).reshape(R, -1)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("lengths,dk,dv", [([150, 0, 40], 40, 56), ([6, 16, 1, 9], 40, 56),
                                           ([700, 33], 64, 64), ([70], 128, 128), ([90, 5], 128, 64)])
def test_columns_of_mixed_sizes(tgm, lengths, dk, dv, dtype, reverse):
    """A column of a state keeps its own precision beside one 2^21 times as large."""
    dt, H, G = TYPES[dtype], 2, 1
    seqs = packed(lengths)
    d = make(seqs, H, G, dk, dv, torch.float32, seed=11)
    far = [10.0, -11.0, 0.0, -5.0, 9.0]
    d["v"], d["do"] = sized(d["v"].cpu(), G, far), sized(d["do"].cpu(), H, far[::-1])
    d["k"], d["q"] = sized(d["k"].cpu(), G, [6.0, -4.0, 0.0]), sized(d["q"].cpu(), H, [0.0, 6.0])
    for n in ("q", "k", "v", "do"):
        d[n] = d[n].to(dt).cuda()
    d["state"] = d["dlast"] = None
    # results of fp16's range: o has q k v, dk q v do
    go(tgm, seqs, H, G, dk, dv, dt, reverse=reverse, d=d, scale=2.0 ** -12)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,w", [(31, 32), (16, 16), (60, 64)])
def test_rows_of_mixed_sizes(tgm, n, w, dtype):
    """Rows of a chunk that go to rows of the state of their own (k is 1 in a column of its
    own) keep their precision beside rows 2^22 times as large."""
    dt = TYPES[dtype]
    seqs = packed([n])
    d = make(seqs, 1, 1, w, w, dt, state=False, decay=[-2.0 ** -6])
    k = torch.zeros(n, w)
    k[torch.arange(n), torch.arange(n)] = 1.0
    f = torch.exp2(torch.where(torch.arange(n) % 2 == 0, 11.0, -11.0))[:, None]
    d["k"], d["v"] = k.to(dt).cuda(), (randn(3, n, w) * f).to(dt).cuda()
    d["q"], d["do"] = (randn(4, n, w) * 2.0 ** -6).to(dt).cuda(), k.flip(0).to(dt).cuda()
    go(tgm, seqs, 1, 1, w, w, dt, d=d, scale=1.0)


@pytest.mark.parametrize("n", [9, 40])
def test_states_far_above(tgm, n):
    """fp16 rows that read a first state above 2^116 (fp32 holds it) by a small scale."""
    dt, w = torch.float16, 16
    seqs = packed([n] * 4)
    d = make(seqs, 1, 1, w, w, dt, decay=[-2.0 ** -8])
    d["state"], d["dlast"] = d["state"] * 2.0 ** 117, d["dlast"] * 2.0 ** 117
    go(tgm, seqs, 1, 1, w, w, dt, d=d, scale=2.0 ** -112, what=())


@pytest.mark.parametrize("rows,H,G", [(200, 2, 2), (5000, 4, 1), (0, 2, 1)])
def test_rows_of_no_sequence_alone(tgm, rows, H, G):
    """Not one sequence: nothing is written, and a capture of the calls goes through."""
    seqs = packed([], behind=rows)
    d, out, _ = both(tgm, seqs, H, G, 16, 8, torch.bfloat16, state=False)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = torch.full_like(out["o"], 7.0)
        tgm.tgm_decay_attn(d["q"], d["k"], d["v"], d["decay"], o, 0,
                           work(tgm, rows, 0, H, 16, 8, torch.bfloat16, G, False), kv_heads=G,
                           **seqs[0])
    g.replay()
    torch.cuda.synchronize()
    for t in [o] + [out[n] for n in ("o", "dq", "dk", "dv")]:
        assert (t.float() == 7).all()


# ---- states handed along many cells
def walk_is_wide(rows, S, H, size):
    """Whether the walk over the cells' states has the work for which it takes 2,048 elements a
    workgroup: over sequences or cells, whichever it goes by, at least so many workgroups of
    512."""
    cells = -(-rows // min(4096, max(64, -(-int((2 * rows * H) ** 0.5) // 64) * 64)))
    by_sequence = S <= 4 * cells
    return by_sequence, (S if by_sequence else cells) * H * -(-size // 512) > 4096


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_walk_by_sequences(tgm, dtype, reverse):
    """Wide states of many heads: uneven sequences over several cells of rows, and states that
    are no whole number of a workgroup's elements."""
    lengths = [20 + (37 * i) % 300 for i in range(24)]
    lengths[3], lengths[9], lengths[20] = 2900, 0, 1500
    seqs, H, dk, dv = packed(lengths, before=30, behind=3), 16, 64, 100
    assert walk_is_wide(seqs[3], len(lengths), H, dk * dv) == (True, True)
    go(tgm, seqs, H, 16, dk, dv, TYPES[dtype], reverse=reverse)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_walk_by_cells(tgm, dtype, reverse):
    """More than four sequences to a cell, most of them short, two of them over several cells."""
    short = [(7 * i) % 5 for i in range(60)]
    seqs = packed(short[:40] + [1900] + short[40:] + [950, 1, 3], behind=40)
    H, dk, dv = 16, 128, 126
    assert walk_is_wide(seqs[3], len(seqs[1]), H, dk * dv) == (False, True)
    go(tgm, seqs, H, 16, dk, dv, TYPES[dtype], reverse=reverse)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_sequences_alone(tgm, dtype):
    """Each sequence's results are those of a call with that sequence alone, within both calls'
    tolerances (how its rows come into chunks and cells may differ)."""
    dt, lengths, H, G, d = TYPES[dtype], [64, 0, 90, 10, 700], 2, 1, 64
    how, begin, end, rows = packed(lengths)
    m, out, ref = go(tgm, (how, begin, end, rows), H, G, d, d, dt)
    for s, (b, e) in enumerate(zip(begin, end)):
        alone = {n: m[n][b:e] for n in ("q", "k", "v", "do")}
        alone.update(decay=m["decay"], state=m["state"][s:s + 1], dlast=m["dlast"][s:s + 1])
        _, got, _ = both(tgm, packed([e - b]), H, G, d, d, dt, d=alone)
        for n in got:
            tol = decayref.tolerance(n, ref, dt)
            tol = tol + rounded(ref[n].abs() + tol, torch.float32 if "state" in n else dt)
            at = slice(s, s + 1) if "state" in n else slice(b, e)
            check(n, got[n], out[n][at].cpu().to(F64), 2 * tol[at])

"""The sequence operators together, as a layer over event histories uses them:

    t, u = norm(x, res);  z = u W_in^T + b  (gates and candidates, 2D columns)
    h = scan(z[:, :D], z[:, D:]);  out = h W_out^T + t

forward and backward against fp64 autograd, on packed histories and on sampled
neighbours (tgm_sample, newest first, padded); in 8 bits; row by row for
serving; captured into a graph; on two streams; and on rows whose offsets pass
32 bits.

Tolerance of the whole layer in fp32: four stages of at most 100 roundings
(sums of up to 64 terms) each, on sums whose terms' absolute values are about 8
times the result: 4 x 100 x 8 x 2^-24 = 1.9e-4, relative to the largest value."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from opref import CHAIN, F64, U, check, linear, norm, rounded, scan  # noqa: E402

TOL = 2e-4
EPS = 1e-6
D, C = 48, 64   # state and channel widths


@pytest.fixture(scope="module", autouse=True)
def tgm():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2402_15113_amd import tgm as t
    t.lib()
    return t


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).cuda()


def near(name, got, ref, tol=TOL):
    got = got.detach().cpu().to(F64)
    off = float((got - ref).abs().max())
    assert off <= tol * float(ref.abs().max()), f"{name}: off by {off}, scale {float(ref.abs().max())}"


class Layer:
    """Weights, buffers and one work space, which the calls of a stream share."""

    def __init__(self, tgm, rows, S, packed, seed=0):
        self.tgm, self.rows, self.S = tgm, rows, S
        self.w = 1 + 0.1 * randn(seed, C)
        self.w_in, self.b_in = randn(seed + 1, 2 * D, C) / C ** 0.5, randn(seed + 2, 2 * D)
        self.w_out = randn(seed + 3, C, D) / D ** 0.5
        e = lambda *shape: torch.zeros(*shape, device="cuda")
        self.t, self.u, self.z, self.h, self.out = e(rows, C), e(rows, C), e(rows, 2 * D), \
            e(rows, D), e(rows, C)
        self.h_last = e(S, D)
        self.carry = e(tgm.tgm_scan_carry_rows(rows, S, packed), D)
        n = max(tgm.tgm_scan_work_bytes(rows, D, S), tgm.tgm_norm_work_bytes(rows, C),
                *(tgm.tgm_linear_work_bytes(rows, a, b, torch.float32, backward=k)
                  for a, b in ((2 * D, C), (C, D)) for k in (False, True)))
        self.work = torch.empty(n, dtype=torch.uint8, device="cuda")

    def forward(self, x, res, seq):
        T, k = self.tgm, self.work
        T.tgm_norm(x, self.w, self.u, EPS, res=res, total=self.t)
        T.tgm_linear(self.u, self.w_in, self.z, k, bias=self.b_in)
        T.tgm_scan(self.z[:, :D], self.z[:, D:], self.h, self.S, k, h_last=self.h_last,
                   carry=self.carry, **seq)
        T.tgm_linear(self.h, self.w_out, self.out, k, residual=self.t)
        return self.out

    def backward(self, dout, dh_last, seq):
        T, k = self.tgm, self.work
        g = {n: torch.zeros_like(getattr(self, n)) for n in ("w", "w_in", "b_in", "w_out")}
        dh, dz, du, dx = (torch.zeros_like(v) for v in (self.h, self.z, self.u, self.u))
        g["h0"] = torch.zeros_like(self.h_last)
        T.tgm_linear_backward(self.h, self.w_out, dout, k, dx=dh, dw=g["w_out"])
        T.tgm_scan_backward(self.z[:, :D], self.z[:, D:], dh, self.carry, dz[:, :D], dz[:, D:],
                            self.S, k, dh_last=dh_last, dh0=g["h0"], **seq)
        T.tgm_linear_backward(self.u, self.w_in, dz, k, dx=du, dw=g["w_in"], db=g["b_in"])
        T.tgm_norm_backward(self.t, self.w, du, EPS, dx, g["w"], k, dtotal=dout)
        g["x"] = dx
        return g

    def reference(self, x, res, h0, rows_of, dout, dh_last):
        """fp64 autograd; rows_of: each sequence's rows in the scan's order."""
        f = lambda v: v.detach().cpu().to(F64).requires_grad_()
        p = dict(w=f(self.w), w_in=f(self.w_in), b_in=f(self.b_in), w_out=f(self.w_out), x=f(x),
                 h0=f(h0))
        t = p["x"] + res.cpu().to(F64)
        u = t * (t.square().mean(1, keepdim=True) + EPS) ** -0.5 * p["w"]
        z = u @ p["w_in"].t() + p["b_in"]
        a = torch.sigmoid(z[:, :D])
        h, last = [None] * self.rows, []
        for s, rows in enumerate(rows_of):
            v = p["h0"][s]
            for r in rows:
                v = a[r] * v + (1 - a[r]) * z[r, D:]
                h[r] = v
            last.append(v)
        zero = torch.zeros(D, dtype=F64)
        used = torch.tensor([v is not None for v in h])
        h = torch.stack([zero if v is None else v for v in h])
        out, last = h @ p["w_out"].t() + t, torch.stack(last)
        loss = (out * dout.cpu().to(F64)).sum() + (last * dh_last.cpu().to(F64)).sum()
        names = list(p)
        return out.detach(), last.detach(), used, dict(
            zip(names, torch.autograd.grad(loss, [p[n] for n in names])))


def histories(lengths):
    off = torch.cat([torch.zeros(1, dtype=torch.int64),
                     torch.tensor(lengths, dtype=torch.int64).cumsum(0)])
    return off.cuda(), [list(range(off[s], off[s + 1])) for s in range(len(lengths))]


def test_layer_over_packed_histories(tgm):
    off, rows_of = histories([5, 0, 40, 1, 33, 70])
    n = int(off[-1])
    L = Layer(tgm, n, len(rows_of), True)
    x, res, dout = randn(10, n, C), randn(11, n, C), randn(12, n, C)
    h0, dh_last = randn(13, len(rows_of), D), randn(14, len(rows_of), D)
    seq = dict(offsets=off, h0=h0)
    out = L.forward(x, res, seq).clone()
    g = L.backward(dout, dh_last, seq)
    ref, last, used, rg = L.reference(x, res, h0, rows_of, dout, dh_last)
    assert used.all()
    near("out", out, ref)
    near("h_last", L.h_last, last)
    for name in rg:
        near(name, g[name], rg[name])


def sampled(tgm):
    """Neighbours that tgm_sample finds in a small graph: newest first, padded."""
    N, E, nb, R = 30, 400, 7, 25
    gen = torch.Generator().manual_seed(5)
    ids = lambda n: torch.randint(0, N, (n,), generator=gen, dtype=torch.int32).cuda()
    t = torch.sort(torch.rand(E, generator=gen, dtype=F64))[0].cuda()
    src, dst, neg = ids(E), ids(E), ids(E)
    graph = tgm.tgm_graph_create(N, src, dst, t, neg, None)
    root, ts = ids(R), torch.linspace(0, 1, R, dtype=F64).cuda()
    nbr, eid = (torch.empty(R, nb, dtype=torch.int32, device="cuda") for _ in range(2))
    nts, cnt = torch.empty(R, nb, dtype=F64, device="cuda"), torch.empty(R, dtype=torch.int32,
                                                                         device="cuda")
    tgm.tgm_sample(graph, root, ts, R, nb, nbr, eid, nts, cnt)
    torch.cuda.synchronize()
    tgm.tgm_graph_destroy(graph)
    return R, nb, nbr, cnt


def test_layer_over_sampled_neighbours(tgm):
    R, nb, nbr, cnt = sampled(tgm)
    counts = cnt.tolist()
    assert min(counts) == 0 and max(counts) == nb
    L = Layer(tgm, R * nb, R, False)
    table = randn(20, 30, C)
    x = table[nbr.clamp(min=0).long().reshape(-1)]
    hole = (nbr.reshape(-1) < 0)
    x[hole] = float("nan")   # what padding holds does not matter
    res, dout = randn(21, R * nb, C), randn(22, R * nb, C)
    h0, dh_last = randn(23, R, D), randn(24, R, D)
    seq = dict(length=cnt, h0=h0, reverse=True)   # oldest first: from the last row up
    out = L.forward(x, res, seq).clone()
    rows_of = [list(range(s * nb + counts[s] - 1, s * nb - 1, -1)) for s in range(R)]
    ref, last, used, _ = L.reference(torch.where(hole[:, None], torch.zeros_like(x), x), res, h0,
                                     rows_of, dout, dh_last)
    assert torch.equal(used, ~hole.cpu())
    near("out", out[~hole], ref[used])
    near("h_last", L.h_last, last)
    assert torch.isfinite(L.h_last).all()


def test_layer_in_8_bits(tgm):
    """norm to 8 bits and the 8-bit product against fp64 on the stored values."""
    n = 200
    x, w = randn(1, n, C).bfloat16(), (1 + 0.1 * randn(2, C)).bfloat16()
    q, s = torch.empty(n, C, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(n,
                                                                                   device="cuda")
    tgm.tgm_norm(x, w, q, EPS, scale=s)
    wide = randn(3, 2 * D, C)
    sw = wide.abs().amax(1) / 448
    wq = (wide / sw[:, None]).to(torch.float8_e4m3fn)
    for out in (torch.float32, torch.bfloat16):
        y = torch.empty(n, 2 * D, device="cuda", dtype=out)
        k = torch.empty(tgm.tgm_linear_work_bytes(n, 2 * D, C, q.dtype), dtype=torch.uint8,
                        device="cuda")
        tgm.tgm_linear(q, wq, y, k, scale_x=s, scale_w=sw, act="silu")
        _, _, ref, e = linear(q.float(), wq.float(), "silu", scale_x=s, scale_w=sw,
                              cut8=out != torch.float32)
        check("y", y, ref, e + rounded(ref.abs() + e, out))


def test_serving_follows_training(tgm):
    """The histories again, one event of every sequence at a time, with the states
    in a table of nodes: the same outputs as all rows at once."""
    S, L_, N = 9, 6, 20
    rows = S * L_
    L = Layer(tgm, rows, S, False)
    x, res = randn(1, rows, C), randn(2, rows, C)
    state = randn(3, N, D)
    slots = torch.randperm(N, generator=torch.Generator().manual_seed(4))[:S].to(torch.int32).cuda()
    h0 = state[slots.long()].clone()
    whole = L.forward(x, res, dict(h0=h0)).clone()
    one = Layer(tgm, S, S, False)
    for t in range(L_):
        T, k = tgm, one.work
        T.tgm_norm(x[t::L_], one.w, one.u, EPS, res=res[t::L_], total=one.t)
        T.tgm_linear(one.u, one.w_in, one.z, k, bias=one.b_in)
        T.tgm_scan_step(one.z[:, :D], one.z[:, D:], state, one.h, slots=slots)
        T.tgm_linear(one.h, one.w_out, one.out, k, residual=one.t)
        near("out", one.out, whole[t::L_].cpu().to(F64))
    near("state", state[slots.long()], L.h_last.cpu().to(F64))


def test_row_count_of_a_node_set(tgm):
    """n_rows as *n_nodes leaves it: rows past it stay as they were."""
    n, cap = 37, 90
    L = Layer(tgm, cap, cap, False)
    x, res = randn(1, cap, C), randn(2, cap, C)
    x[n:] = float("nan")
    count = torch.tensor([n], dtype=torch.int32, device="cuda")
    state = torch.full((cap, D), 7.0, device="cuda")
    for v in (L.t, L.u, L.z, L.h, L.out):
        v.fill_(7)
    tgm.tgm_norm(x, L.w, L.u, EPS, res=res, total=L.t, n_rows=count)
    tgm.tgm_linear(L.u, L.w_in, L.z, L.work, bias=L.b_in, n_rows=count)
    tgm.tgm_scan_step(L.z[:, :D], L.z[:, D:], state, L.h, n_rows=count)
    tgm.tgm_linear(L.h, L.w_out, L.out, L.work, residual=L.t, n_rows=count)
    for v in (L.t, L.u, L.z, L.h, L.out, state):
        assert (v[n:] == 7).all() and torch.isfinite(v[:n]).all()
    near("t", L.t[:n], norm(x[:n], L.w, EPS, res[:n])[0])


def test_captured_into_a_graph(tgm):
    """A forward and a backward pass captured once and replayed on new inputs, with
    eager calls and synchronizations between the replays."""
    off, rows_of = histories([300, 0, 700, 40])
    n, S = int(off[-1]), len(rows_of)
    L, eager = Layer(tgm, n, S, True), Layer(tgm, n, S, True)
    x, res, dout = randn(10, n, C), randn(11, n, C), randn(12, n, C)
    h0, dh_last = randn(13, S, D), randn(14, S, D)
    seq = dict(offsets=off, h0=h0)
    before = tgm.alloc_count()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        L.forward(x, res, seq)
        L.backward(dout, dh_last, seq)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = L.forward(x, res, seq)
        g = L.backward(dout, dh_last, seq)
    for k in range(4):
        x.copy_(randn(30 + k, n, C))
        h0.copy_(randn(40 + k, S, D))
        want = eager.forward(x, res, seq).clone()
        wg = eager.backward(dout, dh_last, seq)
        if k % 2:
            torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(L.h_last, eager.h_last), k
        for name in wg:
            assert torch.equal(g[name], wg[name]), (k, name)
    assert tgm.alloc_count() == before


def test_two_streams_at_once(tgm):
    """Calls that run at the same time, each with its own work space."""
    off, rows_of = histories([4000, 1, 5000])
    n, S = int(off[-1]), len(rows_of)
    x, res = randn(10, n, C), randn(11, n, C)
    seq = dict(offsets=off, h0=randn(13, S, D))
    want = Layer(tgm, n, S, True).forward(x, res, seq).clone()
    layers = [Layer(tgm, n, S, True) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    for _ in range(5):
        for L, s in zip(layers, streams):
            with torch.cuda.stream(s):
                L.forward(x, res, seq)
    torch.cuda.synchronize()
    for L in layers:
        assert torch.equal(L.out, want)


def test_a_stream_by_argument(tgm):
    x, w = randn(1, 50, C), randn(2, C)
    y, s = torch.empty_like(x), torch.cuda.Stream()
    torch.cuda.synchronize()
    tgm.tgm_norm(x, w, y, EPS, stream=s)
    s.synchronize()
    ref = norm(x, w, EPS)[1]
    check("y", y, ref, rounded(ref, y.dtype) + CHAIN * U * ref.abs())


def test_offsets_past_32_bits(tgm):
    """The last rows of matrices of more than 2^31 elements and 2^32 bytes."""
    cols, n, k = 4096, 700_000, 40
    x = torch.zeros(n, cols, device="cuda", dtype=torch.bfloat16)
    y = torch.zeros(n, cols, device="cuda", dtype=torch.bfloat16)
    x[-k:] = randn(1, k, cols).bfloat16()
    w = randn(2, cols).bfloat16()
    tgm.tgm_norm(x, w, y, EPS)
    ref = norm(x[-k:], w, EPS)[1]
    check("norm", y[-k:], ref, rounded(ref, y.dtype) + CHAIN * U * ref.abs())
    # a product whose rows lie 4,096 apart, read and written
    W = randn(3, 64, 32).bfloat16()
    tgm.tgm_linear(x[:, :32], W, y[:, 64:128], torch.empty(
        max(16, tgm.tgm_linear_work_bytes(n, 64, 32, W.dtype)), dtype=torch.uint8, device="cuda"))
    ref, _, _, e = linear(x[-k:, :32], W, "none")
    check("linear", y[-k:, 64:128], ref, e + rounded(ref.abs() + e, y.dtype))
    # a scan of the last rows behind one that ends before them
    off = torch.tensor([0, n - k, n], device="cuda")
    work = torch.empty(tgm.tgm_scan_work_bytes(n, 64, 2), dtype=torch.uint8, device="cuda")
    tgm.tgm_scan(x[:, :64], x[:, 64:128], y[:, :64], 2, work, offsets=off)
    ref, err = scan(x[-k:, :64], x[-k:, 64:128], [0], [k])
    check("scan", y[-k:, :64], ref["y"], err["y"] + rounded(ref["y"], y.dtype))


def test_8_bit_nan(tgm):
    """A NaN code spreads over its row or column and no further."""
    for rows in (8, 300):
        x, w = (randn(s, *shape).to(torch.float8_e4m3fn) for s, shape in
                ((1, (rows, 70)), (2, (150, 70))))
        x.view(torch.uint8)[3, 69], w.view(torch.uint8)[100, 0] = 0x7f, 0xff
        sx, sw = torch.ones(rows, device="cuda"), torch.ones(150, device="cuda")
        for out in (torch.float32, torch.bfloat16):
            y = torch.empty(rows, 150, device="cuda", dtype=out)
            tgm.tgm_linear(x, w, y, torch.empty(max(16, tgm.tgm_linear_work_bytes(
                rows, 150, 70, x.dtype)), dtype=torch.uint8, device="cuda"), scale_x=sx, scale_w=sw)
            bad = torch.isnan(y)
            assert bad[3].all() and bad[:, 100].all()
            bad[3], bad[:, 100] = False, False
            assert not bad.any()

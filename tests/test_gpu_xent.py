"""tgm_xent and tgm_xent_backward against fp64: sizes around the tiles, one row and one
class, odd strides, biases that leave classes out, rows without a target, row counts on the
device, tables in several pieces, infinities and NaN, captured and on two streams.

Tolerances, with U = 2^-24.  A logit is a sum of K exact products added in fp32, by the
matrix instructions 4 to 32 at a time and in no more than K / 4 + 8 sums one after another:
e_z = (K / 4 + 8) U sum|x w| + U |z|.  An exponential of d = z - max is off by (2 |d| + 4) U
of itself; a row's N of them add up in at most N / 16 + 40 sums one after another, and the
logarithm rounds once.  dz has the errors of its logit, of lse and of the exponential, one
product, and one rounding to the operands' type; dx and dW are sums of n such."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from opref import F64, TYPES, U, check, half_step, rounded  # noqa: E402


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


def untouched(got, cols):
    return got._base is None or (got._base[:, cols:].float() == 7).all()


def work(tgm, rows, N, K, dtype, backward):
    n = tgm.tgm_xent_work_bytes(rows, N, K, dtype, backward=backward)
    return torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)


def reference(x, w, target, bias, dloss):
    """Results and tolerances before the type's rounding, on the GPU in fp64."""
    x64, w64, rows, N, K = x.to(F64), w.to(F64), x.shape[0], w.shape[0], x.shape[1]
    z = x64 @ w64.t().contiguous()
    a = x64.abs() @ w64.abs().t().contiguous()
    if bias is not None:
        z, a = z + bias.to(F64), a + torch.where(bias.isinf(), 0.0, bias.to(F64).abs())
    ez = (K / 4 + 8) * U * a + U * torch.where(z.isinf(), 0.0, z.abs())
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    d = torch.where(z.isinf(), 0.0, (z - z.amax(1, keepdim=True)).abs())
    el = (p * (ez + 2 * U * d)).sum(1) + (N / 16 + 44) * U + 2 * U * lse.abs()
    t = target.long()
    used = (t >= 0) & (t < N)
    at = t.clamp(0, N - 1)[:, None]
    zt, ezt = z.gather(1, at)[:, 0], ez.gather(1, at)[:, 0]
    zero = torch.zeros_like(lse)
    out = dict(lse=(lse, el), loss=(torch.where(used, lse - zt, zero),
                                    torch.where(used, el + ezt + U * (lse.abs() + zt.abs()), zero)))
    if dloss is None:
        return out
    dl = torch.where(used, dloss.to(F64), zero)[:, None]
    on = torch.zeros_like(z).scatter_(1, at, 1.0)
    dz = dl * (p - on)
    far = torch.where(z.isinf(), 0.0, (z - lse[:, None]).abs())
    ep = p * (ez + el[:, None] + U * (3 * far + lse.abs()[:, None] + 8))
    edz = dl.abs() * (ep + 2 * U * (p - on).abs())
    # the rounding for the products, with fp16's smallest step 2^-24 at 2^14 or more of scale
    top = float(dl.abs().max()) if rows else 0.0
    er = edz + half_step(x.dtype) * (dz.abs() + edz) + \
        (2.0 ** -25 * 2.0 ** -13 * top if x.dtype == torch.float16 else 0.0)
    r = dz.abs() + er
    c = lambda n: (n / 4 + 80) * U
    out["dx"] = (dz @ w64, er @ w64.abs() + c(N) * (r @ w64.abs()))
    out["dw"] = (dz.t().contiguous() @ x64,
                 er.t().contiguous() @ x64.abs() + c(rows) * (r.t().contiguous() @ x64.abs()))
    out["db"] = (dz.sum(0), edz.sum(0) + c(rows) * (dz.abs() + edz).sum(0))
    return out


def go(tgm, rows, N, K, dtype, seed=0, pad=0, bias=True, ignore=True, masked=False, n_rows=None,
       what=("dx", "dw", "db"), spread=2.0):
    x = strided(randn(seed, rows, K), dtype, pad)
    w = strided(randn(seed + 1, N, K) * spread / K ** 0.5, dtype, 2 * pad)
    g = torch.Generator().manual_seed(seed + 2)
    t = torch.randint(0, N, (rows,), generator=g).to(torch.int32)
    b = randn(seed + 3, N).to(dtype) if bias else None
    if masked:
        out = torch.rand(N, generator=g) < 0.4
        out[0] = False
        b[out] = -math.inf
        t = torch.where(out[t.long()], torch.zeros_like(t), t)
    if ignore:
        bad = torch.tensor([-1, N, -2 ** 31, 2 ** 31 - 1], dtype=torch.int64)
        pick = torch.rand(rows, generator=g) < 0.3
        t = torch.where(pick, bad[torch.randint(0, 4, (rows,), generator=g)], t.long()).to(
            torch.int32)
    t, b = t.cuda(), None if b is None else b.cuda()
    dl = (randn(seed + 4, rows) * (100.0 if dtype == torch.float16 else 0.01)).cuda()
    nr = None if n_rows is None else torch.tensor([n_rows], dtype=torch.int32, device="cuda")
    m = rows if n_rows is None else max(0, min(rows, n_rows))
    loss, lse = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
    tgm.tgm_xent(x, w, t, loss, work(tgm, rows, N, K, dtype, False), lse=lse, bias=b, n_rows=nr)
    ref = reference(x[:m], w, t[:m], b, dl[:m])
    cpu = lambda v: v.cpu()
    for name, got in (("loss", loss), ("lse", lse)):
        r, e = map(cpu, ref[name])
        check(name, got[:m], r, e)
        assert (got[m:] == 7).all()
    outs = dict(dx=strided(torch.full((rows, K), 7.0), dtype, pad),
                dw=strided(torch.full((N, K), 7.0), dtype, pad),
                db=torch.full((N,), 7.0, device="cuda").to(dtype))
    tgm.tgm_xent_backward(x, w, t, lse, dl, work(tgm, rows, N, K, dtype, True), bias=b, n_rows=nr,
                          **{k: outs[k] for k in what})
    for name in what:
        r, e = map(cpu, ref[name])
        got = outs[name][:m] if name == "dx" else outs[name]
        check(name, got, r, e + rounded(r.abs() + e, dtype))
    for name in set(outs) - set(what):
        assert (outs[name].float() == 7).all()
    assert (outs["dx"][m:].float() == 7).all(), "rows past the count were written"
    assert untouched(outs["dx"], K) and untouched(outs["dw"], K)
    return loss, lse, outs


SIZES = [(1, 1, 1), (1, 2, 8), (3, 5, 3), (17, 63, 64), (64, 64, 128), (65, 130, 37),
         (200, 1000, 100), (129, 257, 300), (600, 9228, 100)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,N,K", SIZES)
def test_sizes(tgm, rows, N, K, dtype):
    go(tgm, rows, N, K, TYPES[dtype], seed=rows)
    go(tgm, rows, N, K, TYPES[dtype], seed=rows + 9, pad=3, bias=False, ignore=False)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_aligned_and_not(tgm, dtype):
    for K in (64, 65, 72, 128):
        go(tgm, 140, 264, K, TYPES[dtype], seed=K)
        go(tgm, 140, 265, K, TYPES[dtype], seed=K, pad=8)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_classes_left_out(tgm, dtype):
    _, _, out = go(tgm, 70, 300, 40, TYPES[dtype], masked=True)
    go(tgm, 70, 3000, 40, TYPES[dtype], masked=True, pad=1)


@pytest.mark.parametrize("n", [-1, 0, 1, 63, 64, 65, 128, 200, 500])
def test_row_count_on_the_device(tgm, n):
    go(tgm, 200, 150, 48, torch.bfloat16, n_rows=n)
    go(tgm, 200, 150, 48, torch.float32, n_rows=n)


@pytest.mark.parametrize("what", [("dx",), ("dw",), ("db",), ("dx", "db"), ()])
def test_some_gradients(tgm, what):
    go(tgm, 100, 200, 64, torch.float16, what=what)


@pytest.mark.parametrize("dtype,rows,N", [("f32", 8192, 9001), ("bf16", 16384, 9001),
                                          ("f16", 16384, 8201)])
def test_pieces(tgm, dtype, rows, N):
    """dz of all classes is more than a piece: dx adds the pieces."""
    go(tgm, rows, N, 64, TYPES[dtype])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_large_tiles(tgm, dtype):
    go(tgm, 3600, 3700, 1032, TYPES[dtype], bias=False)


def test_no_rows(tgm):
    w = torch.ones(20, 8, device="cuda")
    x, t = torch.empty(0, 8, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    loss, k = torch.empty(0, device="cuda"), work(tgm, 0, 20, 8, torch.float32, True)
    dw, db = torch.ones_like(w), torch.ones(20, device="cuda")
    tgm.tgm_xent(x, w, t, loss, None)
    tgm.tgm_xent_backward(x, w, t, loss, loss, k, dx=x.clone(), dw=dw, db=db)
    assert (dw == 0).all() and (db == 0).all()


def test_nothing_left(tgm):
    """Every class left out: no distribution, no gradient; and a target that is left out."""
    x, w = randn(1, 6, 16).cuda(), randn(2, 40, 16).cuda()
    t = torch.arange(6, dtype=torch.int32, device="cuda")
    loss, lse = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    b = torch.full((40,), -math.inf, device="cuda")
    dl = torch.ones(6, device="cuda")
    k, kb = work(tgm, 6, 40, 16, torch.float32, False), work(tgm, 6, 40, 16, torch.float32, True)
    out = dict(dx=torch.ones(6, 16).cuda(), dw=torch.ones(40, 16).cuda(), db=torch.ones(40).cuda())
    tgm.tgm_xent(x, w, t, loss, k, lse=lse, bias=b)
    assert (loss == math.inf).all() and (lse == -math.inf).all()
    tgm.tgm_xent_backward(x, w, t, lse, dl, kb, bias=b, **out)
    assert all((v == 0).all() for v in out.values())
    b[3:] = 0
    tgm.tgm_xent(x, w, t, loss, k, lse=lse, bias=b)
    assert (loss[:3] == math.inf).all() and torch.isfinite(loss[3:]).all()
    tgm.tgm_xent_backward(x, w, t, lse, dl, kb, bias=b, **out)
    assert torch.equal(out["db"][:3], -torch.ones(3, device="cuda"))
    assert all(torch.isfinite(v).all() for v in out.values())
    # the lowest finite value is a number like others, and leaves nothing of its class either
    low = torch.where(b.isinf(), torch.finfo(torch.float32).min, b)
    l2 = torch.empty(6, device="cuda")
    tgm.tgm_xent(x, w, t, loss, k, lse=l2, bias=low)
    assert torch.equal(l2, lse)


def test_not_finite(tgm):
    """A row with NaN or an infinite logit keeps it to itself."""
    x, w = randn(1, 40, 24).cuda(), randn(2, 70, 24).cuda()
    t = torch.arange(40, dtype=torch.int32, device="cuda")
    k = work(tgm, 40, 70, 24, torch.float32, False)
    a, b = torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
    tgm.tgm_xent(x, w, t, a, k)
    x[3, 5], x[20, 0] = math.nan, math.inf
    tgm.tgm_xent(x, w, t, b, k)
    rest = torch.ones(40, dtype=torch.bool, device="cuda")
    rest[[3, 20]] = False
    assert torch.isnan(b[3]) and not torch.isfinite(b[20]) and torch.equal(a[rest], b[rest])
    # a bias of +infinity: all the probability
    bias = torch.zeros(70, device="cuda")
    bias[9] = math.inf
    x[3, 5], x[20, 0] = 0.0, 0.0
    tgm.tgm_xent(x, w, t, b, k, lse=a, bias=bias)
    assert (a == math.inf).all() and torch.isnan(b[9]) and (b[:9] == math.inf).all()


def test_far_logits(tgm):
    """Logits of some thousand: nothing overflows, and the far ones vanish."""
    go(tgm, 50, 200, 16, torch.float32, spread=2000.0)
    go(tgm, 50, 200, 16, torch.bfloat16, spread=2000.0)


def test_differences(tgm):
    """The gradient against central differences of the loss, in fp32: with steps of 2^-7 the
    third derivative (at most 0.1 sum|v|^3 a row) and the loss's rounding are what is off."""
    rows, N, K, h = 9, 33, 12, 2.0 ** -7
    x, w, b = randn(1, rows, K).cuda(), randn(2, N, K).cuda() / K ** 0.5, randn(3, N).cuda()
    t = torch.arange(rows, dtype=torch.int32, device="cuda")
    t[4] = -1
    dl = randn(5, rows).cuda()
    k, kb = work(tgm, rows, N, K, torch.float32, False), work(tgm, rows, N, K, torch.float32, True)
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")

    def total(x, w, b):
        tgm.tgm_xent(x, w, t, loss, k, lse=lse, bias=b)
        return float((loss.double() * dl.double()).sum())

    total(x, w, b)
    out = dict(dx=torch.empty_like(x), dw=torch.empty_like(w), db=torch.empty_like(b))
    tgm.tgm_xent_backward(x, w, t, lse, dl, kb, bias=b, **out)
    for i, name in enumerate(("dx", "dw", "db")):
        p = [x, w, b]
        v = randn(30 + i, *p[i].shape).cuda()
        v = v / v.norm()
        up, down = list(p), list(p)
        up[i], down[i] = p[i] + h * v, p[i] - h * v
        slope = (total(*up) - total(*down)) / (2 * h)
        mine = float((out[name].double() * v.double()).sum())
        # logits move by at most 3 h along v (rows of x and W have norms near 1 to 4)
        third = float(dl.abs().sum()) * 64 * h * h / 6
        rounding = float(dl.abs().sum()) * 64 * U / h
        assert abs(slope - mine) <= third + rounding, name


def test_captured_and_two_streams(tgm):
    rows, N, K = 300, 1100, 72
    dt = torch.bfloat16
    x, w = randn(1, rows, K).cuda().to(dt), randn(2, N, K).cuda().to(dt)
    b = randn(3, N).cuda().to(dt)
    t = torch.randint(0, N, (rows,), generator=torch.Generator().manual_seed(4)).to(
        torch.int32).cuda()
    dl = randn(5, rows).cuda()

    def call(k, o, stream=None):
        tgm.tgm_xent(x, w, t, o["loss"], k, lse=o["lse"], bias=b, stream=stream)
        tgm.tgm_xent_backward(x, w, t, o["lse"], dl, k, bias=b, dx=o["dx"], dw=o["dw"],
                              db=o["db"], stream=stream)

    new = lambda: dict(loss=torch.zeros(rows, device="cuda"), lse=torch.zeros(rows, device="cuda"),
                       dx=torch.zeros_like(x), dw=torch.zeros_like(w), db=torch.zeros_like(b))
    n = max(tgm.tgm_xent_work_bytes(rows, N, K, dt), tgm.tgm_xent_work_bytes(rows, N, K, dt, True))
    ks = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(3)]
    outs = [new() for _ in range(3)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(ks[0], outs[0])
    for i in range(4):
        x.copy_(randn(10 + i, rows, K))
        t.copy_(torch.randint(-3, N + 3, (rows,), generator=torch.Generator().manual_seed(i)))
        torch.cuda.synchronize()
        g.replay()
        side = torch.cuda.Stream()
        call(ks[1], outs[1], side)
        call(ks[2], outs[2])
        torch.cuda.synchronize()
        for name in outs[0]:
            assert torch.equal(outs[0][name], outs[1][name]), name
            assert torch.equal(outs[0][name], outs[2][name]), name


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N", [40, 700])
def test_infinite_logit_beside_large_ones(tgm, dtype, N):
    """exp(-300) is zero in 32 bits: nothing, beside an infinite sum, and not NaN."""
    dt, rows, K = TYPES[dtype], 70, 16
    x, w = torch.zeros(rows, K, device="cuda", dtype=dt), torch.zeros(N, K, device="cuda", dtype=dt)
    bias = torch.zeros(N, device="cuda", dtype=dt)
    bias[3], bias[N - 1] = math.inf, 300.0
    target = torch.full((rows,), N - 1, device="cuda", dtype=torch.int32)
    target[0] = 3
    loss, lse = (torch.zeros(rows, device="cuda") for _ in range(2))
    tgm.tgm_xent(x, w, target, loss, work(tgm, rows, N, K, dt, False), lse=lse, bias=bias)
    assert (lse == math.inf).all() and (loss[1:] == math.inf).all() and torch.isnan(loss[0])
    # NaN goes through all the same, wherever it is
    w[N // 2, 0], x[5, 0] = math.nan, 1.0
    tgm.tgm_xent(x, w, target, loss, work(tgm, rows, N, K, dt, False), lse=lse, bias=bias)
    assert torch.isnan(lse).all()


def test_very_many_rows(tgm):
    """More rows than a launch has groups of 16 of: two classes of one channel, whose loss is
    log(1 + e^-z) for the first."""
    rows, f32 = (1 << 26) + 100, torch.float32
    x = (torch.arange(rows, device="cuda") % 1024 / 256.0)[:, None].contiguous()
    w = torch.tensor([[1.0], [0.0]], device="cuda")
    target = torch.zeros(rows, device="cuda", dtype=torch.int32)
    loss, lse = (torch.full((rows,), -1.0, device="cuda") for _ in range(2))
    tgm.tgm_xent(x, w, target, loss, work(tgm, rows, 2, 1, f32, False), lse=lse)
    for some in (slice(0, 1 << 20), slice(rows - (1 << 20), rows)):
        z = x[some, 0].double()
        # two exponentials, their sum, a logarithm and a difference, of values below 5
        tol = torch.full_like(z, 40 * U)
        check("lse", lse[some], torch.log(1 + z.exp()).cpu(), tol.cpu())
        check("loss", loss[some], torch.log(1 + (-z).exp()).cpu(), tol.cpu())
    assert (loss >= 0).all() and (lse > 0).all()
    dx = torch.full_like(x, 7.0)
    tgm.tgm_xent_backward(x, w, target, lse, torch.ones_like(lse),
                          work(tgm, rows, 2, 1, f32, True), dx=dx)
    z = x[-1000:, 0].double()
    check("dx", dx[-1000:, 0], (-1 / (1 + z.exp())).cpu(), torch.full((1000,), 60 * U).double())
    assert (dx < 0).all() and (dx > -0.6).all()


# ---- rows that have no part in the loss
def spoil(x, rows_of_x, seed):
    """What is not finite in one column of some of the rows, in all columns of others."""
    for i, r in enumerate(rows_of_x):
        if i % 3 == 0:
            x[r] = (math.nan, math.inf, -math.inf)[i // 3 % 3]
        elif i % 3 == 1:
            x[r, (seed + i) % x.shape[1]] = (math.nan, math.inf)[i // 3 % 2]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,N,K,pad", [(1, 5, 3, 0), (70, 130, 40, 0), (200, 1000, 100, 3),
                                          (130, 300, 65, 1), (3600, 3700, 264, 0)])
def test_rows_without_a_target_may_hold_anything(tgm, rows, N, K, pad, dtype):
    """Loss 0 and no gradient, whatever their x holds: the same results as of zeros there."""
    dt = TYPES[dtype]
    x, w = strided(randn(1, rows, K), dt, pad), strided(randn(2, N, K) / K ** 0.5, dt, pad)
    t = torch.randint(0, N, (rows,), generator=torch.Generator().manual_seed(3)).to(torch.int32)
    out_rows = list(range(0, rows, 3))
    t[out_rows] = torch.tensor([-1, N, -2 ** 31, 2 ** 31 - 1]).to(torch.int32)[
        torch.arange(len(out_rows)) % 4]
    t, dl = t.cuda(), randn(4, rows).cuda()
    dl[out_rows[0]] = math.nan
    bias = randn(5, N).cuda().to(dt)
    got = []
    for some in (False, True):
        x[out_rows] = 0
        if some:
            spoil(x, out_rows, 7)
        loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        tgm.tgm_xent(x, w, t, loss, work(tgm, rows, N, K, dt, False), lse=lse, bias=bias)
        o = dict(loss=loss, dx=strided(torch.full((rows, K), 7.0), dt, pad),
                 dw=strided(torch.full((N, K), 7.0), dt, pad), db=torch.full_like(bias, 7.0))
        tgm.tgm_xent_backward(x, w, t, lse, dl, work(tgm, rows, N, K, dt, True), bias=bias,
                              dx=o["dx"], dw=o["dw"], db=o["db"])
        assert (loss[out_rows] == 0).all() and (o["dx"][out_rows] == 0).all()
        assert untouched(o["dx"], K) and untouched(o["dw"], K)
        got.append(o)
    for name in got[0]:
        assert torch.isfinite(got[1][name]).all(), name
        assert torch.equal(got[0][name], got[1][name]), name


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_of_nothing_left_may_hold_anything(tgm, dtype):
    """A row whose every logit is -infinity by its own x has no gradient either."""
    dt, rows, N, K = TYPES[dtype], 40, 60, 16
    x, w = randn(1, rows, K).cuda().to(dt), randn(2, N, K).abs().cuda().to(dt) + 0.5
    x[5] = -math.inf
    t = torch.arange(rows, dtype=torch.int32, device="cuda")
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    tgm.tgm_xent(x, w, t, loss, work(tgm, rows, N, K, dt, False), lse=lse)
    assert lse[5] == -math.inf and loss[5] == math.inf
    dw, dx = torch.empty_like(w), torch.empty_like(x)
    tgm.tgm_xent_backward(x, w, t, lse, torch.ones(rows, device="cuda"),
                          work(tgm, rows, N, K, dt, True), dx=dx, dw=dw)
    assert torch.isfinite(dw).all() and (dx[5] == 0).all()


def test_what_is_not_finite_elsewhere_goes_through(tgm):
    """NaN in a row that has a target is in that column of dW; a row behind the count is not."""
    rows, N, K = 90, 70, 24
    x, w = randn(1, rows, K).cuda(), randn(2, N, K).cuda()
    t = (torch.arange(rows, dtype=torch.int32, device="cuda") % N)
    t[3] = -1
    x[3] = math.nan
    nr = torch.tensor([80], dtype=torch.int32, device="cuda")
    x[85] = math.nan
    for bad in (False, True):
        if bad:
            x[11, 4] = math.nan
        loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        tgm.tgm_xent(x, w, t, loss, work(tgm, rows, N, K, torch.float32, False), lse=lse,
                     n_rows=nr)
        dw = torch.empty_like(w)
        tgm.tgm_xent_backward(x, w, t, lse, torch.ones(rows, device="cuda"),
                              work(tgm, rows, N, K, torch.float32, True), dw=dw, n_rows=nr)
        # (the row's logits are NaN, so all columns are)
        assert torch.isnan(dw).all() if bad else torch.isfinite(dw).all()


def test_captured_with_ignored_rows(tgm):
    """Whether rows have to be kept out is found anew in every replay."""
    dt, rows, N, K = torch.bfloat16, 300, 500, 64
    x, w = randn(1, rows, K).cuda().to(dt), randn(2, N, K).cuda().to(dt)
    t = torch.randint(0, N, (rows,), generator=torch.Generator().manual_seed(3)).to(
        torch.int32).cuda()
    lse, dl = torch.zeros(rows, device="cuda"), randn(4, rows).cuda()
    n = max(tgm.tgm_xent_work_bytes(rows, N, K, dt), tgm.tgm_xent_work_bytes(rows, N, K, dt, True))
    ks = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    dws = [torch.zeros_like(w) for _ in range(2)]

    def call(i):
        tgm.tgm_xent(x, w, t, None, ks[i], lse=lse)
        tgm.tgm_xent_backward(x, w, t, lse, dl, ks[i], dw=dws[i])

    call(0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(0)
    for i in range(4):
        x.copy_(randn(20 + i, rows, K))
        t.copy_(torch.randint(0, N, (rows,), generator=torch.Generator().manual_seed(i)))
        if i % 2:
            t[i::7] = -1
            x[i::7] = math.nan
        torch.cuda.synchronize()
        g.replay()
        call(1)
        torch.cuda.synchronize()
        assert torch.isfinite(dws[0]).all() and torch.equal(dws[0], dws[1])


# ---- tables of several pieces
def in_pieces(tgm, rows, N, K, dtype):
    """Whether the work space is too small for dz of all classes."""
    return tgm.tgm_xent_work_bytes(rows, N, K, dtype, backward=True) < \
        rows * N * torch.finfo(dtype).bits // 8


@pytest.mark.parametrize("dtype,rows,N,K,n_rows", [
    ("f32", 16384, 12809, 65, 16001), ("bf16", 32768, 12809, 65, 32001),
    ("f16", 32768, 12809, 65, 32001), ("f32", 16384, 17160, 64, None),
    ("bf16", 32768, 11456, 72, None), ("f16", 32768, 17161, 64, None)])
def test_several_pieces(tgm, dtype, rows, N, K, n_rows):
    """dx adds the pieces, and every piece has its own targets, bias and rows of dW."""
    assert in_pieces(tgm, rows, N, K, TYPES[dtype]), "all classes are one piece"
    go(tgm, rows, N, K, TYPES[dtype], n_rows=n_rows, pad=K % 2)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_many_pieces(tgm, dtype):
    """Many rows: pieces of 1,024 classes, the last one of a few; rows that are kept out too."""
    rows, N, K = 300000, 2 * 1024 + 37, 8
    dt = TYPES[dtype]
    assert in_pieces(tgm, rows, N, K, dt), "all classes are one piece"
    go(tgm, rows, N, K, dt, n_rows=299990)


@pytest.mark.parametrize("dtype,rows", [("f32", 140001), ("bf16", 280001), ("f16", 280001)])
def test_pieces_with_rows_kept_out(tgm, dtype, rows):
    """Every piece's dW takes the rows of x that have a part in the loss, and no others."""
    N, K, dt = 1500, 9, TYPES[dtype]
    assert in_pieces(tgm, rows, N, K, dt), "all classes are one piece"
    x, w = randn(1, rows, K).cuda().to(dt), randn(2, N, K).cuda().to(dt)
    t = torch.randint(0, N, (rows,), generator=torch.Generator().manual_seed(3)).to(
        torch.int32).cuda()
    t[5::11] = -1
    dl, got = randn(4, rows).cuda(), []
    for fill in (0.0, math.nan):
        x[5::11] = fill
        lse = torch.empty(rows, device="cuda")
        tgm.tgm_xent(x, w, t, None, work(tgm, rows, N, K, dt, False), lse=lse)
        dw, dx = torch.full_like(w, 7.0), torch.full_like(x, 7.0)
        tgm.tgm_xent_backward(x, w, t, lse, dl, work(tgm, rows, N, K, dt, True), dw=dw, dx=dx)
        got.append((dw, dx))
    assert torch.isfinite(got[1][0]).all() and torch.equal(got[0][0], got[1][0])
    assert (got[1][1][5::11] == 0).all() and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N", [40, 700])
def test_every_class_at_the_lowest_value(tgm, dtype, N):
    """A mask of the type's lowest value over all classes: equal logits of that size are finite,
    as is everything that is made of them; one class that is not masked has all the probability."""
    dt, rows, K = TYPES[dtype], 70, 16
    x, w = randn(1, rows, K).cuda().to(dt), randn(2, N, K).cuda().to(dt)
    low = torch.finfo(dt).min
    t = torch.full((rows,), 7, dtype=torch.int32, device="cuda")
    dl = torch.ones(rows, device="cuda")
    for open_class in (None, 7):
        bias = torch.full((N,), low, device="cuda", dtype=dt)
        if open_class is not None:
            bias[open_class] = 0.5
        loss, lse = (torch.empty(rows, device="cuda") for _ in range(2))
        tgm.tgm_xent(x, w, t, loss, work(tgm, rows, N, K, dt, False), lse=lse, bias=bias)
        out = dict(dx=torch.empty_like(x), dw=torch.empty_like(w), db=torch.empty_like(bias))
        tgm.tgm_xent_backward(x, w, t, lse, dl, work(tgm, rows, N, K, dt, True), bias=bias, **out)
        ref = reference(x, w, t, bias, dl)
        for name, got in (("lse", lse), ("loss", loss)):
            r, e = (v.cpu() for v in ref[name])
            check(name, got, r, e)
        assert all(torch.isfinite(v.float()).all() for v in out.values())

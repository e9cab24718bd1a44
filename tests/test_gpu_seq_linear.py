"""tgm_linear and tgm_linear_backward against fp64: sizes around the tiles, the
vectors and the matrix instructions, odd strides, 8-bit inputs with scales, row
counts on the device, infinities next to a tail, in place.

Tolerances (opref): one rounding of the output's type, the fp32 sums' error in
any order, the activations' evaluation, and in the gradient the rounding of dz
to the operands' type."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from opref import F64, TYPES, check, linear, linear_grads, rounded  # noqa: E402

E4M3 = torch.float8_e4m3fn
ACTS = ["none", "relu", "silu", "gelu"]


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
    whole = got._base if got._base is not None else got
    return (whole[:, cols:].float() == 7).all()


def work(tgm, rows, N, K, dtype, act="none", backward=False):
    n = tgm.tgm_linear_work_bytes(rows, N, K, dtype, act=act, backward=backward)
    return torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)


def forward(tgm, rows, N, K, dt, act, seed=0, pad=0, bias=True, res=True, z=True, out=None):
    out = out or dt
    x, w = strided(randn(seed, rows, K), dt, pad), strided(randn(seed + 1, N, K) / K ** 0.5, dt,
                                                           2 * pad)
    b = randn(seed + 2, N).to(out).cuda() if bias else None
    r = strided(randn(seed + 3, rows, N), out, pad) if res else None
    s = dict(scale_x=torch.exp(randn(seed + 4, rows)).cuda(),
             scale_w=torch.exp(randn(seed + 5, N)).cuda()) if dt == E4M3 else {}
    y = strided(torch.full((rows, N), 7.0), out, pad)
    zz = strided(torch.full((rows, N), 7.0), out, 3 * pad) if z else None
    k = work(tgm, rows, N, K, dt, act)
    tgm.tgm_linear(x, w, y, k, act=act, bias=b, residual=r, z=zz, **s)
    xs, ws = (x.float(), w.float()) if dt == E4M3 else (x, w)
    rz, ez, ry, ey = linear(xs, ws, act, b, r, cut8=dt == E4M3 and out != torch.float32, **s)
    check("y", y, ry, ey + rounded(ry.abs() + ey, out))
    assert untouched(y, N), "columns past the row were written"
    if z:
        check("z", zz, rz, ez + rounded(rz.abs() + ez, out))
        assert untouched(zz, N)
    return y


def backward(tgm, rows, N, K, dt, act, seed=0, pad=0, n_rows=None):
    x, w = strided(randn(seed, rows, K), dt, pad), strided(randn(seed + 1, N, K) / K ** 0.5, dt,
                                                           2 * pad)
    dy = strided(randn(seed + 2, rows, N), dt, pad)
    z = strided(randn(seed + 3, rows, N) * 2, dt, 3 * pad) if act != "none" else None
    dx, dw = (strided(torch.full(s, 7.0), dt, pad) for s in ((rows, K), (N, K)))
    db = torch.full((N,), 7.0, device="cuda").to(dt)
    k = work(tgm, rows, N, K, dt, act, backward=True)
    nr = None if n_rows is None else torch.tensor([n_rows], dtype=torch.int32, device="cuda")
    tgm.tgm_linear_backward(x, w, dy, k, act=act, z=z, dx=dx, dw=dw, db=db, n_rows=nr)
    m = rows if n_rows is None else max(0, min(rows, n_rows))
    ref = linear_grads(x[:m], w, dy[:m], act, None if z is None else z[:m])
    for name, got in (("dx", dx[:m]), ("dw", dw), ("db", db)):
        r, e = ref[name]
        check(name, got, r, e + rounded(r.abs() + e, dt))
    assert (dx[m:].float() == 7).all(), "rows past the count were written"
    assert untouched(dx, K) and untouched(dw, K)
    return dx, dw, db


SIZES = [(1, 1, 1), (1, 17, 33), (3, 4, 8), (5, 15, 7), (16, 16, 32), (16, 64, 64), (17, 20, 31),
         (33, 129, 65), (64, 100, 472), (65, 16, 128), (100, 200, 129), (129, 127, 64),
         (130, 260, 100), (300, 520, 200), (257, 130, 1000), (520, 300, 96)]


@pytest.mark.parametrize("dtype", list(TYPES) + ["e4m3"])
@pytest.mark.parametrize("size", SIZES)
def test_forward(tgm, size, dtype):
    k = SIZES.index(size)
    dt = TYPES.get(dtype, E4M3)
    out = torch.bfloat16 if dt == E4M3 else None
    forward(tgm, *size, dt, ACTS[k % 4], pad=k % 3, out=out)
    forward(tgm, *size, dt, ACTS[(k + 1) % 4], pad=0, bias=k % 2 == 0, res=k % 2 == 1, z=False,
            out=out)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_activations(tgm, dtype, act):
    forward(tgm, 20, 40, 24, TYPES[dtype], act)
    forward(tgm, 20, 40, 24, E4M3, act, out=TYPES[dtype])
    backward(tgm, 20, 40, 24, TYPES[dtype], act)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", SIZES)
def test_gradient(tgm, size, dtype):
    k = SIZES.index(size)
    backward(tgm, *size, TYPES[dtype], ACTS[k % 4], pad=k % 3)
    backward(tgm, *size, TYPES[dtype], ACTS[(k + 2) % 4])


def test_long_sums(tgm):
    for dt in TYPES.values():
        forward(tgm, 40, 48, 9000, dt, "none")
        backward(tgm, 9000, 24, 40, dt, "silu")
        backward(tgm, 30, 5000, 40, dt, "none")
    forward(tgm, 40, 48, 9001, E4M3, "none", out=torch.float32)


@pytest.mark.parametrize("size", [(1500, 1030, 136), (1024, 2048, 512), (2049, 513, 264)])
def test_many_tiles(tgm, size):
    for dt in (torch.bfloat16, torch.float32):
        forward(tgm, *size, dt, "gelu")
        backward(tgm, *size, dt, "silu")
    forward(tgm, *size, E4M3, "none", out=torch.bfloat16)
    forward(tgm, *size, torch.float16, "silu", pad=1)


@pytest.mark.parametrize("K", [1, 37, 64, 75, 129, 300])
@pytest.mark.parametrize("dtype", list(TYPES) + ["e4m3"])
def test_ragged_tiles(tgm, dtype, K):
    """More workgroups than a product without tiles takes; the sums end inside a step,
    rows and columns inside a tile."""
    dt = TYPES.get(dtype, E4M3)
    out = torch.float16 if dt == E4M3 else None
    forward(tgm, 601, 1101, K, dt, ACTS[K % 4], pad=K % 3, out=out)
    forward(tgm, 513, 1160, K, dt, "none", pad=0, bias=False, res=True, z=False, out=out)


@pytest.mark.parametrize("rows,N,K", [(601, 1101, 75), (130, 96, 2100), (17, 64, 9000)])
def test_tiles_beside_what_is_not_read(tgm, rows, N, K):
    """A row count on the device, infinities in one row and NaN in one column, and a
    residual in place, where tiles (in one part or several) take the product."""
    for dt in TYPES.values():
        x, w, r = (randn(s, *shape).to(dt).cuda() for s, shape in
                   ((1, (rows, K)), (2, (N, K)), (3, (rows, N))))
        k = work(tgm, rows, N, K, dt)
        y = torch.full_like(r, 7.0)
        m = rows - 9
        bad = x.clone()
        bad[m:] = float("nan")
        nr = torch.tensor([m], dtype=torch.int32, device="cuda")
        tgm.tgm_linear(bad, w, y, k, n_rows=nr)
        ref, _, _, e = linear(x[:m], w, "none")
        check("y", y[:m], ref, e + rounded(ref.abs() + e, dt))
        assert (y[m:] == 7).all()
        tgm.tgm_linear(x, w, y, k, residual=r)
        own = r.clone()
        tgm.tgm_linear(x, w, own, k, residual=own)
        assert torch.equal(y, own)
        x[3, K - 1], w[5, 0] = float("inf"), float("nan")
        tgm.tgm_linear(x, w, y, k)
        assert torch.isnan(y[:, 5]).all()
        rest = torch.isfinite(y)
        rest[3], rest[:, 5] = True, True
        assert rest.all() and not torch.isfinite(y[3]).any()


@pytest.mark.parametrize("size", [(17, 64, 512), (700, 40, 300), (512, 512, 700), (768, 256, 1),
                                  (100, 4096, 65), (16, 8200, 130)])
def test_without_tiles(tgm, size):
    for dt in list(TYPES.values()) + [E4M3]:
        out = torch.bfloat16 if dt == E4M3 else None
        forward(tgm, *size, dt, "gelu", pad=1, out=out)
        forward(tgm, *size, dt, "none", pad=0, z=False, out=out)


@pytest.mark.parametrize("n", [-3, 0, 1, 16, 63, 64, 100, 300])
def test_row_count_on_the_device(tgm, n):
    rows, N, K = 200, 72, 40
    for dt in (torch.float32, torch.bfloat16):
        x, w = randn(1, rows, K).to(dt).cuda(), randn(2, N, K).to(dt).cuda()
        y = torch.full((rows, N), 7.0, device="cuda", dtype=dt)
        nr = torch.tensor([n], dtype=torch.int32, device="cuda")
        x[max(0, min(rows, n)):] = float("nan")   # rows that are not read
        tgm.tgm_linear(x, w, y, work(tgm, rows, N, K, dt), n_rows=nr)
        m = max(0, min(rows, n))
        ref, _, _, e = linear(x[:m], w, "none")
        check("y", y[:m], ref, e + rounded(ref.abs() + e, dt))
        assert (y[m:] == 7).all()
        backward(tgm, rows, N, K, dt, "silu", n_rows=n)


def test_row_count_hides_nan_from_sums(tgm):
    """Rows past the count reach neither dW nor db, whatever they hold."""
    rows, N, K, n = 150, 70, 33, 97
    for dt in (torch.float32, torch.bfloat16):
        x, dy, w = (randn(s, *shape).to(dt).cuda()
                    for s, shape in ((1, (rows, K)), (2, (rows, N)), (3, (N, K))))
        x[n:], dy[n:] = float("nan"), float("inf")
        nr = torch.tensor([n], dtype=torch.int32, device="cuda")
        dw, db = torch.empty(N, K, device="cuda", dtype=dt), torch.empty(N, device="cuda", dtype=dt)
        tgm.tgm_linear_backward(x, w, dy, work(tgm, rows, N, K, dt, backward=True), dw=dw, db=db,
                                n_rows=nr)
        ref = linear_grads(x[:n], w, dy[:n], "none")
        for name, got in (("dw", dw), ("db", db)):
            check(name, got, ref[name][0], ref[name][1] + rounded(ref[name][0].abs() + ref[name][1],
                                                                  dt))


def test_optional_gradients(tgm):
    rows, N, K = 70, 90, 50
    for dt in (torch.float32, torch.float16):
        dx, dw, db = backward(tgm, rows, N, K, dt, "gelu")
        x, w, dy, z = (randn(s, *shape).to(dt).cuda() for s, shape in
                       ((0, (rows, K)), (1, (N, K)), (2, (rows, N)), (3, (rows, N))))
        x, w, z = x, (randn(1, N, K) / K ** 0.5).to(dt).cuda(), (randn(3, rows, N) * 2).to(dt).cuda()
        k = work(tgm, rows, N, K, dt, "gelu", backward=True)
        for name, want in (("dx", dx), ("dw", dw), ("db", db)):
            got = torch.empty_like(want).contiguous()
            tgm.tgm_linear_backward(x, w, dy, k, act="gelu", z=z, **{name: got})
            assert torch.equal(got, want), name


def test_no_rows(tgm):
    x, w = torch.empty(0, 5, device="cuda"), torch.ones(6, 5, device="cuda")
    y = torch.empty(0, 6, device="cuda")
    dw, db = torch.full((6, 5), 7.0, device="cuda"), torch.full((6,), 7.0, device="cuda")
    tgm.tgm_linear(x, w, y, None)
    tgm.tgm_linear_backward(x, w, y, None, dx=x, dw=dw, db=db)
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("K", [1, 33, 100, 129])
def test_infinities_stay_in_their_rows_and_columns(tgm, K):
    """Also in the last columns of the sum, next to what pads it."""
    for rows, N in ((20, 24), (300, 300)):
        for dt in TYPES.values():
            x, w = randn(1, rows, K).to(dt).cuda(), randn(2, N, K).to(dt).cuda()
            x[3, K - 1], w[5, 0] = float("inf"), float("nan")
            y = torch.empty(rows, N, device="cuda", dtype=dt)
            tgm.tgm_linear(x, w, y, work(tgm, rows, N, K, dt))
            assert torch.isnan(y[:, 5]).all()
            rest = torch.isfinite(y)
            rest[3], rest[:, 5] = True, True
            assert rest.all() and not torch.isfinite(y[3]).any()


def test_in_place_residual(tgm):
    for rows in (9, 300):
        x, w, r = (randn(s, *shape).bfloat16().cuda() for s, shape in
                   ((1, (rows, 64)), (2, (130, 64)), (3, (rows, 130))))
        y, k = torch.empty_like(r), work(tgm, rows, 130, 64, torch.bfloat16)
        tgm.tgm_linear(x, w, y, k, residual=r)
        tgm.tgm_linear(x, w, r, k, residual=r)
        assert torch.equal(y, r)


def test_reproducible(tgm):
    for size in ((4, 300, 2000), (500, 300, 200)):
        a = forward(tgm, *size, torch.bfloat16, "silu")
        assert torch.equal(a, forward(tgm, *size, torch.bfloat16, "silu"))
        a = backward(tgm, *size, torch.bfloat16, "silu")
        for u, v in zip(a, backward(tgm, *size, torch.bfloat16, "silu")):
            assert torch.equal(u, v)


def test_against_differences(tgm):
    """The gradient of a whole layer's loss against central differences in fp64."""
    rows, N, K = 6, 5, 7
    x, w, b, dy = (randn(s, *shape).cuda() for s, shape in
                   ((1, (rows, K)), (2, (N, K)), (3, (N,)), (4, (rows, N))))
    for act in ("silu", "gelu"):
        y, z = torch.empty(rows, N, device="cuda"), torch.empty(rows, N, device="cuda")
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
        tgm.tgm_linear(x, w, y, work(tgm, rows, N, K, torch.float32), act=act, bias=b, z=z)
        tgm.tgm_linear_backward(x, w, dy, work(tgm, rows, N, K, torch.float32, act, True),
                                act=act, z=z, dx=dx, dw=dw, db=db)
        ins = [v.cpu().to(F64) for v in (x, w, b)]
        f = lambda a: float((linear(a[0], a[1], act, a[2])[2] * dy.cpu().to(F64)).sum())
        h = 1e-6
        for k, grad, at in ((0, dx, (2, 3)), (1, dw, (4, 6)), (1, dw, (0, 0)), (2, db, (1,))):
            lo, hi = [v.clone() for v in ins], [v.clone() for v in ins]
            lo[k][at] -= h
            hi[k][at] += h
            n = (f(hi) - f(lo)) / (2 * h)
            assert abs(float(grad[at]) - n) <= 2e-5 * (1 + abs(n))

"""tgm_linear and tgm_linear_backward at sizes that take the large tiles (256 x 256; fp32 128
x 128) and two parts of them, ragged in every dimension: bias, activation, residual in
place, z, row counts inside a tile, infinities and NaN.  Against fp64 at the tiles'
edges and at random, whole rows and whole columns; tolerances as in
test_gpu_seq_linear."""
import ctypes as C

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from opref import TYPES, check, linear, linear_grads, rounded  # noqa: E402

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def tgm():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2402_15113_amd import tgm as t
    t.lib()
    return t


def randn(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def plan(tgm, M, N, K, dtype):
    """(large, parts) of a product, by the library's own rule."""
    f = tgm.lib()._ZN3tgm11linear_planEllli
    f.argtypes, f.restype = [C.c_int64, C.c_int64, C.c_int64, C.c_int32], C.c_uint64
    v = f(M, N, K, tgm.dtype_code(dtype))
    return bool(v & 0xff), v >> 32


def some(n, seed):
    """Places of n: both sides of the tiles' and blocks' edges, the ends, random ones."""
    at = {0, 1, 15, 16, 31, 32, 63, 64, 127, 128, 129, 255, 256, 257, n - 257, n - 129, n - 33,
          n - 17, n - 9, n - 8, n - 5, n - 4, n - 3, n - 2, n - 1, n // 256 * 256,
          n // 256 * 256 - 1, n // 128 * 128, n // 128 * 128 - 1}
    g = torch.Generator().manual_seed(seed)
    at |= set(torch.randint(n, (20,), generator=g).tolist())
    return torch.tensor(sorted(k for k in at if 0 <= k < n))


def work(tgm, rows, N, K, dtype, act="none", backward=False):
    n = tgm.tgm_linear_work_bytes(rows, N, K, dtype, act=act, backward=backward)
    return torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)


FORWARD = [("f32", "f32", 2000, 4092, 100), ("f32", "f32", 2000, 4092, 1036),
           ("bf16", "bf16", 3600, 3592, 1032), ("f16", "f16", 3847, 3331, 1096),
           ("bf16", "bf16", 3600, 3592, 1024), ("e4m3", "bf16", 3600, 3591, 2064),
           ("e4m3", "f16", 3847, 3592, 2192), ("e4m3", "f32", 3600, 3592, 2064)]


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dtype,out,rows,N,K", FORWARD)
def test_forward(tgm, dtype, out, rows, N, K, act):
    dt, ot = TYPES.get(dtype, E4M3), TYPES[out]
    assert plan(tgm, rows, N, K, dt) == (True, 1)
    m = rows - 13 if act in ("relu", "gelu") else rows
    nr = torch.tensor([m], dtype=torch.int32, device="cuda") if m < rows else None
    x, w = randn(1, rows, K).to(dt), (randn(2, N, K) / K ** 0.5).to(dt)
    if m < rows:
        x.view(torch.uint8 if dt == E4M3 else dt)[m:] = 0x7f if dt == E4M3 else float("nan")
    b, res = randn(3, N).to(ot), randn(4, rows, N).to(ot)
    s = dict(scale_x=torch.exp(randn(5, rows)), scale_w=torch.exp(randn(6, N))) \
        if dt == E4M3 else {}
    y, z = res.clone(), torch.full((rows, N), 7.0, device="cuda", dtype=ot)
    tgm.tgm_linear(x, w, y, work(tgm, rows, N, K, dt, act), act=act, bias=b, residual=y, z=z,
                   n_rows=nr, **s)
    assert torch.equal(y[m:], res[m:]) and (z[m:] == 7).all()
    cut8 = dt == E4M3 and ot != torch.float32
    cast = (lambda v: v.float()) if dt == E4M3 else (lambda v: v)
    for r, c in ((some(m, 1), torch.arange(N)), (torch.arange(m), some(N, 2))):
        r, c = r.cuda(), c.cuda()
        sc = dict(scale_x=s["scale_x"][r], scale_w=s["scale_w"][c]) if s else {}
        rz, ez, ry, ey = linear(cast(x)[r], cast(w)[c], act, b[c], res[r][:, c], cut8=cut8, **sc)
        check("z", z[r][:, c], rz, ez + rounded(rz.abs() + ez, ot))
        check("y", y[r][:, c], ry, ey + rounded(ry.abs() + ey, ot))
    # results without z and a residual are the same sums
    plain = torch.empty_like(y)
    tgm.tgm_linear(x, w, plain, work(tgm, rows, N, K, dt), bias=b, **s)
    assert torch.equal(plain[:m], z[:m])


@pytest.mark.parametrize("dtype,out,rows,N,K", FORWARD[1:4] + FORWARD[5:])
def test_infinities_and_nan_stay_in_their_rows_and_columns(tgm, dtype, out, rows, N, K):
    dt, ot = TYPES.get(dtype, E4M3), TYPES[out]
    x, w = randn(1, rows, K).to(dt), randn(2, N, K).to(dt)
    s = dict(scale_x=torch.ones(rows, device="cuda"), scale_w=torch.ones(N, device="cuda")) \
        if dt == E4M3 else {}
    if dt == E4M3:
        x.view(torch.uint8)[rows - 2, K - 1], w.view(torch.uint8)[300, 0] = 0x7f, 0xff
    else:
        x[rows - 2, K - 1], w[300, 0] = float("inf"), float("nan")
    y = torch.empty(rows, N, device="cuda", dtype=ot)
    tgm.tgm_linear(x, w, y, work(tgm, rows, N, K, dt), **s)
    fine = torch.isfinite(y)
    assert torch.isnan(y[:, 300]).all() and not fine[rows - 2].any()
    fine[rows - 2], fine[:, 300] = True, True
    assert fine.all()


# rows, N, K; (large, parts) of dx and of dW
BACKWARD = [("f32", 2000, 100, 4092, (True, 1), None), ("f32", 300, 2000, 4092, None, (True, 1)),
            ("bf16", 3600, 1032, 3592, (True, 1), None), ("f16", 3847, 1096, 3336, (True, 1), None),
            ("bf16", 1029, 3600, 3592, None, (True, 1)), ("f16", 1096, 3848, 3336, None, (True, 1)),
            ("bf16", 8203, 2568, 2696, None, (True, 2)),
            ("f16", 8256, 2568, 2696, None, (True, 2))]


@pytest.mark.parametrize("counted", [False, True])
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("dtype,rows,N,K,dx_plan,dw_plan", BACKWARD)
def test_gradient(tgm, dtype, rows, N, K, dx_plan, dw_plan, act, counted):
    dt = TYPES[dtype]
    assert dx_plan is None or plan(tgm, rows, K, N, dt) == dx_plan
    assert dw_plan is None or plan(tgm, N, K, rows, dt) == dw_plan
    m = rows - 13 if counted else rows
    nr = torch.tensor([m], dtype=torch.int32, device="cuda") if counted else None
    x, w, dy = randn(1, rows, K).to(dt), (randn(2, N, K) / K ** 0.5).to(dt), randn(3, rows, N).to(dt)
    z = (2 * randn(4, rows, N)).to(dt) if act != "none" else None
    for v in (x, dy) + (() if z is None else (z,)):
        v[m:] = float("nan")
    dx, dw, db = (torch.full(s, 7.0, device="cuda", dtype=dt) for s in ((rows, K), (N, K), (N,)))
    tgm.tgm_linear_backward(x, w, dy, work(tgm, rows, N, K, dt, act, True), act=act, z=z, dx=dx,
                            dw=dw, db=db, n_rows=nr)
    assert (dx[m:] == 7).all()
    x, dy, z = x[:m], dy[:m], None if z is None else z[:m]
    rs, ns, ks = (some(n, 5).cuda() for n in (m, N, K))
    of = lambda a, b: None if z is None else z[a][:, b]
    every = torch.arange(m, device="cuda"), torch.arange(N, device="cuda")
    for name, got, ref in (
            ("dx", dx[rs], linear_grads(x[rs], w, dy[rs], act, of(rs, every[1]))["dx"]),
            ("dx", dx[:m][:, ks], linear_grads(x[:, ks], w[:, ks], dy, act, z)["dx"]),
            ("dw", dw[ns], linear_grads(x, w[ns], dy[:, ns], act, of(every[0], ns))["dw"]),
            ("dw", dw[:, ks], linear_grads(x[:, ks], w[:, ks], dy, act, z)["dw"]),
            ("db", db, linear_grads(x[:, :1], w[:, :1], dy, act, z)["db"])):
        r, e = ref
        check(name, got, r, e + rounded(r.abs() + e, dt))

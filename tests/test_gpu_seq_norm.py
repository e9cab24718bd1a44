"""tgm_norm and tgm_norm_backward against fp64, at the widths where their lanes
and vectors change, odd widths and strides, empty and partial row counts, rows
of zeros, infinities and NaN, and in place.

Tolerances: one rounding of the output's type, plus the fp32 sums' error
(opref.CHAIN roundings of the terms' absolute sum at most)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from opref import CHAIN, F64, STEP, TYPES, U, check, cpu64, norm, norm_grads, rounded  # noqa: E402

E4M3 = torch.float8_e4m3fn
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def tgm():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2402_15113_amd import tgm as t
    t.lib()
    return t


def make(rows, D, dtype, seed=0, pad=0):
    """[rows x D] with rows of different size, in rows of D + pad."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, D + pad, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))
    return x.to(dtype).cuda()[:, :D]


def check_y(y, scale, ref, name="y"):
    if y.dtype != E4M3:
        check(name, y, ref, rounded(ref, y.dtype) + CHAIN * U * ref.abs())
        return
    top = ref.abs().amax(1)
    s = torch.maximum(top / 448, torch.tensor(2.0 ** -126, dtype=F64))
    check("scale", scale, s, (CHAIN + 2) * U * s)
    # half a step of the 8-bit value times the scale, and of the smallest one
    tol = (2.0 ** -4 * ref.abs() + STEP[E4M3] / 2 * s[:, None]) * (1 + 1e-4)
    check(name, y.float().cpu().to(F64) * s[:, None], ref, tol + 2 * (CHAIN + 4) * U * ref.abs())


WIDTHS = [1, 3, 7, 8, 9, 100, 128, 129, 255, 512, 513, 1025, 2049, 4099, 8191, 16390, 32768]


@pytest.mark.parametrize("out", ["same", "8bit"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D", WIDTHS)
def test_forward(tgm, D, dtype, out):
    dt = TYPES[dtype]
    for rows in (1, 5, 37):
        x, res = make(rows, D, dt, 1, pad=3), make(rows, D, dt, 2)
        w = make(1, D, dt, 3)[0].contiguous()
        ref_t, ref = norm(x, w, EPS, res)
        y = torch.zeros(rows, D + 5, device="cuda", dtype=E4M3 if out == "8bit" else dt)
        y.fill_(2.0) if out != "8bit" else y.view(torch.uint8).fill_(0x40)
        total = torch.empty(rows, D, device="cuda", dtype=dt)
        scale = torch.empty(rows, device="cuda") if out == "8bit" else None
        tgm.tgm_norm(x, w, y[:, :D], EPS, res=res, total=total, scale=scale)
        check("total", total, ref_t, rounded(ref_t, dt) + U * ref_t.abs())
        check_y(y[:, :D], scale, ref)
        assert (y[:, D:].float() == 2.0).all(), "columns past the row were written"


def test_no_residual_keeps_total_apart(tgm):
    x, w = make(9, 100, torch.float32), torch.ones(100, device="cuda")
    y = torch.empty_like(x)
    total = torch.empty_like(x)
    tgm.tgm_norm(x, w, y, EPS)
    tgm.tgm_norm(x, w, y, EPS, total=total)
    assert torch.equal(total, x)
    check_y(y, None, norm(x, w, EPS)[1])


@pytest.mark.parametrize("D", [100, 513, 5000])
def test_in_place(tgm, D):
    for dt in (torch.float32, torch.bfloat16):
        x, res, w = make(33, D, dt, 1), make(33, D, dt, 2), make(1, D, dt, 3)[0].contiguous()
        y, total = torch.empty_like(x), torch.empty_like(x)
        tgm.tgm_norm(x, w, y, EPS, res=res, total=total)
        a, b = x.clone(), res.clone()
        tgm.tgm_norm(a, w, a, EPS, res=b, total=b)
        assert torch.equal(a, y) and torch.equal(b, total)
        dy = make(33, D, dt, 4)
        dx, work = torch.empty_like(x), torch.empty(tgm.tgm_norm_work_bytes(33, D),
                                                    dtype=torch.uint8, device="cuda")
        dw = torch.empty_like(w)
        tgm.tgm_norm_backward(total, w, dy, EPS, dx, dw, work)
        c = dy.clone()
        tgm.tgm_norm_backward(total, w, c, EPS, c, dw, work)
        assert torch.equal(c, dx)


@pytest.mark.parametrize("n", [-5, 0, 1, 16, 17, 20, 99])
def test_row_count_on_the_device(tgm, n):
    rows, D = 20, 100
    x, w = make(rows, D, torch.bfloat16), make(1, D, torch.bfloat16, 3)[0].contiguous()
    dy = make(rows, D, torch.bfloat16, 4)
    y, dx, dw = (torch.full_like(v, 7) for v in (x.contiguous(), x.contiguous(), w))
    n_rows = torch.tensor([n], dtype=torch.int32, device="cuda")
    work = torch.empty(tgm.tgm_norm_work_bytes(rows, D), dtype=torch.uint8, device="cuda")
    tgm.tgm_norm(x, w, y, EPS, n_rows=n_rows)
    tgm.tgm_norm_backward(x, w, dy, EPS, dx, dw, work, n_rows=n_rows)
    m = max(0, min(rows, n))
    assert (y[m:] == 7).all() and (dx[m:] == 7).all()
    rdx, rdw, sx, sw = norm_grads(x[:m], w, dy[:m], EPS)
    check_y(y[:m], None, norm(x[:m], w, EPS)[1])
    check("dx", dx[:m], rdx, rounded(rdx, dx.dtype) + CHAIN * U * sx)
    check("dw", dw, rdw, rounded(rdw, dw.dtype) + CHAIN * U * sw)


def test_no_rows(tgm):
    x, w = torch.empty(0, 8, device="cuda"), torch.ones(8, device="cuda")
    dw = torch.full((8,), 3.0, device="cuda")
    tgm.tgm_norm(x, w, torch.empty_like(x), EPS)
    tgm.tgm_norm_backward(x, w, x, EPS, torch.empty_like(x), dw, None)
    assert (dw == 0).all()


@pytest.mark.parametrize("D", [4, 100, 4099])
def test_infinities_nan_and_zeros(tgm, D):
    x, w = make(6, D, torch.float32), torch.ones(D, device="cuda")
    x[1, 2], x[2, 0], x[3, 3] = float("nan"), float("inf"), float("-inf")
    x[4] = 0
    y = torch.empty_like(x)
    tgm.tgm_norm(x, w, y, 0.0)   # a row of zeros: 0 * inf
    check_y(y, None, norm(x, w, 0.0)[1])
    q, scale = torch.empty(6, D, device="cuda", dtype=E4M3), torch.empty(6, device="cuda")
    tgm.tgm_norm(x, w, q, EPS, scale=scale)
    f = q.float()
    assert torch.isnan(f[1]).all()
    assert torch.isnan(f[2, 0]) and (f[2, 1:] == 0).all()
    assert torch.isnan(f[3, 3]) and torch.isnan(f[3]).sum() == 1
    assert (f[4] == 0).all() and float(scale[4]) == 2.0 ** -126
    fine = [0, 5]
    check_y(q[fine], scale[fine], norm(x[fine], w, EPS)[1])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D", WIDTHS)
def test_gradient(tgm, D, dtype):
    dt = TYPES[dtype]
    for rows, with_total in ((1, False), (37, True), (1500, True)):
        if rows * D > 3_000_000:
            continue
        t, dy = make(rows, D, dt, 1, pad=1), make(rows, D, dt, 2)
        w, dtotal = make(1, D, dt, 3)[0].contiguous(), make(rows, D, dt, 4, pad=2)
        dx, dw = torch.empty(rows, D + 1, device="cuda", dtype=dt)[:, :D], torch.empty_like(w)
        work = torch.empty(tgm.tgm_norm_work_bytes(rows, D), dtype=torch.uint8, device="cuda")
        args = dict(dtotal=dtotal if with_total else None)
        tgm.tgm_norm_backward(t, w, dy, EPS, dx, dw, work, **args)
        rdx, rdw, sx, sw = norm_grads(t, w, dy, EPS, **args)
        check("dx", dx, rdx, rounded(rdx, dt) + CHAIN * U * sx)
        check("dw", dw, rdw, rounded(rdw, dt) + CHAIN * U * sw)
        again = torch.empty_like(dw)
        tgm.tgm_norm_backward(t, w, dy, EPS, dx, again, work, **args)
        assert torch.equal(again, dw), "dw is not reproducible"
        none = torch.empty_like(dx)
        tgm.tgm_norm_backward(t, w, dy, EPS, none, None, None, **args)
        assert torch.equal(none, dx)


def test_against_differences(tgm):
    """dx and dw against central differences of the fp64 formula."""
    t, dy = make(3, 20, torch.float32, 5), make(3, 20, torch.float32, 6)
    w = make(1, 20, torch.float32, 7)[0].contiguous()
    dx, dw = torch.empty_like(t), torch.empty_like(w)
    work = torch.empty(tgm.tgm_norm_work_bytes(3, 20), dtype=torch.uint8, device="cuda")
    tgm.tgm_norm_backward(t, w, dy, EPS, dx, dw, work)
    T, W, G = cpu64(t, w, dy)
    f = lambda T, W: float((norm(T, W, EPS)[1] * G).sum())
    h = 1e-6
    for r, c in ((0, 0), (1, 7), (2, 19)):
        d = torch.zeros_like(T)
        d[r, c] = h
        n = (f(T + d, W) - f(T - d, W)) / (2 * h)
        # rounding of the differences: 2^-53 |f| / h; truncation: h^2; fp32 as above
        assert abs(float(dx[r, c]) - n) <= 1e-5 * (1 + abs(n))
        d = torch.zeros_like(W)
        d[c] = h
        n = (f(T, W + d) - f(T, W - d)) / (2 * h)
        assert abs(float(dw[c]) - n) <= 1e-5 * (1 + abs(n)) + CHAIN * U * float(
            norm_grads(t, w, dy, EPS)[3][c])

"""tgm_rotary against fp64: types, layouts, parts of the head, odd heads and strides, far
places and event times, in place, row counts on the device, and its gradient.

Tolerance: cos and sin are off by at most 4 U from their series and the reduced angle's two
roundings, and by the fp64 angle's own error (2^-52 of it, and once more in the reference);
two products, a sum and the amplitude round once each; then one rounding of the type."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

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


def reference(x, heads, omega, pos, layout, amplitude, inverse):
    """(y, tolerance before the type's rounding)"""
    rows, W = x.shape
    x = x.detach().cpu().to(F64).view(rows, heads, -1)
    h = omega.numel()
    at = (torch.arange(h), torch.arange(h) + h) if layout == "half" else \
        (2 * torch.arange(h), 2 * torch.arange(h) + 1)
    angle = (pos.cpu().to(F64)[:, None] * omega.cpu()[None])[:, None]
    c, s = torch.cos(angle) * amplitude, torch.sin(angle) * amplitude * (-1 if inverse else 1)
    a, b = x[..., at[0]], x[..., at[1]]
    y, tol = x.clone(), torch.zeros_like(x)
    y[..., at[0]], y[..., at[1]] = a * c - b * s, b * c + a * s
    e = amplitude * (a.abs() + b.abs()) * (8 * U + 2.0 ** -51 * angle.abs())
    tol[..., at[0]], tol[..., at[1]] = e, e
    return y.view(rows, W), tol.view(rows, W)


def go(tgm, rows, heads, d, rot, dtype, layout="half", pos=None, amplitude=1.0, inverse=False,
       pad=0, place="out", n_rows=None, omega=None):
    x = strided(randn(rows, rows, heads * d), dtype, pad)
    if omega is None:
        omega = 10000.0 ** (-2 * torch.arange(rot // 2, dtype=F64) / rot)
    omega = omega.cuda()
    where = torch.arange(rows) if pos is None else pos
    ref, tol = reference(x, heads, omega, where, layout, amplitude, inverse)
    y = x if place == "in" else strided(torch.full((rows, heads * d), 7.0), dtype, 2 * pad)
    before = y.clone()
    nr = None if n_rows is None else torch.tensor([n_rows], dtype=torch.int32, device="cuda")
    tgm.tgm_rotary(x, y, heads, omega, None if pos is None else pos.cuda(), layout=layout,
                   amplitude=amplitude, inverse=inverse, n_rows=nr)
    m = rows if n_rows is None else max(0, min(rows, n_rows))
    check("y", y[:m], ref[:m], (tol + rounded(ref.abs() + tol, dtype))[:m])
    assert torch.equal(y[m:], before[m:]), "rows past the count were written"
    if y._base is not None:
        assert (y._base[:, heads * d:].float() == 7).all(), "columns past the row were written"
    return y


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("heads,d,rot", [(1, 2, 2), (2, 50, 50), (3, 64, 32), (5, 17, 6),
                                         (40, 128, 128), (2, 1024, 1024), (7, 101, 26)])
def test_heads(tgm, heads, d, rot, dtype, layout):
    for rows, pad, place in ((1, 0, "out"), (19, 3, "out"), (130, 0, "in"), (5, 5, "in")):
        go(tgm, rows, heads, d, rot, TYPES[dtype], layout, pad=pad, place=place)


@pytest.mark.parametrize("kind", [torch.int32, torch.int64, F64])
def test_positions(tgm, kind):
    pos = (torch.rand(300, generator=torch.Generator().manual_seed(3), dtype=F64) * 1.7e9)
    pos[:4] = torch.tensor([0.0, 1.0, -5.0, 2.0 ** 31 - 1], dtype=F64)
    for layout in ("half", "interleaved"):
        go(tgm, 300, 2, 64, 64, torch.float32, layout, pos=pos.to(kind))
    go(tgm, 300, 2, 64, 64, torch.bfloat16, "half", pos=pos.to(kind), amplitude=1.25,
       inverse=True)


def test_places_past_32_bits(tgm):
    pos = torch.tensor([2 ** 33 + 1, -2 ** 35, 2 ** 31, 7])
    go(tgm, 4, 1, 8, 8, torch.float32, pos=pos)


@pytest.mark.parametrize("n", [-3, 0, 1, 64, 100, 1000])
def test_row_count_on_the_device(tgm, n):
    go(tgm, 100, 4, 32, 16, torch.bfloat16, n_rows=n)
    go(tgm, 100, 4, 32, 16, torch.float32, place="in", n_rows=n)


def test_no_rows(tgm):
    x = torch.empty(0, 64, device="cuda")
    tgm.tgm_rotary(x, x.clone(), 2, torch.ones(8, dtype=F64, device="cuda"))


def test_large_grid(tgm):
    # more row blocks than the grid has, and heads split over workgroups where there are few rows
    go(tgm, 300001, 1, 512, 512, torch.bfloat16)
    go(tgm, 2, 4096, 16, 8, torch.float32)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_gradient(tgm, layout):
    """<dy, rotary(x)> changes along v as <inverse(dy), v>; and there and back again."""
    rows, H, d, rot, A = 33, 3, 40, 24, 1.25
    omega = (100.0 ** (-torch.arange(rot // 2, dtype=F64) / 12)).cuda()
    pos = torch.arange(rows).cuda() * 3
    x, dy, v = (randn(k, rows, H * d).cuda() for k in (1, 2, 3))
    f = lambda t, **kw: (tgm.tgm_rotary(t, o := torch.empty_like(t), H, omega, pos, layout=layout,
                                        amplitude=A, **kw), o)[1]
    dx = f(dy, inverse=True)
    xr = x.cpu().to(F64).requires_grad_()
    ref, _ = reference(x, H, omega, pos, layout, A, False)
    # the operator is linear: differences are exact up to rounding
    left = ((f(x + v) - f(x)).double() * dy.double()).sum()
    right = (dx.double() * v.double()).sum()
    scale = float((dy.abs().double() * v.abs().double()).sum())
    assert abs(float(left - right)) <= 64 * U * scale
    back = f(f(x), inverse=True)
    want = x.cpu().to(F64).view(rows, H, d).clone()
    want[..., :rot] *= A * A
    tol = 64 * U * A * A * (want.abs() + want.abs().amax(-1, keepdim=True))
    check("there and back", back, want.view(rows, -1), tol.view(rows, -1))


def test_not_finite(tgm):
    """An angle without a value makes NaN of its pair alone, a NaN or infinity in x too."""
    x = torch.ones(3, 8, device="cuda")
    x[2, 1] = math.inf
    pos = torch.tensor([math.inf, math.nan, 1.0], dtype=F64, device="cuda")
    y = torch.empty_like(x)
    tgm.tgm_rotary(x, y, 1, torch.tensor([1.0, 0.5], dtype=F64, device="cuda"), pos)
    assert torch.isnan(y[:2, :4]).all() and (y[:2, 4:] == 1).all()
    assert torch.isinf(y[2, [1, 3]]).all() and torch.isfinite(y[2, [0, 2, 4, 5, 6, 7]]).all()


def test_slices_of_one_matrix(tgm):
    """q and k turned in place where tgm_linear left them, v untouched."""
    H, d, rows = 4, 32, 50
    qkv = randn(5, rows, 3 * H * d).cuda().to(torch.bfloat16)
    before, qk = qkv.clone(), qkv[:, :2 * H * d]
    omega = (100.0 ** (-torch.arange(16, dtype=F64) / 16)).cuda()
    ref, tol = reference(qk, 2 * H, omega, torch.arange(rows), "half", 1.0, False)
    tgm.tgm_rotary(qk, qk, 2 * H, omega)
    check("qk", qk, ref, tol + rounded(ref.abs() + tol, torch.bfloat16))
    assert torch.equal(qkv[:, 2 * H * d:], before[:, 2 * H * d:])


def test_captured(tgm):
    x = randn(9, 64, 256).cuda()
    omega = (100.0 ** (-torch.arange(32, dtype=F64) / 32)).cuda()
    pos = torch.arange(64, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        tgm.tgm_rotary(x, y, 4, omega, pos)
    for k in range(4):
        x.copy_(randn(20 + k, 64, 256))
        pos.add_(1000)
        g.replay()
        tgm.tgm_rotary(x, z, 4, omega, pos)
        torch.cuda.synchronize()
        assert torch.equal(y, z)


def test_more_rows_than_the_grid(tgm):
    """Every workgroup takes a row, and the first ones a second one, whose angles come in the
    place of the first one's: both ends against fp64."""
    rows, d, some = (1 << 20) + 100, 512, 300
    x = torch.randn(rows, d, device="cuda", generator=torch.Generator("cuda").manual_seed(5)).to(
        torch.bfloat16)
    omega = (10000.0 ** (-2 * torch.arange(d // 2, dtype=F64) / d)).cuda()
    for layout in ("half", "interleaved"):
        y = torch.full_like(x, 7.0)
        tgm.tgm_rotary(x, y, 1, omega, layout=layout)
        for at in (slice(0, some), slice((1 << 20) - some, (1 << 20) + 100)):
            ref, tol = reference(x[at], 1, omega, torch.arange(rows)[at], layout, 1.0, False)
            check("y", y[at], ref, tol + rounded(ref.abs() + tol, torch.bfloat16))

"""Products past the range of their types: 8-bit scales whose product leaves fp32, and
tgm_linear_backward in fp16 where dy times the activation's derivative leaves fp16's range
and the gradients do not: large and small dy, both in one call, infinities and row counts.
Against fp64; tolerances (opref): the rounding of dz, held times a power of two of at least
65,504 / (2.26 max|dy|), the sums' error in any order, one rounding of the result."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from opref import F64, STEP, U, act, act_grad_err, check, cut, half_step, rounded  # noqa: E402

F16 = torch.float16


@pytest.fixture(scope="module", autouse=True)
def tgm():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2402_15113_amd import tgm as t
    t.lib()
    return t


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def run(tgm, x, w, z, dy, name, n_rows=None):
    x, w, z, dy = (v.to(F16) for v in (x, w, z, dy))
    rows, (N, K) = x.shape[0], w.shape
    m = rows if n_rows is None else n_rows
    k = torch.empty(tgm.tgm_linear_work_bytes(rows, N, K, F16, act=name, backward=True),
                    dtype=torch.uint8, device="cuda").fill_(255)
    dx, dw = torch.full((rows, K), 7.0).to(F16).cuda(), torch.empty(N, K).to(F16).cuda()
    db = torch.empty(N).to(F16).cuda()
    nr = None if n_rows is None else torch.tensor([n_rows], dtype=torch.int32, device="cuda")
    tgm.tgm_linear_backward(x.cuda(), w.cuda(), dy.cuda(), k, act=name, z=z.cuda(), dx=dx, dw=dw,
                            db=db, n_rows=nr)
    x, w, z, dy = (v.to(F64) for v in (x, w, z, dy))
    x, z, dy = x[:m], z[:m], dy[:m]
    dz = dy * act(z, name)[1]
    off = dy.abs() * act_grad_err(z)
    finite = dy[torch.isfinite(dy)].abs()
    scale = 65504 / 2.26 / float(finite.max()) if finite.numel() and finite.max() > 0 else 1.0
    e = off + half_step(F16) * (dz.abs() + off) + STEP[F16] / 2 / scale
    for key, got, ref, err in (
            ("dx", dx[:m], dz @ w, e @ w.abs() + (N + 8) * U * ((dz.abs() + e) @ w.abs())),
            ("dw", dw, dz.t() @ x, e.t() @ x.abs() + (m + 8) * U * ((dz.abs() + e).t() @ x.abs())),
            ("db", db, dz.sum(0), (off + (m + 8) * U * (dz.abs() + off)).sum(0))):
        # past fp16's largest value a result is infinite
        ref = torch.where(ref.abs() >= 65520, float("inf") * ref.sign(), ref)
        check(key, got, ref, err + rounded(ref.abs() + err, F16))
    assert (dx[m:] == 7).all()
    return dx, dw, db


SIZES = [(40, 24, 16), (300, 260, 200), (9, 3, 5), (1, 1, 1), (700, 1030, 264)]


@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("size", SIZES)
def test_dz_past_the_largest_value(tgm, size, name):
    """|dy| near 65,504 where the derivative is above 1; x and W bring the sums back."""
    rows, N, K = size
    z = randn(1, rows, N) * 0.2 + (2.4 if name == "silu" else 1.4)
    dy = 60000 + 5000 * torch.rand(rows, N, generator=torch.Generator().manual_seed(2))
    dx, dw, _ = run(tgm, randn(3, rows, K) * 1e-3, randn(4, N, K) * 1e-3, z, dy, name)
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()


@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("size", SIZES)
def test_dz_below_the_smallest_value(tgm, size, name):
    """dz of 1e-7 and less, which fp16 has two bits of or none; W of some thousands."""
    rows, N, K = size
    z = randn(1, rows, N) * 0.5 - 4
    dy = randn(2, rows, N) * 2e-5
    run(tgm, randn(3, rows, K) * 1000, randn(4, N, K) * 20000, z, dy, name)


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_both_at_once(tgm, name):
    rows, N, K = 200, 96, 72
    dy = randn(2, rows, N) * torch.logspace(-6, 4, rows)[:, None]
    for n in (None, 0, 1, 130, 200):
        run(tgm, randn(3, rows, K), randn(4, N, K) / 10, randn(1, rows, N) * 2, dy, name, n_rows=n)


def test_zeros_and_infinities(tgm):
    rows, N, K = 70, 40, 24
    x, w, z = randn(3, rows, K), randn(4, N, K), randn(1, rows, N)
    run(tgm, x, w, z, torch.zeros(rows, N), "gelu")
    dy = randn(2, rows, N)
    want = run(tgm, x, w, z, dy, "silu")
    dy[5, 7] = float("inf")
    dx, dw, db = run(tgm, x, w, z, dy, "silu")
    rest = [r for r in range(rows) if r != 5]
    assert torch.equal(dx[rest], want[0][rest]) and not torch.isfinite(dx[5]).any()
    rest = [n for n in range(N) if n != 7]
    assert torch.equal(dw[rest], want[1][rest]) and torch.equal(db[rest], want[2][rest])
    dy[5, 7] = float("nan")
    assert torch.isnan(run(tgm, x, w, z, dy, "silu")[2][7])


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("rows,N,K", [(20, 24, 64), (700, 264, 128)])
def test_scales_whose_product_leaves_fp32(tgm, rows, N, K, out):
    """8-bit products with scales of 2^-126 and 2^-24, and of 2^100 each where the sum is
    zero: the results are ordinary fp32 values, their scales' product is not."""
    E4M3, ot = torch.float8_e4m3fn, dict(f32=torch.float32, bf16=torch.bfloat16)[out]
    x, w = (256 * randn(1, rows, K)).clamp(-448, 448).to(E4M3), torch.full((N, K), 448.0).to(E4M3)
    x.view(torch.uint8)[rows // 2:] = 0
    sx, sw = torch.full((rows,), 2.0 ** -126), torch.full((N,), 2.0 ** -24)
    sx[rows // 2:], sw[N // 2:] = 2.0 ** 100, 2.0 ** 100
    y = torch.empty(rows, N, device="cuda", dtype=ot)
    k = torch.empty(max(16, tgm.tgm_linear_work_bytes(rows, N, K, E4M3)), dtype=torch.uint8,
                    device="cuda")
    tgm.tgm_linear(x.cuda(), w.cuda(), y, k, scale_x=sx.cuda(), scale_w=sw.cuda())
    x, w = x.to(F64), w.to(F64)
    s = sx.to(F64)[:, None] * sw.to(F64)[None]
    ref, size = (x @ w.t()) * s, (x.abs() @ w.abs().t()) * s
    lost = 0 if ot == torch.float32 else cut(x, w) * s
    # the sum, and a product below 2^-126, which keeps no more than steps of 2^-149
    err = (K + 8) * U * size + lost + 2.0 ** -149
    check("y", y, ref, err + rounded(ref.abs() + err, ot))
    assert (y[rows // 2:] == 0).all() and (y[:rows // 2, :N // 2] != 0).any()


def test_captured_with_other_sizes_of_dy(tgm):
    """The scale of dz and the row count are the replay's, not the capture's."""
    rows, N, K = 150, 64, 40
    x, w, z, dy = (v.to(F16).cuda() for v in (randn(3, rows, K), randn(4, N, K) / 8,
                                              randn(1, rows, N), randn(2, rows, N)))
    nr = torch.tensor([rows], dtype=torch.int32, device="cuda")
    size = tgm.tgm_linear_work_bytes(rows, N, K, F16, act="gelu", backward=True)
    out, want = ([torch.zeros(rows, K), torch.zeros(N, K), torch.zeros(N)] for _ in range(2))
    out, want = ([v.to(F16).cuda() for v in o] for o in (out, want))
    works = [torch.empty(size, dtype=torch.uint8, device="cuda").fill_(255) for _ in range(2)]

    def call(o, k):
        tgm.tgm_linear_backward(x, w, dy, k, act="gelu", z=z, dx=o[0], dw=o[1], db=o[2], n_rows=nr)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call(out, works[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(out, works[0])
    for k, (scale, n) in enumerate(((1e-6, rows), (1.0, 77), (9000.0, rows), (0.0, 5), (1e-3, 0))):
        dy.copy_((randn(20 + k, rows, N) * scale).clamp(-60000, 60000))
        nr.fill_(n)
        for o in (out, want):
            o[0].zero_()
        call(want, works[1])
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(out, want):
            assert torch.equal(u, v), k

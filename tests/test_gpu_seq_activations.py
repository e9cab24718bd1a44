"""The activations of tgm_linear and their derivatives, value by value, against fp64, with
tolerances relative to each value: where they are small as well as where they are not.

A sum of one product with 1 gives z exactly. In units of U = 2^-24, relative:
  GELU in fp32, of a factor that does not cancel: t = 1 / (1 + c x) has 4 roundings (the
    reciprocal's one step is two of them), which the fitted function's slope of at most 2.3
    makes 10; its 9 coefficients, of alternating signs and twice the result in sum, 18; the
    fit 1; the exponential, with its argument's rounding made up for, 4; products 4: 40.
  SiLU in fp32: expf 2, 1 + e, the reciprocal after a step of Newton's 2, two products: 10.
  16-bit results: half a step of theirs and the rounded argument of the exponential (its
    size of at most z^2 or |z|, times 2), of the rest 60 (the fit's slope 3.4, its error 2).
The exponentials end at 2^-126; up to |z| times that much is lost there."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from opref import F64, TYPES, U, act, check, rounded  # noqa: E402

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def tgm():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2402_15113_amd import tgm as t
    t.lib()
    return t


def values(dtype, name):
    top = 14.0 if name == "gelu" else 80.0
    z = torch.cat([torch.linspace(-top, top, 4001), torch.linspace(-1, 1, 801),
                   torch.logspace(-6, 0, 97), -torch.logspace(-6, 0, 97)])
    return z.to(dtype)


def bound(z, name, dtype):
    """Relative error of a factor sigmoid or Phi before the output's rounding."""
    if dtype == torch.float32:
        return torch.full_like(z, (40 if name == "gelu" else 10) * U)
    return (2 * (z * z if name == "gelu" else z.abs()) + 60) * U


def work(tgm, rows, N, K, dtype, name, backward):
    n = tgm.tgm_linear_work_bytes(rows, N, K, dtype, act=name, backward=backward)
    return torch.empty(max(16, n), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_value(tgm, dtype, name):
    dt = TYPES[dtype]
    z = values(dt, name)[:, None]
    y = torch.empty(z.shape[0], 5, device="cuda", dtype=dt)
    one = torch.ones(5, 1, device="cuda", dtype=dt)
    tgm.tgm_linear(z.cuda(), one, y, work(tgm, z.shape[0], 5, 1, dt, name, False), act=name)
    z = z.to(F64)
    ref = act(z, name)[0].expand(-1, 5)
    tol = bound(z, name, dt) * ref.abs() + z.abs() * 2.0 ** -126
    check(name, y, ref, tol + rounded(ref.abs() + tol, dt))


@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_derivative(tgm, dtype, name):
    dt = TYPES[dtype]
    z = values(dt, name)[:, None]
    one, dy = torch.ones(1, 1, device="cuda", dtype=dt), torch.ones_like(z, device="cuda")
    dx = torch.empty_like(dy)
    tgm.tgm_linear_backward(z.cuda(), one, dy, work(tgm, z.shape[0], 1, 1, dt, name, True),
                            act=name, z=z.cuda(), dx=dx)
    z = z.to(F64)
    ref = act(z, name)[1]
    # the sum's two terms: p and z p (1 - p), or Phi and z phi
    p = torch.sigmoid(z) if name == "silu" else torch.erfc(-z / 2 ** 0.5) / 2
    other = z * p * torch.sigmoid(-z) if name == "silu" else \
        z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    size = p + other.abs()
    tol = 2 * bound(z, name, dt) * size + (1 + z.abs()) * 2.0 ** -126
    if name == "silu" and dt != torch.float32:   # 1 - p is formed from p
        tol = tol + 4 * U * z.abs() * p
    # dz in the type, and dx
    check(name, dx, ref, tol + 2 * rounded(ref.abs() + tol, dt))


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_8_bit_inputs_in_full(tgm, name):
    """z of 8-bit values and scales, results in fp32."""
    x = torch.arange(256, dtype=torch.uint8).view(E4M3)
    x = x[torch.isfinite(x.float())][:, None]
    sx = torch.full((x.shape[0],), 2.0 ** -5)
    y = torch.empty(x.shape[0], 4, device="cuda")
    one = torch.ones(4, 1, device="cuda").to(E4M3)
    tgm.tgm_linear(x.cuda(), one, y, work(tgm, x.shape[0], 4, 1, E4M3, name, False), act=name,
                   scale_x=sx.cuda(), scale_w=torch.ones(4, device="cuda"))
    z = x.to(F64) * 2.0 ** -5
    ref = act(z, name)[0].expand(-1, 4)
    tol = bound(z, name, torch.float32) * ref.abs() + z.abs() * 2.0 ** -126
    check(name, y, ref, tol + rounded(ref.abs() + tol, torch.float32))

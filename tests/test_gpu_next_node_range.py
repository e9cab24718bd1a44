"""Rotary positions, linear attention and cross entropy over rows, tables and states that lie more
than 2^32 elements apart: the same results as of rows side by side, whose offsets are small."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def tgm():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2402_15113_amd import tgm as t
    t.lib()
    yield t
    torch.cuda.empty_cache()


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).cuda()


def apart(t, ld):
    """The rows of t with a stride of ld; what lies between them is not written."""
    w = torch.empty((t.shape[0] - 1) * ld + t.shape[1], dtype=t.dtype, device="cuda")
    v = w.as_strided(t.shape, (ld, 1))
    v.copy_(t)
    return v


LD = (1 << 24) - 8      # 300 rows of it: 5.0e9 elements
ROWS = 300


def test_rotary(tgm):
    x = randn(1, ROWS, 256).to(BF16)
    omega = torch.linspace(0.1, 1.0, 32, dtype=torch.float64, device="cuda")
    y = torch.empty_like(x)
    tgm.tgm_rotary(x, y, 4, omega)
    far = apart(x, LD)
    tgm.tgm_rotary(far, far, 4, omega)
    assert torch.equal(far, y)


@pytest.mark.parametrize("reverse", [False, True])
def test_decay_attn(tgm, reverse):
    H, d, S = 2, 64, 3
    q, k, v, do = (randn(i, ROWS, H * d).to(BF16) for i in range(4))
    decay = torch.tensor([-0.01, -0.3], device="cuda")
    how = dict(scale=0.125, offsets=torch.tensor([0, 7, 250, ROWS - 3], device="cuda"),
               reverse=reverse)
    got = []
    for lay in (lambda t: t, lambda t: apart(t, LD)):
        work = [torch.empty(max(16, tgm.tgm_decay_attn_work_bytes(ROWS, S, H, d, d, BF16,
                                                                  backward=b)),
                            dtype=torch.uint8, device="cuda") for b in (False, True)]
        a = [lay(t) for t in (q, k, v)]
        o = lay(torch.zeros_like(q))
        tgm.tgm_decay_attn(*a, decay, o, S, work[0], **how)
        o = o.clone()
        g = [lay(torch.zeros_like(q)) for _ in range(3)]
        tgm.tgm_decay_attn_backward(*a, decay, lay(do), *g, S, work[1], **how)
        got.append([o] + [t.clone() for t in g])
        del a, g
        torch.cuda.empty_cache()
    for x, y in zip(*got):
        assert torch.equal(x, y)


def test_decay_step(tgm):
    """States past 2^32 elements of their table."""
    H, d, S, rows = 8, 128, 36000, 5
    state = torch.empty(S, H, d, d, device="cuda")
    q, k, v = (randn(i, rows, H * d).to(BF16) for i in range(3))
    decay = torch.linspace(-0.5, -0.01, H, device="cuda")
    slots = torch.tensor([35999, 3, 33000, 34000, 0], dtype=torch.int32, device="cuda")
    first = randn(5, rows, H, d, d)
    state[slots.long()] = first
    near, o, o2 = first.clone(), torch.empty_like(q), torch.empty_like(q)
    tgm.tgm_decay_attn_step(q, k, v, decay, state, o, slots=slots)
    tgm.tgm_decay_attn_step(q, k, v, decay, near, o2)
    assert torch.equal(o, o2) and torch.equal(state[slots.long()], near)


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_xent(tgm, dtype):
    """dW's rows, x's and W's, and a row without a target that is not finite."""
    N, K = 300, 64
    x, w = randn(1, ROWS, K).to(dtype), randn(2, N, K).to(dtype)
    x[17] = float("nan")
    t = torch.arange(ROWS, dtype=torch.int32, device="cuda") % N
    t[17] = -1
    dl, got = randn(3, ROWS), []
    for lay in (lambda m: m, lambda m: apart(m, LD)):
        a, b = lay(x), lay(w)
        loss, lse = torch.empty(ROWS, device="cuda"), torch.empty(ROWS, device="cuda")
        work = torch.empty(max(tgm.tgm_xent_work_bytes(ROWS, N, K, dtype, backward=b)
                               for b in (False, True)), dtype=torch.uint8, device="cuda")
        tgm.tgm_xent(a, b, t, loss, work, lse=lse)
        dx, dw = lay(torch.zeros_like(x)), lay(torch.zeros_like(w))
        tgm.tgm_xent_backward(a, b, t, lse, dl, work, dx=dx, dw=dw)
        got.append([loss, dx.clone(), dw.clone()])
        del a, b, dx, dw
        torch.cuda.empty_cache()
    for i, (p, q) in enumerate(zip(*got)):
        assert torch.isfinite(p).all() and torch.equal(p, q), i

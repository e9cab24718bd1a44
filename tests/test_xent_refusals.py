"""What the cross entropy's calls refuse, on the host and without a device: the addresses
below are never followed."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_2402_15113_amd import tgm  # noqa: E402

X = 4096   # stands for an address
BIG = 1 << 50


def desc(**kw):
    d = dict(rows=8, N=100, K=64, dtype=tgm.TGM_BF16, ld_x=0, ld_w=0, ld_dx=0, ld_dw=0)
    d.update(kw)
    return C.byref(tgm.XentDesc(*[d[n] for n, _ in tgm.XentDesc._fields_]))


BAD = [dict(rows=-1), dict(N=0), dict(K=0), dict(N=(1 << 20) + 1), dict(K=(1 << 20) + 1),
       dict(dtype=3), dict(dtype=-1), dict(ld_x=63), dict(ld_w=1 << 24), dict(ld_dx=-64),
       dict(ld_dw=1), dict(rows=(1 << 31) - 1, K=129), dict(rows=(1 << 31) - 1, N=129, K=64),
       dict(N=1 << 19, K=1 << 19)]


@pytest.mark.parametrize("bad", BAD)
def test_sizes(bad):
    L, E = tgm.lib(), tgm.TGM_EINVAL
    assert L.tgm_xent(desc(**bad), X, X, X, X, None, X, X, X, BIG, None) == E
    assert L.tgm_xent_backward(desc(**bad), X, X, X, X, X, X, None, X, X, X, X, BIG, None) == E


def test_pointers_and_work():
    L, E = tgm.lib(), tgm.TGM_EINVAL
    ok = [desc(), X, X, None, X, None, X, None, X, BIG, None]
    for k in (0, 1, 2, 4, 6, 8):   # neither loss nor lse: nothing is asked for
        assert L.tgm_xent(*[None if j == k else v for j, v in enumerate(ok)]) == E, k
    need = tgm.tgm_xent_work_bytes(8, 100, 64, torch.bfloat16)
    assert L.tgm_xent(*ok[:8], X + 8, BIG, None) == E
    assert L.tgm_xent(*ok[:8], X, need - 1, None) == tgm.TGM_ESIZE
    assert L.tgm_xent(desc(rows=0), None, X, None, None, None, None, None, None, 0, None) == 0
    back = [desc(), X, X, None, X, X, X, None, X, X, X, X, BIG, None]
    for k in (0, 1, 2, 4, 5, 6, 11):
        assert L.tgm_xent_backward(*[None if j == k else v for j, v in enumerate(back)]) == E, k
    need = tgm.tgm_xent_work_bytes(8, 100, 64, torch.bfloat16, backward=True)
    assert L.tgm_xent_backward(*back[:11], X + 4, BIG, None) == E
    assert L.tgm_xent_backward(*back[:11], X, need - 1, None) == tgm.TGM_ESIZE
    assert L.tgm_xent_backward(*back[:8], None, None, None, X, BIG, None) == tgm.TGM_OK


def test_work_bytes():
    for bad in ((-1, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1 << 21, 1), (1, 1, 1 << 21)):
        with pytest.raises(tgm.TgmError):
            tgm.tgm_xent_work_bytes(*bad, torch.float32)
    with pytest.raises(tgm.TgmError):
        tgm.tgm_xent_work_bytes(1, 1, 1, torch.float8_e4m3fn)
    with pytest.raises(ValueError):
        tgm.tgm_xent_work_bytes(1 << 31, 1, 1, torch.float32)
    assert tgm.lib().tgm_xent_work_bytes(1, 1, 1, 0, 0, None) == tgm.TGM_EINVAL
    # the gradient's space does not grow with the classes past a piece
    at = lambda N: tgm.tgm_xent_work_bytes(8192, N, 2048, torch.bfloat16, backward=True)
    assert at(1 << 20) <= 1.1 * at(1 << 17) < 1 << 30


def test_binding():
    x, w, t = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(4, dtype=torch.int32)
    loss = torch.zeros(4)
    with pytest.raises(ValueError, match="GPU"):
        tgm.tgm_xent(x, w, t, loss, None)
    with pytest.raises(ValueError, match="matrix"):
        tgm.tgm_xent(x, w[0], t, loss, None)
    with pytest.raises(ValueError, match="missing"):
        tgm._arg("target", None, torch.int32, (4,), 0)

"""What the sequence operators refuse, on the host and without a device: the
addresses below are never followed."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_2402_15113_amd import tgm  # noqa: E402

X = 4096   # stands for an address
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    import os

    from paper_2402_15113_amd import _build
    if not os.path.exists(tgm.LIB_PATH):
        _build.build(force=False)
    return tgm.lib()


def norm_desc(**kw):
    d = dict(rows=8, D=64, dtype=tgm.TGM_BF16, out_dtype=tgm.TGM_BF16, eps=1e-5, ld_x=0,
             ld_res=0, ld_total=0, ld_y=0)
    d.update(kw)
    return C.byref(tgm.NormDesc(*[d[n] for n, _ in tgm.NormDesc._fields_]))


BAD_NORM = [dict(rows=-1), dict(D=0), dict(D=32769), dict(dtype=3), dict(dtype=7),
            dict(eps=-1.0), dict(eps=float("nan")), dict(ld_x=63), dict(ld_y=1 << 24),
            dict(ld_res=-64), dict(ld_total=5)]


@pytest.mark.parametrize("bad", BAD_NORM + [dict(out_dtype=0), dict(out_dtype=9)])
def test_norm_sizes(L, bad):
    assert L.tgm_norm(norm_desc(**bad), X, X, X, None, X, X, None, None) == tgm.TGM_EINVAL


def test_norm_pointers(L):
    E = tgm.TGM_EINVAL
    assert L.tgm_norm(None, X, X, X, None, X, X, None, None) == E
    assert L.tgm_norm(norm_desc(), None, X, X, None, X, X, None, None) == E
    assert L.tgm_norm(norm_desc(), X, X, None, None, X, X, None, None) == E
    assert L.tgm_norm(norm_desc(), X, X, X, None, X, None, None, None) == E
    # a scale goes with 8 bits, and with nothing else
    assert L.tgm_norm(norm_desc(), X, X, X, None, X, X, X, None) == E
    assert L.tgm_norm(norm_desc(out_dtype=3), X, X, X, None, X, X, None, None) == E


@pytest.mark.parametrize("bad", BAD_NORM)
def test_norm_backward_sizes(L, bad):
    assert L.tgm_norm_backward(norm_desc(**bad), X, X, X, X, None, X, X, X, BIG,
                               None) == tgm.TGM_EINVAL


def test_norm_backward_work(L):
    call = lambda work, n: L.tgm_norm_backward(norm_desc(), X, X, X, X, None, X, X, work, n, None)
    need = tgm.tgm_norm_work_bytes(8, 64)
    assert need == 8 * 64 * 4
    assert call(None, need) == tgm.TGM_EINVAL
    assert call(X + 4, need) == tgm.TGM_EINVAL
    assert call(X, need - 1) == tgm.TGM_ESIZE
    assert L.tgm_norm_work_bytes(8, 64, None) == tgm.TGM_EINVAL
    assert L.tgm_norm_backward(norm_desc(), X, X, X, X, None, None, X, X, BIG,
                               None) == tgm.TGM_EINVAL


def test_binding_checks_tensors():
    x, w = torch.zeros(4, 8), torch.ones(8)
    with pytest.raises(ValueError, match="GPU"):
        tgm.tgm_norm(x, w, torch.empty_like(x), 1e-5)
    with pytest.raises(ValueError, match="type"):
        tgm._arg("w", w.half(), torch.float32, (8,), x.device)
    with pytest.raises(ValueError, match="no operator takes"):
        tgm.dtype_code(torch.int8)


def test_binding_checks_strides():
    m = tgm._arg
    dev = torch.device("cpu")
    for bad in (torch.zeros(8, 4).t(), torch.zeros(1, 8).expand(4, 8)):
        with pytest.raises(ValueError):
            m("x", bad, torch.float32, (4, 8), dev)
    with pytest.raises(ValueError, match="shape"):
        m("x", torch.zeros(4, 9), torch.float32, (4, 8), dev)

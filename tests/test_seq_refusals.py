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


def linear_desc(**kw):
    d = dict(rows=8, N=32, K=64, dtype=tgm.TGM_BF16, out_dtype=tgm.TGM_BF16, act=0, ld_x=0,
             ld_w=0, ld_res=0, ld_z=0, ld_y=0, ld_dx=0, ld_dw=0)
    d.update(kw)
    return C.byref(tgm.LinearDesc(*[d[n] for n, _ in tgm.LinearDesc._fields_]))


BAD_LINEAR = [dict(rows=-1), dict(N=0), dict(K=0), dict(N=(1 << 20) + 1), dict(K=(1 << 20) + 1),
              dict(act=4), dict(act=-1), dict(dtype=0), dict(out_dtype=2), dict(dtype=5),
              dict(ld_x=63), dict(ld_w=-64), dict(ld_y=31), dict(ld_z=1 << 24), dict(ld_res=1),
              dict(rows=(1 << 31) - 1, K=129), dict(N=1 << 19, K=1 << 19)]


@pytest.mark.parametrize("bad", BAD_LINEAR + [dict(ld_dx=63), dict(ld_dw=1)])
def test_linear_sizes(L, bad):
    E = tgm.TGM_EINVAL
    assert L.tgm_linear(linear_desc(**bad), X, None, X, None, X, X, None, X, X, X, BIG, None) == E
    assert L.tgm_linear_backward(linear_desc(**bad), X, X, X, X, None, X, X, X, X, BIG, None) == E


def test_linear_pointers_and_scales(L):
    E = tgm.TGM_EINVAL
    ok = [linear_desc(), X, None, X, None, None, None, None, None, X, X, BIG, None]
    for k in (0, 1, 3, 9):
        assert L.tgm_linear(*[None if j == k else v for j, v in enumerate(ok)]) == E, k
    # scales go with 8 bits, and with nothing else
    for k in (2, 4):
        assert L.tgm_linear(*[X if j == k else v for j, v in enumerate(ok)]) == E, k
    ok[0], ok[2], ok[4] = linear_desc(dtype=tgm.TGM_E4M3), X, X
    for k in (1, 2, 3, 4, 9):
        assert L.tgm_linear(*[None if j == k else v for j, v in enumerate(ok)]) == E, k
    ok[0] = linear_desc(dtype=tgm.TGM_E4M3, out_dtype=tgm.TGM_E4M3)
    assert L.tgm_linear(*ok) == E


def test_linear_backward_pointers_and_work(L):
    E = tgm.TGM_EINVAL
    ok = [linear_desc(act=2), X, X, X, X, None, X, X, X, X, BIG, None]
    for k in (0, 1, 2, 3, 4, 9):
        assert L.tgm_linear_backward(*[None if j == k else v for j, v in enumerate(ok)]) == E, k
    assert L.tgm_linear_backward(*ok[:9], X + 2, BIG, None) == E
    need = tgm.tgm_linear_work_bytes(8, 32, 64, torch.bfloat16, act="silu", backward=True)
    assert need >= 8 * 32 * 2
    assert L.tgm_linear_backward(*ok[:10], need - 1, None) == tgm.TGM_ESIZE
    ok[0] = linear_desc(dtype=tgm.TGM_E4M3, out_dtype=tgm.TGM_E4M3)
    assert L.tgm_linear_backward(*ok) == E


def test_linear_work_bytes():
    for bad in ((-1, 1, 1, 0, 0, 0), (1, 0, 1, 0, 0, 0), (1, 1, 0, 0, 0, 0), (1, 1, 1, 4, 0, 0),
                (1, 1, 1, 0, 4, 0), (1, 1, 1, 3, 0, 1)):
        with pytest.raises(tgm.TgmError):
            tgm._bytes("tgm_linear_work_bytes", *bad)
    assert tgm.lib().tgm_linear_work_bytes(1, 1, 1, 0, 0, 0, None) == tgm.TGM_EINVAL
    with pytest.raises(ValueError, match="act"):
        tgm.tgm_linear_work_bytes(1, 1, 1, torch.float32, act="tanh")


def scan_desc(**kw):
    d = dict(rows=96, S=3, D=64, dtype=tgm.TGM_BF16, reverse=0, ld_g=0, ld_x=0, ld_y=0, ld_dg=0,
             ld_dx=0)
    d.update(kw)
    return C.byref(tgm.ScanDesc(*[d[n] for n, _ in tgm.ScanDesc._fields_]))


BAD_SCAN = [dict(rows=-1), dict(rows=1 << 31), dict(S=-1), dict(D=0), dict(D=65537),
            dict(dtype=3), dict(dtype=-1), dict(ld_g=63), dict(ld_x=-64), dict(ld_y=1 << 24)]


@pytest.mark.parametrize("off", [None, X])
@pytest.mark.parametrize("bad", BAD_SCAN + [dict(ld_dg=1), dict(ld_dx=-1)])
def test_scan_sizes(L, bad, off):
    E = tgm.TGM_EINVAL
    assert L.tgm_scan(scan_desc(**bad), X, X, off, X, X, X, X, X, X, BIG, None) == E
    assert L.tgm_scan_backward(scan_desc(**bad), X, X, off, X, X, X, X, X, X, X, X, X, BIG,
                               None) == E


def test_scan_pointers_and_work(L):
    E = tgm.TGM_EINVAL
    ok = [scan_desc(), X, X, X, None, None, X, None, None, X, BIG, None]
    for k in (0, 1, 2, 6, 9):
        assert L.tgm_scan(*[None if j == k else v for j, v in enumerate(ok)]) == E, k
    assert L.tgm_scan(*ok[:9], X + 8, BIG, None) == E
    assert L.tgm_scan(*ok[:9], X, 3 * 64 * 12 - 1, None) == tgm.TGM_ESIZE
    back = [scan_desc(), X, X, X, None, None, X, X, None, X, X, None, X, BIG, None]
    for k in (0, 1, 2, 6, 7, 9, 10, 12):
        assert L.tgm_scan_backward(*[None if j == k else v for j, v in enumerate(back)]) == E, k
    assert L.tgm_scan_backward(*back[:12], X, 10, None) == tgm.TGM_ESIZE
    # padded sequences divide the rows
    for bad in (dict(rows=97), dict(S=0)):
        assert L.tgm_scan(scan_desc(**bad), X, X, None, None, None, X, None, None, X, BIG,
                          None) == E


def test_scan_sizes_of_buffers():
    assert tgm.tgm_scan_carry_rows(100, 7, True) == 4
    assert tgm.tgm_scan_carry_rows(0, 0, True) == 0
    assert tgm.tgm_scan_carry_rows(200, 2, False) == 8     # 100 rows: 4 tiles each
    assert tgm.tgm_scan_carry_rows(70, 7, False) == 3      # 10 rows: 3 sequences a tile
    for bad in ((-1, 1, True), (10, 3, False), (1 << 31, 1, True), (5, 0, False), (5, -1, True)):
        with pytest.raises(tgm.TgmError):
            tgm.tgm_scan_carry_rows(*bad)
    with pytest.raises(tgm.TgmError):
        tgm.tgm_scan_work_bytes(10, 0, 1)
    assert tgm.lib().tgm_scan_carry_rows(5, 1, 1, None) == tgm.TGM_EINVAL
    assert tgm.lib().tgm_scan_work_bytes(5, 1, 1, None) == tgm.TGM_EINVAL


@pytest.mark.parametrize("bad", BAD_SCAN)
def test_scan_step_sizes(L, bad):
    assert L.tgm_scan_step(scan_desc(**bad), X, X, X, X, X, X, None) == tgm.TGM_EINVAL


def test_scan_step_pointers(L):
    ok = [scan_desc(), X, X, None, None, X, X, None]
    for k in (0, 1, 2, 5):
        assert L.tgm_scan_step(*[None if j == k else v
                                 for j, v in enumerate(ok)]) == tgm.TGM_EINVAL, k


def test_binding_checks_tensors():
    x, w = torch.zeros(4, 8), torch.ones(8)
    with pytest.raises(ValueError, match="GPU"):
        tgm.tgm_norm(x, w, torch.empty_like(x), 1e-5)
    with pytest.raises(ValueError, match="type"):
        tgm._arg("w", w.half(), torch.float32, (8,), 0)
    with pytest.raises(ValueError, match="no operator takes"):
        tgm.dtype_code(torch.int8)


def test_binding_checks_strides():
    m = lambda t: tgm._arg("x", t, torch.float32, (4, 8), 0)
    with pytest.raises(ValueError, match="contiguous"):
        m(torch.zeros(8, 4).t())
    with pytest.raises(ValueError, match="overlap"):
        m(torch.zeros(1, 8).expand(4, 8))
    with pytest.raises(ValueError, match="shape"):
        m(torch.zeros(4, 9))
    with pytest.raises(ValueError, match="missing"):
        m(None)
    with pytest.raises(ValueError, match="GPU"):
        m(torch.zeros(4, 8))

"""The largest sizes that the sequence operators take, on the host and without a
device: a work space that is too small ends every call before it launches."""
import pytest

torch = pytest.importorskip("torch")

from paper_2402_15113_amd import tgm  # noqa: E402
from test_seq_refusals import L, X, scan_desc  # noqa: E402, F401


def scan_calls(L, packed, **d):
    d = scan_desc(**d)
    off = X if packed else None
    return (L.tgm_scan(d, X, X, off, None, None, X, None, X, X, 1, None),
            L.tgm_scan_backward(d, X, X, off, None, None, X, X, None, X, X, None, X, 1, None))


@pytest.mark.parametrize("rows,S,D,packed", [
    (1 << 30, 1, 1, True), (1 << 30, 1, 64, True), (1 << 29, 9, 128, True),
    (33 * 16_000_000, 16_000_000, 64, False), (1 << 20, 1, 65536, True)])
def test_scan_takes_forward_and_back(L, rows, S, D, packed):
    T = tgm.tgm_scan_carry_rows(rows, S, packed)
    assert T * -(-D // 64) <= 2 ** 26 - 2 ** 15
    for dtype in (tgm.TGM_F32, tgm.TGM_BF16, tgm.TGM_F16):
        assert scan_calls(L, packed, rows=rows, S=S, D=D, dtype=dtype) == (tgm.TGM_ESIZE,) * 2
    assert tgm.tgm_scan_work_bytes(rows, D, S) > 0


@pytest.mark.parametrize("rows,S,D,packed", [
    (1 << 30, 1, 257, True), (1 << 30, 1, 65536, True), (33 * 32_000_000, 32_000_000, 129, False)])
def test_scan_refuses_forward_and_back(L, rows, S, D, packed):
    for dtype in (tgm.TGM_F32, tgm.TGM_BF16, tgm.TGM_F16):
        assert scan_calls(L, packed, rows=rows, S=S, D=D, dtype=dtype) == (tgm.TGM_EINVAL,) * 2
    if packed:
        with pytest.raises(tgm.TgmError):
            tgm.tgm_scan_work_bytes(rows, D, S)


@pytest.mark.parametrize("wide", [1 << 31, (1 << 32) + 3, -(1 << 32) + 3])
def test_binding_cuts_no_size_short(wide):
    """3 plus a multiple of 2^32 is not 3."""
    f32 = torch.float32
    for call in (lambda: tgm.tgm_norm_work_bytes(wide, 64), lambda: tgm.tgm_norm_work_bytes(3, wide),
                 lambda: tgm.tgm_linear_work_bytes(wide, 3, 3, f32),
                 lambda: tgm.tgm_linear_work_bytes(3, wide, 3, f32, backward=True),
                 lambda: tgm.tgm_linear_work_bytes(3, 3, wide, f32),
                 lambda: tgm.tgm_scan_work_bytes(96, 64, wide),
                 lambda: tgm.tgm_scan_work_bytes(96, wide, 3),
                 lambda: tgm.tgm_scan_carry_rows(96, wide, False)):
        with pytest.raises(ValueError, match="out of range"):
            call()
    g = torch.zeros(96, 64)
    for call in (lambda: tgm.tgm_scan(g, g, g, wide, None),
                 lambda: tgm.tgm_scan_backward(g, g, g, None, g, g, wide, None)):
        with pytest.raises(ValueError, match="S is"):
            call()

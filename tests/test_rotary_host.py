"""Frequencies of tgm_rotary from their formulas, and what the rotary calls refuse, on the
host and without a device: the addresses below are never followed."""
import ctypes as C
import math

import pytest

np = pytest.importorskip("numpy")
torch = pytest.importorskip("torch")

from paper_2402_15113_amd import tgm  # noqa: E402

X = 4096   # stands for an address


def desc(**kw):
    d = dict(rows=8, H=4, d=64, rot=32, dtype=tgm.TGM_BF16, pos_type=0, layout=0, inverse=0,
             amplitude=1.0, ld_x=0, ld_y=0)
    d.update(kw)
    return C.byref(tgm.RotaryDesc(*[d[n] for n, _ in tgm.RotaryDesc._fields_]))


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(H=0), dict(H=4097), dict(d=1, rot=0), dict(d=1025), dict(rot=0),
    dict(rot=31), dict(rot=66), dict(rot=-2), dict(dtype=3), dict(dtype=-1), dict(pos_type=3),
    dict(pos_type=-1), dict(layout=2), dict(layout=-1), dict(ld_x=255), dict(ld_y=1 << 24),
    dict(ld_y=-256)])
def test_sizes(bad):
    assert tgm.lib().tgm_rotary(desc(**bad), X, X, X, None, X, None) == tgm.TGM_EINVAL


def test_pointers_and_strides_in_place():
    L, E = tgm.lib(), tgm.TGM_EINVAL
    ok = [desc(), X, X, X, None, X, None]
    for k in (0, 1, 2, 5):
        assert L.tgm_rotary(*[None if j == k else v for j, v in enumerate(ok)]) == E, k
    assert L.tgm_rotary(desc(ld_x=256, ld_y=300), X, X, X, None, X, None) == E
    # nothing to do, and nothing asked for
    assert L.tgm_rotary(desc(rows=0), None, X, None, None, None, None) == tgm.TGM_OK


def test_binding():
    x, w = torch.zeros(4, 24), torch.ones(4, dtype=torch.float64)
    call = lambda **kw: tgm.tgm_rotary(**{**dict(x=x, y=x, heads=3, omega=w), **kw})
    with pytest.raises(ValueError, match="GPU"):
        call()
    for kw, words in ((dict(heads=5), "heads"), (dict(heads=0), "heads"),
                      (dict(omega=torch.ones(5, dtype=torch.float64)), "pairs"),
                      (dict(omega=None), "vector"), (dict(x=x[0]), "matrix"),
                      (dict(pos=torch.zeros(4)), "type")):
        with pytest.raises(ValueError, match=words):
            call(**kw)


@pytest.mark.parametrize("rot", [2, 4, 50, 128, 1024])
def test_frequencies(rot):
    j = np.arange(rot // 2)
    plain = 10000.0 ** (-2 * j / rot)
    w, a = tgm.tgm_rotary_frequencies(rot)
    assert a == 1 and np.allclose(w, plain, rtol=1e-14, atol=0)
    w, a = tgm.tgm_rotary_frequencies(rot, "linear", base=500.0, factor=4.0)
    assert a == 1 and np.allclose(w, 500.0 ** (-2 * j / rot) / 4, rtol=1e-14, atol=0)
    w, a = tgm.tgm_rotary_frequencies(rot, "base", factor=8.0)
    assert a == 1 and w[0] == 1
    if rot > 2:   # the lowest one is divided by the factor
        assert math.isclose(w[-1], plain[-1] / 8, rel_tol=1e-12)
    w, a = tgm.tgm_rotary_frequencies(rot, "parts", factor=8.0, original=4096.0)
    assert math.isclose(a, 0.1 * math.log(8) + 1, rel_tol=1e-6)
    turns = 4096 * plain / (2 * math.pi)
    often, seldom = turns >= 32, turns <= 1
    assert np.allclose(w[often], plain[often], rtol=1e-14, atol=0)
    assert np.allclose(w[seldom], plain[seldom] / 8, rtol=1e-14, atol=0)
    keep = (turns - 1) / 31
    mid = plain * keep + plain / 8 * (1 - keep)
    assert np.allclose(w[~often & ~seldom], mid[~often & ~seldom], rtol=1e-13, atol=0)


@pytest.mark.parametrize("rot", [2, 4, 64, 1024])
@pytest.mark.parametrize("base,factor", [(1e300, 1e10), (10000.0, 1e300), (1e-300, 1e308)])
def test_base_past_the_numbers(rot, base, factor):
    """base factor^(rot / (rot - 2)) may be more than fp64 holds where its roots are not."""
    w, a = tgm.tgm_rotary_frequencies(rot, "base", base=base, factor=factor)
    j = np.arange(rot // 2)
    grow = math.log(factor) / (rot - 2) if rot > 2 else 0.0
    # (exponents of some hundred: their rounding is that many steps of the result)
    want = -2 * j * (math.log(base) / rot + grow)
    assert a == 1 and w[0] == 1 and (w > 0).all()
    assert np.allclose(np.log(w), want, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("bad", [
    dict(rot=3), dict(rot=0), dict(rot=-2), dict(rot=1026), dict(base=0.0), dict(base=-1.0),
    dict(base=math.inf), dict(base=math.nan), dict(scaling="linear", factor=0.5),
    dict(scaling="base", factor=math.nan), dict(scaling="parts", factor=2.0),
    dict(scaling="parts", factor=2.0, original=100.0, often=1.0, seldom=1.0),
    dict(scaling="parts", factor=2.0, original=100.0, seldom=-1.0)])
def test_frequencies_refused(bad):
    with pytest.raises(tgm.TgmError):
        tgm.tgm_rotary_frequencies(**{**dict(rot=64), **bad})


def test_frequencies_words():
    with pytest.raises(ValueError, match="scaling"):
        tgm.tgm_rotary_frequencies(64, "other")
    with pytest.raises(ValueError, match="range"):
        tgm.tgm_rotary_frequencies(1 << 32)
    out, a = (C.c_double * 4)(), C.c_float()
    f = tgm.lib().tgm_rotary_frequencies
    assert f(8, 0, 1e4, 1.0, 0.0, 32.0, 1.0, None, C.byref(a)) == tgm.TGM_EINVAL
    assert f(8, 0, 1e4, 1.0, 0.0, 32.0, 1.0, out, None) == tgm.TGM_EINVAL
    assert f(8, 4, 1e4, 1.0, 0.0, 32.0, 1.0, out, C.byref(a)) == tgm.TGM_EINVAL

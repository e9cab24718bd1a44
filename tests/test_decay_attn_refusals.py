"""What the linear attention's calls refuse, on the host and without a device: the addresses
below are never followed."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_2402_15113_amd import tgm  # noqa: E402

X = 4096   # stands for an address
BIG = 1 << 50


def desc(**kw):
    d = dict(rows=96, S=3, H=4, H_kv=2, d_k=32, d_v=16, dtype=tgm.TGM_BF16, reverse=0, scale=1.0,
             ld_q=0, ld_k=0, ld_v=0, ld_o=0, ld_dq=0, ld_dk=0, ld_dv=0)
    d.update(kw)
    return C.byref(tgm.DecayAttnDesc(*[d[n] for n, _ in tgm.DecayAttnDesc._fields_]))


BAD = [dict(rows=-1), dict(rows=(1 << 30) + 1), dict(S=-1), dict(H=0), dict(H=4097, H_kv=1),
       dict(H_kv=0), dict(H_kv=3), dict(H_kv=8), dict(d_k=0), dict(d_k=129), dict(d_v=0),
       dict(d_v=129), dict(dtype=3), dict(dtype=-1), dict(ld_q=127), dict(ld_k=63),
       dict(ld_v=-32), dict(ld_o=1 << 24)]


@pytest.mark.parametrize("off", [None, X])
@pytest.mark.parametrize("bad", BAD + [dict(ld_dq=1), dict(ld_dk=63), dict(ld_dv=-1)])
def test_sizes(bad, off):
    L, E = tgm.lib(), tgm.TGM_EINVAL
    assert L.tgm_decay_attn(desc(**bad), X, X, X, X, off, X, X, X, X, X, BIG, None) == E
    assert L.tgm_decay_attn_backward(desc(**bad), X, X, X, X, off, X, X, X, X, X, X, X, X, X, BIG,
                                     None) == E


@pytest.mark.parametrize("bad", BAD)
def test_step_sizes(bad):
    assert tgm.lib().tgm_decay_attn_step(desc(**bad), X, X, X, X, X, X, X, X,
                                         None) == tgm.TGM_EINVAL


def test_padded_rows_are_divided():
    L, E = tgm.lib(), tgm.TGM_EINVAL
    for bad in (dict(rows=97), dict(S=0)):
        assert L.tgm_decay_attn(desc(**bad), X, X, X, X, None, X, X, X, X, X, BIG, None) == E
        assert L.tgm_decay_attn_backward(desc(**bad), X, X, X, X, None, X, X, X, X, X, X, X, X, X,
                                         BIG, None) == E


def test_pointers_and_work():
    L, E = tgm.lib(), tgm.TGM_EINVAL
    ok = [desc(), X, X, X, X, X, None, None, X, None, X, BIG, None]
    for k in (0, 1, 2, 3, 4, 8):
        assert L.tgm_decay_attn(*[None if j == k else v for j, v in enumerate(ok)]) == E, k
    back = [desc(), X, X, X, X, X, None, None, X, None, X, X, X, None, X, BIG, None]
    for k in (0, 1, 2, 3, 4, 8):
        assert L.tgm_decay_attn_backward(*[None if j == k else v
                                           for j, v in enumerate(back)]) == E, k
    for backward, fn, args, at in ((False, L.tgm_decay_attn, ok, 10),
                                   (True, L.tgm_decay_attn_backward, back, 14)):
        need = tgm.tgm_decay_attn_work_bytes(96, 3, 4, 32, 16, torch.bfloat16, kv_heads=2,
                                             backward=backward)
        if need:
            swap = lambda p, n: args[:at] + [p, n] + args[at + 2:]
            assert fn(*swap(None, BIG)) == E
            assert fn(*swap(X + 4, BIG)) == E
            assert fn(*swap(X, need - 1)) == tgm.TGM_ESIZE
    step = [desc(), X, X, X, X, None, None, X, None, None]
    for k in (0, 1, 2, 3, 4, 7):
        assert L.tgm_decay_attn_step(*[None if j == k else v for j, v in enumerate(step)]) == E, k
    assert L.tgm_decay_attn_step(desc(rows=0), None, None, None, X, None, None, None, None,
                                 None) == tgm.TGM_OK


def test_states_are_two_tables():
    """A sequence's last state may be written before another workgroup has read its first."""
    L, E = tgm.lib(), tgm.TGM_EINVAL
    other = 2 * X
    work = lambda b: tgm.tgm_decay_attn_work_bytes(96, 3, 4, 32, 16, torch.bfloat16, kv_heads=2,
                                                   backward=b)
    for last, want in ((X, E), (other, tgm.TGM_ESIZE)):
        assert work(False) and L.tgm_decay_attn(desc(), X, X, X, X, X, None, X, X, last, X,
                                                work(False) - 1, None) == want
        assert L.tgm_decay_attn_backward(desc(), X, X, X, X, X, None, X, X, X, X, X, X, last, X,
                                         work(True) - 1, None) == want


def test_work_bytes():
    f = tgm.tgm_decay_attn_work_bytes
    for bad in ((-1, 1, 1, 1, 1), (1, -1, 1, 1, 1), (1, 1, 0, 1, 1), (1, 1, 1, 0, 1),
                (1, 1, 1, 1, 129)):
        with pytest.raises(tgm.TgmError):
            f(*bad, torch.float32)
    with pytest.raises(tgm.TgmError):
        f(1, 1, 4, 8, 8, torch.float32, kv_heads=3)
    with pytest.raises(ValueError):
        f(1, 1 << 31, 4, 8, 8, torch.float32)
    assert tgm.lib().tgm_decay_attn_work_bytes(1, 1, 1, 1, 1, 1, 0, 0, None) == tgm.TGM_EINVAL


def test_binding():
    q, k, v, g = torch.zeros(6, 8), torch.zeros(6, 4), torch.zeros(6, 6), torch.zeros(4)
    o = torch.zeros(6, 12)
    call = lambda **kw: tgm.tgm_decay_attn(**{**dict(q=q, k=k, v=v, decay=g, o=o, S=2, work=None,
                                                     kv_heads=2), **kw})
    with pytest.raises(ValueError, match="GPU"):
        call()
    for kw, words in ((dict(kv_heads=3), "share"), (dict(decay=g[None]), "vector"),
                      (dict(decay=None), "vector"), (dict(q=torch.zeros(6, 9)), "heads"),
                      (dict(k=torch.zeros(6, 6)), "heads"), (dict(v=v[0]), "matrix")):
        with pytest.raises(ValueError, match=words):
            call(**kw)
    with pytest.raises(ValueError, match="state"):
        tgm._state("state", torch.zeros(2, 4, 2, 2), (2, 4, 2, 3), 0)
    with pytest.raises(ValueError, match="S is"):
        tgm._sequences(-1, None, None, 0)


@pytest.mark.parametrize("kw", [dict(rows=200), dict(rows=200, H=2), dict(rows=0),
                                dict(rows=1 << 20, H_kv=4)])
def test_no_sequences(kw):
    """Packed rows of no sequence at all: nothing to do, and nothing that is launched."""
    L, kw = tgm.lib(), dict(dict(S=0), **kw)
    assert L.tgm_decay_attn(desc(**kw), X, X, X, X, X, None, X, X, None, X, BIG,
                            None) == tgm.TGM_OK
    assert L.tgm_decay_attn_backward(desc(**kw), X, X, X, X, X, None, X, X, X, X, X, X, None, X,
                                     BIG, None) == tgm.TGM_OK
    # what the calls ask for is checked all the same
    if kw["rows"]:
        assert L.tgm_decay_attn(desc(**kw), None, X, X, X, X, None, X, X, None, X, BIG,
                                None) == tgm.TGM_EINVAL
        assert L.tgm_decay_attn_backward(desc(**kw), X, X, X, X, X, None, X, None, X, X, X, X,
                                         None, X, BIG, None) == tgm.TGM_EINVAL

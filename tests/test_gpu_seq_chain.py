"""The scan's chain of workgroups: more channels than runners fit the chip.

Tolerances as in test_gpu_seq_scan."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from opref import TYPES  # noqa: E402
from test_gpu_seq_scan import Batch  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def tgm():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2402_15113_amd import tgm as t
    t.lib()
    return t


@pytest.mark.parametrize("dtype,D", [("f32", 700), ("bf16", 1101), ("f32", 33000),
                                     ("f16", 65536)])
def test_wide_rows(tgm, dtype, D):
    """Up to 32 slices of channel blocks, each with chains of two or three workgroups
    forward and five back, in both directions."""
    for reverse in (False, True):
        Batch(tgm, D, TYPES[dtype], lengths=[330, 0, 200], extra=2, reverse=reverse).run()


def test_wide_rows_on_two_streams(tgm):
    """Two such calls at once, each with its own work space."""
    D = 33000
    batches = [Batch(tgm, D, torch.float32, lengths=[330, 0, 200], seed=s) for s in (0, 9)]
    want = []
    for b in batches:
        b.forward()
        b.backward()
        want.append([v.clone() for v in (b.y, b.h_last, b.dg, b.dx, b.dh0)])
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    for _ in range(3):
        for b, s in zip(batches, streams):
            with torch.cuda.stream(s):
                b.forward()
                b.backward()
    torch.cuda.synchronize()
    for b, w in zip(batches, want):
        for u, v in zip(w, (b.y, b.h_last, b.dg, b.dx, b.dh0)):
            assert torch.equal(u, v)

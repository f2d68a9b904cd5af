"""Dense weight gradients against their 64-bit statements, every tile with whole and cut pieces.

Tolerance: (terms + 32) * 2^-24 times the sum of the terms' magnitudes, an fp32 sum in any order: a
term a row, of 8-bit rows three, whose factor scale * dy is rounded once (2 units more)."""
import pytest

torch = pytest.importorskip("torch")

import paper_1706_01307_amd as spc  # noqa: E402
from tests.linear_weight_variants import TILES  # noqa: E402
from tests.rows_ref import U  # noqa: E402
from tests.test_rows_dense_gpu import _off, _operands  # noqa: E402
from tests.test_rows_gpu import _f64, _gen, _gpu, _shifted  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def _poison():
    """Leave NaN in the memory that the next allocations are given: a sum that is not written, or a
    part that is read before it is, shows."""
    torch.cuda.empty_cache()
    blocks = [torch.full((2 ** 24,), float("nan"), device="cuda") for _ in range(3)]
    blocks += [torch.full((2 ** b,), float("nan"), device="cuda") for b in range(8, 18)]
    del blocks


@pytest.mark.parametrize("dt,n,ci,co,tile,whole,several", TILES)
def test_every_tile(dt, n, ci, co, tile, whole, several):
    x, xv, _, _, d = _operands(dt, n, ci, co, n + co)
    dy = _gen(n + 2)(n, co, dtype=d)
    dv = _f64(dy)
    want, mag = xv.t() @ dv, xv.abs().t() @ dv.abs()
    terms, views = n, [(x, dy.cuda())]
    if dt == "e4m3":
        terms = 3 * n + 2
        views += [(spc.Rows8(_shifted(x.q.cpu().view(torch.uint8)).view(x.q.dtype), x.scale), _shifted(dy))]
    elif whole:
        views += [(_shifted(x.cpu()), dy.cuda()), (x, _shifted(dy))]
    for i, (a, b) in enumerate(views):
        _poison()
        dw, db = spc.linear_backward_weight(a, b)
        _off(dw, want, (terms + 32) * U * mag, ("dw", i))
        _off(db, dv.sum(0), (n + 32) * U * dv.abs().sum(0), ("db", i))
        again, none = spc.linear_backward_weight(a, b, bias=False)
        assert none is None and torch.equal(again, dw), i

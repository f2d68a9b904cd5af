"""Weight gradients of 8-bit rows wherever their factors lie.

scale * dy is rounded once (U of it) and enters as three bf16 numbers that add up to it exactly;
products of e4m3 and bf16 numbers are exact; so an fp32 sum of 3 rows' terms: (3 rows + 34) U of the
terms' magnitudes, whatever the other rows and columns hold."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_1706_01307_amd as spc  # noqa: E402
from tests import rows_dense_ref as ref  # noqa: E402
from tests.rows_ref import U  # noqa: E402
from tests.test_rows_dense_gpu import _off, _rows8, _same  # noqa: E402
from tests.test_rows_gpu import _f64, _gen, _gpu, _shifted  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def _check(q, s, dy, what):
    n, xv, dv = len(q), ref.stands_for(q, s), _f64(dy)
    want, bound = xv.t() @ dv, (3 * n + 34) * U * (xv.abs().t() @ dv.abs())
    for rows in (_rows8(q, s), spc.Rows8(_shifted(q.view(torch.uint8)).view(ref.F8), s.cuda())):
        dw, db = spc.linear_backward_weight(rows, dy.cuda())
        _off(dw, want, bound, what)
        _off(db, dv.sum(0), (n + 32) * U * dv.abs().sum(0), "db")


def test_factors_whose_product_is_near_1():
    """A row of 1e37 under a gradient of 1e-37 beside ordinary rows, and the other way round."""
    r = _gen(1)
    for size in (1e37, 1e-25):
        for n in (1, 70, 300):
            x, dy = r(n, 40), r(n, 24).bfloat16()
            x[::3] *= size
            dy[::3] *= 1 / size
            _check(*ref.packed(x), dy, (size, n))
            _check(*ref.packed(x[::3]), dy[::3], (size, n, "alone"))


@pytest.mark.parametrize("ci,co", [(40, 70), (33, 65), (136, 264), (131, 300)])
def test_rows_and_columns_of_very_different_sizes(ci, co):
    """Columns of the gradient and rows of either factor over 2^60, and features that only some rows
    have: what is small beside its neighbours keeps its own bits."""
    n, r = 2000, _gen(ci)
    x = r(n, ci) * torch.exp2(25 * torch.sin(torch.arange(n) / 40.0))[:, None]
    x[:, ::2] = x[:, ::2].clamp(min=0)
    x[::2, 1::4] = 0
    dy = r(n, co) * torch.exp2(-60.0 * torch.arange(co) / co) * torch.exp2(20 * torch.cos(torch.arange(n) / 77.0))[:, None]
    _check(*ref.packed(x), dy.bfloat16(), (ci, co))


def test_scales_of_either_sign():
    r = _gen(6)
    q, s = ref.packed(r(500, 48))
    s = torch.where(torch.arange(500) % 3 == 0, -s, s)
    _check(q, s, r(500, 40).bfloat16(), "mixed")
    _check(q, -s.abs(), r(500, 40).bfloat16(), "negative")


def test_gradients_that_are_not_finite():
    """An infinity reaches its column alone, as the infinity, or with a factor of 0 the NaN, that it
    is there; a scale that is not finite every column."""
    r = _gen(9)
    for n, ci, co in ((200, 40, 24), (3000, 33, 65)):
        q, s = ref.packed(r(n, ci))
        dy = r(n, co).bfloat16()
        clean, _ = spc.linear_backward_weight(_rows8(q, s), dy.cuda())
        bad = dy.clone()
        bad[7, 3], bad[n - 1, 5], bad[11, 9], bad[90, 12] = math.inf, -math.inf, math.nan, 3.3e38
        got, _ = spc.linear_backward_weight(_rows8(q, s), bad.cuda())
        want = (ref.stands_for(q, s).t() @ _f64(bad)).float()
        rest = [c for c in range(co) if c not in (3, 5, 9, 12)]
        assert torch.equal(got[:, rest], clean[:, rest])
        assert bool(torch.isinf(want[:, 3]).any()) and bool(torch.isnan(want[:, 9]).all())
        for c in (3, 5, 9):
            _same(got[:, c], want[:, c], c)
        # (one factor is 3.3e38: what leaves fp32 is infinite on both sides; the rest is that one term,
        # rounded four times, and the sum of the others, below 1e33)
        out, w12 = got[:, 12].cpu().double(), want[:, 12].double()
        past = torch.isinf(w12)
        assert torch.equal(out[past], w12[past])
        assert bool(((out - w12).abs()[~past] <= 4 * U * w12.abs()[~past] + 1e33).all())
        s2 = s.clone()
        s2[5] = math.nan
        got, _ = spc.linear_backward_weight(_rows8(q, s2), dy.cuda())
        assert torch.isnan(got).all()

"""Every kernel variant of the grouped products and their weight gradient against the 64-bit
formulas, at sizes that test_rows_plan_cpu.py holds to the variants (rows_variants.py).
Tolerances are test_rows_gpu.py's."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_1706_01307_amd as spc  # noqa: E402
from tests import rows_ref as ref  # noqa: E402
from tests import rows_variants as v  # noqa: E402
from tests.test_rows_gpu import DT, _close, _f64, _gen  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.init()


def _case(sizes, seed):
    """offsets, their number of positions with those behind the last group, gathered rows"""
    off = np.concatenate([[0], np.cumsum(sizes)])
    m = int(off[-1]) + v.TAIL
    g = torch.Generator().manual_seed(seed)
    n_x = m // 2 + 1
    rows = torch.randint(0, n_x, (m,), generator=g)
    rows[0], rows[m // 3] = -1, n_x                 # rows of zeros
    return off, torch.from_numpy(off).int().cuda(), m, n_x, rows


def _ids(case):
    return "-".join(str(p) for p in (case[0], *case[-1], *case[3:-1], "back" if case[1] is True
                                     else "")).rstrip("-")


@pytest.mark.parametrize("case", v.PRODUCTS, ids=_ids)
def test_products(case):
    dtype, backward, sizes, red, cols, _ = case
    dt, r = DT[dtype], _gen(red + cols)
    off, offd, m, n_x, rows = _case(sizes, red)
    E = len(sizes)
    w = r(E, red, cols, std=1 / math.sqrt(red), dtype=dt)
    if backward:
        x = r(m, red, dtype=dt)
        want, mag = ref.grouped(_f64(x), _f64(w), off, None, None, False)
        wt = w.transpose(1, 2).contiguous().cuda()
        for odt in DT.values():
            g = spc.grouped_backward_data(x.cuda(), wt, offd, out_dtype=odt)
            _close(g, want, mag, red, "dx")
            mask = r(m, cols, dtype=odt)
            mask[m // 2, 0], mask[m - 4, cols - 1] = math.nan, -0.0
            g = spc.grouped_backward_data(x.cuda(), wt, offd, mask=mask.cuda(), out_dtype=odt)
            _close(g, torch.where(mask.double() <= 0, 0.0, want), mag, red, "dx with a mask")
        return
    x, b = r(n_x, red, dtype=dt), r(E, cols)
    want, mag = ref.grouped(_f64(x), _f64(w), off, rows, _f64(b), False)
    xd, wd, rd = x.cuda(), w.cuda(), rows.int().cuda()
    for odt in DT.values():
        for relu in (False, True):
            y = spc.grouped_forward(xd, wd, offd, rows=rd, bias=b.cuda(), relu=relu, out_dtype=odt)
            _close(y, torch.where(want < 0, 0.0, want) if relu else want, mag, red + 1, "y")


@pytest.mark.parametrize("case", v.WEIGHTS, ids=_ids)
def test_weight_gradients(case):
    dtype, sizes, ci, co, _ = case
    dt, r = DT[dtype], _gen(ci + co)
    off, offd, m, n_x, rows = _case(sizes, ci)
    x, dy = r(n_x, ci, dtype=dt), r(m, co, dtype=dt)
    dy[-v.TAIL:] = math.nan                         # no group's
    xs = ref.take(_f64(x), rows, m)
    xd, dyd, rd = x.cuda(), dy.cuda(), rows.int().cuda()
    gw, gb = spc.grouped_backward_weight(xd, dyd, offd, rows=rd)
    for e, (a, b) in enumerate(zip(off[:-1], off[1:])):
        d = _f64(dy[a:b])
        _close(gw[e], xs[a:b].T @ d, xs[a:b].abs().T @ d.abs(), b - a, ("dw", e))
        _close(gb[e], d.sum(0), d.abs().sum(0), b - a, ("db", e))
    again, none = spc.grouped_backward_weight(xd, dyd, offd, rows=rd, bias=False)
    assert none is None and torch.equal(gw, again)

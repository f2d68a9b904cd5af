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


def _check(got, x, w, off, bias, finish, terms, what):
    """Every position of `got` against finish(64-bit product, its positions), some rows at a time
    on the device; x: the rows read, float64 on the device."""
    E, m = len(off) - 1, len(x)
    for e, a, b in ref.groups(off, m) + [(E, int(off[-1]), m)]:
        for p in range(a, b, 50000):
            q = min(p + 50000, b)
            if e == E:                              # behind the last group
                assert not got[p:q].any(), what
                continue
            want, mag = x[p:q] @ w[e], x[p:q].abs() @ w[e].abs()
            if bias is not None:
                want, mag = want + bias[e], mag + bias[e].abs()
            want = finish(want, slice(p, q))
            bound = (terms + 32) * ref.U * mag + 1e-36
            if got.dtype == torch.bfloat16:
                bound += ref.BF16 * want.abs()
            bad = ~((got[p:q].double() - want).abs() <= bound)
            assert not bool(bad.any()), (what, e, p, int(bad.sum()))


@pytest.mark.parametrize("case", v.PRODUCTS, ids=_ids)
def test_products(case):
    dtype, backward, sizes, red, cols, _ = case
    dt, r = DT[dtype], _gen(red + cols)
    off, offd, m, n_x, rows = _case(sizes, red)
    E = len(sizes)
    w = r(E, red, cols, std=1 / math.sqrt(red), dtype=dt).cuda()
    w64 = w.double()
    if backward:
        x = r(m, red, dtype=dt).cuda()
        x64, wt = x.double(), w.transpose(1, 2).contiguous()
        for odt in DT.values():
            g = spc.grouped_backward_data(x, wt, offd, out_dtype=odt)
            _check(g, x64, w64, off, None, lambda t, s: t, red, "dx")
            mask = torch.randn(m, cols, device="cuda").to(odt)
            mask[m // 2, 0], mask[m - 4, cols - 1] = math.nan, -0.0
            g = spc.grouped_backward_data(x, wt, offd, mask=mask, out_dtype=odt)
            _check(g, x64, w64, off, None, lambda t, s: torch.where(mask[s] <= 0, 0.0, t), red,
                   "dx with a mask")
        return
    x, b = r(n_x, red, dtype=dt), r(E, cols).cuda()
    x64, b64 = ref.take(x.double(), rows, m).cuda(), b.double()
    x, rows = x.cuda(), rows.int().cuda()
    for odt in DT.values():
        for relu in (False, True):
            y = spc.grouped_forward(x, w, offd, rows=rows, bias=b, relu=relu, out_dtype=odt)
            _check(y, x64, w64, off, b64, lambda t, s: t.clamp(min=0) if relu else t, red + 1, "y")


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

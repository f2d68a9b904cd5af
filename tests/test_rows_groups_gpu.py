"""Grouped products of groups whose offsets are not what a routing gives: descending, negative
or past the end.  An offset counts as the largest of it and those before it, within [0, m]."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_1706_01307_amd as spc  # noqa: E402
from tests import rows_ref as ref  # noqa: E402
from tests.test_rows_gpu import DT, _close, _f64, _gen  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.init()


def _offsets(kind, E, m):
    g = np.random.default_rng(E + m)
    off = np.sort(g.integers(0, m + 1, E + 1))
    off[0], off[E] = 0, m
    if kind == "up and down":                       # 0, m, 0, m, ...
        off = np.where(np.arange(E + 1) % 2, m, 0)
    elif kind == "one down":                        # late, so that whole runs of groups ascend
        off[E - 1] = m // 3
    elif kind == "anywhere":
        off = g.integers(-m, 2 * m, E + 1)
        off[0] = 0
    elif kind == "falling":                         # one group, and positions behind it
        off = np.concatenate([[0], np.arange(E, 0, -1) * (m // (E + 2))])
    return off


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["up and down", "one down", "anywhere", "falling"])
@pytest.mark.parametrize("E,m,ci,co", [
    (4, 65536, 64, 96), (8, 59520, 96, 200),        # sums of many chunks of positions
    (3, 50, 16, 16), (5, 20, 512, 64),              # few positions
    (70, 900, 33, 24), (200, 3000, 40, 72), (129, 20000, 64, 136)])   # groups past the first 64
def test_groups_do_not_overlap(E, m, ci, co, kind, dtype):
    r, dt = _gen(E + m), DT[dtype]
    off = _offsets(kind, E, m)
    cut = np.maximum.accumulate(np.clip(off, 0, m))
    x, w, b, dy = r(m, ci, dtype=dt), r(E, ci, co, dtype=dt), r(E, co), r(m, co, dtype=dt)
    offd = torch.from_numpy(off).int().cuda()
    xd, wd, dyd = x.cuda(), w.cuda(), dy.cuda()
    want, mag = ref.grouped(_f64(x), _f64(w), cut, None, _f64(b), False)
    (dx, dw, db), (mx, mw, mb) = ref.grouped_grad(_f64(x), _f64(dy), _f64(w), cut, None, None)
    y = torch.full((m, co), float("nan"), dtype=dt, device="cuda")
    spc.grouped_forward(xd, wd, offd, bias=b.cuda(), out=y)
    _close(y, want, mag, ci + 1, "y")
    g = torch.full((m, ci), float("nan"), dtype=dt, device="cuda")
    spc.grouped_backward_data(dyd, wd, offd, out=g)
    _close(g, dx, mx, co, "dx")
    gw, gb = spc.grouped_backward_weight(xd, dyd, offd)
    _close(gw, dw, mw, int(np.diff(cut).max()), "dw")
    _close(gb, db, mb, int(np.diff(cut).max()), "db")
    again = spc.grouped_backward_weight(xd, dyd, offd)
    assert torch.equal(gw, again[0]) and torch.equal(gb, again[1])


def test_sizes_past_32_bits_are_refused():
    """A width of 2^32 + 8 is not taken for one of 8 (tensors without elements)."""
    wide = 2 ** 32 + 8

    def empty(*shape):
        return torch.empty(shape, device="cuda")
    off0, off1 = (torch.zeros(e, dtype=torch.int32, device="cuda") for e in (1, 2))
    for call in (lambda: spc.grouped_forward(empty(0, wide), empty(0, wide, 4), off0),
                 lambda: spc.grouped_forward(empty(0, 8), empty(0, 8, wide), off0),
                 lambda: spc.grouped_backward_data(empty(0, wide), empty(0, 8, wide), off0),
                 lambda: spc.grouped_backward_data(empty(0, 4), empty(0, wide, 4), off0),
                 lambda: spc.grouped_backward_weight(empty(0, wide), empty(0, 4), off1),
                 lambda: spc.grouped_backward_weight(empty(0, 8), empty(0, wide), off1)):
        with pytest.raises(ValueError):
            call()

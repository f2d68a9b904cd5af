"""GPU parity of the operators on feature rows against their 64-bit statements.

Tolerance of every result: (terms + 32) * 2^-24 times the sum of the absolute
values of its terms (an fp32 evaluation in any order), plus one rounding to bf16
where the result is bf16 (rows_ref.U, rows_ref.BF16).  Indices, and which elements
are dropped, are compared exactly.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_1706_01307_amd as spc  # noqa: E402
from tests import rows_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.init()


def _gen(seed):
    g = torch.Generator().manual_seed(seed)

    def r(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g) * std + mean).to(dtype)
    return r


def _close(got, want, mag, terms, what):
    assert tuple(got.shape) == tuple(want.shape), what
    bound = (terms + 32) * ref.U * mag + (ref.BF16 * want.abs() if got.dtype == torch.bfloat16
                                          else 0.0) + 1e-36
    g = got.detach().cpu().double()
    bad = ~((g - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(((g - want).abs() / bound).max()))


def _dev(t):
    return None if t is None else t.cuda()


def _f64(t):
    return None if t is None else t.double()


def _shifted(t):
    """The same tensor one element into a buffer: contiguous, aligned to its element only."""
    buf = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    buf[1:] = t.cuda().reshape(-1)
    return buf[1:].view(t.shape)


# ---------------------------------------------------------------------------
# Layer norm
# ---------------------------------------------------------------------------
NORM = [(1, 1), (1, 7), (5, 8), (461, 16), (33, 24), (100, 64), (7, 100), (3, 129), (257, 145),
        (2, 512), (9, 513), (4, 1000), (3, 2048), (2, 2050), (3, 4100), (2, 8192), (2, 8200),
        (1, 20001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", NORM)
def test_layer_norm(n, C, dtype):
    r, dt = _gen(n * 31 + C), DT[dtype]
    x, dy = r(n, C, std=1.5, mean=0.7, dtype=dt), r(n, C, dtype=dt)
    for affine in (True, False):
        ga, be = (r(C, mean=1.0, std=0.3), r(C)) if affine else (None, None)
        y, mean, rstd = spc.layer_norm_forward(x.cuda(), _dev(ga), _dev(be), 1e-5)
        wy, wm, wr, mag = ref.layer_norm(_f64(x), _f64(ga), _f64(be), 1e-5)
        # (a row of one element: x - mean is exactly 0, rstd 1 / sqrt(eps))
        _close(y, wy, mag, C, "y")
        _close(mean, wm, x.double().abs().mean(1), C, "mean")
        _close(rstd, wr, wr * (1 + (x.double().abs().mean(1) * wr) ** 2), 2 * C, "rstd")
        m, s = wm.float(), wr.float()
        (dx, dg, db), (mx, mg, mb) = ref.layer_norm_grad(_f64(dy), _f64(x), m.double(), s.double(),
                                                         _f64(ga))
        for params in (True, False):
            gx, gg, gb = spc.layer_norm_backward(dy.cuda(), x.cuda(), m.cuda(), s.cuda(), _dev(ga),
                                                 params=params)
            _close(gx, dx, mx, 2 * C, "dx")
            assert (gg is None) == (gb is None) == (not params)
        gx, gg, gb = spc.layer_norm_backward(dy.cuda(), x.cuda(), m.cuda(), s.cuda(), _dev(ga),
                                             params=True)
        _close(gg, dg, mg, n, "dgamma")
        _close(gb, db, mb, n, "dbeta")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_of_many_rows_sums_their_gradients(dtype):
    """More rows than the gradient has workgroups, at several widths."""
    for n, C in ((40001, 12), (40001, 64), (20003, 200)):
        r, dt = _gen(C), DT[dtype]
        x, dy, ga = r(n, C, dtype=dt), r(n, C, dtype=dt), r(C, mean=1.0)
        _, m, s, _ = ref.layer_norm(_f64(x), None, None, 1e-5)
        m, s = m.float(), s.float()
        want, mag = ref.layer_norm_grad(_f64(dy), _f64(x), m.double(), s.double(), _f64(ga))
        got = spc.layer_norm_backward(dy.cuda(), x.cuda(), m.cuda(), s.cuda(), ga.cuda())
        again = spc.layer_norm_backward(dy.cuda(), x.cuda(), m.cuda(), s.cuda(), ga.cuda())
        for g, g2, w, a, t in zip(got, again, want, mag, (2 * C, n, n)):
            _close(g, w, a, t, (n, C))
            assert torch.equal(g, g2)


def test_layer_norm_constant_and_nonfinite_rows():
    x = torch.full((4, 70), 3.25)
    x[1, 5], x[2, 69] = math.inf, math.nan
    y, mean, rstd = spc.layer_norm_forward(x.cuda(), eps=1e-5)
    y, rstd = y.cpu(), rstd.cpu()
    assert torch.equal(y[0], torch.zeros(70)) and torch.equal(y[3], torch.zeros(70))
    assert abs(float(rstd[0]) * math.sqrt(1e-5) - 1) < 1e-6
    assert not torch.isfinite(y[1]).any() and torch.isnan(y[2]).all()
    # with eps = 0 a constant row is 0 * infinity, and no other row is touched
    x = torch.randn(3, 64)
    x[1] = 2.0
    y = spc.layer_norm_forward(x.cuda(), eps=0.0)[0].cpu()
    assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2]).all()


def test_layer_norm_without_rows():
    x = torch.empty(0, 24, device="cuda")
    y, mean, rstd = spc.layer_norm_forward(x)
    assert y.shape == (0, 24) and mean.shape == rstd.shape == (0,)
    dx, dg, db = spc.layer_norm_backward(x, x, mean, rstd, torch.ones(24, device="cuda"))
    assert dx.shape == (0, 24) and not dg.any() and not db.any()
    assert spc.dropout_forward(x, 0.5, 1).shape == (0, 24)


# ---------------------------------------------------------------------------
# Dropout
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1,), (3,), (8,), (5, 7), (33, 65), (461, 16), (4099,)])
def test_dropout(shape, dtype):
    r, dt = _gen(len(shape) + shape[-1]), DT[dtype]
    x, res = r(*shape, dtype=dt), r(*shape, dtype=dt)
    for p, seed, offset in ((0.0, 1, 0), (0.1, 2 ** 64 - 3, 5), (0.5, 77, 2 ** 40 + 1),
                            (0.9, 0, 2 ** 64 - 1), (1 - 1e-12, 3, 3)):
        keep = torch.from_numpy(ref.kept(0, x.numel(), p, seed, offset)).view(x.shape)
        d = torch.where(keep, x.double() / (1 - p), 0.0)
        y = spc.dropout_forward(x.cuda(), p, seed, offset)
        assert torch.equal((y != 0).cpu() | (x == 0), keep | (x == 0))
        _close(y, d, d.abs(), 4, (p, "y"))
        y = spc.dropout_forward(x.cuda(), p, seed, offset, residual=res.cuda())
        _close(y, res.double() + d, res.double().abs() + d.abs(), 4, (p, "y with residual"))
        dx = spc.dropout_backward(x.cuda(), p, seed, offset)
        _close(dx, d, d.abs(), 4, (p, "dx"))
        step = torch.tensor([7], device="cuda")
        a = spc.dropout_forward(x.cuda(), p, seed, offset - 7, step=step)
        assert torch.equal(a, spc.dropout_forward(x.cuda(), p, seed, offset))


def test_dropout_of_nonfinite_elements_in_place_and_views():
    x = torch.full((64, 33), math.nan)
    keep = torch.from_numpy(ref.kept(0, x.numel(), 0.5, 9, 1)).view(x.shape)
    y = spc.dropout_forward(x.cuda(), 0.5, 9, 1).cpu()
    assert torch.equal(torch.isnan(y), keep) and torch.equal(y[~keep], torch.zeros(int((~keep).sum())))
    for dt in DT.values():
        x, res = torch.randn(50, 33).to(dt), torch.randn(50, 33).to(dt)
        want = spc.dropout_forward(x.cuda(), 0.5, 9, 1, residual=res.cuda())
        for out in ("x", "res"):
            a, b = x.cuda(), res.cuda()
            spc.dropout_forward(a, 0.5, 9, 1, residual=b, out=a if out == "x" else b)
            assert torch.equal(a if out == "x" else b, want)
        assert torch.equal(spc.dropout_forward(_shifted(x), 0.5, 9, 1, residual=_shifted(res)), want)
        # rows of a wider tensor, and a transposed one, are copied
        wide = torch.zeros(50, 40, dtype=dt, device="cuda")
        wide[:, 3:36] = x.cuda()
        assert torch.equal(spc.dropout_forward(wide[:, 3:36], 0.5, 9, 1, residual=res.cuda()), want)
        assert torch.equal(spc.dropout_forward(x.cuda().t().contiguous().t(), 0.5, 9, 1,
                                               residual=res.cuda()), want)


# ---------------------------------------------------------------------------
# Routing
# ---------------------------------------------------------------------------
ROUTE = [(1, 1, 1), (1, 2, 2), (3, 5, 3), (70, 8, 2), (300, 8, 8), (129, 9, 4), (461, 16, 2),
         (600, 33, 1), (257, 64, 6), (90, 100, 16), (65, 256, 8), (40, 257, 3), (33, 600, 5),
         (20, 1024, 16), (0, 8, 2)]


def _check_route(x, k, normalize):
    n, E = x.shape
    got = spc.route_forward(x.cuda(), k, normalize)
    experts, weights, offsets, rows, pos = ref.route(x.double().numpy(), k, normalize)
    for name, want in (("experts", experts), ("offsets", offsets), ("rows", rows), ("pos", pos)):
        assert np.array_equal(getattr(got, name).cpu().numpy(), want), (name, n, E, k)
    w = torch.from_numpy(weights)
    fin = x.double()[torch.isfinite(x)]
    size = float(fin.abs().max()) if fin.numel() else 0.0
    ok = torch.isfinite(w)
    g = got.weights.cpu()
    assert torch.equal(torch.isnan(g), torch.isnan(w))
    # exp of a difference of up to 2 * size, rounded
    _close(torch.where(ok, g, 0.0), torch.where(ok, w, 0.0), torch.where(ok, w, 0.0),
           E + 2 * size, (n, E, k, "weights"))
    return got, experts, weights


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,E,k", ROUTE)
def test_route(n, E, k, dtype):
    r, dt = _gen(n + E + k), DT[dtype]
    for kind in ("plain", "ties", "masked"):
        x = r(n, E, std=2.0)
        if kind == "ties":
            x = torch.round(x)                      # many equal logits, zeros of both signs
        if kind == "masked" and n:
            g = torch.Generator().manual_seed(3)
            x[torch.rand(n, E, generator=g) < 0.4] = -math.inf
            x[torch.rand(n, E, generator=g) < 0.1] = torch.finfo(torch.float32).min
            x[::3] = -math.inf                      # rows without an expert
        x = x.to(dt)
        if kind == "masked" and n > 1:
            x[1] = torch.finfo(dt).min              # the lowest value is a value
        for normalize in (True, False):
            got, experts, weights = _check_route(x, k, normalize)
            dw = r(n, k)
            d = spc.route_backward(dw.cuda(), x.cuda(), got.experts, got.weights, normalize)
            want = torch.from_numpy(ref.route_grad(dw.double().numpy(), x.double().numpy(), experts,
                                                   weights, normalize)).view(n, E)
            # |dlogits| <= p (|dw| + D); D is a sum of k terms, the weights are off by E + 2 size
            mag = torch.full_like(want, 2 * float(dw.abs().max()) if n else 0.0)
            _close(d, want, mag, 3 * (E + k + 40), (n, E, k, kind, "dlogits"))


def test_route_nonfinite_rows_stay_to_themselves():
    x = torch.randn(40, 12)
    x[3, 7] = math.nan
    x[5, 2], x[5, 9] = math.inf, math.nan
    x[8, 4] = math.inf
    x[9] = math.nan
    for normalize in (True, False):
        got, _, _ = _check_route(x, 3, normalize)
        e = got.experts.cpu()
        assert e[3, 0] == 7 and e[5, 0] == 9 and e[8, 0] == 4 and e[9].tolist() == [0, 1, 2]


def test_route_of_many_workgroups_is_stable():
    """All pairs, in order, of 70,000 rows (several workgroups, the scan's carry)."""
    for E, k in ((3, 2), (64, 2), (200, 5)):
        x = torch.randint(-6, 7, (70001, E)).float()
        x[::7] = -math.inf
        got = spc.route_forward(x.cuda(), k)
        v, e = torch.sort(x, dim=1, descending=True, stable=True)
        e = torch.where(v[:, :k] > -math.inf, e[:, :k], -1)
        assert torch.equal(got.experts.cpu().long(), e)
        flat = torch.where(e < 0, E, e).reshape(-1)
        order = torch.sort(flat, stable=True).indices
        total = int((flat < E).sum())
        assert got.offsets.cpu().tolist() == [int((flat < b).sum()) for b in range(E)] + [total]
        rows, pos = got.rows.cpu().long(), got.pos.cpu().long().reshape(-1)
        assert torch.equal(rows[:total], order[:total] // k)
        assert (rows[total:] == -1).all()
        assert torch.equal(pos[order[:total]], torch.arange(total))
        assert (pos[flat == E] == -1).all()


# ---------------------------------------------------------------------------
# Grouped products
# ---------------------------------------------------------------------------
# group sizes, C_in, C_out
GROUPED = [([1], 1, 1), ([1], 512, 96), ([0, 1, 0], 8, 16), ([3, 0, 5], 16, 24),
           ([7, 1, 2, 30], 33, 17), ([130, 0, 1, 64], 64, 64), ([65, 200], 96, 200),
           ([129, 127, 128, 0, 300], 128, 136), ([40, 0, 700], 100, 72), ([0, 0], 16, 16),
           ([513], 7, 300), ([1] * 70, 40, 48), ([2, 0, 3] * 30, 24, 8), ([1500, 20], 72, 130)]


def _groups_case(sizes, ci, co, dt, seed, gather, tail):
    r = _gen(seed)
    off = np.concatenate([[0], np.cumsum(sizes)])
    m = int(off[-1]) + tail
    g = torch.Generator().manual_seed(seed)
    n_x = max(1, m // 2) if gather else m
    rows = torch.randint(0, n_x, (m,), generator=g) if gather else None
    if gather and m > 4:
        rows[2], rows[4] = -1, n_x                  # rows of zeros
    x = r(n_x, ci, dtype=dt)
    w = r(len(sizes), ci, co, std=1 / math.sqrt(ci), dtype=dt)
    return r, off, m, rows, x, w, r(len(sizes), co)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,ci,co", GROUPED)
def test_grouped(sizes, ci, co, dtype):
    dt = DT[dtype]
    for gather, tail in ((False, 0), (True, 0), (True, 5), (False, 3)):
        r, off, m, rows, x, w, b = _groups_case(sizes, ci, co, dt, ci + co, gather, tail)
        offd = torch.from_numpy(off).int().cuda()
        rd = None if rows is None else rows.int().cuda()
        for bias, relu, odt in ((b, True, dt), (None, False, torch.float32),
                                (b, False, torch.bfloat16)):
            y = spc.grouped_forward(x.cuda(), w.cuda(), offd, rows=rd, bias=_dev(bias), relu=relu,
                                    out_dtype=odt)
            want, mag = ref.grouped(_f64(x), _f64(w), off, rows, _f64(bias), relu)
            _close(y, want, mag, ci + 1, "y")
        dy, mask = r(m, co, dtype=dt), r(m, ci, dtype=dt)
        (dx, dw, db), (mx, mw, mb) = ref.grouped_grad(_f64(x), _f64(dy), _f64(w), off, rows,
                                                      _f64(mask))
        g = spc.grouped_backward_data(dy.cuda(), w.cuda(), offd, mask=mask.cuda())
        _close(g, dx, mx, co, "dx")
        (dx2, _, _), _ = ref.grouped_grad(_f64(x), _f64(dy), _f64(w), off, rows, None)
        odt = torch.float32 if dt == torch.bfloat16 else torch.bfloat16
        g = spc.grouped_backward_data(dy.cuda(), w.cuda(), offd, out_dtype=odt)
        _close(g, dx2, mx, co, "dx of another type")
        gw, gb = spc.grouped_backward_weight(x.cuda(), dy.cuda(), offd, rows=rd)
        _close(gw, dw, mw, max(sizes), "dw")
        _close(gb, db, mb, max(sizes), "db")
        gw2, none = spc.grouped_backward_weight(x.cuda(), dy.cuda(), offd, rows=rd, bias=False)
        assert none is None and torch.equal(gw, gw2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_grouped_large_groups_are_summed_in_chunks(dtype):
    """Enough positions for the weight gradient's chunks, in groups of very different sizes."""
    dt = DT[dtype]
    for sizes, ci, co in (([30000, 1, 0, 999, 5000], 64, 96), ([9001, 9001], 130, 65)):
        r, off, m, rows, x, w, b = _groups_case(sizes, ci, co, dt, 5, True, 0)
        offd, rd = torch.from_numpy(off).int().cuda(), rows.int().cuda()
        dy = r(m, co, dtype=dt)
        (dx, dw, db), (mx, mw, mb) = ref.grouped_grad(_f64(x), _f64(dy), _f64(w), off, rows, None)
        y = spc.grouped_forward(x.cuda(), w.cuda(), offd, rows=rd, bias=b.cuda())
        want, mag = ref.grouped(_f64(x), _f64(w), off, rows, _f64(b), False)
        _close(y, want, mag, ci + 1, "y")
        g = spc.grouped_backward_data(dy.cuda(), w.cuda(), offd)
        _close(g, dx, mx, co, "dx")
        gw, gb = spc.grouped_backward_weight(x.cuda(), dy.cuda(), offd, rows=rd)
        _close(gw, dw, mw, max(sizes), "dw")
        _close(gb, db, mb, max(sizes), "db")
        again = spc.grouped_backward_weight(x.cuda(), dy.cuda(), offd, rows=rd)
        assert torch.equal(gw, again[0]) and torch.equal(gb, again[1])


@pytest.mark.parametrize("sizes,ci,co,dtype", [
    # reductions of one to four stages kept in registers, several column tiles
    ([9000, 0, 1, 8500, 127], 40, 136, "bf16"), ([17001, 60], 64, 264, "bf16"),
    ([300, 16500], 128, 520, "bf16"), ([8192, 8193], 168, 200, "bf16"),
    ([5000, 12000, 77], 256, 392, "bf16"),
    # tiles of 256 x 256, and the fp32 kernels at the same sizes
    ([70000, 61000, 300], 264, 144, "bf16"), ([17000, 90], 264, 144, "f32"),
    ([20000, 513], 200, 328, "bf16")])
def test_grouped_many_rows(sizes, ci, co, dtype):
    dt = DT[dtype]
    odt = torch.float32 if dt == torch.bfloat16 else torch.bfloat16
    r, off, m, rows, x, w, b = _groups_case(sizes, ci, co, dt, 3, True, 70)
    offd, rd = torch.from_numpy(off).int().cuda(), rows.int().cuda()
    dy, mask = r(m, co, dtype=dt), r(m, ci, dtype=dt)
    plain, mag = ref.grouped(_f64(x), _f64(w), off, rows, _f64(b), False)
    (dx, dw, db), (mx, mw, mb) = ref.grouped_grad(_f64(x), _f64(dy), _f64(w), off, rows, None)
    y = spc.grouped_forward(x.cuda(), w.cuda(), offd, rows=rd, bias=b.cuda(), relu=True)
    _close(y, torch.where(plain < 0, 0.0, plain), mag, ci + 1, "y")
    y = spc.grouped_forward(x.cuda(), w.cuda(), offd, rows=rd, bias=b.cuda(), out_dtype=odt)
    _close(y, plain, mag, ci + 1, "y of another type")
    # the same widths the other way: as an input gradient
    wt = w.transpose(1, 2).contiguous()
    back, mag = ref.grouped(_f64(dy), _f64(wt), off, None, None, False)
    g = spc.grouped_backward_data(dy.cuda(), w.cuda(), offd, mask=mask.cuda())
    _close(g, torch.where(mask.double() <= 0, 0.0, dx), mx, co, "dx")
    g = spc.grouped_backward_data(dy.cuda(), w.cuda(), offd, out_dtype=odt)
    _close(g, dx, mx, co, "dx of another type")
    fwd_mask = r(m, co, dtype=dt)
    xs = ref.take(x, rows, m)
    (dx2, _, _), (mx2, _, _) = ref.grouped_grad(_f64(dy), _f64(xs), _f64(wt), off, None, None)
    g = spc.grouped_backward_data(xs.cuda(), wt.cuda(), offd, mask=fwd_mask.cuda())
    _close(g, torch.where(fwd_mask.double() <= 0, 0.0, dx2), mx2, ci, "dx, wide")
    y = spc.grouped_forward(dy.cuda(), wt.cuda(), offd)
    _close(y, back, mag, co, "y, narrow")
    gw, gb = spc.grouped_backward_weight(x.cuda(), dy.cuda(), offd, rows=rd)
    _close(gw, dw, mw, max(sizes), "dw")
    _close(gb, db, mb, max(sizes), "db")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,ci,co", [
    ([300, 0, 77], 133, 72), ([40000, 9000], 66, 72), ([9000, 12000], 390, 264),
    ([66000, 66001], 261, 264), ([66000, 66001], 256, 264)])
def test_grouped_masks_of_cut_and_whole_rows(sizes, ci, co, dtype):
    """The input gradient's mask in tiles of every size, with results of either type."""
    r, off, m, _, _, w, _ = _groups_case(sizes, ci, co, DT[dtype], 11, False, 3)
    dy = r(m, co, dtype=DT[dtype])
    want, mag = ref.grouped(_f64(dy), _f64(w.transpose(1, 2).contiguous()), off, None, None, False)
    offd, dyd, wd = torch.from_numpy(off).int().cuda(), dy.cuda(), w.cuda()
    for odt in DT.values():
        mask = r(m, ci, dtype=odt)
        mask[m // 2, 0], mask[m - 4, ci - 1] = math.nan, -0.0
        g = spc.grouped_backward_data(dyd, wd, offd, mask=mask.cuda(), out_dtype=odt)
        _close(g, torch.where(mask.double() <= 0, 0.0, want), mag, co, (sizes, ci, co, odt))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_grouped_few_rows(dtype):
    """Up to a few dozen positions: one, several and all of them in a group, long reductions."""
    for sizes, ci, co in (([0, 1, 0, 0, 2], 512, 200), ([32], 1030, 64), ([5, 0, 9, 1], 7, 2048),
                          ([4, 4], 2500, 136), ([33], 96, 64)):
        r, off, m, rows, x, w, b = _groups_case(sizes, ci, co, DT[dtype], 8, True, 1)
        offd = torch.from_numpy(off).int().cuda()
        for relu in (False, True):
            y = spc.grouped_forward(x.cuda(), w.cuda(), offd, rows=rows.int().cuda(),
                                    bias=b.cuda(), relu=relu)
            want, mag = ref.grouped(_f64(x), _f64(w), off, rows, _f64(b), relu)
            _close(y, want, mag, ci + 1, (sizes, ci, co))


def test_grouped_no_rows_and_many_groups():
    for dt in DT.values():
        w = torch.randn(5, 16, 24).to(dt).cuda()
        off = torch.zeros(6, dtype=torch.int32, device="cuda")
        x, dy = torch.empty(0, 16, dtype=dt, device="cuda"), torch.empty(0, 24, dtype=dt,
                                                                         device="cuda")
        assert spc.grouped_forward(x, w, off).shape == (0, 24)
        assert spc.grouped_backward_data(dy, w, off).shape == (0, 16)
        dw, db = spc.grouped_backward_weight(x, dy, off)
        assert not dw.any() and not db.any() and dw.shape == (5, 16, 24)
        # a group index past the first 64, and past 1024
        E = 1500
        sizes = [0] * E
        sizes[3], sizes[70], sizes[1100], sizes[1499] = 2, 1, 40, 5
        r, o, m, rows, x, w, b = _groups_case(sizes, 12, 8, dt, 1, False, 2)
        y = spc.grouped_forward(x.cuda(), w.cuda(), torch.from_numpy(o).int().cuda(), bias=b.cuda())
        want, mag = ref.grouped(_f64(x), _f64(w), o, rows, _f64(b), False)
        _close(y, want, mag, 13, "y")


def test_grouped_nonfinite_values_stay_with_their_rows_and_groups():
    for dt in DT.values():
        r, off, m, rows, x, w, b = _groups_case([70, 60, 3], 40, 72, dt, 2, False, 0)
        x[5, 3], x[72, 0] = math.nan, math.inf
        w[2, 1, 1] = math.inf
        y = spc.grouped_forward(x.cuda(), w.cuda(), torch.from_numpy(off).int().cuda()).cpu()
        bad = ~torch.isfinite(y)
        rows_bad = bad.any(1).nonzero()[:, 0].tolist()
        assert set(rows_bad) == {5, 72, 130, 131, 132}
        assert bad[5].all() and bad[130:133, 1].all() and int(bad[130:133].sum()) == 3
        # weight gradients: only the group of a row that holds one
        dy = r(m, 72, dtype=dt)
        dw, db = spc.grouped_backward_weight(x.cuda(), dy.cuda(),
                                             torch.from_numpy(off).int().cuda())
        assert torch.isfinite(db).all() and torch.isfinite(dw[2]).all()
        assert not torch.isfinite(dw[0, 3]).any() and torch.isfinite(dw[0, :3]).all()


def test_grouped_offsets_out_of_order_stay_in_bounds():
    """Offsets that descend or leave [0, m] make empty or cut groups, nothing else."""
    x, w = torch.randn(50, 16).cuda(), torch.randn(3, 16, 16).cuda()
    off = torch.tensor([0, 30, 20, 90], dtype=torch.int32).cuda()
    y = spc.grouped_forward(x, w, off)
    want = torch.cat([x[:30] @ w[0], x[30:50] @ w[2]])
    assert torch.allclose(y[:20], want[:20], atol=1e-4)
    assert torch.allclose(y[30:], want[30:], atol=1e-4)


# ---------------------------------------------------------------------------
# Combine
# ---------------------------------------------------------------------------
COMBINE = [(1, 1, 1), (1, 4, 512), (5, 2, 7), (64, 2, 64), (33, 3, 33), (20, 4, 130), (9, 8, 1000),
           (3, 16, 24), (2, 2, 5000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,C", COMBINE)
def test_combine(n, k, C, dtype):
    r, dt = _gen(n + k + C), DT[dtype]
    g = torch.Generator().manual_seed(n)
    m = n * k
    for holes in (False, True):
        pos = torch.randperm(m, generator=g)
        used = m
        if holes:
            used = m - m // 3
            pos = torch.where(pos < used, pos, -1 - pos % 2 * (1 - 2 * m - 1))  # -1, or far beyond
        pos = pos.view(n, k)
        y, w, res, do = r(m, C, dtype=dt), r(n, k), r(n, C, dtype=dt), r(n, C, dtype=dt)
        for wt, rs in ((w, res), (None, None), (w, None)):
            out = spc.combine_forward(y.cuda(), pos.int().cuda(), _dev(wt), residual=_dev(rs))
            want, mag = ref.combine(_f64(y), pos, _f64(wt), _f64(rs))
            _close(out, want, mag, k + 1, "out")
        off = torch.tensor([0, used], dtype=torch.int32).cuda()
        for wt in (w, None):
            dy, dw = spc.combine_backward(do.cuda(), y.cuda(), pos.int().cuda(), _dev(wt),
                                          offsets=off if holes else None)
            wy, ww, mag = ref.combine_grad(_f64(do), _f64(y), pos, _f64(wt))
            _close(dy, wy, wy.abs(), 1, "dy")
            if wt is None:
                assert dw is None
            else:
                _close(dw, ww, mag, C, "dweights")


def test_combine_in_place_and_without_rows():
    y, pos = torch.randn(6, 8).cuda(), torch.tensor([[0, 5], [2, -1]], dtype=torch.int32).cuda()
    res = torch.randn(2, 8).cuda()
    want = spc.combine_forward(y, pos, residual=res)
    assert spc.combine_forward(y, pos, residual=res, out=res) is res and torch.equal(res, want)
    none = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    assert spc.combine_forward(y, none).shape == (0, 8)
    # every position is behind the count
    dy, dw = spc.combine_backward(torch.empty(0, 8, device="cuda"), y, none,
                                  torch.empty(0, 2, device="cuda"),
                                  offsets=torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert not dy.any() and dw.shape == (0, 2)
    # a slot without a position hides whatever its weight holds
    w = torch.tensor([[0.5, 2.0], [1.0, math.nan]]).cuda()
    assert torch.isfinite(spc.combine_forward(y, pos, w)).all()


# ---------------------------------------------------------------------------
# All of them
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_at_any_element_offset(dtype):
    """Inputs that start one element into a buffer give what aligned ones give."""
    r, dt = _gen(9), DT[dtype]
    n, C, E, k, co = 150, 40, 6, 2, 56
    x, w, lg = r(n, C, dtype=dt), r(E, C, co, dtype=dt), r(n, E, dtype=dt)
    ga, be, b = r(C), r(C), r(E, co)
    dy = r(n, C, dtype=dt)
    res = []
    for put in (lambda t: t.cuda(), _shifted):
        y, m, s = spc.layer_norm_forward(put(x), put(ga), put(be))
        grads = spc.layer_norm_backward(put(dy), put(x), put(m), put(s), put(ga))
        q = spc.route_forward(put(lg), k, False)
        dl = spc.route_backward(put(q.weights), put(lg), put(q.experts), put(q.weights), False)
        h = spc.grouped_forward(put(y), put(w), put(q.offsets), rows=put(q.rows), bias=put(b))
        dh = spc.grouped_backward_data(put(h), put(w), put(q.offsets))
        dw = spc.grouped_backward_weight(put(y), put(h), put(q.offsets), rows=put(q.rows))
        o = spc.combine_forward(put(h), put(q.pos), put(q.weights))
        c = spc.combine_backward(put(o), put(h), put(q.pos), put(q.weights), offsets=put(q.offsets))
        res.append([y, m, s, *grads, q.weights, q.pos, dl, h, dh, *dw, o, *c])
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_calls_on_another_stream_are_ordered_there():
    s = torch.cuda.Stream()
    x = torch.randn(4000, 64, device="cuda")
    lg, w = torch.randn(4000, 8, device="cuda"), torch.randn(8, 64, 32, device="cuda")
    q = spc.route_forward(lg, 2)
    want = spc.combine_forward(spc.grouped_forward(x, w, q.offsets, rows=q.rows), q.pos, q.weights)
    torch.cuda.synchronize()
    q = spc.route_forward(lg.t().contiguous().t(), 2, stream=s)     # (copied there)
    h = spc.grouped_forward(x, w, q.offsets, rows=q.rows, stream=s)
    o = spc.combine_forward(h, q.pos, q.weights, stream=s)
    s.synchronize()
    assert torch.equal(o, want)


def test_whole_block_in_a_captured_graph():
    """Forward and gradients captured once and replayed on new inputs and new dropped elements,
    with eager work between the replays."""
    n, C, E, k = 700, 48, 5, 2
    x, lg = torch.empty(n, C, device="cuda"), torch.empty(n, E, device="cuda")
    ga, be = torch.randn(C, device="cuda"), torch.randn(C, device="cuda")
    w, b = torch.randn(E, C, C, device="cuda"), torch.randn(E, C, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def block():
        y, m, s = spc.layer_norm_forward(x, ga, be)
        q = spc.route_forward(lg, k)
        h = spc.grouped_forward(y, w, q.offsets, rows=q.rows, bias=b, relu=True)
        u = spc.combine_forward(h, q.pos, q.weights)
        o = spc.dropout_forward(u, 0.3, 11, 5, residual=x, step=step)
        du = spc.dropout_backward(o, 0.3, 11, 5, step=step)
        dh, dwt = spc.combine_backward(du, h, q.pos, q.weights, offsets=q.offsets)
        dy = spc.combine_forward(spc.grouped_backward_data(dh, w, q.offsets), q.pos)
        dw, db = spc.grouped_backward_weight(y, dh, q.offsets, rows=q.rows)
        dl = spc.route_backward(dwt, lg, q.experts, q.weights)
        return [o, *spc.layer_norm_backward(dy, x, m, s, ga), dw, db, dl]

    x.normal_()
    lg.normal_()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        block()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = block()
    seen = []
    for i in range(4):
        x.normal_()
        lg.normal_()
        step.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        out = [t.clone() for t in got]
        want = block()
        torch.cuda.synchronize()
        for a, c in zip(out, want):
            assert torch.equal(a, c), i
        seen.append(out[0] == x)
    assert not torch.equal(seen[0], seen[1])


@pytest.mark.parametrize("dtype", ["bf16"])
def test_element_offsets_past_32_bits(dtype):
    """Tensors of more than 2^32 elements: the far rows are read and written."""
    dt, C = DT[dtype], 1024
    m = 2 ** 22 + 50
    y = torch.empty((m, C), dtype=dt, device="cuda")
    at = torch.tensor([[0, m - 1], [2 ** 21 + 3, 2 ** 22 + 1], [m - 7, 5]])
    r = _gen(4)
    v = r(6, C, dtype=dt)
    y[at.view(-1).cuda()] = v.cuda()
    w = r(3, 2)
    out = spc.combine_forward(y, at.int().cuda(), w.cuda())
    want, mag = ref.combine(_f64(v), torch.arange(6).view(3, 2), _f64(w), None)
    _close(out, want, mag, 3, "combine")
    # gathered and plain rows of the same tensor
    wt = r(1, C, 8, std=1 / 32, dtype=dt)
    rows = at.view(-1).int().cuda()
    off = torch.tensor([0, 6], dtype=torch.int32).cuda()
    z = spc.grouped_forward(y, wt.cuda(), off, rows=rows)
    want, mag = ref.grouped(_f64(v), _f64(wt), np.array([0, 6]), None, None, False)
    _close(z, want, mag, C, "grouped")
    # the last positions of a gradient that long
    y[-6:] = v.cuda()
    d = spc.layer_norm_forward(y)[0][-6:]
    want, _, _, mag = ref.layer_norm(_f64(v), None, None, 1e-5)
    _close(d, want, mag, C, "layer norm")
    y.fill_(1.0)
    d = spc.dropout_forward(y, 0.5, 3, 4)
    n = 4 * C
    for first in (0, 2 ** 32 - n // 2, m * C - n):
        keep = torch.from_numpy(ref.kept(first, n, 0.5, 3, 4))
        assert torch.equal(d.view(-1)[first:first + n].cpu().float(), keep.float() * 2)
    # positions far into dx and dy
    off = torch.tensor([0, m - 3, m], dtype=torch.int32).cuda()
    wt = r(2, 8, C, dtype=dt)
    del d
    small = spc.grouped_backward_data(y, wt.cuda(), off)          # y: all ones
    want = wt.double().sum(2)
    _close(small[-3:], want[1].expand(3, 8), wt.double().abs().sum(2)[1].expand(3, 8), C, "dx")
    _close(small[:3], want[0].expand(3, 8), wt.double().abs().sum(2)[0].expand(3, 8), C, "dx")


def test_binding_refuses_what_does_not_fit():
    x = torch.randn(6, 8, device="cuda")
    w = torch.randn(2, 8, 4, device="cuda")
    off = torch.tensor([0, 2, 6], dtype=torch.int32, device="cuda")
    pos = torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    bad = [(TypeError, lambda: spc.layer_norm_forward(x.half())),
           (TypeError, lambda: spc.layer_norm_forward(x.cpu())),
           (ValueError, lambda: spc.layer_norm_forward(x[0])),
           (ValueError, lambda: spc.layer_norm_forward(x, torch.ones(7, device="cuda"))),
           (TypeError, lambda: spc.layer_norm_forward(x, torch.ones(8, device="cuda").bfloat16())),
           (spc.SpconvError, lambda: spc.layer_norm_forward(x, eps=-1.0)),
           (spc.SpconvError, lambda: spc.dropout_forward(x, 1.0, 0)),
           (TypeError, lambda: spc.dropout_forward(x, 0.1, 0, residual=x.bfloat16())),
           (ValueError, lambda: spc.dropout_forward(x, 0.1, 0, residual=x[:5])),
           (ValueError, lambda: spc.dropout_forward(x, 0.1, 0, out=x.t())),
           (spc.SpconvError, lambda: spc.route_forward(x, 0)),
           (spc.SpconvError, lambda: spc.route_forward(x, 9)),
           (ValueError, lambda: spc.grouped_forward(x[:, :7], w, off)),
           (TypeError, lambda: spc.grouped_forward(x, w.bfloat16(), off)),
           (TypeError, lambda: spc.grouped_forward(x, w, off.long())),
           (ValueError, lambda: spc.grouped_forward(x, w, off[:2])),
           (ValueError, lambda: spc.grouped_backward_data(x, w, off)),
           (ValueError, lambda: spc.grouped_backward_weight(x[:5], x, off)),
           (TypeError, lambda: spc.combine_forward(x, pos.long())),
           (ValueError, lambda: spc.combine_forward(x, pos, torch.ones(3, 1, device="cuda"))),
           (ValueError, lambda: spc.combine_backward(x, x, pos))]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            print("accepted", i)

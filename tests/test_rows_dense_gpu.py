"""GPU parity of the RMS norm, rows in 8 bits, activations and dense products against their 64-bit
statements (rows_dense_ref.py).

Tolerances, in units U = 2^-24 of fp32, counted before the first run:
  sums       (terms + 32) U times the sum of the terms' magnitudes; one rounding to the result's
             type more where that is bf16 (2^-8 of it);
  activation 8 U of |z|: two factors, each of a few roundings and, for the logistic function, of one
             unit of exp2 and of the reciprocal each; the argument's rounding is damped by
             s (1 - s) |u| < 0.28; and 1.13, the steepest slope, times the error of z;
  slope      (32 + 2 |z|) U: 1 - s is off by U / 2, times z;
  8 bits     packed from the same fp32 values bit for bit; from values off by d, half a step of
             e4m3 (2^-4 of the value, 2^-10 of the scale) and d;
  dw of 8-bit rows: 2^-22 more of a term's magnitude (two f16 numbers hold 22 bits), and 2^-39 of the
             row's largest |x| times the largest |scale dy| (what is smaller than f16's range).
"""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_1706_01307_amd as spc  # noqa: E402
from tests import rows_dense_ref as ref  # noqa: E402
from tests.linear_variants import PRODUCTS, SHORT, WEIGHTS  # noqa: E402
from tests.rows_ref import BF16, U  # noqa: E402
from tests.test_rows_gpu import DT, _close, _dev, _f64, _gen, _gpu, _shifted  # noqa: E402,F401

pytestmark = pytest.mark.gpu
ACTS = [None, "relu", "gelu", "silu"]


def _rows8(q, scale):
    return spc.Rows8(q.cuda(), scale.cuda())


def _same(a, b, what=""):
    """Bit for bit, NaN at the same places."""
    a, b = a.cpu(), b.cpu()
    a, b = (t.view(torch.uint8) if t.dtype == ref.F8 else t for t in (a, b))
    assert a.shape == b.shape and a.dtype == b.dtype, what
    assert torch.equal(torch.isnan(a), torch.isnan(b)) if a.is_floating_point() else True, what
    assert bool(((a == b) | (a != a)).all()), what


def _off(got, want, bound, what):
    """|got - want| within the bound (and half a rounding to got's type)."""
    bound = bound + (BF16 * want.abs() if got.dtype == torch.bfloat16 else 0.0) + 1e-36
    d = (got.detach().cpu().double() - want).abs()
    bad = ~(d <= bound)
    assert tuple(got.shape) == tuple(want.shape) and not bad.any(), (
        what, int(bad.sum()), float((d / bound).max()))


# ---------------------------------------------------------------------------
# Rows in 8 bits
# ---------------------------------------------------------------------------
WIDTHS = [(1, 1), (1, 7), (5, 8), (461, 16), (33, 24), (100, 64), (7, 100), (3, 129), (257, 145),
          (2, 512), (9, 513), (4, 1000), (3, 2048), (2, 2050), (3, 4100), (2, 8192), (2, 8200),
          (1, 20001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", WIDTHS)
def test_pack_and_unpack(n, C, dtype):
    r, dt = _gen(n * 31 + C), DT[dtype]
    x = (r(n, C) * torch.exp(4 * r(n, 1))).to(dt)
    q, scale = ref.packed(x)
    for given in (x.cuda(), _shifted(x), x.t().contiguous().cuda().t()):
        got = spc.pack_rows(given)
        _same(got.q, q), _same(got.scale, scale)
    z = ref.stands_for(q, scale)
    for act in ACTS:
        for out in (torch.float32, torch.bfloat16):
            y = spc.unpack_rows(got, out, act=act)
            _off(y, ref.act(z, act), 9 * U * z.abs(), ("unpack", act))
    y = spc.unpack_rows(spc.Rows8(_shifted(q.view(torch.uint8)).view(ref.F8), scale.cuda()))
    _same(y, (q.float() * scale[:, None]).bfloat16(), "unpack shifted")


def test_every_code_of_eight_bits():
    q = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(1, 256).view(ref.F8)
    y = spc.unpack_rows(_rows8(q, torch.ones(1)), torch.float32)
    _same(y, q.float())
    # as an operand: the identity brings every code through the matrix cores and the vector ALU
    eye = torch.eye(256).bfloat16().cuda()
    fine = torch.where(torch.isnan(q.float()), torch.zeros(()), q.float()).to(ref.F8)
    for n in (1, 100):
        y, _ = spc.linear_forward(_rows8(fine.repeat(n, 1), torch.ones(n)), eye,
                                  out_dtype=torch.float32)
        assert torch.equal(y.cpu(), fine.float().repeat(n, 1)), n
    dw, _ = spc.linear_backward_weight(_rows8(fine.t().contiguous(), torch.ones(256)), eye)
    assert torch.equal(dw.cpu(), fine.float())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pack_of_rows_that_are_not_finite_or_tiny(dtype):
    x = torch.randn(8, 40, generator=torch.Generator().manual_seed(1))
    x[1, 7] = math.inf
    x[2, 39] = math.nan
    x[3] = 0
    x[4] *= 2.0 ** -120
    x[5] *= 2.0 ** 120
    x[6, 0] = -math.inf
    x = x.to(DT[dtype])
    q, scale = ref.packed(x)
    assert torch.isnan(scale[[1, 2, 6]]).all() and torch.isfinite(scale[[0, 3, 4, 5, 7]]).all()
    got = spc.pack_rows(x.cuda())
    _same(got.q, q), _same(got.scale, scale)
    y = spc.unpack_rows(got, torch.float32)
    assert torch.isnan(y[[1, 2, 6]]).all() and torch.isfinite(y[[0, 3, 4, 5, 7]]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(1, 1), (3, 7), (461, 16), (100, 64), (257, 145), (5, 1000), (2, 20001)])
def test_activation_backward(n, C, dtype):
    r, dt = _gen(n + C), DT[dtype]
    z, dy = r(n, C, std=3.0, dtype=dt), r(n, C, dtype=dt)
    q, scale = ref.packed(z)
    for act in ACTS:
        for pre, v in ((z.cuda(), _f64(z)), (_shifted(z), _f64(z)),
                       (_rows8(q, scale), (q.float() * scale[:, None]).double())):
            dz = spc.activation_backward(dy.cuda(), pre, act)
            _off(dz, _f64(dy) * ref.slope(v, act), (34 + 2 * v.abs()) * U * _f64(dy).abs(), act)
    d = dy.cuda()
    want = spc.activation_backward(d.clone(), z.cuda(), "gelu")
    assert spc.activation_backward(d, z.cuda(), "gelu", out=d) is d and torch.equal(d, want)
    big = torch.tensor([[-3e38, -1e20, -200.0, -0.0, 0.0, 200.0, 1e20, 3e38]]).to(dt).cuda()
    one = torch.ones_like(big)
    for act in ("gelu", "silu"):
        s = spc.activation_backward(one, big, act).cpu().float()
        assert s[0, :3].abs().max() == 0 and (s[0, 3:5] == 0.5).all() and (s[0, 5:] == 1).all(), act


# ---------------------------------------------------------------------------
# RMS norm
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", WIDTHS)
def test_rms_norm(n, C, dtype):
    r, dt, eps = _gen(n * 37 + C), DT[dtype], 1e-5
    x, res = r(n, C, std=1.5, dtype=dt), (r(n, C) * (0.2 + r(n, 1).abs())).to(dt)
    dy, dh = r(n, C, dtype=dt), r(n, C, dtype=dt)
    for gamma, residual in ((r(C, std=0.3, mean=1.0), res), (None, None), (r(C), None), (None, res)):
        h = x if residual is None else (x.float() + residual.float()).to(dt)
        want, rstd = ref.rms(_f64(h), _f64(gamma), eps)
        # rstd: half the sum's error; y: two products more
        tol = (C / 2 + 24) * U
        given = (x.cuda(), _dev(residual)) if n % 2 else (_shifted(x), residual if residual is None
                                                         else _shifted(residual))
        y, s, rs = spc.rms_norm_forward(given[0], _dev(gamma), eps, residual=given[1])
        assert s is given[0] if residual is None else True
        _same(s, h, "sum")
        _off(rs, rstd, tol * rstd, "rstd")
        _off(y, want, tol * want.abs(), "y")
        y8, s8, rs8 = spc.rms_norm_forward(given[0], _dev(gamma), eps, residual=given[1], packed=True)
        _same(s8, h, "sum, packed")
        _same(rs8, rs, "rstd, packed")
        top = want.abs().amax(1)
        _off(y8.scale, top / ref.TOP, (tol + 2 * U) * top / ref.TOP, "scale")
        back = ref.stands_for(y8.q.cpu(), y8.scale.cpu())
        bound = torch.maximum(want.abs() / 16, (top / ref.TOP)[:, None] / 1024) * (1 + 1e-4)
        assert bool(((back - want).abs() <= bound + 4 * tol * top[:, None]).all()), "8 bits"
        assert y8.q.cpu().float().abs().amax(1).eq(448).all()
        # gradients, for the statistics given
        rstd = rs.cpu()
        h8 = ref.packed(h)
        for kept, hv in ((s, _f64(h)), (_rows8(*h8), ref.stands_for(*h8))):
            for more in (None, dh):
                (dx, dg), (mx, mg) = ref.rms_grad(_f64(dy), hv, _f64(rstd), _f64(gamma), _f64(more))
                gx, gg = spc.rms_norm_backward(dy.cuda(), kept, rs, _dev(gamma), dh=_dev(more),
                                               params=True)
                _close(gx, dx, mx, 2 * C, "dx")
                _close(gg, dg, mg, n, "dgamma")
                gx2, none = spc.rms_norm_backward(dy.cuda(), kept, rs, _dev(gamma), dh=_dev(more),
                                                  params=False)
                assert none is None
                _same(gx2, gx, "dx alone")


def test_rms_norm_of_many_rows_and_none():
    r = _gen(5)
    for n, C, dtype in ((40000, 16, "bf16"), (33333, 20, "f32"), (0, 8, "bf16")):
        dt = DT[dtype]
        x, dy, g = r(n, C, dtype=dt), r(n, C, dtype=dt), r(C)
        y, h, rs = spc.rms_norm_forward(x.cuda(), g.cuda())
        want, _ = ref.rms(_f64(x), _f64(g), 1e-6)
        _off(y, want, (C + 24) * U * want.abs(), "y")
        (dx, dg), (mx, mg) = ref.rms_grad(_f64(dy), _f64(x), _f64(rs.cpu()), _f64(g), None)
        gx, gg = spc.rms_norm_backward(dy.cuda(), h, rs, g.cuda())
        _close(gx, dx, mx, 2 * C, "dx")
        _close(gg, dg, mg, n, "dgamma")
        again = spc.rms_norm_backward(dy.cuda(), h, rs, g.cuda())
        assert torch.equal(gg, again[1]) and torch.equal(gx, again[0])
        q = spc.rms_norm_forward(x.cuda(), packed=True, stats=False)
        assert q[2] is None and tuple(q[0].q.shape) == (n, C) and tuple(q[0].scale.shape) == (n,)
        p = spc.pack_rows(x.cuda())
        assert tuple(spc.unpack_rows(p).shape) == (n, C)


@pytest.mark.parametrize("n,C", [(37, 24), (5, 145), (3, 2048), (2, 9001)])
def test_rms_norm_in_place_of_the_stream(n, C):
    r = _gen(C)
    x, res = r(n, C).cuda(), r(n, C).cuda()
    for packed in (False, True):
        want = spc.rms_norm_forward(x, residual=res, packed=packed)
        for which in range(2):
            a, b = x.clone(), res.clone()
            y, h, rs = spc.rms_norm_forward(a, residual=b, packed=packed, sum_out=(a, b)[which])
            assert h is (a, b)[which]
            _same(h, want[1]), _same(rs, want[2])
            assert torch.equal((b, a)[which], (res, x)[which])
            for p, q in zip((y.q, y.scale) if packed else (y,),
                            (want[0].q, want[0].scale) if packed else (want[0],)):
                _same(p, q)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rms_norm_keeps_what_is_not_finite_in_its_row(dtype):
    r, dt = _gen(8), DT[dtype]
    for C in (24, 300, 5000):
        x = r(6, C, dtype=dt)
        clean = spc.rms_norm_forward(x.cuda(), packed=True)
        plain = spc.rms_norm_forward(x.cuda())[0]
        x[1, 3], x[4, C - 1] = math.nan, math.inf
        got = spc.rms_norm_forward(x.cuda(), packed=True)
        y = spc.rms_norm_forward(x.cuda())[0]
        rest = [0, 2, 3, 5]
        assert torch.equal(y[rest], plain[rest])
        assert torch.equal(got[0].q[rest].view(torch.uint8), clean[0].q[rest].view(torch.uint8))
        assert torch.isnan(got[0].scale[[1, 4]]).all() and torch.isnan(y[1]).all()
        assert torch.equal(got[0].scale[rest], clean[0].scale[rest])


# ---------------------------------------------------------------------------
# Dense products
# ---------------------------------------------------------------------------
def _operands(dt, n, ci, co, seed):
    """x as given, as float64 with its Rows8 if it has; w, bias, residual."""
    r = _gen(seed)
    d = torch.float32 if dt == "f32" else torch.bfloat16
    x, w, b = r(n, ci, dtype=d), r(ci, co, std=ci ** -0.5, dtype=d), r(co)
    if dt != "e4m3":
        return x.cuda(), _f64(x), w, b, d
    x = x * torch.exp(r(n, 1))
    q, s = ref.packed(x)
    return _rows8(q, s), ref.stands_for(q, s), w, b, d


@pytest.mark.parametrize("backward,n,red,cols,stages,residual", SHORT)
def test_products_that_keep_their_weights(backward, n, red, cols, stages, residual):
    """Sums as in test_products; rows in front of y and behind it stay as they are, a row of infinities
    and NaN reaches no other."""
    ci, co = (cols, red) if backward else (red, cols)
    x, _, w, b, d = _operands("bf16", n, ci, co, n + red)
    rows = (_gen(n)(n, co, dtype=d) if backward else x.cpu()).clone()
    bad = n // 2
    rows[bad, 0], rows[bad, red - 1] = float("inf"), float("nan")
    good = torch.arange(n) != bad
    clean = rows.clone()
    clean[bad] = 0
    rows, w_, b_ = rows.cuda(), w.cuda(), b.cuda()
    frame = torch.full((n + 16, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    y = frame[8:n + 8]
    wt = _f64(w).t() if backward else _f64(w)
    z, mag = _f64(clean) @ wt, _f64(clean).abs() @ wt.abs()
    if backward:
        assert spc.linear_backward_data(rows, w_, out=y) is y
        _off(y[good], z[good], (red + 34) * U * mag[good], "dx")
        assert bool(torch.isnan(y[bad]).any())
    else:
        big = n * cols > 3e6
        res = _gen(n + 1)(n, cols, dtype=d) if residual else None
        calls = [(a, keep, bias) for a in ACTS for keep in (False, True) for bias in (None, b)]
        for act, keep, bias in [(None, False, b), ("gelu", True, b), ("silu", False, None)] if big else calls:
            v, m = (z, mag) if bias is None else (z + _f64(bias), mag + _f64(bias).abs())
            ez, a = (red + 34) * U * m, ref.act(v, act)
            for r in (None, res) if residual else (None,):
                s = a if r is None else a + _f64(r)
                if r is not None and keep:               # in place of the residual
                    y.copy_(r)
                got, pre = spc.linear_forward(rows, w_, None if bias is None else b_, act=act, pre=keep,
                                              residual=None if r is None else y if keep else r.cuda(), out=y)
                assert got is y and (pre is not None) == keep
                _off(y[good], s[good], (1.13 * ez + 8 * U * v.abs() + 2 * U * s.abs())[good], ("y", act))
                if keep:
                    _off(pre[good], v[good], ez[good], "z")
    assert bool((frame[:8] == 7).all()) and bool((frame[n + 8:] == 7).all())


@pytest.mark.parametrize("dt,backward,n,red,cols,want", PRODUCTS)
def test_products(dt, backward, n, red, cols, want):
    ci, co = (cols, red) if backward else (red, cols)
    big = n > 10000
    x, xv, w, b, d = _operands(dt, n, ci, co, n + red)
    r = _gen(n)
    side = r(n, cols)
    outs = [d] if big else [torch.float32, torch.bfloat16]
    if not backward:
        z, mag = ref.linear(xv, _f64(w), _f64(b))
        ez = (red + 34) * U * mag
        for act in ACTS:
            for out in outs:
                res = side.to(out)
                y, pre = spc.linear_forward(x, w.cuda(), b.cuda(), act=act, residual=res.cuda(),
                                            pre=True, out_dtype=out)
                v = ref.act(z, act) + _f64(res)
                _off(pre, z, ez, ("z", act))
                _off(y, v, 1.13 * ez + 8 * U * z.abs() + 2 * U * v.abs(), ("y", act))
                if act == "silu":
                    bare, none = spc.linear_forward(x, w.cuda(), act=act, out_dtype=out)
                    assert none is None
                    z0, mag0 = ref.linear(xv, _f64(w), None)
                    _off(bare, ref.act(z0, act), 1.13 * (red + 34) * U * mag0 + 9 * U * z0.abs(), "bare")
                    o = res.cuda()
                    got, _ = spc.linear_forward(x, w.cuda(), b.cuda(), act=act, residual=o, out=o,
                                                out_dtype=out)
                    assert got is o and torch.equal(o, y), "in place of the residual"
    else:
        dy = r(n, co, dtype=d)
        g, mag = _f64(dy) @ _f64(w).t(), _f64(dy).abs() @ _f64(w).abs().t()
        eg = (red + 34) * U * mag
        for act in ACTS:
            for out in outs:
                p = (3 * side).to(out)
                q, s = ref.packed(p)
                kept = [(None, torch.zeros_like(g))] if act is None else [
                    (p.cuda(), _f64(p)), (_rows8(q, s), (q.float() * s[:, None]).double())]
                for pre, pv in kept:
                    dx = spc.linear_backward_data(dy.cuda(), w.cuda(), act=act, pre=pre, out_dtype=out)
                    sl = ref.slope(pv, act)
                    _off(dx, g * sl, 1.13 * eg + (34 + 2 * pv.abs()) * U * g.abs(), ("dx", act))


@pytest.mark.parametrize("dt", ["f32", "bf16", "e4m3"])
def test_products_of_unaligned_and_strided_operands(dt):
    n, ci, co = 70, 48, 72
    x, xv, w, b, d = _operands(dt, n, ci, co, 4)
    want, z = spc.linear_forward(x, w.cuda(), b.cuda(), act="gelu", pre=True)
    odd = spc.Rows8(_shifted(x.q.cpu().view(torch.uint8)).view(ref.F8), x.scale) if dt == "e4m3" \
        else _shifted(x.cpu())
    zv, mag = ref.linear(xv, _f64(w), _f64(b))
    for xx, ww in ((odd, w.cuda()), (x, _shifted(w)), (odd, _shifted(w)),
                   (x, w.t().contiguous().cuda().t())):
        y, z = spc.linear_forward(xx, ww, b.cuda(), act="gelu", pre=True)
        _off(z, zv, (ci + 34) * U * mag, "z")
    dy = _gen(1)(n, co, dtype=d)
    dx = spc.linear_backward_data(dy.cuda(), w.cuda())
    g, gm = _f64(dy) @ _f64(w).t(), _f64(dy).abs() @ _f64(w).abs().t()
    for a, c in ((dy.cuda(), w.cuda()), (_shifted(dy), w.cuda()), (dy.cuda(), _shifted(w))):
        _off(spc.linear_backward_data(a, c), g, (co + 34) * U * gm, "dx")
    assert dx.shape == (n, ci)


@pytest.mark.parametrize("dt", ["f32", "bf16", "e4m3"])
def test_products_keep_what_is_not_finite_in_its_row(dt):
    for n, ci, co in ((40, 32, 64), (3, 64, 2048), (65600, 16, 160), (50, 33, 70)):
        x, _, w, b, d = _operands(dt, n, ci, co, 9)
        clean, _ = spc.linear_forward(x, w.cuda(), b.cuda(), act="silu")
        if dt == "e4m3":
            x.scale[1] = math.nan
        else:
            x[1, 3] = math.nan
        y, _ = spc.linear_forward(x, w.cuda(), b.cuda(), act="silu")
        assert torch.isnan(y[1]).all()
        assert torch.equal(y[0], clean[0]) and torch.equal(y[2:], clean[2:])


def _weight_bound(xv, dyv, n, x8, scale):
    mag = xv.abs().t() @ dyv.abs()
    bound = (n + 32) * U * mag
    if x8:
        s = scale.double()[:, None]
        q = (xv / s).abs().amax(0)[:, None]
        bound = bound + 2.0 ** -22 * mag + 2.0 ** -39 * n * q * (s * dyv).abs().max()
    return bound


@pytest.mark.parametrize("dt,n,ci,co,tile", WEIGHTS)
def test_weight_gradients(dt, n, ci, co, tile):
    x, xv, _, _, d = _operands(dt, n, ci, co, n + ci)
    dy = _gen(n + 1)(n, co, dtype=d)
    dw, db = spc.linear_backward_weight(x, dy.cuda())
    scale = x.scale.cpu() if dt == "e4m3" else None
    _off(dw, xv.t() @ _f64(dy), _weight_bound(xv, _f64(dy), n, dt == "e4m3", scale), "dw")
    _off(db, _f64(dy).sum(0), (n + 32) * U * _f64(dy).abs().sum(0), "db")
    again, none = spc.linear_backward_weight(x, dy.cuda(), bias=False)
    assert none is None and torch.equal(again, dw)
    if dt != "e4m3":
        odd, _ = spc.linear_backward_weight(_shifted(x.cpu()), _shifted(dy))
        _off(odd, xv.t() @ _f64(dy), _weight_bound(xv, _f64(dy), n, False, None), "dw, unaligned")


def test_weight_gradient_of_8_bit_rows_over_all_sizes_of_factors():
    """Rows that grow and shrink along a chunk, columns of very different sizes, gradients far below
    f16's range, rows and gradients that are not finite."""
    n, ci, co = 1500, 40, 70
    r = _gen(2)
    for shift in (-100.0, -20.0, 0.0, 60.0):
        x = r(n, ci) * torch.exp2(10 * torch.sin(torch.arange(n) / 40.0))[:, None]
        dy = (r(n, co) * torch.exp2(shift - torch.arange(co) / 8.0) *
              torch.exp2(torch.arange(n) / 200.0)[:, None]).bfloat16()
        q, s = ref.packed(x)
        xv = ref.stands_for(q, s)
        dw, db = spc.linear_backward_weight(_rows8(q, s), dy.cuda())
        _off(dw, xv.t() @ _f64(dy), _weight_bound(xv, _f64(dy), n, True, s), shift)
        _off(db, _f64(dy).sum(0), (n + 32) * U * _f64(dy).abs().sum(0), "db")
    # a gradient that is not finite stays in its column
    bad = dy.clone()
    bad[700, 5] = math.inf
    bad[100, 6] = math.nan
    got, _ = spc.linear_backward_weight(_rows8(q, s), bad.cuda())
    rest = [c for c in range(co) if c not in (5, 6)]
    assert torch.equal(got[:, rest], dw[:, rest])
    assert torch.isnan(got[:, 6]).all() and not torch.isfinite(got[:, 5]).any()
    # zeros, and no rows at all
    dw, db = spc.linear_backward_weight(_rows8(q, s), torch.zeros_like(dy).cuda())
    assert not dw.any() and not db.any()
    for d in (torch.float32, torch.bfloat16):
        e = torch.empty(0, 8, dtype=d, device="cuda")
        dw, db = spc.linear_backward_weight(e, torch.empty(0, 12, dtype=d, device="cuda"))
        assert dw.shape == (8, 12) and not dw.any() and not db.any()
        w = torch.ones(8, 12, dtype=d, device="cuda")
        assert spc.linear_forward(e, w)[0].shape == (0, 12)
        assert spc.linear_backward_data(torch.empty(0, 12, dtype=d, device="cuda"), w).shape == (0, 8)


def test_gradients_of_a_layer_against_differences():
    """A norm, two products and an activation in fp32: the gradients the operators give, against
    differences of the 64-bit statements along one direction of every operand.  Each side is off by
    its tolerance's share, below 1e-4 of the sum of the products' magnitudes."""
    r, n, c, m = _gen(12), 30, 24, 40
    x, res, g = r(n, c), r(n, c), r(c, std=0.2, mean=1.0)
    w1, b1, w2 = r(c, m, std=c ** -0.5), r(m), r(m, c, std=m ** -0.5)
    dy = r(n, c)

    def layer(x, res, g, w1, b1, w2):
        h = x + res
        z = ref.rms(h, g, 1e-6)[0] @ w1 + b1
        return ref.act(z, "gelu") @ w2 + h
    dev = [t.cuda() for t in (x, res, g, w1, b1, w2)]
    y1, h, rs = spc.rms_norm_forward(dev[0], dev[2], residual=dev[1])
    a, z = spc.linear_forward(y1, dev[3], dev[4], act="gelu", pre=True)
    out, _ = spc.linear_forward(a, dev[5], residual=h)
    d = dy.cuda()
    dz = spc.linear_backward_data(d, dev[5], act="gelu", pre=z)
    dw2, _ = spc.linear_backward_weight(a, d)
    dw1, db1 = spc.linear_backward_weight(y1, dz)
    dx, dg = spc.rms_norm_backward(spc.linear_backward_data(dz, dev[3]), h, rs, dev[2], dh=d)
    args = [_f64(t) for t in (x, res, g, w1, b1, w2)]
    assert torch.allclose(out.cpu().double(), layer(*args), rtol=1e-4, atol=1e-4)
    for i, grad in enumerate((dx, dx, dg, dw1, db1, dw2)):
        v = torch.randn(args[i].shape, dtype=torch.float64, generator=torch.Generator().manual_seed(i))
        lo, hi = ([t + (e * v if j == i else 0) for j, t in enumerate(args)] for e in (-1e-6, 1e-6))
        num = ((layer(*hi) - layer(*lo)) / 2e-6 * _f64(dy)).sum()
        own = grad.cpu().double() * v
        assert abs(float(own.sum() - num)) <= 1e-4 * float(own.abs().sum()), i


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------
def _block(x, stream, g, w1, b1, w2, b2, wr, balance, we, dy):
    """A dense layer and routed experts beside it, forwards and backwards, kept in 8 bits."""
    n8, h, rs = spc.rms_norm_forward(x, g, residual=stream, packed=True)
    lg, _ = spc.linear_forward(n8, wr, out_dtype=torch.float32)
    q = spc.route_scores_forward(lg, 2, bias=balance, groups=4, top_groups=2, scale=2.5)
    a, z = spc.linear_forward(n8, w1, b1, act="silu", pre=True)
    y, _ = spc.linear_forward(a, w2, b2, residual=h)
    n = spc.unpack_rows(n8)
    e = spc.grouped_forward(n, we, q.offsets, rows=q.rows)
    y = spc.combine_forward(e, q.pos, q.weights, residual=y)
    z8, h8 = spc.pack_rows(z), spc.pack_rows(h)
    de, dwt = spc.combine_backward(dy, e, q.pos, q.weights, offsets=q.offsets)
    dwe, _ = spc.grouped_backward_weight(n, de, q.offsets, rows=q.rows, bias=False)
    dn = spc.combine_forward(spc.grouped_backward_data(de, we, q.offsets), q.pos)
    dl = spc.route_scores_backward(dwt, lg, q.experts, q.weights, scale=2.5)
    a2 = spc.unpack_rows(z8, act="silu")
    dw2, db2 = spc.linear_backward_weight(a2, dy)
    dz = spc.linear_backward_data(dy, w2, act="silu", pre=z8)
    dw1, db1 = spc.linear_backward_weight(n8, dz)
    dwr, _ = spc.linear_backward_weight(n8, dl.bfloat16(), bias=False)
    dn = spc.linear_backward_data(dz, w1) + dn + spc.linear_backward_data(dl.bfloat16(), wr)
    dx, dg = spc.rms_norm_backward(dn, h8, rs, g, dh=dy)
    return [y, h, n8.q, n8.scale, lg, q.experts, q.weights, q.offsets, q.rows, dwe, dl, dw2, db2,
            dw1, db1, dwr, dx, dg]


def _block_operands(n, c, m, E, seed):
    r, bf = _gen(seed), torch.bfloat16
    return [t.cuda() for t in (
        r(n, c, dtype=bf), r(n, c, dtype=bf), r(c, std=0.2, mean=1.0),
        r(c, m, std=c ** -0.5, dtype=bf), r(m), r(m, c, std=m ** -0.5, dtype=bf), r(c),
        r(c, E, std=c ** -0.5, dtype=bf), r(E, std=0.05), r(E, c, c, std=c ** -0.5, dtype=bf),
        r(n, c, dtype=bf))]


def _equal(got, want, what):
    for i, (a, b) in enumerate(zip(got, want)):
        a, b = (t.view(torch.uint8) if t.dtype == ref.F8 else t for t in (a, b))
        assert torch.equal(a, b), (what, i)


@pytest.mark.parametrize("n,c,m,E", [(1, 64, 256, 8), (37, 24, 40, 8), (3000, 64, 200, 16)])
def test_a_block_in_a_captured_graph_and_on_another_stream(n, c, m, E):
    """Captured once and replayed on new inputs, eager work between: every replay equals the eager
    block; and so does the block on a stream of its own, with calls of another on the first."""
    t = _block_operands(n, c, m, E, 1)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _block(*t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _block(*t)
    for i in range(4):
        for a, b in zip(t, _block_operands(n, c, m, E, 10 + i)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        out = [v.clone() for v in got]
        want = _block(*t)
        torch.cuda.synchronize()
        _equal(out, want, ("replay", i))
    other = _block_operands(n, c, m, E, 50)
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = _block(*t)
    b = _block(*other)
    torch.cuda.synchronize()
    _equal(a, want, "side")
    _equal(b, _block(*other), "first")


def test_the_stream_argument():
    t = _block_operands(50, 64, 96, 8, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    n8, h, rs = spc.rms_norm_forward(t[0], t[2], residual=t[1], packed=True, stream=side)
    y, z = spc.linear_forward(n8, t[3], t[4], act="gelu", pre=True, stream=side)
    z8 = spc.pack_rows(z, stream=side)
    dz = spc.activation_backward(y, z8, "gelu", stream=side)
    dw, db = spc.linear_backward_weight(n8, dz, stream=side)
    side.synchronize()
    m8, h2, rs2 = spc.rms_norm_forward(t[0], t[2], residual=t[1], packed=True)
    y2, z2 = spc.linear_forward(m8, t[3], t[4], act="gelu", pre=True)
    dz2 = spc.activation_backward(y2, spc.pack_rows(z2), "gelu")
    _equal([n8.q, h, rs, y, z, dz, dw, db],
           [m8.q, h2, rs2, y2, z2, dz2, *spc.linear_backward_weight(m8, dz2)], "stream")


def test_element_offsets_past_32_bits():
    """Rows beyond 2^32 elements of every operand that can be so long."""
    n, c = 2 ** 22 + 300, 1024
    far = slice(n - 200, n)
    x = torch.zeros((n, c), dtype=torch.bfloat16, device="cuda")
    r = _gen(6)
    v = r(200, c, dtype=torch.bfloat16)
    x[far] = v.cuda()
    q, s = ref.packed(v)
    p = spc.pack_rows(x)
    _same(p.q[far], q), _same(p.scale[far], s)
    y = spc.unpack_rows(p, act="silu")
    z = ref.stands_for(q, s)
    _off(y[far], ref.act(z, "silu"), 9 * U * z.abs(), "unpack")
    del y
    w = r(c, 8, std=1 / 32, dtype=torch.bfloat16)
    got, _ = spc.linear_forward(x, w.cuda())
    want, mag = ref.linear(_f64(v), _f64(w), None)
    _off(got[far], want, (c + 34) * U * mag, "linear")
    got, _ = spc.linear_forward(p, w.cuda())
    want, mag = ref.linear(z, _f64(w), None)
    _off(got[far], want, (c + 34) * U * mag, "linear of 8 bits")
    dy = torch.zeros((n, 8), dtype=torch.bfloat16, device="cuda")
    e = r(200, 8, dtype=torch.bfloat16)
    dy[far] = e.cuda()
    dw, db = spc.linear_backward_weight(x, dy)
    _off(dw, _f64(v).t() @ _f64(e), 232 * U * (_f64(v).abs().t() @ _f64(e).abs()), "dw")
    dw, db = spc.linear_backward_weight(p, dy)
    _off(dw, z.t() @ _f64(e), _weight_bound(z, _f64(e), 200, True, s), "dw of 8 bits")
    dx = spc.linear_backward_data(dy, w.cuda(), act="gelu", pre=x)
    g = _f64(e) @ _f64(w).t()
    vv = _f64(v)
    _off(dx[far], g * ref.slope(vv, "gelu"),
         1.13 * 42 * U * (_f64(e).abs() @ _f64(w).abs().t()) + (34 + 2 * vv.abs()) * U * g.abs(), "dx")
    del dx
    y, h, rs = spc.rms_norm_forward(x, eps=1e-5, residual=x)
    hv = _f64((v.float() * 2).bfloat16())
    want, _ = ref.rms(hv, None, 1e-5)
    _off(y[far], want, (c + 24) * U * want.abs(), "norm")
    dx, _ = spc.rms_norm_backward(x, h, rs, out=y)
    (want, _), (mx, _) = ref.rms_grad(_f64(v), hv, _f64(rs[far].cpu()), None, None)
    _close(dx[far], want, mx, 2 * c, "norm's dx")


def test_binding_refuses_what_does_not_fit():
    x, w = torch.randn(6, 8, device="cuda"), torch.randn(8, 4, device="cuda")
    p, b = spc.pack_rows(x), torch.ones(4, device="cuda")
    half = spc.Rows8(p.q, p.scale.half())
    bad = [(TypeError, lambda: spc.pack_rows(x.half())),
           (TypeError, lambda: spc.pack_rows(x.cpu())),
           (ValueError, lambda: spc.pack_rows(x[0])),
           (TypeError, lambda: spc.unpack_rows(x)),
           (TypeError, lambda: spc.unpack_rows(half)),
           (TypeError, lambda: spc.unpack_rows(spc.Rows8(p.q.view(torch.uint8), p.scale))),
           (ValueError, lambda: spc.unpack_rows(spc.Rows8(p.q, p.scale[:5]))),
           (TypeError, lambda: spc.unpack_rows(p, torch.float16)),
           (ValueError, lambda: spc.unpack_rows(p, act="tanh")),
           (ValueError, lambda: spc.unpack_rows(p, out=x)),
           (TypeError, lambda: spc.activation_backward(x, x.bfloat16(), "relu")),
           (TypeError, lambda: spc.activation_backward(x, p.q, "relu")),
           (ValueError, lambda: spc.activation_backward(x, spc.Rows8(p.q[:3], p.scale[:3]), "relu")),
           (ValueError, lambda: spc.activation_backward(x, x[:5], "relu")),
           (ValueError, lambda: spc.activation_backward(x, x, "swish")),
           (TypeError, lambda: spc.rms_norm_forward(x, residual=x.bfloat16())),
           (ValueError, lambda: spc.rms_norm_forward(x, residual=x[:5])),
           (ValueError, lambda: spc.rms_norm_forward(x, torch.ones(7, device="cuda"))),
           (ValueError, lambda: spc.rms_norm_forward(x, sum_out=x)),
           (ValueError, lambda: spc.rms_norm_forward(x, packed=True, out=x.clone())),
           (spc.SpconvError, lambda: spc.rms_norm_forward(x, eps=-1.0)),
           (TypeError, lambda: spc.rms_norm_backward(x, x.bfloat16(), x[:, 0].contiguous())),
           (ValueError, lambda: spc.rms_norm_backward(x, p, x[0])),
           (TypeError, lambda: spc.linear_forward(x, w.bfloat16())),
           (TypeError, lambda: spc.linear_forward(p, w)),
           (ValueError, lambda: spc.linear_forward(x, w.t())),
           (ValueError, lambda: spc.linear_forward(x, w, b[:3])),
           (TypeError, lambda: spc.linear_forward(x, w, b.bfloat16())),
           (ValueError, lambda: spc.linear_forward(x, w, act="tanh")),
           (TypeError, lambda: spc.linear_forward(x, w, out_dtype=torch.float16)),
           (TypeError, lambda: spc.linear_forward(x, w, residual=torch.ones(6, 4, device="cuda").bfloat16())),
           (ValueError, lambda: spc.linear_forward(x, w, residual=x)),
           (ValueError, lambda: spc.linear_backward_data(x, w)),
           (ValueError, lambda: spc.linear_backward_data(x[:, :4], w, act="relu")),
           (ValueError, lambda: spc.linear_backward_data(x[:, :4], w, pre=x)),
           (ValueError, lambda: spc.linear_backward_data(x[:, :4], w, act="relu", pre=x[:5])),
           (ValueError, lambda: spc.linear_backward_weight(x, x[:5])),
           (TypeError, lambda: spc.linear_backward_weight(p, x)),
           (ValueError, lambda: spc.route_scores_forward(x, 2, score="tanh")),
           (ValueError, lambda: spc.route_scores_forward(x, 2, bias=b)),
           (spc.SpconvError, lambda: spc.route_scores_forward(x, 2, groups=3)),
           (spc.SpconvError, lambda: spc.route_scores_forward(x, 3, groups=4, top_groups=1)),
           (spc.SpconvError, lambda: spc.route_scores_forward(x, 2, scale=0.0))]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            print("accepted", i)

"""Routing by sigmoid scores far from 0: renormalised weights and gradients where the scores
themselves are beyond fp32, and gradients where they are all but 1.

Weights: half a unit each for two arguments and a quotient, a unit for exp, k + 1 for the sum, less
than (k + 16) U of a weight.  Gradients: a weight, k of them in a sum (k + 1 more), a logistic
function and four products, less than (3 k + 48) U of the magnitudes."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_1706_01307_amd as spc  # noqa: E402
from tests.rows_ref import U  # noqa: E402
from tests.test_rows_gpu import DT, _gen, _gpu  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def _check(x, k, scale, dw):
    """x [n, E]: against the chosen scores in 64 bits, 0 from logits of -709.79 on, over their sum."""
    r = spc.route_scores_forward(x.cuda(), k, score="sigmoid", scale=scale)
    e = r.experts.cpu().long()
    assert bool((e >= 0).all())
    c = x.double().gather(1, e)
    s = 1 / (1 + torch.exp(-c))
    total = s.sum(1, keepdim=True)
    share = torch.where(total > 0, s / torch.where(total > 0, total, 1.0), 0.0)
    w, bf = share * scale, x.dtype == torch.bfloat16
    off = (r.weights.cpu().double() - w).abs()
    assert bool((off <= (k + 16) * U * w + 1e-37).all()), float((off / w).max() / U)
    d = spc.route_scores_backward(dw.cuda(), x.cuda(), r.experts, r.weights, score="sigmoid", scale=scale)
    d = d.cpu().double()
    g, back = dw.double() * scale, torch.sigmoid(-c)
    want = share * back * (g - (share * g).sum(1, keepdim=True))
    mag = share * back * (g.abs() + (share * g.abs()).sum(1, keepdim=True))
    got = d.gather(1, e)
    bound = (3 * k + 48) * U * mag + 1e-36 + (2.0 ** -8 * want.abs() if bf else 0.0)
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())
    assert torch.equal(d.scatter(1, e, torch.zeros_like(got)), torch.zeros_like(d))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1.0, 2.5])
def test_logits_far_below_0(scale, dtype):
    dt, r = DT[dtype], _gen(4)
    same = torch.full((1, 8), -100.0).to(dt)
    w = spc.route_scores_forward(same.cuda(), 2, scale=scale).weights
    assert w.cpu().tolist() == [[0.5 * scale] * 2]
    for E, k, lo, hi in ((2, 2, -89, -89), (8, 3, -90, -86), (16, 8, -300, -85), (64, 8, -110, -60),
                         (5, 5, -100, 5), (8, 8, -104, 0), (300, 16, -700, -90), (4, 4, -2000, -800),
                         (16, 4, -30, -15)):
        n = 50
        x = (lo + (hi - lo) * torch.rand(n, E, generator=torch.Generator().manual_seed(E))).to(dt)
        _check(x, k, scale, r(n, k))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite_beside_far_logits(dtype):
    x = torch.tensor([[-200.0, math.nan, -201.0], [-200.0, math.inf, -201.0],
                      [-200.0, -math.inf, -201.0], [-3e38, -200.0, -201.0]]).to(DT[dtype])
    r = spc.route_scores_forward(x.cuda(), 3, score="sigmoid")
    w, e = r.weights.cpu(), r.experts.cpu().tolist()
    assert torch.isnan(w[0]).all() and e[1] == [1, 0, 2] and w[1].tolist() == [1.0, 0.0, 0.0]
    two = torch.softmax(x[2, ::2].double(), 0)
    assert e[2] == [0, 2, -1] and bool(((w[2, :2].double() - two).abs() <= 20 * U).all()) and w[2, 2] == 0
    two = torch.softmax(x[3, 1:].double(), 0)
    assert e[3] == [1, 2, 0] and bool(((w[3, :2].double() - two).abs() <= 20 * U).all()) and w[3, 2] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("normalize", [True, False])
def test_gradient_of_scores_all_but_1(normalize, dtype):
    """The slope s (1 - s) of a score next to 1 keeps the bits of 1 - s."""
    n, E, k, scale = 60, 16, 4, 2.5
    x = (5 + 75 * torch.rand(n, E, generator=torch.Generator().manual_seed(2))).to(DT[dtype])
    dw = _gen(3)(n, k)
    if normalize:
        return _check(x, k, scale, dw)
    r = spc.route_scores_forward(x.cuda(), k, scale=scale, normalize=False)
    d = spc.route_scores_backward(dw.cuda(), x.cuda(), r.experts, r.weights, scale=scale, normalize=False)
    c = x.double().gather(1, r.experts.cpu().long())
    want = dw.double() * scale * torch.sigmoid(c) * torch.sigmoid(-c)
    got = d.cpu().double().gather(1, r.experts.cpu().long())
    bound = (16 * U + (2.0 ** -8 if dtype == "bf16" else 0.0)) * want.abs() + 1e-36
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("normalize", [True, False])
def test_rows_closed_by_the_lowest_number(normalize, dtype):
    """A row of the type's lowest value has scores of 0 and weights of 0; beside an open expert such ones
    weigh nothing; no gradient reaches them."""
    low = torch.finfo(DT[dtype]).min
    x = torch.full((3, 8), low).to(DT[dtype])
    x[1, 5], x[2, 2], x[2, 6] = -95.0, -709.0, -720.0
    r = spc.route_scores_forward(x.cuda(), 2, normalize=normalize)
    w = r.weights.cpu()
    assert r.experts.cpu().tolist() == [[0, 1], [5, 0], [2, 0]]
    assert w.tolist() == ([[0, 0], [1, 0], [1, 0]] if normalize else [[0, 0], [w[1, 0], 0], [0, 0]])
    d = spc.route_scores_backward(torch.ones(3, 2, device="cuda"), x.cuda(), r.experts, r.weights,
                                  normalize=normalize).cpu()
    d[1, 5] = 0
    assert not d.any()

"""GPU parity of the routing by scores: the choice and the order of the pairs exactly, weights and
gradients within fp32's roundings (a score: 4 units for exp and a division; a sum of k of them; a
division: (k + 16) U of the magnitudes)."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_1706_01307_amd as spc  # noqa: E402
from tests import rows_dense_ref as ref  # noqa: E402
from tests.rows_ref import U  # noqa: E402
from tests.test_rows_gpu import DT, _gen, _gpu  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def _check_pairs(r, experts, E):
    n, k = experts.shape
    flat = experts.reshape(-1)
    order = torch.argsort(torch.where(flat < 0, E, flat), stable=True)
    used = int((flat >= 0).sum())
    pos, rows = torch.full_like(flat, -1), torch.full_like(flat, -1)
    pos[order[:used]] = torch.arange(used)
    rows[:used] = order[:used] // k
    off = torch.zeros(E + 1, dtype=torch.int64)
    off[1:] = torch.bincount(flat[flat >= 0], minlength=E).cumsum(0)
    for got, want in ((r.experts, experts), (r.pos, pos.view(n, k)), (r.rows, rows), (r.offsets, off)):
        assert torch.equal(got.cpu().long(), want)


# Both sides have a score in 64 bits, off by at most 4 units of 2^-53 (exp, an addition, a division,
# the bias), and a group's worth, below 4, by 4 units of each of its two and its own sum's: 2 * 4 + 2
# units on either side, 20 in all: within 2^-48 two groups of different scores have no order.
NO_ORDER = 2.0 ** -48


def _settled(want, got, x, bias, kind, groups, top_groups):
    """`want`, with the rows of `got` where 64 bits do not order the groups that decide: there every
    group that was chosen from is worth as much as the last that stays, within NO_ORDER."""
    if groups == 1 or torch.isnan(x).any():
        return want
    v = ref.scores(x, kind) + (0 if bias is None else bias.double())
    v = v.masked_fill(x.double() == -math.inf, -math.inf)
    worth = v.view(len(x), groups, -1).topk(min(2, x.shape[1] // groups), 2).values
    none = worth == -math.inf
    worth = worth.masked_fill(none, 0.0).sum(2).masked_fill(none[:, :, 0], -math.inf)
    ranked = torch.sort(worth, 1, descending=True).values
    last = ranked[:, top_groups - 1]
    open_ = (top_groups < groups) & ((last - ranked[:, min(top_groups, groups - 1)]) <= NO_ORDER)
    of = worth.gather(1, got.clamp(min=0) // (x.shape[1] // groups))
    fits = ((of >= last[:, None] - NO_ORDER) | (got < 0)).all(1)
    return torch.where((open_ & fits)[:, None], got, want)


def _check(x, bias, k, groups=1, top_groups=1, kinds=("sigmoid", "softmax")):
    E = x.shape[1]
    dw = _gen(7)(x.shape[0], k)
    for kind in kinds:
        want = ref.choose(x, bias, kind, groups, top_groups, k)
        for normalize, scale in ((True, 1.0), (False, 2.5)):
            r = spc.route_scores_forward(x.cuda(), k, score=kind, groups=groups, scale=scale,
                                         bias=None if bias is None else bias.cuda(),
                                         top_groups=top_groups, normalize=normalize)
            want = _settled(want, r.experts.cpu().long(), x, bias, kind, groups, top_groups)
            _check_pairs(r, want, E)
            w = ref.weights(x, want, kind, normalize, scale)
            units = k + 16 + (E if kind == "softmax" else 0)
            ok = (r.weights.cpu().double() - w).abs() <= units * U * w.abs() + 1e-37
            assert bool((ok | (torch.isnan(w) & torch.isnan(r.weights.cpu()))).all()), (kind, normalize)
            if torch.isnan(w).any():
                continue
            d = spc.route_scores_backward(dw.cuda(), x.cuda(), r.experts, r.weights, score=kind,
                                          normalize=normalize, scale=scale)
            g, mag = ref.weights_grad(x, want, kind, normalize, scale, dw.double())
            # (1 - s, and s where it is near 1, are off by U: a unit of s, not of 1 - s)
            bound = (2 * units + 32) * U * mag + (U * 8 * scale * dw.double().abs().amax(1, keepdim=True)
                                                  if kind == "sigmoid" else 0)
            if x.dtype == torch.bfloat16:
                bound = bound + 2.0 ** -8 * g.abs()
            assert bool(((d.cpu().double() - g).abs() <= bound + 1e-37).all()), (kind, normalize)


CASES = [(1, 1, 1, 1, 1), (3, 2, 1, 1, 1), (50, 5, 3, 1, 1), (33, 8, 2, 4, 2), (40, 16, 4, 4, 2),
         (20, 24, 6, 8, 3), (64, 30, 8, 5, 3), (9, 64, 8, 8, 4), (7, 66, 8, 6, 2), (5, 64, 16, 64, 20),
         (4, 100, 8, 10, 3), (3, 256, 8, 16, 4), (3, 250, 4, 2, 1), (2, 511, 8, 7, 3),
         (2, 1024, 16, 32, 4), (2, 1023, 3, 33, 9)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,E,k,groups,top_groups", CASES)
def test_choices(n, E, k, groups, top_groups, dtype):
    r = _gen(n * 7 + E)
    x = (r(n, E) * 1.5 + r(E, std=0.7)).to(DT[dtype])
    _check(x, r(E, std=0.1), k, groups, top_groups)
    _check(x, None, k, groups, top_groups)
    x = x.masked_fill(torch.rand(n, E, generator=torch.Generator().manual_seed(E)) < 0.4, -math.inf)
    x[n // 2] = -math.inf
    _check(x, r(E, std=0.1), k, groups, top_groups)


@pytest.mark.parametrize("groups,top_groups", [(1, 1), (4, 2), (16, 5)])
def test_scores_next_to_one_another(groups, top_groups):
    """Logits a few units of fp32 apart, and equal ones: the order is that of 64 bits."""
    n, E, k = 200, 32, 6
    g = torch.Generator().manual_seed(5)
    base = torch.randn(n, 1, generator=g)
    step = torch.randint(-2, 3, (n, E), generator=g)
    x = (base.view(torch.int32) + step.int()).view(torch.float32)
    _check(x, None, k, groups, top_groups)
    _check(x, torch.zeros(E), k, groups, top_groups)
    _check(x, torch.randint(0, 3, (E,), generator=g) * 2.0 ** -24, k, groups, top_groups)
    _check(torch.zeros(n, E), None, k, groups, top_groups)
    _check(torch.zeros(3, 256), None, k, groups, top_groups)
    # scores that 64 bits, but not 32, tell apart; and that neither does
    _check(torch.randn(n, E, generator=g) * 0.5 + 20, torch.zeros(E), k, groups, top_groups)
    _check(torch.randn(n, E, generator=g) + 60, None, k, groups, top_groups, ("sigmoid",))
    # a tie at the last place with a near one behind it
    x = torch.randn(n, E, generator=g)
    x[:, 3] = x[:, 9] = x.max(1).values + 0.5
    x[:, 17] = (x[:, 3].contiguous().view(torch.int32) - 1).view(torch.float32)
    _check(x, None, 1, groups, top_groups)


def test_values_that_are_not_finite():
    r = _gen(3)
    x = r(12, 16)
    x[1, 5] = math.nan
    x[2, 3] = x[2, 9] = math.nan
    x[3, 7] = math.inf
    x[4] = math.nan
    x[5] = -math.inf
    x[6, :15] = -math.inf
    for groups, top in ((1, 1), (4, 2)):
        for bias in (None, r(16, std=0.1)):
            for kind in ("sigmoid", "softmax"):
                want = ref.choose(x, bias, kind, groups, top, 3)
                got = spc.route_scores_forward(x.cuda(), 3, score=kind, groups=groups, top_groups=top,
                                               bias=None if bias is None else bias.cuda())
                _check_pairs(got, want, 16)
    bias = r(16, std=0.1)
    bias[4], bias[11], bias[12] = -math.inf, math.inf, math.inf
    x = r(12, 16)
    _check(x, bias, 3)
    _check(x, bias, 3, 8, 3)


@pytest.mark.parametrize("n,E,k,groups,top_groups,dtype", [
    (5000, 8, 2, 2, 1, "f32"), (20000, 16, 4, 4, 2, "bf16"), (3000, 64, 8, 8, 4, "f32"),
    (300, 1024, 2, 1, 1, "bf16"), (0, 8, 2, 2, 1, "f32"), (257, 3, 1, 3, 2, "f32")])
def test_many_rows(n, E, k, groups, top_groups, dtype):
    """More than one workgroup: ranks over workgroups, counts summed and scanned.  The choice is
    taken from 64-bit torch operations (the statement takes one comparison at a time)."""
    r = _gen(n + E)
    x, bias = (r(n, E) + r(E, std=0.7)).to(DT[dtype]), r(E, std=0.05)
    v = ref.scores(x, "sigmoid") + bias.double()
    if groups > 1:
        worth = v.view(n, groups, E // groups).topk(min(2, E // groups), 2).values.sum(2)
        stay = torch.zeros(n, groups, dtype=torch.bool)
        stay.scatter_(1, torch.sort(worth, dim=1, descending=True, stable=True).indices[:, :top_groups], True)
        v = v.masked_fill(~stay.repeat_interleave(E // groups, 1), -math.inf)
    want = torch.sort(v, dim=1, descending=True, stable=True).indices[:, :k]
    got = spc.route_scores_forward(x.cuda(), k, bias=bias.cuda(), groups=groups, top_groups=top_groups)
    _check_pairs(got, want, E)
    again = spc.route_scores_forward(x.cuda(), k, bias=bias.cuda(), groups=groups,
                                     top_groups=top_groups)
    for name in ("experts", "weights", "offsets", "rows", "pos"):
        assert torch.equal(getattr(got, name), getattr(again, name))


def test_softmax_weights_of_experts_far_below_the_best():
    """The bias can choose experts whose scores are nothing in fp32: their renormalised weights are
    still the softmax over the chosen."""
    x = torch.tensor([[0.0, -150.0, -151.0, -300.0]])
    bias = torch.tensor([0.0, 5.0, 5.0, 0.0])
    r = spc.route_scores_forward(x.cuda(), 2, score="softmax", bias=bias.cuda())
    w = torch.softmax(torch.tensor([-150.0, -151.0], dtype=torch.float64), 0)
    assert r.experts.cpu().tolist() == [[1, 2]]
    assert bool(((r.weights.cpu().double()[0] - w).abs() <= 20 * U).all())

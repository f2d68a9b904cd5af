"""Routing by scores: groups whose two best biased scores cancel, or leave fp32's range, are chosen
as 64-bit arithmetic has them."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_1706_01307_amd as spc  # noqa: E402
from tests import rows_dense_ref as ref  # noqa: E402
from tests.test_rows_gpu import DT, _gen, _gpu  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def _experts(x, bias, k, groups, top_groups, kind="sigmoid"):
    r = spc.route_scores_forward(x.cuda(), k, score=kind, bias=bias.cuda(), groups=groups,
                                 top_groups=top_groups)
    return r.experts.cpu().long()


def test_two_biases_that_cancel():
    x = torch.tensor([[1.36e-5, 0.0, 0.0, 9.6e-6]])
    bias = torch.tensor([64.0, -64.0, 64.0, -64.0])
    assert _experts(x, bias, 1, 2, 1).tolist() == [[0]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
# (groups of whole pieces and of odd widths, which are searched for differently; one lane and more)
@pytest.mark.parametrize("groups,per", [(2, 4), (2, 8), (4, 8), (16, 8), (2, 2), (3, 3), (5, 7), (2, 128)])
def test_groups_whose_best_two_cancel(groups, per, kind, dtype):
    """Group 0's best two are biased by +-size, group 1's by nothing; logits differ so little that the
    two groups' worths lie within a few roundings of `size`.  Rows whose 64-bit worths are closer than
    64 of their own roundings (2^-53 of the size each) are left out."""
    r, E = _gen(groups * 100 + per), groups * per
    for size in (8.0, 32.0, 100.0, 1000.0, 30000.0):
        bias = torch.full((E,), -2 * size)
        bias[0], bias[1], bias[per], bias[per + 1] = size, -size, 0.0, 0.0
        x = (r(400, E) * 2.0 ** -21 * size).to(DT[dtype])
        v = ref.scores(x, kind) + bias.double()
        worth = v.view(400, groups, per).topk(2, 2).values.sum(2)
        x = x[(worth[:, 0] - worth[:, 1]).abs() > 64 * 2.0 ** -53 * size]
        assert len(x) > 300 or dtype == "bf16"
        want = ref.choose(x, bias, kind, groups, 1, 1)
        assert torch.equal(_experts(x, bias, 1, groups, 1, kind), want), size
        assert 0 < int((want == 0).sum()) < len(x)


def test_worths_beyond_fp32():
    x = torch.tensor([[0.5, 0.5, 1.0, 1.0]])
    for b, want in (([3e38, 3e38, 3.2e38, 3.2e38], 2), ([3.2e38, 3.2e38, 3e38, 3e38], 0),
                    ([-3e38, -3e38, -3.2e38, -3.2e38], 0), ([-3.2e38, -3.2e38, -3e38, -3e38], 2),
                    ([3e38, -3.2e38, 1.0, 1.0], 2), ([3.2e38, -3e38, 1.0, 1.0], 0)):
        assert _experts(x, torch.tensor(b), 1, 2, 1).tolist() == [[want]], b
        wide = torch.full((1, 16), -math.inf)
        wide[0, :2], wide[0, 8:10] = x[0, :2], x[0, 2:]
        c = torch.zeros(16)
        c[:2], c[8:10] = torch.tensor(b)[:2], torch.tensor(b)[2:]
        assert _experts(wide, c, 1, 2, 1).tolist() == [[want if want < 2 else 8]], b
    # a group of which nothing is open goes, however far below the other is
    x = torch.tensor([[-math.inf, -math.inf, 0.0, 0.0]])
    assert _experts(x, torch.tensor([9.0, 9.0, -3e38, -3e38]), 2, 2, 1).tolist() == [[2, 3]]


def test_groups_closed_by_the_lowest_number():
    """Biases of the type's lowest value, of one group's experts or of all but one of every group's,
    and infinite ones."""
    r, low = _gen(8), torch.finfo(torch.float32).min
    x = r(200, 32)
    for kind in ("sigmoid", "softmax"):
        for shut in (slice(8, 16), [c for c in range(32) if c % 8 != 3], slice(0, 31), slice(0, 32)):
            for value in (low, -math.inf, math.inf):
                bias = r(32, std=0.1)
                bias[shut] = value
                want = ref.choose(x, bias, kind, 4, 2, 3)
                assert torch.equal(_experts(x, bias, 3, 4, 2, kind), want), (kind, shut, value)

"""SiLU of fp32 rows far below 0, where it is a small number with bits of its own: within 16 U of its
value (the exponent to half a unit of its place, a unit each of exp2 and of the reciprocal, a sum and
three products), and its slope within 32 U of |s| + |z s (1 - s)|, in every kernel that has it.  Down
to z = -80: below, the reciprocal is no normal number."""
import pytest

torch = pytest.importorskip("torch")

import paper_1706_01307_amd as spc  # noqa: E402
from tests import rows_dense_ref as ref  # noqa: E402
from tests.rows_ref import U  # noqa: E402
from tests.test_rows_dense_gpu import _rows8  # noqa: E402
from tests.test_rows_gpu import _gpu  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def _near(got, want, mag, units):
    off = (got.cpu().double() - want).abs()
    assert got.dtype == torch.float32 and bool((off <= units * U * mag).all()), float((off / mag).max() / U)


# (one fp32 row; few; tiles in slices, of 64, cut ones; and of 128)
@pytest.mark.parametrize("n", [1, 16, 100, 5000, 50000])
@pytest.mark.parametrize("C", [64, 61, 232])
def test_silu_of_fp32_rows(n, C):
    z = -80 * torch.rand(n, C, generator=torch.Generator().manual_seed(n + C))
    s = torch.sigmoid(z.double())
    value, slope = z.double() * s, s + z.double() * s * torch.sigmoid(-z.double())
    mag = s + (z.double() * s).abs()
    # as a product's sum: the identity
    y, kept = spc.linear_forward(z.cuda(), torch.eye(C, device="cuda"), act="silu", pre=True)
    assert torch.equal(kept.cpu(), z)
    _near(y, value, value.abs(), 16)
    one = torch.ones(n, C, device="cuda")
    _near(spc.activation_backward(one, z.cuda(), "silu"), slope, mag, 32)
    dx = spc.linear_backward_data(one, torch.eye(C, device="cuda"), act="silu", pre=z.cuda())
    _near(dx, slope, mag, 32)
    q, scale = ref.packed(z)
    v = (q.float() * scale[:, None]).double()
    s = torch.sigmoid(v)
    value, slope, mag = v * s, s + v * s * torch.sigmoid(-v), s + (v * s).abs()
    _near(spc.unpack_rows(_rows8(q, scale), torch.float32, act="silu"), value, value.abs() + 1e-45, 16)
    _near(spc.activation_backward(one, _rows8(q, scale), "silu"), slope, mag, 32)

"""Routings of more workgroups than one step of the scan over them takes (1,024): all pairs in
order, weights and their gradient, against sorted 64-bit ones.  Tolerances are test_rows_gpu.py's."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

import paper_1706_01307_amd as spc  # noqa: E402
from paper_1706_01307_amd import _lib  # noqa: E402
from tests.test_rows_gpu import DT, _close  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.init()


@pytest.mark.parametrize("n,E,k,normalize,dtype", [
    (300001, 16, 2, True, "f32"), (600000, 40, 3, False, "bf16"), (140003, 64, 16, True, "bf16"),
    (262145, 100, 8, False, "f32")])
def test_scan_carries_over_its_steps(n, E, k, normalize, dtype):
    nbytes = ctypes.c_size_t()
    assert _lib.load().spconv_route_workspace(n, E, k, ctypes.byref(nbytes)) == 0
    blocks = nbytes.value // (4 * E) - 1             # counts of every workgroup, and the totals
    assert blocks > 1024 and blocks * E > 8192       # (fewer are added up without the scan)
    g = torch.Generator().manual_seed(n)
    x = torch.round(torch.randn(n, E, generator=g) * 4) / 2 + torch.arange(E) / (2.0 * E)
    x = torch.round(x * 8) / 8                       # ties
    x[torch.rand(n, E, generator=g) < 0.2] = -math.inf
    x[::11] = -math.inf
    x = x.to(DT[dtype])
    got = spc.route_forward(x.cuda(), k, normalize)
    x = x.double()
    v, e = torch.sort(x, dim=1, descending=True, stable=True)
    v, e = v[:, :k], torch.where(v[:, :k] > -math.inf, e[:, :k], -1)
    assert torch.equal(got.experts.cpu().long(), e)
    flat = torch.where(e < 0, E, e).reshape(-1)
    order = torch.sort(flat, stable=True).indices
    count = torch.bincount(flat, minlength=E + 1)[:E]
    total = int(count.sum())
    assert got.offsets.cpu().tolist() == [0] + count.cumsum(0).tolist()
    rows, pos = got.rows.cpu().long(), got.pos.cpu().long().reshape(-1)
    assert torch.equal(rows[:total], order[:total] // k) and (rows[total:] == -1).all()
    assert torch.equal(pos[order[:total]], torch.arange(total)) and (pos[flat == E] == -1).all()
    # weights and gradient
    some, top = e >= 0, torch.where(v[:, :1] > -math.inf, v[:, :1], 0.0)
    p = torch.exp(x - top)
    z = (torch.exp(v - top) if normalize else p).sum(1, keepdim=True)
    z = torch.where(z > 0, z, 1.0)
    w = torch.where(some, torch.exp(v - top) / z, 0.0)
    size = float(x[torch.isfinite(x)].abs().max())
    _close(got.weights, w, w, E + 2 * size, "weights")
    dw = torch.randn(n, k, generator=g)
    d = spc.route_backward(dw.cuda(), x.to(DT[dtype]).cuda(), got.experts, got.weights, normalize)
    dot = (w * dw).sum(1, keepdim=True)
    want = torch.zeros(n, E, dtype=torch.float64) if normalize else -p / z * dot
    want.scatter_add_(1, e.clamp(min=0), torch.where(some, w * (dw - dot if normalize else dw),
                                                     0.0))
    mag = torch.full_like(want, 2 * float(dw.abs().max()))
    _close(d, want, mag, 3 * (E + k + 40), "dlogits")

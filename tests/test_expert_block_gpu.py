"""The expert block of examples/expert_block.py: its output and every gradient against a float64
autograd statement of the same block, its training, and rows taken one at a time."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from examples.expert_block import ExpertBlock, train  # noqa: E402
from tests import rows_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.init()


def _block64(block, x, step, experts, p):
    """The block on the CPU in float64 with the experts given; differentiable."""
    n = torch.nn.functional.layer_norm(x, (x.shape[1],), p["gamma"], p["beta"], 1e-5)
    logits = n @ p["wr"][0]
    w = torch.softmax(logits.gather(1, experts), 1) if block.normalize else \
        torch.softmax(logits, 1).gather(1, experts)
    u = 0
    for s in range(experts.shape[1]):
        e = experts[:, s]
        h = torch.relu(torch.einsum("nc,nch->nh", n, p["w1"][e]) + p["b1"][e])
        z = torch.einsum("nh,nhc->nc", h, p["w2"][e]) + p["b2"][e]
        u = u + w[:, s:s + 1] * z
    keep = torch.from_numpy(ref.kept(0, x.numel(), block.p, block.seed, step)).view(x.shape)
    return x + torch.where(keep, u / (1 - block.p), 0.0)


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("n,C,hidden,experts,k", [(150, 16, 24, 5, 2), (33, 40, 72, 3, 3),
                                                  (1, 8, 8, 4, 1)])
def test_block_and_its_gradients(n, C, hidden, experts, k, normalize):
    block = ExpertBlock(C, hidden, experts, k, p=0.25, seed=7, normalize=normalize)
    g = torch.Generator().manual_seed(n)
    for q in ("gamma", "beta", "b1", "b2"):
        block.params[q] += 0.3 * torch.randn(block.params[q].shape, generator=g).cuda()
    x, dy = torch.randn(n, C, generator=g), torch.randn(n, C, generator=g)
    y, kept = block.forward(x.cuda(), 3)
    dx, grads = block.backward(dy.cuda(), kept)
    chosen = kept[7].experts.cpu().long()
    p = {q: v.cpu().double().requires_grad_() for q, v in block.params.items()}
    x64 = x.double().requires_grad_()
    want = _block64(block, x64, 3, chosen, p)
    want.backward(dy.double())
    # fp32 through five products and a softmax: 1e-4 of a tensor's largest value is a few hundred
    # rounding units
    for name, got, w in [("y", y, want.detach()), ("dx", dx, x64.grad)] + \
            [(q, grads[q], p[q].grad) for q in p]:
        err = float((got.cpu().double() - w).abs().max())
        assert err <= 1e-4 * max(1.0, float(w.abs().max())), (name, err)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_block_trains_and_serves_single_rows(dtype):
    losses, block, x = train(sites=2400, steps=25, dtype=dtype, C=32, hidden=48, experts=4)
    assert np.isfinite(losses).all() and min(losses[-3:]) < 0.7 * losses[0], losses
    whole, none = block.forward(x, 0, train=False)
    assert none is None
    for i in (0, 17, x.shape[0] - 1):
        y, _ = block.forward(x[i:i + 1].contiguous(), 0, train=False)
        assert torch.equal(y[0], whole[i])
    assert torch.equal(block.forward(x, 0, train=False)[0], whole)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_block_is_captured_and_serves_converted_weights(dtype):
    """Forward and gradients in a graph, replayed on new rows between eager ones; weights converted
    once give what converting them in every call gives."""
    block = ExpertBlock(40, 56, 6, 2, p=0.2, dtype=dtype, seed=3)
    x, dy = (torch.randn(130, 40, device="cuda").to(dtype) for _ in range(2))

    def step():
        y, kept = block.forward(x, 5)
        dx, grads = block.backward(dy, kept)
        return [y, dx, *grads.values(), block.forward(x, 0, train=False)[0]]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        x.normal_()
        dy.normal_()
        graph.replay()
        torch.cuda.synchronize()
        out = [t.clone() for t in got]
        for a, b in zip(out, step()):
            assert torch.equal(a, b)
    whole, _ = block.forward(x, 0, train=False)
    block.serve()
    for name in ("wr", "w1", "w2"):
        assert block._w(name) is block.params[name] and block.params[name].dtype == dtype
    assert torch.equal(block.forward(x, 0, train=False)[0], whole)

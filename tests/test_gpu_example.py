"""The example's expert block: its gradients against autograd in 64 bits, and
a few steps of its training."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import expert_block
    return expert_block


def _reference(block, x, dh_out, dy):
    """The block in 64 bits on the CPU, routed as the block was."""
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in block.weights.items()}
    x = x.cpu().double().requires_grad_()
    off = block.offsets.tolist()
    order, place = block.order.cpu(), block.place.cpu()
    rms = lambda v, w: v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt() * w  # noqa: E731
    hp = rms(x, p["w_in"])[order]
    up = torch.cat([torch.relu(hp[a:b] @ p["w1"][e].t()) @ p["w2"][e].t() for e, (a, b) in enumerate(zip(off, off[1:]))])
    u = torch.nn.functional.layer_norm(up[place], (x.shape[1],), eps=1e-5) * p["w_post"]
    y = x + p["scale"] * torch.sigmoid(p["gate"]) * u
    h = rms(y, p["w_out"])
    ((h * dh_out.cpu().double()).sum() + (y * dy.cpu().double()).sum()).backward()
    return h, y, x.grad, {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("rows,C,hidden,E", [(301, 72, 96, 5), (64, 40, 136, 3), (1000, 128, 256, 8)])
def test_gradients(example, rows, C, hidden, E):
    """float32 throughout: every gradient of the whole chain within 2^-12 of
    64 bits in the 2-norm (six products and norms of some hundred terms each,
    2^-24 a term; ReLU signs flip only at sums below their rounding)."""
    b = example.ExpertBlock(rows, C, hidden, E, "f32")
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dh, dy = (torch.randn((rows, C), generator=g, device="cuda") for _ in range(3))
    h = b.forward(x).clone()
    dx = b.backward(dh, dy)
    rh, ry, rdx, rp = _reference(b, x, dh, dy)
    for name, got, want in (("h", h, rh), ("y", b.y, ry), ("dx", dx, rdx), *((k, b.grads[k], rp[k]) for k in rp)):
        want = want.detach()
        err = float((got.cpu().double() - want).norm() / want.norm())
        assert err <= 2.0 ** -12, (name, err)


def test_training(example):
    """bf16: the loss falls, nothing is lost to a NaN, the clipped norm is at most the limit."""
    losses, block = example.train(steps=12, rows=1000, C=128, hidden=256, E=6)
    assert all(v == v for v in losses) and losses[-1] < 0.9 * losses[0]
    norm, c = block.norm.tolist()
    total = sum(float(v.double().square().sum()) for v in block.grads.values()) ** 0.5
    assert total <= 1.0 + 1e-5 and abs(total - norm * c) <= 1e-4 * total
    assert int(block.offsets[-1]) == 1000

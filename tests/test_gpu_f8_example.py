"""The feed-forward block of the examples: its gradients against those of the same block in 64 bits, that it learns, and that its graph serves what
the calls give."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

_at = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "f8_feed_forward.py")
_spec = importlib.util.spec_from_file_location("f8_feed_forward", _at)
ff = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(ff)


def off(x, y):
    return float(torch.linalg.norm(x.double() - y) / torch.linalg.norm(y))


@pytest.mark.parametrize("m,width,hidden", [(300, 256, 200), (129, 130, 257), (1000, 384, 1000)])
def test_gradients(m, width, hidden):
    """Conversions to 3 bits of mantissa are off by 2.6% of the norm (2^-4 at most, evenly spread over it and over where in a power of two a number
    lies), so a product of two converted matrices is off by 3.7%, and what went through three products and four conversions in a row by 3.7 * sqrt(3 +
    0.5) = 7%.  Twice that is allowed."""
    block = ff.FeedForward(width, hidden, seed=m)
    a = ff.Activations(m, width, hidden, True)
    torch.manual_seed(m)
    x, dy = (torch.randn(m, width, device="cuda").bfloat16() for _ in range(2))
    dx = torch.empty_like(x)
    y = block.forward(x, a)
    block.backward(dy, a, dx)
    p = [t.double().cpu().requires_grad_() for t in (x, block.gate_up.master[:hidden], block.gate_up.master[block.up:], block.down.master)]
    want = (torch.nn.functional.silu(p[0] @ p[1].t()) * (p[0] @ p[2].t())) @ p[3].t()
    want.backward(dy.double().cpu())
    got = (y, dx, block.gate_up.grad[:hidden], block.gate_up.grad[block.up:], block.down.grad)
    for g, w in zip(got, (want.detach(), *(t.grad for t in p))):
        assert off(g.cpu(), w) < 0.14
    assert not block.gate_up.grad[hidden:block.up].any()      # the rows between the two halves stay as they were


def test_it_learns_and_serves():
    block, other = ff.FeedForward(256, 300), ff.FeedForward(256, 300, seed=5)
    memory = ff.Activations(512, 256, 300, False)
    losses = ff.train(block, lambda x: other.forward(x, memory).float(), 512, 120)
    assert sum(losses[-5:]) < 0.7 * sum(losses[:5])
    for tokens in (1, 5):
        server, plain = ff.Server(block, tokens), ff.Activations(tokens, 256, 300, False)
        for _ in range(4):
            x = torch.randn(tokens, 256, device="cuda").bfloat16()
            got = server(x).clone()
            assert torch.equal(got, block.forward(x, plain)) and got.isfinite().all()
            torch.cuda.synchronize()

"""The layer of experts of the examples: it runs, its gradients are those of the same layer in 64 bits, and its graph serves what the calls give."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

_at = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "i8_experts.py")
_spec = importlib.util.spec_from_file_location("i8_experts", _at)
ex = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(ex)


def off(x, y):
    return float(torch.linalg.norm(x.double() - y) / torch.linalg.norm(y))


@pytest.mark.parametrize("tokens,width,hidden,experts,each", [(300, 256, 200, 5, 2), (129, 130, 257, 8, 1), (1000, 384, 500, 3, 3), (7, 64, 48, 16, 4)])
def test_gradients(tokens, width, hidden, experts, each):
    """A row whose largest number is 6 times its root of the mean square or less is converted with steps of 6 / 127 of that, so by errors of
    6 / 127 / sqrt(12) = 1.4% of its norm; what has gone through six conversions and the roundings to bfloat16 between them (0.2% each) is
    off by sqrt(6) * 1.4% = 3.4%.  Slopes of the activation are up to 1.1, and twice that is allowed."""
    layer = ex.Experts(experts, width, hidden, seed=tokens)
    torch.manual_seed(tokens)
    x, dy = (torch.randn(tokens, width, device="cuda").bfloat16() for _ in range(2))
    routes, kept = ex.Routes(torch.randn(tokens, experts, device="cuda"), each), {}
    y = layer.forward(x, routes, kept)
    dx = layer.backward(dy, routes, kept)
    assert torch.equal(y, layer.forward(x, routes))
    p = [t.double().cpu().requires_grad_() for t in (x, layer.up.master, layer.down.master)]
    index, weight, bounds = routes.index.cpu().long(), routes.weight.double().cpu(), routes.offsets.tolist()
    parts = []
    for e in range(experts):
        rows = index[bounds[e]:bounds[e + 1]]
        h = torch.nn.functional.silu(p[0][rows] @ p[1][e * hidden:(e + 1) * hidden].t())
        parts.append(h @ p[2][e * width:(e + 1) * width].t())
    want = torch.zeros(tokens, width, dtype=torch.float64).index_add(0, index, torch.cat(parts) * weight)
    want.backward(dy.double().cpu())
    for g, w in zip((y, dx, layer.up.grad, layer.down.grad), (want.detach(), *(t.grad for t in p))):
        assert off(g.cpu(), w) < 0.075


def test_it_trains_and_serves():
    layer, other = ex.Experts(4, 128, 200), ex.Experts(4, 128, 200, seed=5)
    router = torch.randn(128, 4, device="cuda")
    before = layer.up.master.clone()
    losses = ex.train(layer, lambda x, routes: other.forward(x, routes).float(), router, 256, 2, 5)
    assert len(losses) == 5 and all(v == v and v < float("inf") for v in losses) and not torch.equal(before, layer.up.master)
    for tokens in (1, 5):
        server = ex.Server(layer, router, tokens, 2)
        for _ in range(4):
            x = torch.randn(tokens, 128, device="cuda").bfloat16()
            got = server(x).clone()
            torch.cuda.synchronize()
            want = layer.forward(x, ex.Routes(x.float() @ router, 2))
            # (index_add_ adds in any order, so a token's sum of two may be rounded otherwise: a unit of the last place)
            assert off(got, want.double()) < 2.0 ** -7 and got.isfinite().all()

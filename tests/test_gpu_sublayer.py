"""examples/sublayer.py: the whole sublayer, from the residual stream to Q, K and V, through the selection
and the attention and back, and the gradients that the budgets are calibrated with, against float64."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("sublayer_example", os.path.join(ROOT, "examples", "sublayer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def reference(layer, x):
    """The sublayer with dense attention in float64, and its leaves."""
    D = lambda t: t.double().detach().requires_grad_()
    P = {"x": D(x), "w": D(layer.norm[0]), "b": D(layer.norm[1])}
    hn = {n: tuple(D(t) for t in layer.head_norm[n]) for n in "qk"}
    ln = torch.nn.functional.layer_norm
    h = ln(P["x"], (layer.dm,), P["w"], P["b"], layer.eps)
    out, proj = {}, {}
    i = torch.arange(16, device="cuda", dtype=torch.float64)
    angle = torch.cat([layer.pos[:, a:a + 1].double() * 100.0 ** (-i / 16.0) for a in range(2)], 1)
    for n in "qkv":
        proj[n] = h @ layer.W[n].double().T + layer.b[n].double()
        proj[n].retain_grad()
        u = proj[n].view(layer.N, layer.H, 64)
        if n != "v":
            u = ln(u, (64,), *hn[n], layer.eps)
            s = u.view(layer.N, layer.H, 2, 2, 16)
            c, d = (f(angle).view(layer.N, 1, 2, 16) for f in (torch.cos, torch.sin))
            u = torch.stack([s[..., 0, :] * c - s[..., 1, :] * d, s[..., 1, :] * c + s[..., 0, :] * d], -2)
            u = u.reshape(layer.N, layer.H, 64)
        out[n] = u
    A = torch.softmax(torch.einsum("ihc,jhc->hij", out["q"], out["k"]) / 8.0, -1)
    O = (A @ out["v"].transpose(0, 1)).transpose(0, 1).reshape(layer.N, layer.dm)
    return P["x"] + O @ layer.W_o.double().T, P, hn, proj


def far(a, b):
    return float((a.double() - b).norm() / b.norm())


def test_sublayer_and_its_gradients(example):
    layer = example.Sublayer(1, 3, seed=5)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(layer.N, layer.dm, generator=g, device="cuda", dtype=torch.float32).bfloat16()
    dy = (0.1 * torch.randn(layer.N, layer.dm, generator=g, device="cuda", dtype=torch.float32)).bfloat16()
    y, P, hn, proj = reference(layer, x)
    got = layer.forward(x, [layer.candidates] * layer.H)
    # Each of the stages rounds to bf16 once (2^-8 of a value at most, 2^-9.8 in the mean square); the
    # sublayer's contribution goes through four of them (norm, Q and K and V, O, y), and errors of Q and K
    # reach it through logits of size about 8 / 8.  y's own rounding is against y, not the contribution.
    contribution, want = (y - x.double()).detach(), y.detach()
    assert float((got.double() - want).norm()) <= 2.0 ** -6 * float(contribution.norm()) + 2.0 ** -9 * float(want.norm())
    y.backward(dy.double())
    grads = layer.gradients(x, dy)
    # the gradients go through as many roundings again, back through the same stages
    for n in "qkv":
        assert far(grads[n].reshape(layer.N, layer.dm), proj[n].grad) <= 2.0 ** -5, n
    # dx holds the residual branch's gradient as well: its own rounding is against dx, as y's above
    through = float((P["x"].grad - dy.double()).norm())
    assert float((grads["dx"].double() - P["x"].grad).norm()) <= 2.0 ** -4 * through + 2.0 ** -9 * float(P["x"].grad.norm())
    assert far(grads["norm"][0], P["w"].grad) <= 2.0 ** -5 and far(grads["norm"][1], P["b"].grad) <= 2.0 ** -5
    for i, t in enumerate((*hn["q"], *hn["k"])):
        assert far(grads["head_norm"][i], t.grad) <= 2.0 ** -4, i


def test_example_runs(example, capsys):
    layer, budgets, change = example.main(["--views", "2", "--heads", "4"])
    assert len(budgets) == 4 and all(2 <= c <= layer.candidates for c in budgets)
    assert 0.0 < change < 1.0 and "budgets" in capsys.readouterr().out

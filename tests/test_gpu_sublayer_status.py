"""examples/sublayer.py: a failure of any of its calls reaches the caller, and a layer keeps its buffers."""
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


def test_projection_that_gave_up_is_reported(example, monkeypatch):
    """A wait of the projection that ran out leaves its code in the workspace that the call was given: the example
    reads the status of that one before it returns a result."""
    layer, ress = example.Sublayer(1, 2, seed=3), example.ress
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(layer.N, layer.dm, generator=g, device="cuda", dtype=torch.float32).bfloat16()
    budgets = [5] * layer.H
    want = layer.forward(x, budgets)
    project = ress.qkv_proj

    def gives_up(d, h, W_q, W_k, W_v, Q, K, V, ws, **kw):
        project(d, h, W_q, W_k, W_v, Q, K, V, ws, **kw)
        ress.wait_selftest(ws, 1000)

    monkeypatch.setattr(ress, "qkv_proj", gives_up)
    with pytest.raises(ress.RessError) as e:
        layer.forward(x, budgets)
    assert e.value.code == -5
    monkeypatch.setattr(ress, "qkv_proj", project)
    assert torch.equal(layer.forward(x, budgets), want)  # and the next one is not


def test_buffers_are_kept_from_one_forward_to_the_next(example, monkeypatch):
    layer, made, kind = example.Sublayer(1, 2, seed=3), [], example.ress.Buffers
    monkeypatch.setattr(example.ress, "Buffers", lambda *a, **kw: made.append(1) or kind(*a, **kw))
    x = torch.zeros(layer.N, layer.dm, device="cuda", dtype=torch.bfloat16)
    for _ in range(3):
        layer.forward(x, [5] * layer.H)
    assert len(made) == 1

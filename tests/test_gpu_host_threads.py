"""Calls from two host threads on one device, each with its own stream, tensors and workspace: the launch
settings that one call needs must not be those that the other has just made."""
import threading

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ress():
    import paper_2609_35593_gb300 as r
    return r


def together(calls, times):
    """Runs every call `times` times, each call on a thread of its own; the errors that were raised."""
    start, errors = threading.Barrier(len(calls)), []

    def work(call):
        stream = torch.cuda.Stream()
        start.wait()
        try:
            for _ in range(times):
                call(stream)
        except Exception as e:
            errors.append(e)
        stream.synchronize()

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    [t.start() for t in threads]
    [t.join() for t in threads]
    return errors


class NormGradient:
    def __init__(self, ress, rows, width):
        g = torch.Generator(device="cuda").manual_seed(width)
        normal = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float32)
        self.ress, self.dy, self.x = ress, normal(rows, width).bfloat16(), normal(rows, width).bfloat16()
        self.w, self.mean, self.rstd = normal(width), 0.1 * normal(rows), 1 + 0.1 * normal(rows)
        self.out = [torch.empty_like(self.x), torch.empty_like(self.w), torch.empty_like(self.w)]
        self.ws = torch.empty(ress.layer_norm_workspace_bytes(rows, width), dtype=torch.uint8, device="cuda")

    def __call__(self, stream=None):
        dx, dw, db = self.out
        self.ress.layer_norm_bwd(self.dy, self.x, self.w, self.mean, self.rstd, dx, dweight=dw, dbias=db, ws=self.ws,
                                 stream=stream)


@pytest.mark.parametrize("widths", [(16384, 9216), (16383, 5003)])
def test_layer_norm_gradients_of_two_widths(ress, widths):
    # (16383 and 5003 in few rows: element by element)
    layers = [NormGradient(ress, 4, w) for w in widths]
    want = []
    for layer in layers:
        layer()
        want.append([t.clone() for t in layer.out])
        [t.fill_(float("nan")) for t in layer.out]
    assert together(layers, 3000) == []
    for layer, expected in zip(layers, want):
        assert all(torch.equal(a, b) for a, b in zip(layer.out, expected))

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


class Selection:
    """Scoring and restoration of one scene."""

    def __init__(self, ress, views):
        g = torch.Generator(device="cuda").manual_seed(views)
        normal = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float32).bfloat16()
        N, H, dm = views * 1374, 1, 64
        self.ress, self.d, self.c = ress, ress.dims(N, H, views * 5, dm), [20] * H
        self.Q, self.K, self.V = (normal(N, H, 64) for _ in range(3))
        self.buf = ress.Buffers(self.d, self.c)
        ress.prepare_wo(self.d, 0.1 * normal(dm, dm), self.buf.F)
        self.out = [self.buf.J_best, self.buf.row_ptr, self.buf.col_idx]

    def __call__(self, stream=None):
        b = self.buf
        self.ress.score(self.d, self.Q, self.K, self.V, b.F, self.c, b.ws, stream=stream)
        self.ress.restore(self.d, self.c, 3, 0.5, b.ws, b.row_ptr, b.col_idx, b.J_best, stream=stream)


def test_selections_of_two_scenes(ress):
    """Above 2,700 blocks a selection kernel's shared memory needs more than the 48 KB that any launch may have."""
    scenes = [Selection(ress, 2), Selection(ress, 180)]
    want = []
    for s in scenes:
        s()
        want.append([t.clone() for t in s.out])
        [t.fill_(-1) for t in s.out]
    assert together(scenes, 600) == []
    for s, expected in zip(scenes, want):
        ress.status(s.buf.ws)
        assert all(torch.equal(a, b) for a, b in zip(s.out, expected))

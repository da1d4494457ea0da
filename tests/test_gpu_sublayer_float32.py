"""examples/sublayer.py with a float32 residual stream: gradients of the same numbers as a bf16 stream's."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_sublayer import example, far  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def test_gradients_of_a_float32_stream(example):
    layer = example.Sublayer(1, 2, seed=5)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(layer.N, layer.dm, generator=g, device="cuda", dtype=torch.float32).bfloat16()
    dy = (0.1 * torch.randn(layer.N, layer.dm, generator=g, device="cuda", dtype=torch.float32)).bfloat16()
    want = layer.gradients(x, dy)
    got = layer.gradients(x.float(), dy.float())
    assert got["dx"].dtype == torch.float32
    # The norm's sums run in another order for float32 rows (2^-22), which turns a rounding of h to bf16 (2^-8) in one of
    # 2^13 channels, 2^-14 in the mean square; dx of bf16 is rounded once (2^-8 of each value at most).
    for name in want:
        assert far(got[name], want[name].double()) <= 2.0 ** -8, name

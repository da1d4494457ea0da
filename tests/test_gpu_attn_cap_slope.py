"""Gradients of scores several times their cap, where 1 - tanh^2 is far below the rounding of tanh."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from gradients64 import gradients  # noqa: E402
from test_gpu_attn import BF16, F16, R, float32_by_default, normal, run  # noqa: E402,F401
from test_gpu_attn_bwd import grads  # noqa: E402

pytestmark = pytest.mark.gpu


def saturated(kind, times, cap, nq=150, nk=200, heads=4):
    """Scores of about +-times x cap: rows and keys near one direction, rows of both signs."""
    way = normal(1, 1, 1, 64, kind=torch.float32)
    way = way / way.norm()
    near = lambda seed, *s: way + 0.02 * normal(seed, *s, 64, kind=torch.float32)
    size = (8 * times * cap) ** 0.5
    sign = normal(2, nq, heads, 1, kind=torch.float32).sign()
    return (size * sign * near(3, nq, heads)).to(kind), (size * near(4, nk, heads)).to(kind), normal(5, nk, heads, 64, kind=kind)


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("times", [0.4, 1.0, 4.0, 7.0])
@pytest.mark.parametrize("cap", [0.5, 5.0])
@pytest.mark.parametrize("causal", [False, True])
def test_saturated_scores(kind, times, cap, causal):
    q, k, v = saturated(kind, times, cap)
    lens = [q.shape[0]], [k.shape[0]]
    do = normal(9, *q.shape, kind=kind)
    mask = {"causal": causal, "cap": cap}
    o, lse = run(q, k, v, *lens, **mask)
    want, off = gradients(do, q, k, v, o, lse, *lens, **mask)
    for g, w, f, name in zip(grads(do, q, k, v, o, lse, *lens, **mask), want, off, ("dq", "dk", "dv")):
        R.close(g, w, f, name)


def test_scores_past_every_exponential():
    """tanh is 1 and its slope 0 in float32, on both sides: no NaN, and dv as ever."""
    q, k, v = saturated(BF16, 400.0, 1.0)
    lens = [q.shape[0]], [k.shape[0]]
    do = normal(9, *q.shape)
    o, lse = run(q, k, v, *lens, cap=1.0)
    want, off = gradients(do, q, k, v, o, lse, *lens, cap=1.0)
    got = grads(do, q, k, v, o, lse, *lens, cap=1.0)
    assert (got[0] == 0).all() and (got[1] == 0).all()
    R.close(got[2], want[2], off[2], "dv")

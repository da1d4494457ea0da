"""Gradients of the sequences around one whose starts are outside the tensors: that one has none, the others are as ever."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2609_35593_gb300 as ress  # noqa: E402
from test_gpu_attn import BF16, F16, float32_by_default, ints, normal, problem, run, workspace  # noqa: E402,F401
from test_gpu_attn_bwd import grads  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("q_start,k_start,rows,keys", [
    ([0, 60, 40], [0, 60, 100], slice(0, 60), slice(0, 60)),     # the second goes back: no rows
    ([90, 40, 100], [0, 60, 100], slice(40, 100), slice(60, 100)),  # the first goes back
    ([0, 60, 101], [0, 60, 100], slice(0, 60), slice(0, 60)),    # past the tensor
    ([-5, 40, 100], [0, 60, 100], slice(40, 100), slice(60, 100)),  # before it
    ([0, 60, 100], [0, 60, 30], slice(0, 60), slice(0, 60)),     # no keys
])
def test_sequences_next_to_bad_starts(kind, q_start, k_start, rows, keys):
    q, k, v = problem([100], [100], 4, 2, kind)
    do = normal(9, *q.shape, kind=kind, by=0.1)
    n = [rows.stop - rows.start], [keys.stop - keys.start]
    mine = [t[part].contiguous() for t, part in zip((do, q, k, v), (rows, rows, keys, keys))]
    sums = run(*mine[1:], *n)
    want = grads(*mine, *sums, *n)
    o, lse = torch.zeros_like(q), torch.zeros(4, 100, device="cuda")
    o[rows], lse[:, rows] = sums
    out, ws = [torch.full_like(t, 7.0) for t in (q, k, v)], workspace(100, 4, backward=True)
    ress.attn_bwd(do, q, k, v, o, lse, *out, ws, ints(q_start), ints(k_start))
    with pytest.raises(ress.RessError) as e:
        ress.status(ws)
    assert e.value.code == -6
    for got, w, part in zip(out, want, (rows, keys, keys)):
        assert torch.equal(got[part], w)

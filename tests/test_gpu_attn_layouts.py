"""Gradients with heads of larger tensors as inputs and outputs, and batches of very many sequences."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2609_35593_gb300 as ress  # noqa: E402
from test_gpu_attn import BF16, F16, R, float32_by_default, ints, normal, problem, run, workspace  # noqa: E402,F401
from test_gpu_attn_bwd import grads  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("layout", ["one tensor of gradients", "heads outside", "rows of 72"])
def test_gradients_of_strided_heads(kind, layout):
    """The same bits as of contiguous tensors, and what lies between the heads stays."""
    lens, heads, kv = ([130, 70], [130, 70]), 6, 2
    n = 200
    q, k, v = problem(*lens, heads, kv, kind)
    do = normal(9, *q.shape, kind=kind, by=0.1)
    o, lse = run(q, k, v, *lens, causal=True)
    want = grads(do, q, k, v, o, lse, *lens, causal=True)

    def places(*counts):
        """Room for tensors of so many heads, and what surrounds them."""
        if layout == "one tensor of gradients":  # [tokens, heads of all, 64]
            big = torch.full((n, sum(counts) + 1, 64), 7.0, dtype=kind, device="cuda")
            views = list(big[:, :-1].split(counts, 1))
        elif layout == "heads outside":
            big = torch.full((sum(counts) + 1, n, 64), 7.0, dtype=kind, device="cuda")
            views = [t.transpose(0, 1) for t in big[:-1].split(counts, 0)]
        else:
            big = torch.full((n + 1, sum(counts), 72), 7.0, dtype=kind, device="cuda")
            views = [t[..., :64] for t in big[:-1].split(counts, 1)]
        return big, views

    _, ins = places(heads, heads, kv, kv, heads)
    for t, x in zip(ins, (do, q, k, v, o)):
        t.copy_(x)
    big, outs = places(heads, kv, kv)
    ws = workspace(n, heads, backward=True)
    ress.attn_bwd(*ins, lse, *outs, ws, R.starts(lens[0]), R.starts(lens[1]), causal=True)
    ress.status(ws)
    for g, w in zip(outs, want):
        assert torch.equal(g, w)
        g.fill_(7.0)
    assert (big == 7).all()  # nothing else was written


@pytest.mark.parametrize("backward", [False, True])
def test_a_million_sequences(backward):
    """As many as a call takes, empty but for a few; the waits of the others' CTAs last."""
    n, heads = 1 << 20, 2
    some = {0: (70, 90), 3: (1, 40), n // 2: (300, 200), n // 2 + 1: (0, 5), n // 2 + 2: (5, 0), n - 1: (130, 130)}
    q_lens, k_lens = (torch.zeros(n, dtype=torch.int64) for _ in range(2))
    for b, (x, y) in some.items():
        q_lens[b], k_lens[b] = x, y
    starts = [torch.cat([torch.zeros(1, dtype=torch.int64), t.cumsum(0)]).int().cuda() for t in (q_lens, k_lens)]
    lens = [list(t) for t in zip(*some.values())]
    q, k, v = problem(*lens, heads, 1)
    do = normal(9, *q.shape, by=0.1)
    o, lse = run(q, k, v, *lens)
    got, sums, ws = torch.zeros_like(q), torch.zeros_like(lse), workspace(q.shape[0], heads, backward=True)
    ress.attn(q, k, v, got, ws, *starts, lse=sums)
    ress.status(ws)
    assert torch.equal(got, o) and torch.equal(sums, lse)
    if backward:
        want, out = grads(do, q, k, v, o, lse, *lens), [torch.full_like(t, 7.0) for t in (q, k, v)]
        ress.attn_bwd(do, q, k, v, o, lse, *out, ws, *starts)
        ress.status(ws)
        assert all(torch.equal(a, b) for a, b in zip(out, want))

"""f16 has ten binary digits above 2^-14 and loses them below: probabilities and gradients keep them by powers of two that
belong to a row or a sequence, whatever others of the same call hold."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2609_35593_gb300 as ress  # noqa: E402
from gradients64 import gradients  # noqa: E402
from test_gpu_attn import F16, R, float32_by_default, normal, problem, run, workspace  # noqa: E402,F401
from test_gpu_attn_bwd import grads  # noqa: E402

pytestmark = pytest.mark.gpu


def check(q, k, v, do, lens, **mask):
    o, lse = run(q, k, v, *lens, **mask)
    want, off = gradients(do, q, k, v, o, lse, *lens, **mask)
    for g, w, f, name in zip(grads(do, q, k, v, o, lse, *lens, **mask), want, off, ("dq", "dk", "dv")):
        R.close(g, w, f, name)


@pytest.mark.parametrize("lens", [([70, 200, 3], [300, 200, 900]), ([40] * 8, [33, 1, 64, 500, 31, 97, 700, 40]), ([600, 600], [600, 600])],
                         ids=str)
@pytest.mark.parametrize("heads,kv", [(2, 2), (6, 2)])
@pytest.mark.parametrize("causal", [False, True])
def test_sequences_of_other_sizes(lens, heads, kv, causal):
    """dO of packed sequences 2^14 apart, and V 2^6 apart the other way round."""
    q, k, v = problem(*lens, heads, kv, F16)
    do = normal(9, *q.shape, kind=F16)
    a = b = 0
    for i, (nq, nk) in enumerate(zip(*lens)):
        if i % 2 == 0:
            do[a:a + nq] *= 2.0 ** -10
            v[b:b + nk] *= 2.0 ** 3
        else:
            do[a:a + nq] *= 2.0 ** 4
            v[b:b + nk] *= 2.0 ** -3
        a, b = a + nq, b + nk
    check(q, k, v, do, lens, causal=causal)


@pytest.mark.parametrize("rows,keys", [(96, 10992), (700, 700)])
def test_one_row_far_above_the_others(rows, keys):
    """dq of the others keeps its digits, on keys with probabilities near 1e-4 as well."""
    q, k, v = problem([rows], [keys], 2, 1, F16)
    do = normal(9, *q.shape, kind=F16, by=2.0 ** -6)
    do[rows // 2] *= 2.0 ** 12
    check(q, k, v, do, ([rows], [keys]))


@pytest.mark.parametrize("by", [2.0 ** -12, 1.0, 300.0, 2000.0])
def test_values_of_any_size(by):
    """ds is kept times a power of two that comes from V's own size."""
    q, k, v = problem([200, 40], [300, 50], 4, 2, F16)
    do = normal(9, *q.shape, kind=F16, by=2.0 ** -4)
    check(q, k, (v.float() * by).to(F16), do, ([200, 40], [300, 50]), causal=True)


@pytest.mark.parametrize("edge", [0, 15, 16, 150000, 150001, 200003])
def test_the_largest_value_anywhere(edge):
    """V's largest row, which bounds ds, inside a chunk of keys, at its ends and at those of a sequence."""
    lens = ([40, 8], [150001, 50003])
    q, k, v = problem(*lens, 2, 1, F16)
    v[edge] *= 2.0 ** 10
    do = normal(9, *q.shape, kind=F16, by=2.0 ** -6)
    check(q, k, v, do, lens)


def test_gradients_of_nothing():
    """dO of zero, V of zero: zeros, not 0 x infinity."""
    q, k, v = problem([50, 60], [50, 60], 2, 2, F16)
    do = normal(9, *q.shape, kind=F16)
    do[:50] = 0
    v[50:] = 0
    check(q, k, v, do, ([50, 60], [50, 60]))


def test_no_rows_or_no_keys():
    """Alone, and between sequences that have both."""
    for lens in (([0], [70]), ([70], [0]), ([40, 0, 30, 20], [50, 60, 0, 20])):
        q, k, v = problem(*lens, 4, 2, F16)
        check(q, k, v, normal(9, *q.shape, kind=F16), lens)


@pytest.mark.parametrize("bad", [30000.0, -30000.0, math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("causal", [False, True])
def test_neighbours_of_any_size(bad, causal):
    """Not a bit of a sequence's gradients depends on what dO and V of the others are."""
    lens = ([70, 30, 170], [90, 30, 150])
    q, k, v = problem(*lens, 6, 2, F16)
    do = normal(9, *q.shape, kind=F16, by=0.1)
    o, lse = run(q, k, v, *lens, causal=causal)
    want = grads(do, q, k, v, o, lse, *lens, causal=causal)
    do[70:100] = v[90:120] = bad
    got = grads(do, q, k, v, o, lse, *lens, causal=causal)
    for rows, keys in ((slice(0, 70), slice(0, 90)), (slice(100, 270), slice(120, 270))):
        assert torch.equal(got[0][rows], want[0][rows])
        assert torch.equal(got[1][keys], want[1][keys]) and torch.equal(got[2][keys], want[2][keys])




def test_captured_with_other_lengths():
    """A replayed graph finds the powers of the sequences that it has then."""
    heads, n = 4, 500
    q, k, v = problem([n], [n], heads, 2, F16)
    do = normal(9, *q.shape, kind=F16, by=0.1)
    do[n // 2:] *= 2.0 ** -12
    o, lse, out = torch.zeros_like(q), torch.zeros(heads, n, device="cuda"), [torch.zeros_like(t) for t in (q, k, v)]
    starts, ws = R.starts([n, 0]), workspace(n, heads, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ress.attn(q, k, v, o, ws, starts, starts, lse=lse, causal=True)
        ress.attn_bwd(do, q, k, v, o, lse, *out, ws, starts, starts, causal=True)
    for lens in ([500, 0], [250, 250], [77, 423], [0, 500]):
        starts.copy_(R.starts(lens))
        graph.replay()
        ress.status(ws)
        for a, b in zip(grads(do, q, k, v, *run(q, k, v, lens, lens, causal=True), lens, lens, causal=True), out):
            assert torch.equal(a, b)
        want, off = gradients(do, q, k, v, o, lse, lens, lens, causal=True)
        for g, w, f in zip(out, want, off):
            R.close(g, w, f)

"""Gradients of dense attention against the formula in float64, and against differences."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import dense64 as R  # noqa: E402
import paper_2609_35593_gb300 as ress  # noqa: E402
from test_gpu_attn import BF16, F16, ints, masks, normal, problem, run, workspace  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def float32_by_default():
    """Tensors made without a dtype here are float32, whatever other files left as the default."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def grads(do, q, k, v, o, lse, q_lens, k_lens, **mask):
    out = [torch.full_like(t, 7.0) for t in (q, k, v)]
    ws = workspace(*q.shape[:2], backward=True)
    ress.attn_bwd(do, q, k, v, o, lse, *out, ws, R.starts(q_lens), R.starts(k_lens), **mask)
    ress.status(ws)
    return out


def check(q_lens, k_lens, heads, kv, kind=BF16, by=0.1, **mask):
    q, k, v = problem(q_lens, k_lens, heads, kv, kind)
    do = normal(9, *q.shape, kind=kind, by=by)
    o, lse = run(q, k, v, q_lens, k_lens, **mask)
    want, off = R.gradients(do, q, k, v, o, lse, q_lens, k_lens, **mask)
    got = grads(do, q, k, v, o, lse, q_lens, k_lens, **mask)
    for g, w, f, name in zip(got, want, off, ("dq", "dk", "dv")):
        R.close(g, w, f, name)


LENGTHS = [([1], [1]), ([63], [65]), ([128], [64]), ([129], [127]), ([256], [256]), ([1], [700]), ([200], [50]),
           ([5, 0, 1, 300, 64], [5, 7, 0, 300, 1]), ([700, 3, 129], [700, 900, 129])]


@pytest.mark.parametrize("lens", LENGTHS, ids=str)
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (12, 4), (10, 2), (16, 1)])
@pytest.mark.parametrize("causal", [False, True])
def test_gradients_of_packed_sequences(lens, heads, kv, causal):
    check(*lens, heads, kv, causal=causal)


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("causal,prefix,cap,slopes", [(True, True, 0.0, False), (True, False, 30.0, False),
                                                      (False, False, 0.0, True), (True, True, 20.0, True),
                                                      (False, False, 2.0, False), (False, False, 0.0, False)])
@pytest.mark.parametrize("heads,kv", [(4, 4), (6, 2), (48, 1), (64, 1)])
def test_gradients_through_masks_caps_and_slopes(kind, causal, prefix, cap, slopes, heads, kv):
    lens = ([150, 1, 400, 33], [150, 700, 390, 40])
    check(*lens, heads, kv, kind, **masks(heads, lens[1], causal, prefix, cap, slopes))


@pytest.mark.parametrize("by", [1e-4, 1.0, 100.0])
def test_gradients_of_any_size_in_f16(by):
    check([500], [500], 2, 2, F16, by=by)


def test_long_sequences_split_over_ctas():
    check([2500, 2, 1000], [2700, 3000, 1000], 4, 2, causal=True)


def test_slopes_at_positions_past_float32():
    """Distances are those of integers also where a position has more than 24 bits.  Keys 2,000 back and more weigh e^-2000."""
    n, near, rows = (1 << 24) + 2001, 2000, 150
    q, k, v = problem([rows], [near], 2, 1)
    do = normal(9, *q.shape, by=0.1)
    mask = {"causal": True, "slopes": torch.ones(2, device="cuda")}
    far = [torch.zeros(n, 1, 64, dtype=BF16, device="cuda") for _ in range(2)]
    far[0][-near:], far[1][-near:] = k, v
    o, lse = run(q, *far, [rows], [n], **mask)
    want, off = R.gradients(do, q, k, v, o, lse, [rows], [near], **mask)
    dq, dk, dv = grads(do, q, *far, o, lse, [rows], [n], **mask)
    for g, w, f, name in zip((dq, dk[-near:], dv[-near:]), want, off, ("dq", "dk", "dv")):
        R.close(g, w, f, name)
    assert (dk[:-near] == 0).all() and (dv[:-near] == 0).all()


def test_rows_and_keys_behind_the_last_sequence():
    """A padded batch: what is behind is neither read into results nor written."""
    lens, pad = ([130, 70], [130, 70]), 41
    n = sum(lens[0]) + pad
    q, k, v = problem([n], [n], 4, 2, F16)
    do = normal(9, *q.shape, kind=F16)
    o, lse = run(q, k, v, *lens)
    want = grads(*(t[:-pad].contiguous() for t in (do, q, k, v, o)), lse[:, :-pad].contiguous(), *lens)
    for t in (do, q, k, v, o):
        t[-pad:] = math.nan
    lse[:, -pad:] = math.nan
    got = grads(do, q, k, v, o, lse, *lens)
    for g, w in zip(got, want):
        assert torch.equal(g[:-pad], w) and (g[-pad:] == 7).all()


def test_no_rows_or_no_keys():
    q, k, v = problem([0], [70], 2, 2)
    lse = torch.empty(2, 0, device="cuda")
    _, dk, dv = grads(q, q, k, v, q, lse, [0], [70])
    assert (dk == 0).all() and (dv == 0).all()
    q, k, v = problem([70], [0], 2, 2)
    dq = grads(q, q, k, v, torch.zeros_like(q), torch.full((2, 70), -math.inf, device="cuda"), [70], [0])[0]
    assert (dq == 0).all()


def test_many_sequences_without_rows_or_keys():
    n = 1500
    lens = ([70, 300] + [0, 3] * n + [130], [70, 300] + [3, 0] * n + [130])
    q, k, v = problem(*lens, 2, 2)
    do = normal(9, *q.shape)
    o, lse = run(q, k, v, *lens)
    got = grads(do, q, k, v, o, lse, *lens)
    whole = [70, 300, 130]
    keep = torch.cat([torch.arange(370), torch.arange(370 + 3 * n, 500 + 3 * n)]).cuda()
    want = grads(*(t[keep] for t in (do, q, k, v, o)), lse[:, keep].contiguous(), whole, whole)
    for g, w in zip(got, want):
        # other shares of the work: float32 sums in another order, of values below 8
        assert (g[keep].float() - w.float()).abs().max() <= 2.0 ** -7 * w.float().abs().max() and (g[370:370 + 3 * n] == 0).all()


def test_same_bits_again():
    lens = ([300, 1000], [2000, 1000])
    q, k, v = problem(*lens, 4, 2)
    do = normal(9, *q.shape)
    o, lse = run(q, k, v, *lens, causal=True)
    first = grads(do, q, k, v, o, lse, *lens, causal=True)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(grads(do, q, k, v, o, lse, *lens, causal=True), first))


def test_against_differences():
    """sum(do o) along random directions.  The step is exact in the inputs' type (a power of two times signs on
    inputs rounded to coarser steps), the loss is float64's at the two ends; the central difference is off by a third derivative times
    the step's square / 6, bounded by halving the step: a quarter of the change per halving."""
    lens, kind = ([40, 30], [40, 50]), F16
    mask = masks(4, lens[1], True, True, 3.0, True)
    q, k, v = ((t * 64).round().clamp(-127, 127) / 64 for t in problem(*lens, 4, 2, kind))
    do = normal(9, *q.shape, kind=kind)
    o, lse = run(q, k, v, *lens, **mask)
    got = grads(do, q, k, v, o, lse, *lens, **mask)
    _, off = R.gradients(do, q, k, v, o, lse, *lens, **mask)
    loss = lambda *x: (do.double() * R.attention(*(t.to(kind) for t in x), *lens, **mask)[0]).sum()
    for i, t in enumerate((q, k, v)):
        sign = normal(20 + i, *t.shape, kind=torch.float32).sign().to(kind)
        ends = []
        for h in (2.0 ** -7, 2.0 ** -8):
            x = [u.clone() for u in (q, k, v)]
            x[i] = t + h * sign
            up = loss(*x)
            x[i] = t - h * sign
            ends.append(((up - loss(*x)) / (2 * h)).item())
        slope = (got[i].double() * sign.double()).sum().item()
        # o and lse, as the kernel takes them, are rounded: delta = O.dO by u |o do| of each row, times sum p |k| / 8
        rounding = 2.0 ** -11 * (o.double() * do.double()).abs().sum().item() if i < 2 else 0.0
        bound = off[i].sum().item() + abs(ends[0] - ends[1]) + rounding
        assert abs(slope - ends[1]) <= bound, (i, slope, ends, bound)


def test_captured_with_eager_calls_of_other_lengths():
    heads, n = 4, 500
    q, k, v = problem([n], [n], heads, 2)
    do = normal(9, *q.shape)
    o, lse, out = torch.zeros_like(q), torch.zeros(heads, n, device="cuda"), [torch.zeros_like(t) for t in (q, k, v)]
    starts, ws = R.starts([n, 0]), workspace(n, heads, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ress.attn(q, k, v, o, ws, starts, starts, lse=lse, causal=True)
        ress.attn_bwd(do, q, k, v, o, lse, *out, ws, starts, starts, causal=True)
    for lens in ([500, 0], [77, 423], [0, 500]):
        starts.copy_(R.starts(lens))
        graph.replay()
        ress.status(ws)
        eager = run(q, k, v, lens, lens, causal=True)
        assert torch.equal(eager[0], o) and torch.equal(eager[1], lse)
        for a, b in zip(grads(do, q, k, v, *eager, lens, lens, causal=True), out):
            assert torch.equal(a, b)

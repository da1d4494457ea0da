"""What a sequence does not see changes no bit of its results, also where scores are capped: stale rows of pages, keys and rows
of its neighbours, padding."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2609_35593_gb300 as ress  # noqa: E402
from test_gpu_attn import BF16, F16, R, float32_by_default, ints, normal, paged, problem, run, workspace  # noqa: E402,F401
from test_gpu_attn_bwd import grads  # noqa: E402

pytestmark = pytest.mark.gpu

LENS = ([70, 30, 170], [90, 30, 150])
MINE = ((slice(0, 70), slice(0, 90)), (slice(100, 270), slice(120, 270)))  # rows and keys of the first and the last
OTHER, OTHER_KEYS = slice(70, 100), slice(90, 120)
# products of 30,000 with what is near 1 are far above every cap here, and below the types' largest numbers
GARBAGE = (30000.0, -30000.0, math.inf, -math.inf, math.nan)


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("cap,slopes", [(30.0, False), (50.0, True), (2.0, False), (0.0, False)])
@pytest.mark.parametrize("causal", [False, True])
def test_neighbours(kind, cap, slopes, causal):
    heads = 6
    mask = {"causal": causal, "cap": cap, "slopes": torch.logspace(-3, 0, heads, device="cuda") if slopes else None}
    q, k, v = problem(*LENS, heads, 2, kind)
    want = run(q, k, v, *LENS, **mask)
    for bad in GARBAGE:
        x, y, z = q.clone(), k.clone(), v.clone()
        x[OTHER] = y[OTHER_KEYS] = z[OTHER_KEYS] = bad
        o, lse = run(x, y, z, *LENS, **mask)
        for rows, _ in MINE:
            assert torch.equal(lse[:, rows], want[1][:, rows]) and torch.equal(o[rows], want[0][rows]), bad


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("cap,slopes", [(30.0, False), (50.0, True), (2.0, False), (0.0, False)])
@pytest.mark.parametrize("causal", [False, True])
def test_neighbours_in_the_gradient(kind, cap, slopes, causal):
    heads = 6
    mask = {"causal": causal, "cap": cap, "slopes": torch.logspace(-3, 0, heads, device="cuda") if slopes else None}
    q, k, v = problem(*LENS, heads, 2, kind)
    do = normal(9, *q.shape, kind=kind, by=0.1)
    o, lse = run(q, k, v, *LENS, **mask)
    want = grads(do, q, k, v, o, lse, *LENS, **mask)
    for bad in GARBAGE:
        t = [x.clone() for x in (q, k, v, o)]
        for x, part in zip(t, (OTHER, OTHER_KEYS, OTHER_KEYS, OTHER)):
            x[part] = bad
        sums = lse.clone()
        sums[:, OTHER] = bad
        dq, dk, dv = grads(do, *t, sums, *LENS, **mask)
        for rows, keys in MINE:
            assert torch.equal(dq[rows], want[0][rows]), bad
            assert torch.equal(dk[keys], want[1][keys]) and torch.equal(dv[keys], want[2][keys]), bad


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("cap,slopes", [(30.0, False), (50.0, True), (2.0, False), (0.0, False)])
@pytest.mark.parametrize("lens", [([1, 1, 1], [70, 1, 129]), ([17, 130], [100, 130])], ids=str)
def test_stale_rows_of_pages(kind, cap, slopes, lens):
    heads, page = 6, 24
    mask = {"causal": True, "cap": cap, "slopes": torch.logspace(-3, 0, heads, device="cuda") if slopes else None}
    q, k, v = problem(*lens, heads, 2, kind)
    kp, vp, table = paged(k, v, lens[1], page)
    unused = kp.isnan()
    got = []
    for bad in (0.0, *GARBAGE):
        kp[unused], vp[unused] = bad, bad
        o, lse, ws = torch.empty_like(q), torch.empty(heads, sum(lens[0]), device="cuda"), workspace(*q.shape[:2])
        ress.paged_attn(q, kp, vp, table, ints(lens[1]), o, ws, R.starts(lens[0]), lse=lse, **mask)
        ress.status(ws)
        got.append((o, lse))
    for o, lse in got[1:]:
        assert torch.equal(lse, got[0][1]) and torch.equal(o, got[0][0])


@pytest.mark.parametrize("cap", [30.0, 0.0])
def test_padding(cap):
    """Rows and keys behind the last sequence."""
    lens, pad = ([130, 70], [130, 70]), 41
    q, k, v = problem([200 + pad], [200 + pad], 4, 2)
    want = run(q, k, v, *lens, causal=True, cap=cap)
    for bad in GARBAGE:
        for t in (q, k, v):
            t[-pad:] = bad
        o, lse = run(q, k, v, *lens, causal=True, cap=cap)
        assert torch.equal(o[:200], want[0][:200]) and torch.equal(lse[:, :200], want[1][:, :200])
        assert (o[-pad:] == 7).all() and (lse[:, -pad:] == 7).all()

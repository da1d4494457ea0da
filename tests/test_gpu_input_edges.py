"""Layer norm and rotary positions where lanes without channels, or the ends of the ranges, must not show."""
from fractions import Fraction

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DEPTH, U32 = 64, 2.0 ** -24  # of the float32 sums, and of one rounding
ROUND = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
BIG, EPS = 2.0 ** 120, 1e-5  # BIG / sqrt(EPS) is past the largest float32


@pytest.fixture(scope="module")
def ress():
    import paper_2609_35593_gb300 as r
    return r


@pytest.fixture(autouse=True)
def float32_by_default():
    """Tensors made without a dtype here are float32, whatever other files left as the default."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def normal(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def centred_bound(g, r, want, kind):
    """Error of r (g - avg g) in float32 and of its rounding: the mean's, and five roundings on the way."""
    return r * (DEPTH * U32 * g.abs().mean(-1, keepdim=True) + 8 * U32 * (g.abs() + g.mean(-1, keepdim=True).abs())) + \
        1.01 * ROUND[kind] * want.abs()


@pytest.mark.parametrize("width", [24, 33, 72, 136, 264, 1021, 1032, 2049, 4104, 5000, 9001, 16000])
@pytest.mark.parametrize("kind", [BF16, F32])
def test_layer_norm_gradient_of_huge_constant_rows(ress, kind, width):
    """Every h = (x - mean) rstd is 0, and dx = rstd (g - avg g) is finite, although mean rstd is not."""
    for rows in (3, 70):
        x = torch.full((rows, width), BIG, device="cuda", dtype=kind)
        dy, w = normal(width, rows, width).to(kind), 1 + 0.3 * normal(width + 1, width)
        mean = torch.full((rows,), BIG, device="cuda")
        rstd = torch.full((rows,), EPS ** -0.5, device="cuda")
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
        ws = torch.empty(ress.layer_norm_workspace_bytes(rows, width), dtype=torch.uint8, device="cuda")
        ress.layer_norm_bwd(dy, x, w, mean, rstd, dx, dweight=dw, dbias=db, ws=ws)
        g, r = dy.double() * w.double(), rstd.double()[:, None]
        want = r * (g - g.mean(-1, keepdim=True))
        assert bool(((dx.double() - want).abs() <= centred_bound(g, r, want, kind)).all()), rows
        assert not dw.any()
        assert bool(((db.double() - dy.double().sum(0)).abs() <= (rows + 192) * U32 * dy.double().abs().sum(0)).all())


@pytest.mark.parametrize("hd,heads", [(24, 1), (24, 3), (24, 11), (48, 8), (96, 1), (96, 2), (96, 3), (96, 4)])
@pytest.mark.parametrize("layout", ["halves", "interleaved"])
@pytest.mark.parametrize("kind", [BF16, F32])
def test_head_norm_gradient_of_huge_constant_heads(ress, kind, layout, hd, heads):
    """Heads that leave lanes without channels.  (A head's mean is exact: 24, 48 and 96 are 3 times a power of two,
    and 3 times 1/3 in float32 rounds to 1.)"""
    tokens, plan = 50, ress.rope_plan((hd,), head_dim=hd, layout=layout)
    pos = torch.zeros(tokens, 1, dtype=torch.int32, device="cuda")
    x = torch.full((tokens, heads, hd), BIG, device="cuda", dtype=kind)
    dy, w, b = normal(hd + heads, tokens, heads, hd).to(kind), 1 + 0.3 * normal(5, hd), normal(6, hd)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    ws = torch.empty(ress.rope_workspace_bytes(plan, tokens, heads), dtype=torch.uint8, device="cuda")
    ress.rope_bwd(plan, pos, dy, dx, q=x, q_norm=(w, b), q_norm_grads=(dw, db), eps=EPS, ws=ws)
    g, r = dy.double() * w.double(), EPS ** -0.5
    want = r * (g - g.mean(-1, keepdim=True))
    assert bool(((dx.double() - want).abs() <= centred_bound(g, r, want, kind)).all())
    assert not dw.any()
    total = dy.double().sum((0, 1))
    assert bool(((db.double() - total).abs() <= (tokens * heads + 192) * U32 * dy.double().abs().sum((0, 1))).all())


def test_rope_of_given_frequencies_at_the_ends_of_int32(ress):
    """The angle is position times frequency: its turns are good to the position times 2^-64, the kernel takes the
    upper 32 bits, rounds them to float32, and cos and sin are good to two units in the last place."""
    freq = [100.0, 1000.0, -1e-4, -1.0, 1e-9, 0.7, 12345.678, -3e5]
    where = [-2 ** 31, 2 ** 31 - 1, 2 ** 30 + 12345, -77777777, 1, -1, 43968, 0]
    plan = ress.rope_plan((16,), head_dim=16, layout="interleaved", freq=freq)
    pos = torch.tensor(where, device="cuda", dtype=torch.int32)[:, None].contiguous()
    x = torch.zeros(len(where), 1, 16, device="cuda")
    x[..., 0::2] = 1.0
    y = torch.empty_like(x)
    ress.rope(plan, pos, x, y)
    two_pi = Fraction("6.28318530717958647692528676655900576839433879875021164194988918461563281257")
    for i, p in enumerate(where):
        for k, f in enumerate(freq):
            angle = torch.tensor(float(p * Fraction(f) % two_pi), dtype=torch.float64)
            # half turns in [-1, 1], rounded: 2^-25 of them, so pi 2^-25; 2^-32 turns; 2^-32 of them in 2^-64 p
            bound = 3.2 * 2.0 ** -25 + 2 * 6.3 * 2.0 ** -32 + 2 * 2.0 ** -24
            assert abs(float(y[i, 0, 2 * k]) - float(torch.cos(angle))) <= bound, (p, f)
            assert abs(float(y[i, 0, 2 * k + 1]) - float(torch.sin(angle))) <= bound, (p, f)


def test_heads_as_the_library_takes_them(ress):
    """The bytes that the binding makes of tensors are those of the struct that callers with raw pointers pack."""
    x = torch.zeros(7, 10, 64, device="cuda")[:, 1:4]
    y, dx = torch.zeros(7, 3, 64, device="cuda"), torch.zeros(3, 7, 64, device="cuda").transpose(0, 1)
    w, b, dw, db = torch.zeros(4, 64, device="cuda").unbind()
    got = ress._t.rope_heads(y, x, dx, (w, b), (dw, db), 7, 64, 2)
    assert len(got) == ress._ROPE_HEADS.size
    assert ress._ROPE_HEADS.unpack(got) == (3, 1, w.data_ptr(), b.data_ptr(), x.data_ptr(), 640, 64, y.data_ptr(), 192, 64,
                                            dx.data_ptr(), 64, 448, dw.data_ptr(), db.data_ptr())

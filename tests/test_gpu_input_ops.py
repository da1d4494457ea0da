"""The operators that form Q, K and V out of the residual stream, and their gradients, against the
same in float64, with error bounds derived from the float32 sums and the one rounding of a result.

A float32 sum over the threads of a row goes through at most 32 terms in a thread, 5 steps over a
warp and 16 over a CTA's warps: its error is at most DEPTH 2^-24 of the sum of magnitudes."""
import math
from fractions import Fraction

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DEPTH = 64
U32 = 2.0 ** -24
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
E = DEPTH * U32


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


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def rounded(y, kind):
    """Error of one rounding of y to a type: relative, and absolute where it is subnormal."""
    return ROUND[kind] * y.abs() * (1 + 2.0 ** -8) + TINY[kind]


def within(got, want, bound, name=""):
    assert got.shape == want.shape
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (name, int(bad.sum()), float(((got.double() - want).abs() / bound)[bad].max()))


# ---- layer norm ------------------------------------------------------------------------------
def norm64(x, w, b, eps):
    mean = x.mean(-1, keepdim=True)
    c = x - mean
    rstd = (c.square().mean(-1, keepdim=True) + eps).rsqrt()
    return c * rstd, mean, rstd, c * rstd * w + b


def norm_bound(x, h, w, b, rstd):
    """Error of h w + b in float32, h from float32 sums: the mean's error moves every channel alike,
    and the variance by its square."""
    shift = E * x.abs().mean(-1, keepdim=True) * rstd
    err = (h.abs() + shift) * (E + shift.square()) + shift
    return w.abs() * err + 4 * U32 * (w.abs() * h.abs() + b.abs())


WIDTHS = [1, 2, 7, 8, 17, 63, 64, 72, 128, 136, 192, 256, 257, 264, 768, 1021, 1024, 2048, 4096, 4100, 4104,
          5000, 16384]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("x_type,y_type", [(BF16, BF16), (F16, F16), (F32, F32), (F32, BF16), (F32, F16)])
def test_layer_norm_and_gradient(ress, width, x_type, y_type):
    eps = 1e-5
    for rows, params in ((1, F32), (37, x_type), (1030, F32)):
        g = gen(rows * 100003 + width)
        x = (normal(g, rows, width) * (0.5 * normal(g, width)).exp() + 3.0 * normal(g, width)).to(x_type)
        w, b = (1 + 0.3 * normal(g, width)).to(params), (0.2 * normal(g, width)).to(params)
        y = torch.full((rows, width), float("nan"), device="cuda", dtype=y_type)
        mean, rstd = torch.full((2, rows), float("nan"), device="cuda").unbind()
        ress.layer_norm(x, w, b, y, eps=eps, mean=mean, rstd=rstd)
        x64, w64, b64 = x.double(), w.double(), b.double()
        h, m64, r64, y64 = norm64(x64, w64, b64, eps)
        within(mean, m64[:, 0], E * x64.abs().mean(-1), "mean")
        shift = E * x64.abs().mean(-1) * r64[:, 0]
        within(rstd, r64[:, 0], r64[:, 0] * (E + shift.square() + 4 * U32), "rstd")
        within(y, y64, rounded(y64, y_type) + norm_bound(x64, h, w64, b64, r64), "y")

        # the gradient with the statistics that the forward pass saved
        dy, dres = (0.3 * normal(g, rows, width)).to(y_type), normal(g, rows, width).to(x_type)
        m, r = mean.double()[:, None], rstd.double()[:, None]
        h = (x64 - m) * r
        gr = dy.double() * w64
        ag, agh = gr.mean(-1, keepdim=True), (gr * h).mean(-1, keepdim=True)
        core = r * (gr - ag - h * agh)
        err = r * (E * (gr.abs().mean(-1, keepdim=True) + h.abs() * (gr * h).abs().mean(-1, keepdim=True)) +
                   8 * U32 * (gr.abs() + ag.abs() + (h * agh).abs()))
        ws = torch.empty(ress.layer_norm_workspace_bytes(rows, width), dtype=torch.uint8, device="cuda")
        for res in (None, dres):
            dx = torch.full((rows, width), float("nan"), device="cuda", dtype=x_type)
            dw, db = torch.full((2, width), float("nan"), device="cuda").unbind()
            ress.layer_norm_bwd(dy, x, w, mean, rstd, dx, dweight=dw, dbias=db, dres=res, ws=ws)
            want = core if res is None else core + res.double()
            within(dx, want, rounded(want, x_type) + err + (0 if res is None else U32 * res.double().abs()), "dx")
            # rows of a thread, then warps, CTAs and the second kernel's 32 and 32
            depth = (rows + 128 + 64) * U32
            within(dw, (dy.double() * h).sum(0), depth * (dy.double() * h).abs().sum(0) + 1e-30, "dweight")
            within(db, dy.double().sum(0), depth * dy.double().abs().sum(0) + 1e-30, "dbias")


def test_layer_norm_without_parameters_in_place_and_partial_outputs(ress):
    g = gen(5)
    x = normal(g, 300, 520).to(BF16)
    want = norm64(x.double(), 1.0, 0.0, 0.0)[3]
    y = x.clone()
    ress.layer_norm(y, None, None, y, eps=0.0)
    within(y, want, rounded(want, BF16) + 2 * E * (1 + want.abs()))
    # weight alone, bias alone; a gradient of one of the two; none at all, without a workspace
    w, b = normal(g, 520), normal(g, 520)
    y2 = torch.empty_like(x)
    ress.layer_norm(x, w, None, y2, eps=0.0)
    within(y2, want * w.double(), rounded(want * w.double(), BF16) + 2 * E * w.double().abs() * (1 + want.abs()))
    mean, rstd = torch.empty(2, 300, device="cuda").unbind()
    ress.layer_norm(x, None, b, y2, mean=mean, rstd=rstd)
    dy = normal(g, 300, 520).to(BF16)
    ws = torch.empty(ress.layer_norm_workspace_bytes(300, 520), dtype=torch.uint8, device="cuda")
    full, dw, db = torch.empty_like(x), torch.empty(520, device="cuda"), torch.empty(520, device="cuda")
    ress.layer_norm_bwd(dy, x, w, mean, rstd, full, dweight=dw, dbias=db, ws=ws)
    for kw in ({"dweight": torch.empty(520, device="cuda")}, {"dbias": torch.empty(520, device="cuda")}, {}):
        dx = dy.clone()
        ress.layer_norm_bwd(dx, x, w, mean, rstd, dx, ws=ws if kw else None, **kw)  # in place
        assert torch.equal(dx, full)
        for name, t in kw.items():
            assert torch.equal(t, dw if name == "dweight" else db)


@pytest.mark.parametrize("x_type", [BF16, F32])
def test_layer_norm_strides_and_alignment(ress, x_type):
    """Rows of a wider tensor, rows that start off a 16-byte boundary, one row for all."""
    g = gen(9)
    rows, width = 70, 1024
    w, b = 1 + 0.1 * normal(g, width + 1), normal(g, width + 1)
    for off, pitch in ((0, 1040), (8, 1040), (3, 1040), (0, 1031), (16, 1040)):
        wide = normal(g, rows, pitch + 16).to(x_type)
        x = wide[:, off:off + width]
        for xs in (x, x[5:6].expand(rows, width)):
            out = torch.full((rows, pitch + 16), 7.0, device="cuda", dtype=x_type)
            y = out[:, off:off + width]
            ress.layer_norm(xs, w[1:], b[1:], y)  # parameters off a 16-byte boundary too
            h, _, r64, want = norm64(xs.double(), w[1:].double(), b[1:].double(), 1e-5)
            within(y, want, rounded(want, x_type) + norm_bound(xs.double(), h, w[1:].double(), b[1:].double(), r64))
            out[:, off:off + width] = 7.0
            assert bool((out == 7.0).all())  # nothing written beside the rows


@pytest.mark.parametrize("width", [257, 263, 511, 1023, 1025, 2049, 4095, 4097, 8191, 8193, 16383])
@pytest.mark.parametrize("x_type,y_type", [(BF16, BF16), (F32, F32), (F32, F16)])
def test_layer_norm_rows_between_vectors(ress, width, x_type, y_type):
    """Rows that start at any element of a vector, from the number of rows that they are worth it on: all
    tensors at the same one, and not; a row that is not finite, and what lies beside the rows."""
    eps = 1e-5
    for rows, off, pitch, apart in ((63, 0, width, 0), (64, 0, width, 0), (330, 3, width + 6, 0), (330, 1, width, 1)):
        g = gen(rows * 1000003 + width)
        like = lambda kind, o, fill: torch.full((rows * pitch + 16,), fill, device="cuda", dtype=kind)[o:].as_strided(
            (rows, width), (pitch, 1))
        x, y = like(x_type, off, 9.0), like(y_type, off + apart, 9.0)
        x.copy_(normal(g, rows, width) + 2.0)
        x[5, width // 2] = float("nan")
        w, b = 1 + 0.3 * normal(g, width), 0.2 * normal(g, width)
        mean, rstd = torch.full((2, rows), float("nan"), device="cuda").unbind()
        ress.layer_norm(x, w, b, y, eps=eps, mean=mean, rstd=rstd)
        keep = [i for i in range(rows) if i != 5]
        x64, w64, b64 = x.double(), w.double(), b.double()
        h, m64, r64, y64 = norm64(x64, w64, b64, eps)
        within(y[keep], y64[keep], (rounded(y64, y_type) + norm_bound(x64, h, w64, b64, r64))[keep], "y")
        assert bool(y[5].isnan().all())
        y[5] = 0.0
        beside = torch.ones(rows, pitch, device="cuda", dtype=torch.bool)
        beside[:, :width] = False
        assert bool((y.as_strided((rows, pitch), (pitch, 1))[:-1][beside[:-1]] == 9.0).all())

        x[5] = 1.0 + x[4]  # the gradient, of finite rows
        ress.layer_norm(x, w, b, y, eps=eps, mean=mean, rstd=rstd)
        x64, dy, dres, dx = x.double(), like(y_type, off, 9.0), like(x_type, off, 9.0), like(x_type, off + apart, 9.0)
        dy.copy_(0.3 * normal(g, rows, width))
        dres.copy_(normal(g, rows, width))
        m, r = mean.double()[:, None], rstd.double()[:, None]
        h, gr = (x64 - m) * r, dy.double() * w64
        ag, agh = gr.mean(-1, keepdim=True), (gr * h).mean(-1, keepdim=True)
        core = r * (gr - ag - h * agh)
        err = r * (E * (gr.abs().mean(-1, keepdim=True) + h.abs() * (gr * h).abs().mean(-1, keepdim=True))
                   + 8 * U32 * (gr.abs() + ag.abs() + (h * agh).abs()))
        ws = torch.empty(ress.layer_norm_workspace_bytes(rows, width), dtype=torch.uint8, device="cuda")
        dw, db = torch.full((2, width), float("nan"), device="cuda").unbind()
        ress.layer_norm_bwd(dy, x, w, mean, rstd, dx, dweight=dw, dbias=db, dres=dres, ws=ws)
        want = core + dres.double()
        within(dx, want, rounded(want, x_type) + err + U32 * dres.double().abs(), "dx")
        assert bool((dx.as_strided((rows, pitch), (pitch, 1))[:-1][beside[:-1]] == 9.0).all())
        depth = (rows + 128 + 64) * U32
        within(dw, (dy.double() * h).sum(0), depth * (dy.double() * h).abs().sum(0) + 1e-30, "dweight")
        within(db, dy.double().sum(0), depth * dy.double().abs().sum(0) + 1e-30, "dbias")


def test_layer_norm_extreme_rows(ress):
    """Constant rows, a row of zeros, offsets a thousand times the spread, rows with inf and NaN: the
    last only concern themselves."""
    g = gen(3)
    x = normal(g, 64, 1024)
    x[3] = 5.0
    x[4] = 0.0
    x[5] = 1000.0 + x[5]
    x[6, 77] = float("inf")
    x[7, 1] = float("nan")
    x[8] *= 1e-18
    x[9] *= 1e18
    y, mean, rstd = torch.empty_like(x), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    ress.layer_norm(x, None, None, y, mean=mean, rstd=rstd)
    keep = [i for i in range(64) if i not in (6, 7)]
    h, _, r64, want = norm64(x.double(), 1.0, 0.0, 1e-5)
    one = torch.ones((), dtype=torch.float64, device="cuda")
    within(y[keep], want[keep], (norm_bound(x.double(), h, one, 0 * one, r64) + rounded(want, F32))[keep])
    assert bool(y[[6, 7]].isnan().all()) and bool((y[[3, 4]] == 0).all())
    dy = normal(g, 64, 1024)
    dx, dx2 = torch.empty_like(x), torch.empty_like(x)
    ress.layer_norm_bwd(dy, x, None, mean, rstd, dx)
    ress.layer_norm_bwd(dy[:6], x[:6], None, mean[:6], rstd[:6], dx2[:6])
    assert torch.equal(dx[:6], dx2[:6]) and bool(dx[keep].isfinite().all()) and bool(dx[[6, 7]].isnan().any(1).all())


def test_layer_norm_no_rows(ress):
    x = torch.empty(0, 96, device="cuda")
    ress.layer_norm(x, None, None, x.clone())
    ws = torch.empty(ress.layer_norm_workspace_bytes(0, 96), dtype=torch.uint8, device="cuda")
    dw, db = torch.full((2, 96), float("nan"), device="cuda").unbind()
    e = torch.empty(0, device="cuda")
    ress.layer_norm_bwd(x, x, None, e, e, x.clone(), dweight=dw, dbias=db, ws=ws)
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_layer_norm_offsets_past_32_bits(ress):
    """Rows whose elements lie more than 2^32 bytes, and 2^31 elements, apart."""
    width, pitch, rows = 64, 1 << 26, 40  # 2.7e9 elements of 2 bytes
    base = torch.zeros((rows - 1) * pitch + width, device="cuda", dtype=BF16)
    x = base.as_strided((rows, width), (pitch, 1))
    g = gen(2)
    x.copy_(normal(g, rows, width))
    y = torch.empty(rows, width, device="cuda", dtype=BF16)
    ress.layer_norm(x, None, None, y)
    want = norm64(x.double(), 1.0, 0.0, 1e-5)[3]
    within(y, want, rounded(want, BF16) + 4 * E * (1 + want.abs()))
    ress.layer_norm(x, None, None, x)
    assert torch.equal(x, y)


def test_layer_norm_gradient_by_differences(ress):
    """The directional derivative of sum(dy y) in float32, by central differences in float64 of the
    formula: truncation and the gradient's own rounding."""
    g = gen(21)
    rows, width = 50, 200
    x, w, b, dy = normal(g, rows, width), normal(g, width), normal(g, width), normal(g, rows, width)
    mean, rstd = torch.empty(2, rows, device="cuda").unbind()
    ress.layer_norm(x, w, b, torch.empty_like(x), mean=mean, rstd=rstd)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    ws = torch.empty(ress.layer_norm_workspace_bytes(rows, width), dtype=torch.uint8, device="cuda")
    ress.layer_norm_bwd(dy, x, w, mean, rstd, dx, dweight=dw, dbias=db, ws=ws)
    vx, vw, vb = normal(g, rows, width).double(), normal(g, width).double(), normal(g, width).double()
    loss = lambda s: (norm64(x.double() + s * vx, w.double() + s * vw, b.double() + s * vb, 1e-5)[3] * dy.double()).sum()
    numeric = (loss(1e-5) - loss(-1e-5)) / 2e-5
    terms = torch.cat([(dx.double() * vx).flatten(), dw.double() * vw, db.double() * vb])
    # truncation: h^2 times a third derivative of the size of the terms; rounding of the terms
    assert abs(float(terms.sum() - numeric)) <= (1e-8 + 2 * E) * float(terms.abs().sum())


# ---- rotary positions ------------------------------------------------------------------------
def pairs(axes, layout):
    """(axis, first channel, second channel) of each pair."""
    out, start, total = [], 0, sum(axes)
    for t, a in enumerate(axes):
        for i in range(a // 2):
            p = start // 2 + i
            out.append((t,) + {"sections": (start + i, start + a // 2 + i), "halves": (p, total // 2 + p),
                               "interleaved": (2 * p, 2 * p + 1)}[layout])
        start += a
    return out


def rotate64(x, pos, axes, layout, base, sign=1.0, freq=None):
    """x [tokens, heads, channels] in float64 and the sum of the magnitudes that make each channel."""
    y, mag = x.clone(), x.abs().clone()
    k = 0
    counts = [0] * len(axes)
    for t, lo, hi in pairs(axes, layout):
        f = freq[k] if freq is not None else base ** (-2.0 * counts[t] / axes[t])
        counts[t] += 1
        k += 1
        a = pos[:, t].double() * f
        c, s = a.cos()[:, None], sign * a.sin()[:, None]
        y[..., lo] = x[..., lo] * c - x[..., hi] * s
        y[..., hi] = x[..., hi] * c + x[..., lo] * s
        mag[..., lo] = mag[..., hi] = x[..., lo].abs() + x[..., hi].abs()
    return y, mag


# an angle is off by at most pi 2^-25 (rounding to float) and cos and sin by 2 units of 2^-24; the
# products and their sum add two roundings
TURN = 2.0 ** -22

PLANS = [
    (64, (32, 32), "sections"), (64, (16, 24, 24), "halves"), (64, (16, 16), "interleaved"),
    (64, (10, 6, 14), "sections"), (64, (32, 32), "interleaved"), (64, (64,), "halves"), (64, (2,), "sections"),
    (64, (6, 6, 6, 6), "interleaved"), (64, (12, 12), "halves"), (64, (16, 48), "sections"),
    (32, (16, 16), "sections"), (32, (8, 12, 12), "halves"), (80, (32, 32), "sections"), (80, (40, 40), "sections"),
    (128, (32, 48, 48), "halves"), (128, (44, 42, 42), "interleaved"), (128, (128,), "sections"),
    (256, (128, 128), "sections"), (256, (86, 86, 84), "halves"), (6, (2, 2), "sections"), (36, (16, 16), "sections"),
    (2, (2,), "halves"), (160, (64, 32), "halves"),
]


@pytest.mark.parametrize("hd,axes,layout", PLANS)
@pytest.mark.parametrize("kind", [BF16, F16, F32])
def test_rope_and_gradient(ress, hd, axes, layout, kind):
    plan = ress.rope_plan(axes, head_dim=hd, base=50.0, layout=layout)
    eps = 1e-5
    for tokens, hq, hk in ((1, 1, 1), (1, 16, 4), (333, 5, 2), (70, 33, 0), (1100, 4, 4)):
        for norms in ((False, False), (True, True), (True, False)):
            g = gen(tokens * 31 + hq + hd)
            pos = torch.randint(-50, 150, (tokens, len(axes)), generator=g, device="cuda", dtype=torch.int32)
            q = (1.5 * normal(g, tokens, hq, hd) + 0.4 * normal(g, hd)).to(kind)
            k = (normal(g, tokens, hk, hd) + 0.4 * normal(g, hd)).to(kind)
            par = {n: (1 + 0.3 * normal(g, hd), 0.2 * normal(g, hd)) for n in "qk"}
            norm = {n: par[n] if norms[i] else None for i, n in enumerate("qk")}
            out = {n: torch.full_like(x, float("nan")) for n, x in (("q", q), ("k", k))}
            kk = dict(k=k, k_out=out["k"], k_norm=norm["k"]) if hk else {}
            ress.rope(plan, pos, q, out["q"], q_norm=norm["q"], eps=eps, **kk)
            dy = {"q": (0.2 * normal(g, tokens, hq, hd)).to(kind), "k": (0.2 * normal(g, tokens, hk, hd)).to(kind)}
            dx = {n: torch.full_like(dy[n], float("nan")) for n in "qk"}
            grads = {n: torch.full((2, hd), float("nan"), device="cuda").unbind() if norm[n] else None for n in "qk"}
            ws = torch.empty(ress.rope_workspace_bytes(plan, tokens, hq, hk), dtype=torch.uint8, device="cuda")
            kk = dict(dk_out=dy["k"], dk=dx["k"], k_norm=norm["k"], k_norm_grads=grads["k"]) if hk else {}
            if hk and norm["k"]:
                kk["k"] = k
            ress.rope_bwd(plan, pos, dy["q"], dx["q"], q=q if norm["q"] else None, q_norm=norm["q"],
                          q_norm_grads=grads["q"], eps=eps, ws=ws, **kk)
            for n, x in (("q", q), ("k", k)):
                if x.shape[1] == 0:
                    continue
                x64 = x.double()
                if norm[n]:
                    w, b = (p.double() for p in par[n])
                    h, _, rstd, u = norm64(x64, w, b, eps)
                    spread = norm_bound(x64, h, w, b, rstd)
                else:
                    u, spread = x64, torch.zeros_like(x64)
                want, mag = rotate64(u, pos, axes, layout, 50.0)
                err = TURN * mag + rotate_bound(spread, axes, layout)
                within(out[n], want, rounded(want, kind) + err, n)
                # gradients
                d, mag = rotate64(dy[n].double(), pos, axes, layout, 50.0, sign=-1.0)
                derr = TURN * mag
                if norm[n]:
                    gr = d * w
                    ag, agh = gr.mean(-1, keepdim=True), (gr * h).mean(-1, keepdim=True)
                    hw = norm_bound(x64, h, torch.ones_like(w), torch.zeros_like(b), rstd)  # error of h
                    ge = derr * w.abs() + 2 * U32 * gr.abs()
                    big = lambda v: v.mean(-1, keepdim=True)
                    e = rstd * (ge + big(ge) + E * big(gr.abs()) + h.abs() * (big(ge * h.abs() + gr.abs() * hw)
                                + E * big((gr * h).abs())) + hw * agh.abs() + 8 * U32 * (gr.abs() + ag.abs() + (h * agh).abs()))
                    core = rstd * (gr - ag - h * agh)
                    # rstd's own relative error
                    e = e + core.abs() * (E + 4 * U32 + (E * x64.abs().mean(-1, keepdim=True) * rstd).square())
                    within(dx[n], core, rounded(core, kind) + e, "d" + n)
                    depth = (tokens * x.shape[1] / 16 + 256) * U32
                    flat = lambda v: v.flatten(0, 1)
                    within(grads[n][0], flat(d * h).sum(0), flat(depth * (d * h).abs() + derr * h.abs() + d.abs() * hw).sum(0)
                           + 1e-30, "dweight")
                    within(grads[n][1], flat(d).sum(0), flat(depth * d.abs() + derr).sum(0) + 1e-30, "dbias")
                else:
                    within(dx[n], d, rounded(d, kind) + derr, "d" + n)


@pytest.mark.parametrize("hd,axes,layout", [
    (128, (32,), "halves"), (128, (16, 8, 8), "sections"), (80, (8, 12, 12), "interleaved"), (80, (16, 16), "halves"),
    (64, (16, 16), "sections"), (64, (64,), "sections"), (32, (8, 8), "interleaved"), (32, (32,), "halves"),
    (96, (96,), "halves"), (24, (8, 8), "sections")])
@pytest.mark.parametrize("kind", [BF16, F32])
def test_rope_with_few_heads(ress, hd, axes, layout, kind):
    """Heads that leave room for several tokens in a row of a warp, beside heads that do not; gradients
    against those of 16 copies of each head, which fill their rows."""
    plan = ress.rope_plan(axes, head_dim=hd, base=50.0, layout=layout)
    for tokens, hq, hk in ((1, 1, 1), (2, 2, 1), (203, 16, 1), (90, 1, 3), (57, 3, 2), (1500, 4, 1)):
        g = gen(tokens + hd)
        pos = torch.randint(-50, 150, (tokens, len(axes)), generator=g, device="cuda", dtype=torch.int32)
        x = {"q": normal(g, tokens, hq, hd).to(kind), "k": normal(g, tokens, hk, hd).to(kind)}
        dy = {n: (0.2 * normal(g, *t.shape)).to(kind) for n, t in x.items()}
        w, b = 1 + 0.3 * normal(g, hd), 0.2 * normal(g, hd)
        for norm in (None, (w, b)):
            out, dx = ({n: torch.full_like(t, float("nan")) for n, t in x.items()} for _ in range(2))
            grads = torch.full((4, hd), float("nan"), device="cuda")
            ws = torch.empty(ress.rope_workspace_bytes(plan, tokens, hq, hk), dtype=torch.uint8, device="cuda")
            ress.rope(plan, pos, x["q"], out["q"], x["k"], out["k"], q_norm=norm, k_norm=norm)
            kw = {}
            if norm:
                kw = dict(q=x["q"], k=x["k"], q_norm=norm, k_norm=norm, q_norm_grads=(grads[0], grads[1]),
                          k_norm_grads=(grads[2], grads[3]), ws=ws)
            ress.rope_bwd(plan, pos, dy["q"], dx["q"], dy["k"], dx["k"], **kw)
            for i, n in enumerate("qk"):
                u, mag = x[n].double(), 0
                if norm:
                    h, _, rstd, u = norm64(x[n].double(), w.double(), b.double(), 1e-5)
                    spread = norm_bound(x[n].double(), h, w.double(), b.double(), rstd)
                else:
                    spread = torch.zeros_like(u)
                want, mag = rotate64(u, pos, axes, layout, 50.0)
                within(out[n], want, rounded(want, kind) + TURN * mag + rotate_bound(spread, axes, layout), n)
                d, mag = rotate64(dy[n].double(), pos, axes, layout, 50.0, sign=-1.0)
                if not norm:
                    within(dx[n], d, rounded(d, kind) + TURN * mag, "d" + n)
                    continue
                # 16 heads fill their rows: each head beside 15 copies of itself, token by token
                wide, dwide = (t.repeat_interleave(16, 1).contiguous() for t in (x[n], dy[n]))
                dwide_x = torch.empty_like(wide)
                ress.rope_bwd(plan, pos, dwide, dwide_x, q=wide, q_norm=norm)
                ref = dwide_x.view(tokens, -1, 16, hd)[:, :, 0].double()
                # the two may add a row's channels in another order
                size = dx[n].double().abs().mean(-1, keepdim=True) + ref.abs()
                within(dx[n], ref, 2 * rounded(ref, kind) + 8 * E * (size + rstd * (d * w.double()).abs()), "d" + n)
                hw = norm_bound(x[n].double(), h, torch.ones_like(w.double()), torch.zeros_like(b.double()), rstd)
                depth = (tokens * x[n].shape[1] / 16 + 256) * U32
                flat = lambda v: v.flatten(0, 1).sum(0)
                within(grads[2 * i], flat(d * h), flat(depth * (d * h).abs() + TURN * mag * h.abs() + d.abs() * hw) + 1e-30, "dw")
                within(grads[2 * i + 1], flat(d), flat(depth * d.abs() + TURN * mag) + 1e-30, "db")


def rotate_bound(e, axes, layout):
    """Errors of the channels after a rotation of channels with errors e."""
    out = e.clone()
    for _, lo, hi in pairs(axes, layout):
        out[..., lo] = out[..., hi] = e[..., lo] + e[..., hi]
    return out


@pytest.mark.parametrize("kind", [BF16, F32])
@pytest.mark.parametrize("norm", [False, True])
def test_rope_strides_alignment_and_in_place(ress, kind, norm):
    """Heads inside packed rows, heads before tokens, one token for all, odd starts; in place."""
    plan = ress.rope_plan((32, 32))
    g = gen(4)
    tokens, H, hd = 130, 6, 64
    pos = torch.randint(0, 40, (tokens, 2), generator=g, device="cuda", dtype=torch.int32)
    pn = (1 + 0.1 * normal(g, hd), normal(g, hd)) if norm else None
    wide = normal(g, tokens, 20, hd + 5).to(kind)
    flat = normal(g, tokens * H * hd + 9).to(kind)
    cases = {
        "packed": normal(g, tokens, 3 * H, hd).to(kind)[:, H:2 * H],
        "heads first": normal(g, H, tokens, hd).to(kind).transpose(0, 1),
        "padded": wide[:, 2:2 + H, :hd], "odd pitch": wide[:, 1:1 + H, 5:], "one token": wide[3:4, :H, :hd].expand(tokens, H, hd),
        "one head": wide[:, 2:3, :hd].expand(tokens, H, hd), "odd start": flat[3:3 + tokens * H * hd].view(tokens, H, hd),
    }
    for name, x in cases.items():
        want = torch.empty(tokens, H, hd, device="cuda", dtype=kind)
        ress.rope(plan, pos, x.contiguous(), want, q_norm=pn)
        out = torch.empty_like(want)
        ress.rope(plan, pos, x, out, q_norm=pn)
        assert torch.equal(out, want), name
        dwant, dx = torch.empty_like(want), torch.empty_like(want)
        kw = dict(q=x, q_norm=pn) if norm else {}
        ress.rope_bwd(plan, pos, x.contiguous(), dwant, **({**kw, "q": x.contiguous()} if norm else {}))
        ress.rope_bwd(plan, pos, x, dx, **kw)
        assert torch.equal(dx, dwant), name
        if "one" in name:
            continue
        ress.rope(plan, pos, x, x, q_norm=pn)
        assert torch.equal(x, want), name
    # what lies between the heads of an output stays
    out = torch.full((tokens, 20, hd + 5), 7.0, device="cuda", dtype=kind)
    x = normal(g, tokens, H, hd).to(kind)
    ress.rope(plan, pos, x, out[:, 2:2 + H, 3:3 + hd], q_norm=pn)
    out[:, 2:2 + H, 3:3 + hd] = 7.0
    assert bool((out == 7.0).all())


def test_rope_is_exact_at_any_position(ress):
    """Positions up to the ends of int32: angles from the frequencies as fractions of a turn."""
    freq = [1.0, 0.7, 0.01, 3.1e-5]
    plan = ress.rope_plan((4, 4), head_dim=8, layout="interleaved", freq=freq)
    at = [0, 1, -1, 12345678, -(2 ** 31), 2 ** 31 - 1, 99999999, -77777777]
    pos = torch.tensor([[p, -p if p > -2 ** 31 else p] for p in at], device="cuda", dtype=torch.int32)
    x = torch.zeros(len(at), 1, 8, device="cuda")
    x[..., 0::2] = 1.0
    y = torch.empty_like(x)
    ress.rope(plan, pos, x, y)
    two_pi = Fraction("6.28318530717958647692528676655900576839433879875021")
    for i, p in enumerate(pos.cpu().tolist()):
        for k, f in enumerate(freq):
            turns = Fraction(p[k // 2]) * Fraction(f) / two_pi
            a = 2 * math.pi * float(turns - round(turns))
            # the frequency in turns has 53 bits, of which a position loses as many as it has
            tol = TURN + 2 * math.pi * abs(p[k // 2]) * f / (2 * math.pi) * 2.0 ** -52
            assert abs(float(y[i, 0, 2 * k]) - math.cos(a)) <= tol and abs(float(y[i, 0, 2 * k + 1]) - math.sin(a)) <= tol


def test_rope_leaves_other_channels_and_heads_alone(ress):
    """Infinities and NaN reach their own pair (without a norm) or head (with one); channels without a
    pair keep their bits."""
    plan = ress.rope_plan((16, 16))
    g = gen(8)
    x = normal(g, 40, 3, 64)
    x[5, 1, 3], x[6, 2, 50], x[7, 0, 40] = float("inf"), float("inf"), float("nan")
    pos = torch.randint(0, 40, (40, 2), generator=g, device="cuda", dtype=torch.int32)
    y = torch.empty_like(x)
    ress.rope(plan, pos, x, y)
    assert torch.equal(y[..., 32:].view(torch.int32), x[..., 32:].view(torch.int32))
    bad = ~y.isfinite()
    assert bool(bad[5, 1, [3, 11]].all()) and int(bad.sum()) == 4
    ress.rope(plan, pos, x, y, q_norm=(None, None))
    bad = ~y.isfinite()
    assert {tuple(v) for v in bad.any(2).nonzero().tolist()} == {(5, 1), (6, 2), (7, 0)}


def test_rope_no_tokens(ress):
    plan = ress.rope_plan((32, 32))
    pos = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    x = torch.empty(0, 4, 64, device="cuda")
    ress.rope(plan, pos, x, x.clone())
    ws = torch.empty(ress.rope_workspace_bytes(plan, 0, 4), dtype=torch.uint8, device="cuda")
    dw, db = torch.full((2, 64), float("nan"), device="cuda").unbind()
    ress.rope_bwd(plan, pos, x, x.clone(), q=x, q_norm=(None, None), q_norm_grads=(dw, db), ws=ws)
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_rope_gradient_by_differences(ress):
    g = gen(33)
    tokens, H, hd, axes = 30, 3, 64, (16, 24, 24)
    plan = ress.rope_plan(axes, layout="halves", base=50.0)
    pos = torch.randint(0, 60, (tokens, 3), generator=g, device="cuda", dtype=torch.int32)
    x, w, b, dy = normal(g, tokens, H, hd), normal(g, hd), normal(g, hd), normal(g, tokens, H, hd)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    ws = torch.empty(ress.rope_workspace_bytes(plan, tokens, H), dtype=torch.uint8, device="cuda")
    ress.rope_bwd(plan, pos, dy, dx, q=x, q_norm=(w, b), q_norm_grads=(dw, db), ws=ws)
    vx, vw, vb = normal(g, tokens, H, hd).double(), normal(g, hd).double(), normal(g, hd).double()

    def loss(s):
        u = norm64(x.double() + s * vx, w.double() + s * vw, b.double() + s * vb, 1e-5)[3]
        return (rotate64(u, pos, axes, "halves", 50.0)[0] * dy.double()).sum()

    numeric = (loss(1e-5) - loss(-1e-5)) / 2e-5
    terms = torch.cat([(dx.double() * vx).flatten(), dw.double() * vw, db.double() * vb])
    assert abs(float(terms.sum() - numeric)) <= (1e-8 + 4 * E) * float(terms.abs().sum())


# ---- projection to Q, K, V -------------------------------------------------------------------
def qkv_case(ress, N, H, dm, plan_of=None, norms=(True, True), bias=True, seed=0, scale=1.0):
    g = gen(seed * 7919 + N + 13 * H)
    x = (scale * normal(g, N, dm)).to(BF16)
    W = {n: (normal(g, H * 64, dm) / math.sqrt(dm)).to(BF16) for n in "qkv"}
    b = {n: (0.2 * normal(g, H * 64)).to(BF16) if bias else None for n in "qkv"}
    par = {n: (1 + 0.3 * normal(g, 64), 0.2 * normal(g, 64)) for n in "qk"}
    norm = {n: par[n] if norms[i] else None for i, n in enumerate("qk")}
    d = ress.dims(N, H, 0, dm)
    ws = torch.zeros(ress.workspace_bytes(d), dtype=torch.uint8, device="cuda")
    out = {n: torch.full((N, H, 64), float("nan"), device="cuda").to(BF16) for n in "qkv"}
    plan = pos = None
    if plan_of:
        axes, layout = plan_of
        plan = ress.rope_plan(axes, base=50.0, layout=layout)
        pos = torch.randint(0, 100, (N, len(axes)), generator=g, device="cuda", dtype=torch.int32)
    ress.qkv_proj(d, x, W["q"], W["k"], W["v"], out["q"], out["k"], out["v"], ws, b_q=b["q"], b_k=b["k"], b_v=b["v"],
                  plan=plan, pos=pos, q_norm=norm["q"], k_norm=norm["k"])
    ress.status(ws)
    for n in "qkv":
        y = x.double() @ W[n].double().T
        # a float32 sum of dm exact products and the bias
        err = (dm + 2) * U32 * (x.double().abs() @ W[n].double().abs().T)
        if bias:
            y = y + b[n].double()
            err = err + U32 * b[n].double().abs()
        y, err = y.view(N, H, 64), err.view(N, H, 64)
        if n != "v" and norm[n]:
            w, s = (p.double() for p in norm[n])
            h, _, rstd, u = norm64(y, w, s, 1e-5)
            # the product's error through the norm: through the channel itself, the mean and the spread
            through = rstd * (err + err.mean(-1, keepdim=True)) + h.abs() * rstd * (err * h.abs()).mean(-1, keepdim=True)
            err = w.abs() * through * 1.01 + norm_bound(y, h, w, s, rstd)
            y = u
        if n != "v" and plan_of:
            y, mag = rotate64(y, pos, axes, layout, 50.0)
            err = TURN * mag + rotate_bound(err, axes, layout)
        within(out[n], y, rounded(y, BF16) + err, n)


@pytest.mark.parametrize("N,H,dm", [
    (1, 1, 64), (8, 16, 1024), (127, 2, 128), (129, 3, 192), (257, 4, 320), (300, 5, 64), (1000, 7, 512),
    (2748, 4, 256), (5003, 3, 192), (700, 16, 1024), (20000, 4, 256), (130, 32, 128)])
def test_qkv_projection_sizes(ress, N, H, dm):
    qkv_case(ress, N, H, dm, ((32, 32), "sections"))


@pytest.mark.parametrize("axes,layout", [
    ((32, 32), "sections"), ((16, 24, 24), "halves"), ((16, 16), "interleaved"), ((10, 6, 14), "sections"),
    ((64,), "halves"), ((6, 6, 6, 6), "interleaved"), ((2,), "sections"), ((16, 48), "sections"), ((14,), "interleaved"),
    ((12, 12), "halves"), ((16,), "halves")])
@pytest.mark.parametrize("norms,bias", [((True, True), True), ((False, True), False), ((False, False), True)])
def test_qkv_projection_plans(ress, axes, layout, norms, bias):
    qkv_case(ress, 391, 5, 128, (axes, layout), norms, bias, seed=1)


def test_qkv_projection_alone(ress):
    qkv_case(ress, 391, 6, 192, None, (False, False), False, seed=2)
    qkv_case(ress, 391, 6, 192, None, (True, False), True, seed=3, scale=30.0)


def test_qkv_projection_rows_keep_to_themselves(ress):
    """A token with inf and NaN spoils its own rows and no others."""
    g = gen(1)
    N, H, dm = 300, 2, 128
    d = ress.dims(N, H, 0, dm)
    ws = torch.zeros(ress.workspace_bytes(d), dtype=torch.uint8, device="cuda")
    x, W = normal(g, N, dm).to(BF16), [(0.1 * normal(g, H * 64, dm)).to(BF16) for _ in range(3)]
    plan = ress.rope_plan((32, 32))
    pos = torch.randint(0, 30, (N, 2), generator=g, device="cuda", dtype=torch.int32)
    good, bad = ([torch.empty(N, H, 64, device="cuda", dtype=BF16) for _ in range(3)] for _ in range(2))
    kw = dict(plan=plan, pos=pos, q_norm=(None, None))
    ress.qkv_proj(d, x, *W, *good, ws, **kw)
    x2 = x.clone()
    x2[17, 3], x2[200, 5] = float("inf"), float("nan")
    ress.qkv_proj(d, x2, *W, *bad, ws, **kw)
    ress.status(ws)
    keep = [i for i in range(N) if i not in (17, 200)]
    for a, b in zip(good, bad):
        assert torch.equal(a[keep], b[keep]) and not bool(b[[17, 200]].isfinite().all(2).any())


# ---- all of them -------------------------------------------------------------------------------
def test_results_do_not_depend_on_the_run(ress):
    """The same bits each time, on another stream, and in a captured graph replayed on new inputs."""
    g = gen(12)
    N, H, dm = 1374, 4, 256
    d, plan = ress.dims(N, H, 0, dm), ress.rope_plan((32, 32))
    x, dres = normal(g, N, dm).to(BF16), normal(g, N, dm).to(BF16)
    w, b, hw, hb = 1 + 0.1 * normal(g, dm), normal(g, dm), 1 + 0.1 * normal(g, 64), normal(g, 64)
    W = [(normal(g, H * 64, dm) / 16).to(BF16) for _ in range(3)]
    pos = torch.randint(0, 38, (N, 2), generator=g, device="cuda", dtype=torch.int32)
    o = {n: torch.empty(N, dm, device="cuda", dtype=BF16) for n in ("y", "dx")}
    o.update({n: torch.empty(N, H, 64, device="cuda", dtype=BF16) for n in ("Q", "K", "V", "q", "dq")})
    o.update({n: torch.empty(N, device="cuda") for n in ("mean", "rstd")})
    o.update({n: torch.empty(dm, device="cuda") for n in ("dw", "db")})
    o.update({n: torch.empty(64, device="cuda") for n in ("hdw", "hdb")})
    need = max(ress.workspace_bytes(d), ress.layer_norm_workspace_bytes(N, dm), ress.rope_workspace_bytes(plan, N, H))
    ws = torch.zeros(ress.workspace_bytes(d), dtype=torch.uint8, device="cuda")
    ws2, ws3 = (torch.zeros(need, dtype=torch.uint8, device="cuda") for _ in range(2))

    def go():
        ress.layer_norm(x, w, b, o["y"], mean=o["mean"], rstd=o["rstd"])
        ress.qkv_proj(d, o["y"], *W, o["Q"], o["K"], o["V"], ws, plan=plan, pos=pos, q_norm=(hw, hb))
        ress.rope(plan, pos, o["V"], o["q"], q_norm=(hw, hb))
        ress.rope_bwd(plan, pos, o["q"], o["dq"], q=o["V"], q_norm=(hw, hb), q_norm_grads=(o["hdw"], o["hdb"]), ws=ws2)
        ress.layer_norm_bwd(o["dq"].view(N, dm), x, w, o["mean"], o["rstd"], o["dx"], dweight=o["dw"], dbias=o["db"],
                            dres=dres, ws=ws3)

    def bits():
        torch.cuda.synchronize()
        return {n: t.clone() for n, t in o.items()}

    go()
    first = bits()
    for t in o.values():
        t.fill_(float("nan"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    again = bits()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for t in o.values():
        t.fill_(float("nan"))
    graph.replay()
    replayed = bits()
    x.copy_(normal(g, N, dm))
    graph.replay()
    fresh = bits()
    go()
    direct = bits()
    ress.status(ws)
    for n in o:
        assert torch.equal(first[n], again[n]) and torch.equal(first[n], replayed[n]) and torch.equal(fresh[n], direct[n]), n
        assert not torch.equal(first[n], fresh[n]) and bool(first[n].isfinite().all()), n


def test_binding_refuses_tensors(ress):
    """What the binding finds wrong with tensors on the device, and that it says what."""
    z = lambda *shape, dtype=F32: torch.zeros(*shape, device="cuda", dtype=dtype)
    x, w, row = z(4, 64), z(64), z(4)
    ws = torch.empty(ress.layer_norm_workspace_bytes(4, 64), dtype=torch.uint8, device="cuda")
    ln, lb = ress.layer_norm, ress.layer_norm_bwd
    for error, text, call in (
            (TypeError, "x has dtype", lambda: ln(x.double(), None, None, x)),
            (ValueError, "y must live", lambda: ln(x, None, None, x.cpu())),
            (ValueError, "y has shape", lambda: ln(x, None, None, z(4, 63))),
            (ValueError, "y must be contiguous", lambda: ln(x, None, None, z(64, 4).t())),
            (ValueError, "x has shape", lambda: ln(z(4, 0), None, None, z(4, 0))),
            (ValueError, "x has shape", lambda: ln(z(1)[0], None, None, x)),
            (TypeError, "y must be a torch.Tensor", lambda: ln(x, None, None, None)),
            (TypeError, "weight or bias has dtype", lambda: ln(x, w.double(), None, z(4, 64))),
            (ValueError, "weight has 63", lambda: ln(x, z(63), None, z(4, 64))),
            (ValueError, "bias must be contiguous", lambda: ln(x, w, z(128)[::2], z(4, 64))),
            (TypeError, "different dtypes", lambda: ln(x, w, w.half(), z(4, 64))),
            (TypeError, "mean has dtype", lambda: ln(x, w, w, z(4, 64), mean=row.half())),
            (ValueError, "rstd has 3", lambda: ln(x, w, w, z(4, 64), rstd=z(3))),
            (TypeError, "dx and dres", lambda: lb(x, x, w, row, row, x.half())),
            (TypeError, "dx and dres", lambda: lb(x, x, w, row, row, z(4, 64), dres=x.half())),
            (ValueError, "dres has shape", lambda: lb(x, x, w, row, row, z(4, 64), dres=z(3, 64))),
            (ValueError, "mean and rstd", lambda: lb(x, x, w, None, row, z(4, 64))),
            (ValueError, "ws must be contiguous", lambda: lb(x, x, w, row, row, z(4, 64), dweight=z(64), ws=ws[::2])),
            (ress.RessError, "EWORKSPACE", lambda: lb(x, x, w, row, row, z(4, 64), dweight=z(64), ws=ws[:256]))):
        with pytest.raises(error, match=text):
            call()

    plan, pos, q, p = ress.rope_plan((32, 32)), z(4, 2, dtype=torch.int32), z(4, 2, 64), z(64)
    rope, rb = ress.rope, ress.rope_bwd
    for error, text, call in (
            (TypeError, "q has dtype", lambda: rope(plan, pos, q.double(), q.double())),
            (TypeError, "has dtype", lambda: rope(plan, pos, q, q.half())),
            (ValueError, "shape", lambda: rope(plan, pos, z(5, 2, 64), z(5, 2, 64))),
            (ValueError, "shape", lambda: rope(plan, pos, z(4, 2, 32), z(4, 2, 32))),
            (ValueError, "shape", lambda: rope(plan, pos, q, z(4, 3, 64))),
            (ValueError, "contiguous", lambda: rope(plan, pos, q, z(4, 64, 2).transpose(1, 2))),
            (ValueError, "must live", lambda: rope(plan, pos, q, q.cpu())),
            (TypeError, "torch.Tensor", lambda: rope(plan, pos, q, [0.0])),
            (TypeError, "pos has dtype", lambda: rope(plan, pos.long(), q, z(4, 2, 64))),
            (ValueError, "pos has shape", lambda: rope(plan, z(4, 3, dtype=torch.int32), q, z(4, 2, 64))),
            (ValueError, "pos must be contiguous", lambda: rope(plan, z(2, 4, dtype=torch.int32).t(), q, z(4, 2, 64))),
            (ValueError, "has 63", lambda: rope(plan, pos, q, z(4, 2, 64), q_norm=(z(63), None))),
            (TypeError, "has dtype", lambda: rope(plan, pos, q, z(4, 2, 64), q_norm=(p, p.double()))),
            (TypeError, "different dtypes", lambda: rope(plan, pos, q, z(4, 2, 64), q_norm=(p, p.half()))),
            (ValueError, "too many values", lambda: rope(plan, pos, q, z(4, 2, 64), q_norm=(p, p, p))),
            (TypeError, "has dtype", lambda: rb(plan, pos, q, z(4, 2, 64), q=q, q_norm=(p, p), q_norm_grads=(p.half(), None))),
            (ValueError, "has 65", lambda: rb(plan, pos, q, z(4, 2, 64), q=q, q_norm=(p, p), q_norm_grads=(None, z(65)))),
            (ress.RessError, "ws is NULL", lambda: rb(plan, pos, q, z(4, 2, 64), q=q, q_norm=(p, p), q_norm_grads=(z(64), z(64))))):
        with pytest.raises(error, match=text):
            call()

    d = ress.dims(100, 2, 0, 128)
    t = z(100, 128, dtype=BF16)
    wt, o, space = z(128, 128, dtype=BF16), z(100, 2, 64, dtype=BF16), torch.empty(ress.workspace_bytes(d), dtype=torch.uint8, device="cuda")
    for error, text, call in (
            (TypeError, "x has dtype", lambda: ress.qkv_proj(d, t.half(), wt, wt, wt, o, o.clone(), o.clone(), space)),
            (ValueError, "W_v has", lambda: ress.qkv_proj(d, t, wt, wt, wt[:64], o, o.clone(), o.clone(), space)),
            (ValueError, "K must be contiguous",
             lambda: ress.qkv_proj(d, t, wt, wt, wt, o, z(2, 100, 64, dtype=BF16).transpose(0, 1), o.clone(), space)),
            (ValueError, "ws must live", lambda: ress.qkv_proj(d, t, wt, wt, wt, o, o.clone(), o.clone(), space.cpu()))):
        with pytest.raises(error, match=text):
            call()
    torch.cuda.synchronize()

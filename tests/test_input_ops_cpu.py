"""The operators that form Q, K and V: what they refuse before any launch, the rotary plan's numbers, and
rules that their sources keep.  No GPU: every call below is refused or only computes on the host."""
import ctypes
import glob
import math
import os
import re
from fractions import Fraction

import pytest

import __graft_entry__

__graft_entry__._build_module().build()
import paper_2609_35593_gb300 as ress  # noqa: E402

OK, EINVAL, EWORKSPACE, EUNSUPPORTED = 0, -1, -2, -3
lib = ress._lib
A = 1 << 40  # never dereferenced
BF16, F16, F32 = 0, 1, 2


def norm(rows=10, width=64, x=BF16, y=BF16, params=F32, eps=1e-5, strides=None):
    s = strides or (width, width, width, width)
    return ress._NORM.pack(rows, width, x, y, params, eps, *s)


def ln(n, x=A, w=A, b=A, y=A, mean=A, rstd=A):
    return lib.ress_layer_norm(n, x, w, b, y, mean, rstd, None)


def ln_bwd(n, dy=A, x=A, w=A, mean=A, rstd=A, dres=A, dx=A, dw=A, db=A, ws=A, size=1 << 30):
    return lib.ress_layer_norm_bwd(n, dy, x, w, mean, rstd, dres, dx, dw, db, ws, size, None)


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), EINVAL), (dict(width=0), EUNSUPPORTED), (dict(width=16385), EUNSUPPORTED), (dict(x=3), EUNSUPPORTED),
    (dict(y=-1), EUNSUPPORTED), (dict(params=7), EUNSUPPORTED), (dict(x=BF16, y=F32), EUNSUPPORTED),
    (dict(x=F16, y=BF16), EUNSUPPORTED), (dict(eps=-1.0), EINVAL), (dict(eps=math.nan), EINVAL),
    (dict(eps=math.inf), EINVAL), (dict(strides=(-1, 64, 64, 64)), EINVAL), (dict(strides=(64, 63, 64, 64)), EINVAL),
    (dict(rows=1 << 50), EINVAL), (dict(rows=1 << 40, strides=(1 << 40, 64, 64, 64)), EINVAL)])
def test_layer_norm_refuses(change, code):
    assert ln(norm(**change)) == code and lib.ress_last_error()
    if change.get("strides") != (64, 63, 64, 64):  # dy is an input: its rows may overlap
        assert ln_bwd(norm(**change)) == code
    if "strides" not in change and change.get("rows", 0) >= 0:
        assert lib.ress_layer_norm_workspace_bytes(norm(**change)) == 0


def test_layer_norm_refuses_pointers():
    n = norm()
    for name in ("x", "y"):
        assert ln(n, **{name: 0}) == EINVAL and ln(n, **{name: A + 1}) == EINVAL
    assert ln(norm(x=F32, y=F32), x=A + 2) == EINVAL
    for name in ("w", "b", "mean", "rstd"):
        assert ln(n, **{name: A + 2}) == EINVAL
    assert lib.ress_layer_norm(None, A, A, A, A, A, A, None) == EINVAL
    for name in ("dy", "x", "mean", "rstd", "dx"):
        assert ln_bwd(n, **{name: 0}) == EINVAL, name
    assert ln_bwd(n, dres=A + 1) == EINVAL and ln_bwd(n, dw=A + 2) == EINVAL
    assert ln_bwd(n, ws=0) == EINVAL and ln_bwd(n, ws=A + 16) == EINVAL
    need = lib.ress_layer_norm_workspace_bytes(n)
    assert need >= 10 * 2 * 64 * 4 and ln_bwd(n, size=need - 1) == EWORKSPACE
    assert ln_bwd(norm(strides=(64, 64, 63, 64))) == EINVAL  # dx is an output
    assert ln_bwd(norm(strides=(64, 64, 64, -64))) == EINVAL
    assert ln(norm(rows=0), x=0, y=0) == OK  # no rows: nothing to read or write


def plan(axes=(32, 32), hd=64, layout="sections", **kw):
    return ress.rope_plan(axes, head_dim=hd, layout=layout, **kw)


def heads(n=4, enabled=0, w=0, b=0, x=(A, 256, 64), y=(A, 256, 64), dx=(A, 256, 64), dw=0, db=0):
    return ress._ROPE_HEADS.pack(n, enabled, w, b, *x, *y, *dx, dw, db)


def rope(q=None, k=None, p=None, tokens=10, pos=A, kind=BF16, params=F32, eps=1e-5):
    return lib.ress_rope(p or plan(), tokens, pos, kind, params, eps, heads() if q is None else q, k, None)


def rope_bwd(q=None, k=None, p=None, tokens=10, pos=A, ws=A, size=1 << 30):
    return lib.ress_rope_bwd(p or plan(), tokens, pos, BF16, F32, 1e-5, heads() if q is None else q, k, ws, size, None)


def test_rope_refuses():
    assert lib.ress_rope(None, 10, A, 0, 2, 0.0, heads(), None, None) == EINVAL
    assert lib.ress_rope(plan(), 10, A, 0, 2, 0.0, None, None, None) == EINVAL
    assert rope(tokens=-1) == EINVAL and rope(tokens=1 << 60) == EINVAL
    assert rope(pos=0) == EINVAL and rope(pos=A + 2) == EINVAL
    assert rope(kind=3) == EUNSUPPORTED and rope(params=-1) == EUNSUPPORTED and rope(eps=-1.0) == EINVAL
    assert rope(heads(n=0)) == EUNSUPPORTED and rope(heads(n=4097)) == EUNSUPPORTED
    assert rope(heads(x=(0, 256, 64))) == EINVAL and rope(heads(x=(A + 1, 256, 64))) == EINVAL
    assert rope(heads(y=(0, 256, 64))) == EINVAL
    assert rope(heads(x=(A, -1, 64))) == EINVAL and rope(heads(x=(A, 256, 1 << 61))) == EINVAL
    assert rope(heads(y=(A, 255, 64))) == EINVAL and rope(heads(y=(A, 256, 63))) == EINVAL  # heads overlap
    assert rope(heads(y=(A, 64, 639))) == EINVAL  # heads first: 10 tokens of 64
    assert rope(heads(enabled=1, w=A + 2)) == EINVAL and rope(heads(enabled=1, b=A + 2)) == EINVAL
    assert rope(heads(), heads(y=(0, 256, 64))) == EINVAL  # k
    assert b"k.y" in lib.ress_last_error()
    assert rope_bwd(heads(dx=(0, 256, 64))) == EINVAL and rope_bwd(heads(dx=(A, 0, 64))) == EINVAL
    assert rope_bwd(heads(dw=A)) == EINVAL  # a gradient of no norm
    assert rope_bwd(heads(enabled=1, x=(0, 256, 64))) == EINVAL
    assert rope_bwd(heads(enabled=1, dw=A), ws=0) == EINVAL
    need = lib.ress_rope_workspace_bytes(plan(), 10, 4, 0)
    assert rope_bwd(heads(enabled=1, db=A), size=need - 1) == EWORKSPACE
    assert lib.ress_rope_workspace_bytes(plan(), -1, 4, 0) == 0


@pytest.mark.parametrize("kw", [
    dict(axes=(32, 34)), dict(axes=(31, 32)), dict(axes=(0, 64)), dict(axes=()), dict(axes=(2,) * 5), dict(hd=65),
    dict(hd=258, axes=(2,)), dict(hd=0, axes=(2,)), dict(base=0.0), dict(base=-2.0), dict(base=math.nan),
    dict(axes=(4,), freq=[1.0, math.inf])])
def test_rope_plan_refuses(kw):
    with pytest.raises(ress.RessError):
        plan(**kw)
    bad = plan()
    bad.n_pairs = 31  # a plan that was not made by ress_rope_plan_init
    assert rope(p=bad) == EINVAL
    bad = plan()
    bad.axis_dims[1] = 200
    assert rope(p=bad) == EINVAL
    with pytest.raises(KeyError):
        plan(layout="spiral")
    with pytest.raises(ValueError):
        plan(axes=(4, 4), freq=[1.0])


def test_rope_plan_frequencies():
    """Turns per position as 64-bit fractions: of base^(-2i / channels), within the 53 bits of the
    frequency; negative ones and ones above a turn wrap around."""
    two_pi = Fraction("6.28318530717958647692528676655900576839433879875021")
    p = plan((16, 48), base=10000.0)
    want = [10000.0 ** (-2.0 * i / a) for a in (16, 48) for i in range(a // 2)]
    assert p.n_pairs == 32
    for k, f in enumerate(want):
        off = Fraction(p.turns[k], 2 ** 64) - Fraction(f) / two_pi
        assert abs(off) <= Fraction(2) ** -53 * 4 * Fraction(f)
    q = plan((6,), freq=[-1.0, 100.0, 0.0])
    for k, f in enumerate((-1.0, 100.0, 0.0)):
        off = (Fraction(q.turns[k], 2 ** 64) - Fraction(f) / two_pi) % 1
        assert min(off, 1 - off) <= Fraction(2) ** -45


def test_qkv_proj_refuses():
    d = ress.dims(100, 4, 0, 256)
    need = ress.workspace_bytes(d)
    norm_off = ress._HEAD_NORM.pack(0, 0, 0)

    def call(x=A, W=(A, A, A), b=(0, 0, 0), p=None, pos=0, qn=norm_off, kn=None, params=F32, eps=1e-5, out=(A, A, A), ws=A,
             size=need, dims=d):
        return lib.ress_qkv_proj(dims, x, *W, *b, p, pos, qn, kn, params, eps, *out, ws, size, None)

    assert call(x=0) == EINVAL and call(x=A + 8) == EINVAL
    for i in range(3):
        for bad in (0, A + 8):
            t = [A, A, A]
            t[i] = bad
            assert call(W=t) == EINVAL and call(out=t) == EINVAL
        t = [0, 0, 0]
        t[i] = A + 2
        assert call(b=t) == EINVAL
    assert call(p=plan()) == EINVAL and call(pos=A) == EINVAL  # a plan and positions belong together
    assert call(p=plan((16, 16), 32), pos=A) == EUNSUPPORTED  # heads of 32
    assert call(qn=ress._HEAD_NORM.pack(1, A + 2, 0)) == EINVAL
    assert call(params=5) == EUNSUPPORTED and call(eps=math.inf) == EINVAL
    assert call(size=need - 1) == EWORKSPACE and call(ws=A + 16) == EINVAL
    assert call(dims=ress.dims(100, 4, 0, 250)) == EUNSUPPORTED  # d_model no multiple of 64
    assert call(dims=ress.dims(0, 4, 0, 256)) == EINVAL


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):  # host tensors
        ress.layer_norm(x, None, None, x)
    with pytest.raises(TypeError):
        ress.layer_norm([1.0], None, None, x)
    with pytest.raises(ValueError):
        ress.layer_norm_bwd(x, x, None, None, None, x)
    pos = torch.zeros(4, 2, dtype=torch.int32)
    h = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):
        ress.rope(plan(), pos, h, h)
    with pytest.raises(ValueError):
        ress.rope(plan(), pos, h, h, k=h)
    with pytest.raises(ValueError):
        ress.rope(plan(), pos, torch.zeros(4, 2, 32), h)
    with pytest.raises(ValueError):
        ress.rope_bwd(plan(), pos, h, h, q_norm=(None, None))
    with pytest.raises(ValueError):
        ress.qkv_proj(ress.dims(4, 1, 0, 64), x, x, x, x, x, x, x, x)


# ---- sources ---------------------------------------------------------------------------------
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_35593_gb300", "csrc")
FILES = ["k_norm.cu", "k_rope.cuh", "k_rope.cu", "k_rope_bwd.cu", "k_rope_few.cu", "k_qkv.cu", "row_ops.cuh"]


def code(name):
    text = re.sub(r"/\*.*?\*/", " ", open(os.path.join(CSRC, name)).read(), flags=re.S)
    return re.sub(r"//[^\n]*", "", text)


def kernels(name):
    text = code(name)
    for m in re.finditer(r"__global__[^{;]*?\b(k_\w+)\(", text):
        depth, at = 0, text.index("{", m.end())
        for k in range(at, len(text)):
            depth += (text[k] == "{") - (text[k] == "}")
            if depth == 0:
                yield m.group(1), text[m.end():at], text[at:k]
                break


def test_overlapped_kernels_wait_before_they_touch_memory_and_promise_nothing():
    """Kernels that may start before the one ahead has ended: they wait for it (stream_acquire) before they
    read a parameter, an element or a position, and release the next one at the end."""
    found = {}
    for f in FILES:
        assert "__restrict__" not in code(f) and "__ldg" not in code(f)
        for name, params, body in kernels(f):
            found[name] = body
            first = body.index("stream_acquire()")
            assert body.index("stream_release()") > first, name
            for touch in ("param_at(", "params_at<", "load_row<", "load_vec<", "p.pos[", "p.partial[", "tma_load", "tma_store"):
                at = body.find(touch)
                assert at == -1 or at > first, (name, touch)
    assert set(found) == {"k_layer_norm", "k_layer_norm_bwd", "k_fold_parts", "k_rope", "k_rope_fold", "k_qkv"}


def test_every_wait_of_the_projection_is_bounded():
    body = code("k_qkv.cu")
    assert "kQWaitNs" in body and not re.search(r"while\s*\(\s*!\s*mbar_try_wait", body)
    assert len(re.findall(r"mbar_wait\(", body)) == len(re.findall(r"mbar_wait\([^;]*?(?:kQWaitNs|kQDrainNs)\)", body))


def test_sources_of_the_new_operators_are_built():
    build = __graft_entry__._build_module()
    assert {f for f in FILES if f.endswith(".cu")} <= set(build.SOURCES)
    assert {os.path.basename(f) for f in glob.glob(os.path.join(CSRC, "*.cu"))} == set(build.SOURCES)

"""Refusals of the dense attention and of the cache, at the C ABI and in the binding: nothing is launched."""
import ctypes

import pytest

import __graft_entry__

torch = pytest.importorskip("torch")
__graft_entry__._build_module().build()
import paper_2609_35593_gb300 as ress  # noqa: E402

EINVAL, EWORKSPACE, EUNSUPPORTED = -1, -2, -3
P, I32, I64, F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class Heads(ctypes.Structure):
    _fields_ = [("data", P), ("token_stride", I64), ("head_stride", I64)]


class Args(ctypes.Structure):
    _fields_ = [("type", I32), ("n_seqs", I32), ("q_heads", I32), ("kv_heads", I32), ("causal", I32), ("cap", F32),
                ("rows", I64), ("keys", I64), ("q_start", P), ("k_start", P), ("prefix", P), ("slopes", P),
                ("q", Heads), ("k", Heads), ("v", Heads), ("o", Heads), ("lse", P)]


class Pages(ctypes.Structure):
    _fields_ = [("table", P), ("lens", P), ("table_stride", I64), ("table_cols", I32), ("page", I32), ("n_pages", I64),
                ("k_page_stride", I64), ("v_page_stride", I64)]


class Grads(ctypes.Structure):
    _fields_ = [("d_o", Heads), ("dq", Heads), ("dk", Heads), ("dv", Heads)]


class Tables(ctypes.Structure):
    _fields_ = [("n_seqs", I32), ("page", I32), ("table_cols", I32), ("table_stride", I64), ("n_free", I64), ("n_slots", I64)] + [
        (n, P) for n in ("have", "add", "free", "taken", "table", "lens", "q_start", "slots", "pos", "taken_out")]


AT = 1 << 20  # an address that is never looked at
WS = 1 << 30


def heads(n, at=AT):
    return Heads(at, 64 * n, 64)


def args(**changed):
    a = Args(0, 2, 4, 2, 1, 0.0, 100, 200, AT, AT, None, None, heads(4), heads(2), heads(2), heads(4), AT)
    for name, value in changed.items():
        setattr(a, name, value)
    return a


def call(name, *a, ws=WS, size=1 << 40):
    return getattr(ress._lib, name)(*(ctypes.byref(x) if isinstance(x, ctypes.Structure) else x for x in a), ws, size, None)


BAD = [("type", 2, EUNSUPPORTED), ("type", -1, EUNSUPPORTED), ("q_heads", 0, EUNSUPPORTED), ("q_heads", 5, EUNSUPPORTED),
       ("q_heads", 130, EUNSUPPORTED), ("kv_heads", 0, EUNSUPPORTED), ("n_seqs", -1, EINVAL), ("n_seqs", (1 << 20) + 1, EINVAL), ("causal", 2, EINVAL),
       ("cap", -1.0, EINVAL), ("cap", float("nan"), EINVAL), ("cap", float("inf"), EINVAL), ("cap", 1e-31, EINVAL),
       ("rows", -1, EINVAL), ("rows", 1 << 31, EINVAL), ("q_start", None, EINVAL), ("q_start", AT + 2, EINVAL),
       ("prefix", AT + 1, EINVAL), ("slopes", AT + 1, EINVAL), ("lse", AT + 2, EINVAL), ("q", Heads(None, 256, 64), EINVAL),
       ("q", Heads(AT + 8, 256, 64), EINVAL), ("q", Heads(AT, 260, 64), EINVAL), ("q", Heads(AT, 256, 4), EINVAL),
       ("q", Heads(AT, 256, 0), EINVAL), ("k", Heads(AT, 0, 64), EINVAL), ("v", Heads(AT, -128, 64), EINVAL),
       ("o", Heads(AT, 128, 64), EINVAL), ("o", Heads(AT, 256, 32), EINVAL)]


@pytest.mark.parametrize("field,value,code", BAD + [("keys", -1, EINVAL), ("keys", 1 << 31, EINVAL), ("keys", (1 << 31) - 255, EINVAL), ("k_start", None, EINVAL)])
def test_attention_refuses(field, value, code):
    assert call("ress_attn", args(**{field: value})) == code
    assert ress._lib.ress_last_error()
    # in the gradient o is an input, so its heads may overlap
    if field != "o":
        assert call("ress_attn_bwd", args(**{field: value}), Grads(heads(4), heads(4), heads(2), heads(2))) == code


@pytest.mark.parametrize("field,value,code", BAD)
def test_paged_attention_refuses(field, value, code):
    pages = Pages(AT, AT, 8, 8, 64, 100, 64 * 128, 64 * 128)
    assert call("ress_paged_attn", args(**{field: value}), pages) == code


def test_a_prefix_needs_the_causal_mask():
    assert call("ress_attn", args(causal=0, prefix=AT)) == EINVAL


@pytest.mark.parametrize("field,value,code", [("page", 4, EUNSUPPORTED), ("page", 12, EUNSUPPORTED), ("page", 0, EUNSUPPORTED),
                                              ("n_pages", 0, EINVAL), ("n_pages", 1 << 26, EINVAL), ("table_cols", -1, EINVAL),
                                              ("table_cols", (1 << 25) - 3, EINVAL),
                                              ("table", None, EINVAL), ("lens", None, EINVAL), ("lens", AT + 2, EINVAL),
                                              ("k_page_stride", 12, EINVAL), ("v_page_stride", 0, EINVAL),
                                              ("table_stride", -1, EINVAL)])
def test_pages_that_are_refused(field, value, code):
    pages = Pages(AT, AT, 8, 8, 64, 100, 64 * 128, 64 * 128)
    setattr(pages, field, value)
    assert call("ress_paged_attn", args(), pages) == code


def test_the_gradient_needs_lse_and_outputs_that_do_not_overlap():
    good = Grads(heads(4), heads(4), heads(2), heads(2))
    assert call("ress_attn_bwd", args(lse=None), good) == EINVAL
    for name, h in (("d_o", Heads(None, 256, 64)), ("dq", Heads(AT, 128, 64)), ("dk", Heads(AT, 128, 32)), ("dv", Heads(AT, 64, 64))):
        bad = Grads(heads(4), heads(4), heads(2), heads(2))
        setattr(bad, name, h)
        assert call("ress_attn_bwd", args(), bad) == EINVAL, name


def test_workspaces():
    for backward in (False, True):
        need = ress.attn_workspace_bytes(100, 4, backward)
        name, a = ("ress_attn_bwd", (args(), Grads(heads(4), heads(4), heads(2), heads(2)))) if backward else ("ress_attn", (args(),))
        assert call(name, *a, size=need - 1) == EWORKSPACE
        assert call(name, *a, ws=WS + 128, size=need) == EINVAL
        assert call(name, *a, ws=None, size=need) == EINVAL
    assert ress.attn_workspace_bytes(10 ** 6, 16, True) >= ress.attn_workspace_bytes(10, 16, True) + 8 * 16 * (10 ** 6 - 10)
    for rows, heads_ in ((-1, 4), (1 << 31, 4), (5, 0)):
        with pytest.raises(ress.RessError):
            ress.attn_workspace_bytes(rows, heads_)


def test_a_workspace_of_another_device(monkeypatch):
    class On:
        def __init__(self, n):
            self.device = f"cuda:{n}"
            self.get_device = lambda: n

    monkeypatch.setattr(ress, "_scratch", lambda ws: (0, 0))
    assert ress._scratch_beside(On(0), On(0)) == (0, 0) == ress._scratch_beside(None, On(1))
    with pytest.raises(ValueError, match="cuda:1"):
        ress._scratch_beside(On(1), On(0))


def test_outputs_are_not_inputs():
    assert call("ress_attn", args()) == EINVAL
    assert call("ress_paged_attn", args(), Pages(AT, AT, 8, 8, 64, 100, 64 * 128, 64 * 128)) == EINVAL
    assert b"o must not be an input" in ress._lib.ress_last_error()
    for name in ("dq", "dk", "dv"):
        g = Grads(heads(4), *(heads(n, AT + (i << 24)) for i, n in ((1, 4), (2, 2), (3, 2))))
        setattr(g, name, heads(4 if name == "dq" else 2))
        assert call("ress_attn_bwd", args(), g) == EINVAL
        assert name.encode() + b" must not be an input" in ress._lib.ress_last_error()


def test_nothing_to_do_launches_nothing():
    before = ress.kernel_launches()
    assert call("ress_attn", args(rows=0)) == 0
    assert call("ress_attn", args(n_seqs=0)) == 0
    assert call("ress_attn_bwd", args(rows=0, keys=0), Grads()) == 0
    assert call("ress_paged_attn", args(rows=0), Pages(page=8)) == 0
    none = ress._lib.ress_cache_write(0, 2, *(ctypes.byref(heads(2)),) * 2, None, *(ctypes.byref(heads(2)),) * 2, 64, 64, 8, 1, WS,
                                      256, None)
    assert none == 0 and ress.kernel_launches() == before


@pytest.mark.parametrize("field,value,code", [("n_seqs", -1, EUNSUPPORTED), ("n_seqs", 8193, EUNSUPPORTED), ("page", 0, EINVAL),
                                              ("table_stride", 3, EINVAL), ("n_free", -1, EINVAL), ("n_slots", 1 << 31, EINVAL),
                                              ("have", None, EINVAL), ("taken", None, EINVAL), ("slots", AT + 2, EINVAL),
                                              ("lens", AT, EINVAL), ("taken_out", AT + 8, EINVAL)])
def test_tables_that_are_refused(field, value, code):
    t = Tables(2, 16, 4, 4, 10, 20, *(AT + 4 * i for i in range(10)))
    assert t.taken == AT + 12
    if field == "taken_out":
        value = t.taken
    if field == "lens":
        value = t.have
    setattr(t, field, value)
    assert call("ress_cache_tables", t, size=256) == code


@pytest.mark.parametrize("change,code", [({"tokens": -1}, EINVAL), ({"kv": 0}, EUNSUPPORTED), ({"slots": None}, EINVAL),
                                         ({"page": 0}, EINVAL), ({"pages": 1 << 28}, EINVAL), ({"stride": 4}, EINVAL),
                                         ({"k": Heads(AT + 2, 128, 64)}, EINVAL), ({"kc": Heads(AT, 64, 64)}, EINVAL)])
def test_writes_that_are_refused(change, code):
    c = {"tokens": 5, "kv": 2, "slots": AT, "page": 16, "pages": 10, "stride": 16 * 128, "k": heads(2), "kc": heads(2), **change}
    rc = ress._lib.ress_cache_write(c["tokens"], c["kv"], ctypes.byref(c["k"]), ctypes.byref(heads(2)), c["slots"],
                                    ctypes.byref(c["kc"]), ctypes.byref(heads(2)), c["stride"], c["stride"], c["page"], c["pages"], WS, 256,
                                    None)
    assert rc == code


def test_the_binding_refuses_host_tensors():
    """Before the library is called: with the tensor's name."""
    q, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    ws = torch.zeros(256, dtype=torch.uint8)
    with pytest.raises(ValueError, match="q must live on a CUDA device"):
        ress.attn(q, q, q, q, ws)
    with pytest.raises(ValueError, match="lse"):
        ress.attn_bwd(q, q, q, q, q, None, q, q, q, ws)
    with pytest.raises(ValueError, match="q must"):
        ress.paged_attn(q, q, q, i, i, q, ws)
    with pytest.raises(ValueError, match="table must"):
        ress.cache_tables(i, i, i, i, i.view(1, 2), 16, i, i, i, i, i, ws)
    with pytest.raises(ValueError, match="k must"):
        ress.cache_write(q, q, i, q[None], q[None], ws)
    with pytest.raises(TypeError):
        ress.attn(None, q, q, q, ws)


def test_structs_are_as_the_header_has_them():
    """Sizes that the C++ binding packs and this file's structures agree on (natural alignment, no packing)."""
    assert ctypes.sizeof(Args) == 24 + 16 + 4 * 8 + 4 * 24 + 8
    assert ctypes.sizeof(Pages) == 16 + 8 + 8 + 3 * 8 and ctypes.sizeof(Grads) == 4 * 24
    assert ctypes.sizeof(Tables) == 16 + 3 * 8 + 10 * 8

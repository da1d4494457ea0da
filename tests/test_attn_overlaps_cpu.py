"""Outputs that share memory with one another or with inputs are refused before anything is launched; views that lie between
one another are not.  Without a GPU such a call fails at its launch, and the addresses are never looked at."""
import ctypes
import random

import pytest

from test_attn_cpu import AT, EINVAL, WS, Args, Grads, Heads, Pages, Tables, args, call, heads, ress

FAR = 1 << 24  # bytes between tensors of their own


def apart(**changed):
    a = args(q=heads(4, AT), k=heads(2, AT + FAR), v=heads(2, AT + 2 * FAR), o=heads(4, AT + 3 * FAR), lse=AT + 4 * FAR)
    for name, value in changed.items():
        setattr(a, name, value)
    return a


def gradients(**changed):
    g = Grads(heads(4, AT + 5 * FAR), heads(4, AT + 6 * FAR), heads(2, AT + 7 * FAR), heads(2, AT + 8 * FAR))
    for name, value in changed.items():
        setattr(g, name, value)
    return g


def overlaps(name, *a):
    """Whether the call is refused for an overlap."""
    rc, text = call(name, *a), ress._lib.ress_last_error().decode()
    assert rc == EINVAL or "must not" not in text
    return rc == EINVAL and "must not" in text


def at(a, which):
    return getattr(a, which).data if isinstance(getattr(a, which), Heads) else getattr(a, which)


@pytest.fixture(autouse=True)
def no_gpu():
    """Calls that are not refused would launch on these addresses."""
    import torch

    if torch.cuda.is_available():
        pytest.skip("a GPU would read the addresses")


def test_tensors_of_their_own_are_not_refused():
    assert not overlaps("ress_attn", apart())
    assert not overlaps("ress_attn_bwd", apart(), gradients())


@pytest.mark.parametrize("which", ["q", "k", "v"])
@pytest.mark.parametrize("by", [0, 16, 128, -128, 512, 99 * 512 // 2])
def test_o_within_an_input(which, by):
    """Starting anywhere in its rows: heads of 128 bytes, rows of 512 (256 of k and v, 200 of them)."""
    a = apart()
    a.o = heads(4, at(a, which) + by) if which == "q" else Heads(at(a, which) + by, 128, 64)
    if which != "q":  # as many heads as k: rows of 256 bytes
        a.q_heads, a.q = 2, Heads(AT, 128, 64)
    assert overlaps("ress_attn", a)


def test_lse_is_an_output_too():
    a = apart()
    for which in ("q", "k", "v", "o"):
        for by in (0, 4, 128):
            assert overlaps("ress_attn", apart(lse=at(a, which) + by)), which
    # and in the gradient an input
    assert overlaps("ress_attn_bwd", a, gradients(dq=heads(4, a.lse + 16)))


@pytest.mark.parametrize("one,two", [("dk", "dv"), ("dq", "dk"), ("dq", "dv")])
def test_gradients_that_are_one_another(one, two):
    for by in (0, 128):
        a, g = apart(), gradients()
        if one == "dq":  # as many heads
            a.kv_heads, a.k, a.v = 4, heads(4, AT + FAR), heads(4, AT + 2 * FAR)
            g.dk, g.dv = heads(4, g.dk.data), heads(4, g.dv.data)
        assert not overlaps("ress_attn_bwd", a, g)
        setattr(g, two, Heads(getattr(g, one).data + by, getattr(g, one).token_stride, 64))
        assert overlaps("ress_attn_bwd", a, g), by


@pytest.mark.parametrize("which", ["q", "k", "v", "o", "d_o"])
def test_gradients_within_inputs(which):
    a, g = apart(), gradients()
    src = g.d_o if which == "d_o" else getattr(a, which)
    out = "dk" if which in "kv" else "dq"
    setattr(g, out, Heads(src.data + src.token_stride * 2, src.token_stride, 64))  # a row later
    assert overlaps("ress_attn_bwd", a, g)


def test_views_between_one_another():
    """dq, dk, dv as heads of one tensor of rows, as planes, and as rows of one tensor after another."""
    rows = 8 * 64 + 64
    base = AT + 6 * FAR
    g = gradients(dq=Heads(base, rows, 64), dk=Heads(base + 4 * 128, rows, 64), dv=Heads(base + 6 * 128, rows, 64))
    assert not overlaps("ress_attn_bwd", apart(), g)
    # the same a head short: dk's first is dq's last
    g.dk = Heads(base + 3 * 128, rows, 64)
    assert overlaps("ress_attn_bwd", apart(), g)
    # heads outside: planes of 200 rows
    planes = gradients(dq=Heads(base, 64, 200 * 64), dk=Heads(base + 4 * 200 * 128, 64, 200 * 64), dv=Heads(base + 6 * 200 * 128, 64, 200 * 64))
    assert not overlaps("ress_attn_bwd", apart(), planes)
    planes.dv = Heads(base + 5 * 200 * 128 + 128, 64, 200 * 64)
    assert overlaps("ress_attn_bwd", apart(), planes)
    # o between the heads of a larger q (rows of 8 heads, of which q has the first four)
    assert not overlaps("ress_attn", apart(q=Heads(AT, 512, 64), o=Heads(AT + 512, 512, 64)))
    assert overlaps("ress_attn", apart(q=Heads(AT, 512, 64), o=Heads(AT + 384, 512, 64)))
    # every other row
    assert not overlaps("ress_attn", apart(q=Heads(AT, 512, 64), o=Heads(AT + 512, 512, 64), rows=100))


def test_any_strides_as_their_bytes_say():
    """o against q, and keys against values, of random strides and places near one another: as the sets of their bytes."""
    rng = random.Random(3)
    seen = set()
    for _ in range(600):
        rows, n = rng.randint(1, 6), rng.randint(1, 4)

        def layout():
            inner = 64 + 8 * rng.choice([0, 0, 1, 9])
            if rng.random() < 0.5:
                return n * inner + 8 * rng.choice([0, 0, 3, 8, 70]), inner
            return inner, rows * inner + 8 * rng.choice([0, 0, 3, 8, 70])

        one = layout()
        two = one if rng.random() < 0.5 else layout()
        by = 16 * rng.randint(-rows * n * 10, rows * n * 10)
        at_ = lambda base, s: {base + 2 * (i * s[0] + j * s[1]) // 16 * 16 + c for i in range(rows) for j in range(n) for c in range(0, 128, 16)}
        want = bool(at_(0, one) & at_(by, two))
        seen.add(want)
        a = apart(rows=rows, n_seqs=1, q_heads=n, kv_heads=n, lse=None)
        a.q, a.o = Heads(AT, *one), Heads(AT + by, *two)
        a.k, a.v = Heads(AT + FAR, 64 * n, 64), Heads(AT + 2 * FAR, 64 * n, 64)
        assert overlaps("ress_attn", a) == want, (rows, n, one, two, by)
    assert seen == {True, False}


def test_o_within_a_paged_cache():
    pages = Pages(AT, AT, 8, 8, 64, 100, 64 * 128, 64 * 128)
    a = apart()
    assert not overlaps("ress_paged_attn", a, pages)
    a.q_heads, a.q = 2, Heads(AT, 128, 64)
    for by in (0, 128, 64 * 128 * 2 * 3 + 256):
        a.o = Heads(a.k.data + by, 128, 64)
        assert overlaps("ress_paged_attn", a, pages), by


def write(kc, vc, stride=16 * 128, pages=10, page=16):
    k, v = heads(2, AT), heads(2, AT + FAR)
    rc = ress._lib.ress_cache_write(5, 2, ctypes.byref(k), ctypes.byref(v), AT + 2 * FAR, ctypes.byref(kc), ctypes.byref(vc), stride,
                                    stride, page, pages, WS, 256, None)
    text = ress._lib.ress_last_error().decode()
    return rc == EINVAL and "must not" in text


def test_pages_of_keys_and_values():
    kc = heads(2, AT + 4 * FAR)
    assert not write(kc, heads(2, AT + 5 * FAR))
    for by in (0, 16, 128, 256, 16 * 256, 9 * 16 * 256):
        assert write(kc, heads(2, kc.data + by)), by
    assert not write(kc, heads(2, kc.data + 10 * 16 * 256))
    # interleaved: a page of keys, a page of values; or heads of one row
    assert not write(kc, heads(2, kc.data + 16 * 256), stride=2 * 16 * 128)
    assert write(kc, heads(2, kc.data + 15 * 256), stride=2 * 16 * 128)
    assert not write(Heads(kc.data, 256, 64), Heads(kc.data + 256, 256, 64), stride=16 * 256)


NAMES = ("have", "add", "free", "taken", "table", "lens", "q_start", "slots", "pos", "taken_out")
SIZES = dict(zip(NAMES, (2, 2, 10, 1, 8, 2, 3, 20, 20, 1)))


def tables(**changed):
    t = Tables(2, 16, 4, 4, 10, 20, *(AT + FAR * i for i in range(10)))
    for name, value in changed.items():
        setattr(t, name, value)
    return t


def refused(t):
    rc = call("ress_cache_tables", t, size=256)
    return rc == EINVAL and b"must not" in ress._lib.ress_last_error()


def test_outputs_of_the_tables():
    assert not refused(tables())
    outs = NAMES[4:]
    for out in outs:
        for other in NAMES:
            if other == out:
                continue
            where = getattr(tables(), other)
            for at_ in (where, where + 4 * (SIZES[other] - 1), where - 4 * (SIZES[out] - 1)):
                assert refused(tables(**{out: at_})), (out, other)
            for at_ in (where + 4 * SIZES[other], where - 4 * SIZES[out]):
                assert not refused(tables(**{out: at_})), (out, other)


def test_numbers_between_the_rows_of_a_table():
    t = tables(table_stride=8)
    t.lens = t.table + 16
    assert not refused(t)
    t.lens = t.table + 12
    assert refused(t)
    t.lens = t.table + 28  # the second one is the second row's first column
    assert refused(t)

"""Dense attention over packed sequences and over a paged cache, and the cache, against float64."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import dense64 as R  # noqa: E402
import paper_2609_35593_gb300 as ress  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def float32_by_default():
    """Tensors made without a dtype here are float32, whatever other files left as the default."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def normal(seed, *shape, kind=BF16, by=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (by * torch.randn(*shape, generator=g, device="cuda")).to(kind)


def ints(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def workspace(rows, heads, backward=False):
    ws = torch.full((ress.attn_workspace_bytes(rows, heads, backward),), 0xA5, dtype=torch.uint8, device="cuda")
    ws[:256] = 0  # the status word; nothing else needs a value
    return ws


def problem(q_lens, k_lens, heads, kv, kind=BF16, seed=1):
    q = normal(seed, sum(q_lens), heads, 64, kind=kind, by=1.5)
    k, v = normal(seed + 1, sum(k_lens), kv, 64, kind=kind), normal(seed + 2, sum(k_lens), kv, 64, kind=kind)
    return q, k, v


def masks(heads, k_lens, causal, prefix, cap, slopes):
    return {"causal": causal, "prefix": ints([n // 3 for n in k_lens]) if prefix else None, "cap": cap,
            "slopes": torch.logspace(-3, 0, heads, device="cuda") if slopes else None}


def run(q, k, v, q_lens, k_lens, **mask):
    o, lse = torch.full_like(q, 7.0), torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
    ws = workspace(*q.shape[:2])
    ress.attn(q, k, v, o, ws, R.starts(q_lens), R.starts(k_lens), lse=lse, **mask)
    ress.status(ws)
    return o, lse


def check(q, k, v, q_lens, k_lens, got, **mask):
    o, lse, o_off, lse_off = R.attention(q, k, v, q_lens, k_lens, **mask)
    R.close(got[1], lse, lse_off, "lse")
    R.close(got[0], o, o_off, "o")


LENGTHS = [([1], [1]), ([63], [65]), ([128], [64]), ([129], [127]), ([256], [256]), ([257], [300]), ([1], [1500]),
           ([5, 0, 1, 300, 64], [5, 7, 0, 300, 1]), ([200], [50]), ([700, 3, 129], [700, 900, 129])]


@pytest.mark.parametrize("lens", LENGTHS, ids=str)
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (12, 4), (10, 2), (16, 1)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_of_packed_sequences(lens, heads, kv, causal):
    q, k, v = problem(*lens, heads, kv)
    check(q, k, v, *lens, run(q, k, v, *lens, causal=causal), causal=causal)


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("causal,prefix,cap,slopes", [(True, True, 0.0, False), (True, False, 30.0, False),
                                                      (False, False, 0.0, True), (True, True, 20.0, True),
                                                      (False, False, 2.0, False), (False, False, 0.0, False)])
@pytest.mark.parametrize("heads,kv", [(4, 4), (6, 2), (48, 1), (64, 1)])
def test_masks_caps_and_slopes(kind, causal, prefix, cap, slopes, heads, kv):
    lens = ([150, 1, 400, 33], [150, 700, 390, 40])
    q, k, v = problem(*lens, heads, kv, kind)
    mask = masks(heads, lens[1], causal, prefix, cap, slopes)
    check(q, k, v, *lens, run(q, k, v, *lens, **mask), **mask)


def test_long_sequences_split_over_ctas():
    """Items that many CTAs share, and more work than one round."""
    lens = ([300, 2, 1000], [9000, 5000, 1000])
    q, k, v = problem(*lens, 4, 2)
    for causal in (False, True):
        check(q, k, v, *lens, run(q, k, v, *lens, causal=causal), causal=causal)


def test_one_sequence_needs_no_starts_and_lse_is_optional():
    q, k, v = problem([300], [200], 2, 1)
    want = run(q, k, v, [300], [200])[0]
    o, ws = torch.empty_like(q), workspace(300, 2)
    ress.attn(q, k, v, o, ws)
    ress.status(ws)
    assert torch.equal(o, want)


def test_strided_heads_and_rows_behind_the_last_sequence():
    """Heads of one tensor of projections, an output inside a larger one, and a padded batch."""
    lens, pad = ([130, 70], [130, 70]), 41
    n = sum(lens[0]) + pad
    x = normal(3, n, 3, 4, 64)
    x[-pad:] = math.nan
    q, k, v = x.unbind(1)
    big = torch.full((n, 6, 72), 5.0, dtype=BF16, device="cuda")
    o, lse = big[:, 1:5, :64], torch.full((4, n), 5.0, device="cuda")
    ws = workspace(n, 4)
    ress.attn(q, k, v, o, ws, R.starts(lens[0]), R.starts(lens[1]), lse=lse, causal=True)
    ress.status(ws)
    check(q[:-pad], k[:-pad], v[:-pad], *lens, (o[:-pad], lse[:, :-pad]), causal=True)
    assert (o[-pad:] == 5).all() and (lse[:, -pad:] == 5).all()
    assert (big[:, 0] == 5).all() and (big[:, 5] == 5).all() and (big[:, :, 64:] == 5).all()


def test_neighbours_that_are_not_finite():
    """A sequence does not see what its neighbours hold, nor what a tile reads past its end."""
    lens = ([70, 30, 70], [70, 30, 70])
    q, k, v = problem(*lens, 2, 2)
    want = run(q, k, v, *lens)
    for t in (k, v):
        t[70:100] = math.nan
        t[170 - 70:][:0] = 0
    got = run(q, k, v, *lens)
    for a, b in ((slice(0, 70), slice(0, 70)), (slice(100, 170), slice(100, 170))):
        assert torch.equal(got[0][a], want[0][b]) and torch.equal(got[1][:, a], want[1][:, b])


def test_large_scores():
    """One key far above the others, late in the row: the accumulator is rescaled."""
    q, k, v = problem([200], [1000], 2, 2)
    k[777] = 20 * q[5, 0]
    k[100:200] *= 8
    check(q, k, v, [200], [1000], run(q, k, v, [200], [1000]))


def test_many_sequences_without_keys():
    """Between others: items without tiles end while the last tiles before them are worked on."""
    lens = ([70, 300] + [3] * 3000 + [130], [70, 300] + [0] * 3000 + [130])
    q, k, v = problem(*lens, 2, 2)
    o, lse = run(q, k, v, *lens)
    for a, b, n in ((0, 0, 70), (70, 70, 300), (9370, 370, 130)):
        part = slice(b, b + n)
        check(q[a:a + n], k[part], v[part], [n], [n], (o[a:a + n], lse[:, a:a + n]))
    assert (o[370:9370] == 0).all() and (lse[:, 370:9370] == -math.inf).all()


def test_same_bits_again():
    lens = ([300, 1000], [9000, 1000])
    q, k, v = problem(*lens, 4, 2)
    first = run(q, k, v, *lens, causal=True)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(q, k, v, *lens, causal=True), first))


@pytest.mark.parametrize("q_start,k_start", [([0, 60, 101], [0, 60, 100]), ([0, 60, 40], [0, 60, 100]),
                                             ([0, 60, 100], [0, 60, 101]), ([0, 60, 100], [0, 60, 30])])
def test_bad_starts_are_told(q_start, k_start):
    """The sequence before them is as ever; rows outside are not written, rows without keys are 0."""
    q, k, v = problem([100], [100], 2, 2)
    o, ws = torch.full_like(q, 7.0), workspace(100, 2)
    ress.attn(q, k, v, o, ws, ints(q_start), ints(k_start))
    with pytest.raises(ress.RessError) as e:
        ress.status(ws)
    assert e.value.code == -6
    assert torch.equal(o[:60], run(q[:60], k[:60], v[:60], [60], [60])[0])
    assert (o[60:] == (7 if q_start[2] != 100 else 0)).all()


def test_two_streams_and_a_graph_of_other_lengths():
    """A captured call serves other lengths; two calls at once have workspaces of their own."""
    heads, n = 4, 600
    q, k, v = problem([n], [n], heads, 2)
    starts, o, lse, ws = R.starts([n, 0]), torch.zeros_like(q), torch.zeros(heads, n, device="cuda"), workspace(n, heads)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        ress.attn(q, k, v, o, ws, starts, starts, lse=lse, causal=True)
    for lens in ([600, 0], [100, 500], [1, 599], [0, 600]):
        starts.copy_(R.starts(lens))
        graph.replay()
        ress.status(ws)
        check(q, k, v, lens, lens, (o, lse), causal=True)
    other = torch.zeros_like(q), workspace(n, heads)
    side.wait_stream(torch.cuda.current_stream())
    ress.attn(q, k, v, other[0], other[1], starts, starts, causal=True, stream=side)
    ress.attn(q, k, v, o, ws, starts, starts, causal=True)
    torch.cuda.synchronize()
    assert torch.equal(o, other[0])


# ---- the cache ----------------------------------------------------------------------------
def paged(k, v, k_lens, page, seed=5, spare=3):
    """Pages in any order that hold the keys; NaN wherever no key is."""
    need = [-(-n // page) for n in k_lens]
    order = torch.randperm(sum(need) + spare, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((len(k_lens), max(need, default=0) + 1), -1, dtype=torch.int32)
    kp, vp = (torch.full((sum(need) + spare, page, *k.shape[1:]), math.nan, dtype=k.dtype, device="cuda") for _ in range(2))
    at = 0
    for b, n in enumerate(k_lens):
        for i in range(need[b]):
            table[b, i] = id = order.pop()
            rows = slice(at + i * page, at + min(n, (i + 1) * page))
            kp[id, :rows.stop - rows.start], vp[id, :rows.stop - rows.start] = k[rows], v[rows]
        at += n
    return kp, vp, table.cuda()


@pytest.mark.parametrize("page", [8, 16, 24, 64, 72, 128, 256])
@pytest.mark.parametrize("lens", [([1] * 6, [1, 63, 64, 65, 700, 0]), ([17, 1, 130], [500, 3, 130]), ([1], [5000])], ids=str)
@pytest.mark.parametrize("heads,kv", [(16, 16), (12, 4), (16, 1)])
def test_attention_over_a_paged_cache(page, lens, heads, kv):
    q, k, v = problem(*lens, heads, kv)
    kp, vp, table = paged(k, v, lens[1], page)
    o, lse, ws = torch.empty_like(q), torch.empty(heads, sum(lens[0]), device="cuda"), workspace(*q.shape[:2])
    ress.paged_attn(q, kp, vp, table, ints(lens[1]), o, ws, R.starts(lens[0]), lse=lse, causal=True)
    ress.status(ws)
    check(q, k, v, *lens, (o, lse), causal=True)


@pytest.mark.parametrize("layout", ["heads outside", "k and v interleaved"])
def test_layouts_of_pages(layout):
    lens = ([3, 40], [100, 77])
    q, k, v = problem(*lens, 6, 2, F16)
    kp, vp, table = paged(k, v, lens[1], 32)
    if layout == "heads outside":
        kp, vp = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (kp, vp))
    else:
        kp, vp = torch.stack([kp, vp], 1).unbind(1)
    mask = masks(6, lens[1], True, True, 50.0, True)
    o, lse, ws = torch.empty_like(q), torch.empty(6, sum(lens[0]), device="cuda"), workspace(*q.shape[:2])
    ress.paged_attn(q, kp, vp, table, ints(lens[1]), o, ws, R.starts(lens[0]), lse=lse, **mask)
    ress.status(ws)
    check(q, k, v, *lens, (o, lse), **mask)


def test_bad_pages_are_told():
    """A page that is none counts as zeros; a length past the table leaves no keys."""
    lens = ([2, 2], [100, 100])
    q, k, v = problem(*lens, 2, 2)
    kp, vp, table = paged(k, v, lens[1], 32)
    for t in (kp, vp):
        t.nan_to_num_(0.0)
    bad = table.clone()
    bad[0, 1] = kp.shape[0]
    o, ws = torch.empty_like(q), workspace(4, 2)
    ress.paged_attn(q, kp, vp, bad, ints(lens[1]), o, ws, R.starts(lens[0]))
    with pytest.raises(ress.RessError):
        ress.status(ws)
    k, v = k.clone(), v.clone()
    k[32:64] = v[32:64] = 0
    check(q, k, v, *lens, (o, run(q, k, v, *lens)[1]))
    ress.paged_attn(q, kp, vp, table, ints([100, 32 * table.shape[1] + 1]), o, ws, R.starts(lens[0]))
    with pytest.raises(ress.RessError):
        ress.status(ws)
    assert (o[2:] == 0).all() and (o[:2] != 0).any()


def test_a_cache_past_32_bit_offsets():
    """2.1 million rows of 16 heads: 2^31 elements and more, pages of the sequences at both ends; and K, V written there."""
    page, kv, pages = 256, 16, 8300
    kp, vp = (torch.zeros(pages, page, kv, 64, dtype=BF16, device="cuda") for _ in range(2))
    assert kp.numel() > 2 ** 31
    lens = ([3, 70], [600, 300])
    q, k, v = problem(*lens, 16, kv)
    table = ints([pages - 1, 0, pages - 3, 1, pages - 2, 2]).view(2, 3)
    at = torch.cat([table[b, torch.arange(n, device="cuda") // page] * page + torch.arange(n, device="cuda") % page
                    for b, n in enumerate(lens[1])]).int()
    ws, ws2 = workspace(73, 16), torch.zeros(256, dtype=torch.uint8, device="cuda")
    ress.cache_write(k, v, at, kp, vp, ws2)
    ress.status(ws2)
    assert torch.equal(kp.view(-1, kv, 64)[at.long()], k) and torch.equal(vp.view(-1, kv, 64)[at.long()], v)
    o, lse = torch.empty_like(q), torch.empty(16, 73, device="cuda")
    ress.paged_attn(q, kp, vp, table, ints(lens[1]), o, ws, R.starts(lens[0]), lse=lse, causal=True)
    ress.status(ws)
    check(q, k, v, *lens, (o, lse), causal=True)


def test_packed_rows_past_32_bit_offsets():
    """Two sequences at the ends of tensors of more than 2^31 elements."""
    n, heads = (1 << 25) + 300, 1
    q, k, v, o = (torch.zeros(n, heads, 64, dtype=BF16, device="cuda") for _ in range(4))
    a, b = 130, n - 170
    for i, t in enumerate((q, k, v)):
        t[:a], t[b:] = normal(i, a, heads, 64), normal(9 + i, n - b, heads, 64)
    # between them keys without rows, and rows without keys
    starts, k_starts = ints([0, a, a, b, n]), ints([0, a, b, b, n])
    lse, ws = torch.zeros(heads, n, device="cuda"), workspace(n, heads)
    ress.attn(q, k, v, o, ws, starts, k_starts, lse=lse)
    ress.status(ws)
    for part in (slice(0, a), slice(b, n)):
        m = part.stop - part.start
        check(q[part], k[part], v[part], [m], [m], (o[part], lse[:, part]))
    assert (o[a:b] == 0).all()


def tables_of(have, add, free, taken, table, page):
    """What cache_tables is to give, one token after another."""
    table, slots, pos, starts = table.tolist(), [], [], [0]
    for row, h, a in zip(table, have, add):
        for p in range(h, h + a):
            if p % page == 0:
                row[p // page] = free[taken]
                taken += 1
            slots.append(row[p // page] * page + p % page)
            pos.append(p)
        starts.append(len(slots))
    return table, starts, slots, pos, taken


@pytest.mark.parametrize("page", [1, 8, 16, 48])
@pytest.mark.parametrize("have,add", [([0], [1]), ([5, 0, 16, 31], [1, 0, 1, 1]), ([0, 7, 100, 3000], [1700, 0, 48, 1]),
                                      (list(range(400)), [1] * 400), ([0] * 3, [0] * 3)], ids=lambda x: str(x)[:20])
def test_tables_of_the_next_tokens(page, have, add):
    need = [-(-(a + b) // page) for a, b in zip(have, add)]
    held = [-(-a // page) for a in have]
    ids = torch.randperm(sum(need) + 5, generator=torch.Generator().manual_seed(3)).int()
    table = torch.full((len(have), max(need) + 2), -1, dtype=torch.int32)
    at = 0
    for row, n in zip(table, held):
        row[:n] = ids[at:at + n]
        at += n
    free, pad = torch.cat([ids[:2], ids[at:]]), 9
    want = tables_of(have, add, free.tolist(), 2, table, page)
    n = sum(add) + pad
    dev, lens, q_start, slots, pos, out = (table.cuda(), ints([0] * len(have)), ints([0] * (len(have) + 1)), ints([7] * n),
                                           ints([7] * n), ints([0]))
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    ress.cache_tables(ints(have), ints(add), free.cuda(), ints([2]), dev, page, lens, q_start, slots, pos, out, ws)
    ress.status(ws)
    assert dev.tolist() == want[0] and q_start.tolist() == want[1] and out.item() == want[4]
    assert slots.tolist() == want[2] + [-1] * pad and pos.tolist() == want[3] + [-1] * pad
    assert lens.tolist() == [a + b for a, b in zip(have, add)]


def test_tables_without_room_are_told():
    """Too few free pages, too few columns, too few slots, a negative length: no token is placed outside."""
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    for have, add, free, cols, n in (([8], [20], [4, 5], 9, 20), ([8], [20], [4, 5, 6], 2, 20), ([8], [20], [4, 5, 6], 9, 7),
                                     ([-1], [4], [4], 9, 4), ([8], [-4], [4], 9, 4), ([16], [1], [4], 9, 1)):
        table = torch.full((1, cols), -1, dtype=torch.int32, device="cuda")
        if have == [8]:
            table[0, 0] = 2
        guard = ints([7] * (n + 4))
        slots, pos = guard[:n], ints([0] * n)
        ress.cache_tables(ints(have), ints(add), ints(free), ints([0]), table, 8, ints([0]), ints([0, 0]), slots, pos, ints([0]),
                          ws)
        if (have, add) == ([16], [1]):  # a page begins: its entry comes from the free ones, held entries are not looked at
            ress.status(ws)
            assert slots.tolist() == [32]
            continue
        with pytest.raises(ress.RessError) as e:
            ress.status(ws)
        assert e.value.code == -6 and (guard[n:] == 7).all()
        places = [s for s in slots.tolist() if s != -1]
        assert len(set(places)) == len(places) and all(s // 8 in [2] + free for s in places)


@pytest.mark.parametrize("heads", [1, 2, 3, 16, 40])
def test_rows_written_into_pages(heads):
    tokens, page, pages = 77, 24, 9
    k, v = normal(1, tokens, heads, 64), normal(2, tokens, 2, heads, 64)[:, 1]
    kp, vp = (torch.full((pages, page, heads, 64), 3.0, dtype=BF16, device="cuda") for _ in range(2))
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(1))[:tokens].int().cuda()
    slots[5] = slots[76] = -1
    want = []
    for pool, new in ((kp, k), (vp, v)):
        w = pool.clone()
        w.view(-1, heads, 64)[slots[slots >= 0].long()] = new[slots >= 0]
        want.append(w)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    ress.cache_write(k, v, slots, kp, vp, ws)
    ress.status(ws)
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1])
    slots[3], slots[4] = pages * page, -2
    ress.cache_write(k, v, slots, kp, vp, ws)
    with pytest.raises(ress.RessError):
        ress.status(ws)
    assert torch.equal(kp, want[0])


def test_views_one_after_another():
    """Tables, writes and attention as they are used: the cached result is that of all tokens at once."""
    heads, kv, page, scenes, steps = 6, 2, 32, 3, [(40, 1, 90), (1, 1, 1), (70, 0, 5), (1, 1, 1)]
    total = [sum(s[b] for s in steps) for b in range(scenes)]
    data = [problem([n], [n], heads, kv, seed=10 * b + 1) for b, n in enumerate(total)]
    pages = sum(-(-n // page) for n in total)
    kp, vp = (torch.full((pages, page, kv, 64), math.nan, dtype=BF16, device="cuda") for _ in range(2))
    free = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).int().cuda()
    table = torch.full((scenes, max(-(-n // page) for n in total)), -1, dtype=torch.int32, device="cuda")
    have, taken = [0] * scenes, ints([0])
    lens, out = ints(have), ints([0])
    ws, ws2 = workspace(200, heads), torch.zeros(256, dtype=torch.uint8, device="cuda")
    outs = [[] for _ in range(scenes)]
    for add in steps:
        new = [torch.cat([d[i][h:h + a] for d, h, a in zip(data, have, add)]) for i in range(3)]
        n = sum(add)
        old, lens, q_start, slots, pos = lens, ints([0] * scenes), ints([0] * (scenes + 1)), ints([0] * n), ints([0] * n)
        ress.cache_tables(old, ints(add), free, taken, table, page, lens, q_start, slots, pos, out, ws2)
        taken, out = out, taken
        ress.cache_write(new[1], new[2], slots, kp, vp, ws2)
        o = torch.empty_like(new[0])
        ress.paged_attn(new[0], kp, vp, table, lens, o, ws, q_start, causal=True)
        for b, part in enumerate(o.split(list(add))):
            outs[b].append(part)
        have = [h + a for h, a in zip(have, add)]
    ress.status(ws), ress.status(ws2)
    assert taken.item() == pages
    for b, (q, k, v) in enumerate(data):
        want, _, off, _ = R.attention(q, k, v, [total[b]], [total[b]], causal=True)
        R.close(torch.cat(outs[b]), want, off)

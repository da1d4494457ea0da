"""Performance cases of dense attention over packed sequences, its gradient, and attention over a paged
cache of keys and values: what a user of this package calls for a backbone's frame attention, to
fine-tune a layer or calibrate head budgets, and to take views one after another, over the sizes it is
used at, each with its inputs, one pass of it, its work and its result in float64.

An operation is one of
  attn      attention of packed sequences, each on its own keys: softmax of cap tanh(scale q.k / cap)
            - slope |distance| over the keys that a row sees (all of its sequence's, or those up to its
            own position and the first `prefix` ones); the last row and the last key of a sequence stand at the
            same position
  attn_bwd  its gradients with respect to Q, K and V
  paged     the same attention of new tokens over the pages of a cache that holds them already
  append    pages and slots for the next tokens of every sequence, and their keys and values written there

`own` False computes them from elementary torch operations in float32, rounded once at the end.

Sizes are those of 3D-ViT attention (views of 37 x 37 patch and 5 special tokens, heads of 64 channels, every
view a sequence of its own in frame attention) and generic ragged lengths, with fewer heads for K and V.
"""
import math
import random

import torch

own = False

VIEW = 37 * 37 + 5  # tokens of one view
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
PAIRS = 8 * VIEW * 8 * VIEW * 16  # (row, key, head) triples of the largest listed case


def listed():
    attn = {"op": "attn", "type": "bf16", "heads": 16, "kv_heads": 16, "seqs": 1, "q_len": VIEW, "k_len": VIEW,
            "ragged": False, "causal": False, "prefix": False, "cap": 0.0, "slopes": False}
    bwd = {**attn, "op": "attn_bwd"}
    paged = {**attn, "op": "paged", "page": 64}
    append = {"op": "append", "type": "bf16", "kv_heads": 16, "seqs": 8, "have": 20000, "add": 1, "ragged": True,
              "page": 64}
    return [
        # the camera token of every view reads its view in a refining head: latency
        {**attn, "name": "attn_cameras", "seqs": 8, "q_len": 1},
        # packed documents of many lengths in half precision: causal, capped scores, fewer heads for K and V
        {**attn, "name": "attn_documents_f16", "type": "f16", "heads": 12, "kv_heads": 4, "seqs": 37, "q_len": 2531,
         "k_len": 2531, "ragged": True, "causal": True, "cap": 30.0},
        # frame attention of 32 images
        {**attn, "name": "attn_frames_v32", "seqs": 32},
        # dense global attention of 8 images, the largest
        {**attn, "name": "attn_global_v8", "q_len": 8 * VIEW, "k_len": 8 * VIEW},
        # gradients of a cropped pair of images in a small model
        {**bwd, "name": "bwd_crops", "heads": 3, "kv_heads": 3, "seqs": 2, "q_len": 333, "k_len": 333},
        # fine-tuning on packed documents: a prefix that every row sees, distances, fewer heads for K and V
        {**bwd, "name": "bwd_documents", "heads": 8, "kv_heads": 2, "seqs": 23, "q_len": 3001, "k_len": 3001,
         "ragged": True, "causal": True, "prefix": True, "slopes": True},
        # calibration of head budgets on 8 images
        {**bwd, "name": "bwd_global_v8", "q_len": 8 * VIEW, "k_len": 8 * VIEW},
        # one token for each of several scenes whose caches are long and of different lengths
        {**paged, "name": "paged_tokens", "seqs": 8, "q_len": 1, "k_len": 32 * VIEW, "ragged": True, "causal": True},
        # chunks of many short requests in half precision, small pages
        {**paged, "name": "paged_chunks_f16", "type": "f16", "heads": 16, "kv_heads": 4, "seqs": 48, "q_len": 509,
         "k_len": 8191, "ragged": True, "causal": True, "cap": 50.0, "page": 16},
        # the 32nd image of a scene sees the 31 before it and itself
        {**paged, "name": "paged_view", "k_len": 32 * VIEW},
        # the next token of every scene: latency
        {**append, "name": "append_tokens"},
        # the next image of 16 scenes
        {**append, "name": "append_views", "seqs": 16, "add": VIEW, "ragged": False, "have": 4 * VIEW},
    ]


def _log_int(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn_bwd", "attn_bwd", "paged", "paged", "append"])
    heads, kv = rng.choice([(16, 16), (16, 16), (12, 4), (8, 2), (3, 3), (16, 1), (10, 2), (8, 8)])
    case = {"op": op, "type": rng.choice(["bf16", "bf16", "f16"]), "kv_heads": kv, "seqs": _log_int(rng, 1, 64),
            "ragged": rng.random() < 0.6}
    if op == "append":
        case.update(page=rng.choice([16, 32, 64, 128, 256]), have=_log_int(rng, 1, 20000), add=_log_int(rng, 1, VIEW))
        while case["seqs"] * (case["have"] + case["add"]) * kv > 8 * 20001 * 16:
            case["seqs"] -= 1
            case["have"] = 1 + case["have"] // 2
        return case
    k = _log_int(rng, 1, 8 * VIEW)
    q = k
    case["causal"] = rng.random() < 0.5
    if op == "paged":
        k = _log_int(rng, 16, 32 * VIEW)
        q = min(k, rng.choice([1, 1, _log_int(rng, 2, VIEW)]))
        case["page"] = rng.choice([16, 32, 64, 128, 256])
    elif op == "attn" and rng.random() < 0.2:
        q = 1
    most = PAIRS // (3 if op == "paged" else 1)
    while case["seqs"] * q * k * heads > most or case["seqs"] * k * kv > 8 * 32 * VIEW * 16:
        if case["seqs"] > 1:
            case["seqs"] -= 1
        else:
            q, k = (q + 1) // 2, (k + 1) // 2
    case.update(heads=heads, q_len=q, k_len=k, prefix=case["causal"] and rng.random() < 0.4,
                cap=rng.choice([0.0, 0.0, 20.0, 50.0]), slopes=rng.random() < 0.25)
    return case


# ---- sizes ---------------------------------------------------------------------------------
def _spread(case, what, n, top):
    """n lengths up to top: all of them, or the first and others anywhere below on a log scale."""
    if not case["ragged"]:
        return [top] * n
    rng = random.Random("%s %d %d" % (what, n, top))
    return [top] + [min(top, _log_int(rng, max(1, top // 50), top)) for _ in range(n - 1)]


def _lengths(case):
    """Rows and keys of every sequence."""
    n = case["seqs"]
    ks = _spread(case, "keys", n, case["k_len"])
    if case["op"] != "paged" and case["q_len"] == case["k_len"]:
        return ks, ks
    if case["q_len"] == 1:
        return [1] * n, ks
    return [min(q, k) for q, k in zip(_spread(case, "rows", n, case["q_len"]), ks)], ks


def _prefixes(case):
    return [k // 3 for k in _lengths(case)[1]]


def _counts(case):
    """Tokens that every sequence of append has and gets."""
    n = case["seqs"]
    return _spread(case, "have", n, case["have"]), _spread(case, "add", n, case["add"])


def _seen(case):
    """Keys that all rows of every sequence see, added up."""
    out = []
    for q, k, p in zip(*_lengths(case), _prefixes(case)):
        if not case["causal"]:
            out.append(q * k)
            continue
        p = p if case["prefix"] else 0
        first, at = k - q + 1, max(0, min(q, p - (k - q + 1)))  # rows whose own position is inside the prefix
        out.append(at * p + (q - at) * (first + at + k) // 2)
    return out


def work(case):
    kv = case["kv_heads"] * 128  # bytes of the heads of K of one token
    if case["op"] == "append":
        have, add = _counts(case)
        return {"bytes": 4 * kv * sum(add) + 8 * sum(add) + 16 * case["seqs"], "flops": 0.0}
    qs, ks = _lengths(case)
    rows, keys, pairs = sum(qs), sum(ks), sum(_seen(case)) * case["heads"]
    q, k = rows * case["heads"] * 128, keys * kv
    if case["op"] == "attn_bwd":
        return {"bytes": 4 * q + 4 * k + 4 * rows * case["heads"], "flops": 640.0 * pairs}
    return {"bytes": 2 * q + 2 * k + 4 * rows * case["heads"], "flops": 256.0 * pairs}


# ---- inputs --------------------------------------------------------------------------------
def _starts(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return s


def _int32(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _heads(g, n, h, kind):
    return torch.randn(n, h, 64, generator=g, device="cuda").to(kind)


def _tables(g, tokens, room, page):
    """Pages of every sequence, in any order over the cache, and the pages that are left."""
    need = [-(-t // page) for t in tokens]
    ids = torch.randperm(sum(need) + room, generator=g, device="cuda").int()
    starts = _starts(need)
    return [ids[a:b] for a, b in zip(starts, starts[1:])], ids[starts[-1]:]


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, hk = TYPES[case["type"]], case["kv_heads"]
    s = {}
    if case["op"] == "append":
        have, add = _counts(case)
        page = case["page"]
        room = sum(-(-(a + b) // page) - -(-a // page) for a, b in zip(have, add)) + 3
        held, s["free"] = _tables(g, have, room, page)
        s["table"] = torch.full((case["seqs"], max(-(-(a + b) // page) for a, b in zip(have, add)) + 2), -1,
                                dtype=torch.int32, device="cuda")
        for row, ids in zip(s["table"], held):
            row[:len(ids)] = ids
        pages = sum(map(len, held)) + room
        s["have"], s["add"], s["taken"] = _int32(have), _int32(add), _int32([1])
        s["k"], s["v"] = (_heads(g, sum(add), hk, kind) for _ in range(2))
        s["k_pages"], s["v_pages"] = (_heads(g, pages * page, hk, kind).view(pages, page, hk, 64) for _ in range(2))
        return s
    qs, ks = _lengths(case)
    s["q"] = (1.5 * torch.randn(sum(qs), case["heads"], 64, generator=g, device="cuda")).to(kind)
    s["q_start"], s["k_start"] = _int32(_starts(qs)), _int32(_starts(ks))
    s["prefix"] = _int32(_prefixes(case)) if case["prefix"] else None
    s["slopes"] = None
    if case["slopes"]:  # from strong to weak, other ones for other seeds
        h = torch.arange(case["heads"], device="cuda", dtype=torch.float32)
        s["slopes"] = torch.exp2(-8.0 * (h + torch.rand(1, generator=g, device="cuda")) / case["heads"])
    if case["op"] == "paged":
        page = case["page"]
        held, _ = _tables(g, ks, 5, page)
        s["table"] = torch.zeros(len(ks), max(map(len, held)) + 1, dtype=torch.int32, device="cuda")
        for row, ids in zip(s["table"], held):
            row[:len(ids)] = ids
        pages = sum(map(len, held)) + 5
        s["lens"] = _int32(ks)
        s["k_pages"], s["v_pages"] = (_heads(g, pages * page, hk, kind).view(pages, page, hk, 64) for _ in range(2))
        return s
    s["k"], s["v"] = (_heads(g, sum(ks), hk, kind) for _ in range(2))
    if case["op"] == "attn_bwd":
        s["do"] = 0.1 * _heads(g, sum(qs), case["heads"], kind)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "append":
        n = case["seqs"]
        s["lens"], s["q_start"], s["taken_out"] = (torch.empty(m, dtype=torch.int32, device="cuda") for m in (n, n + 1, 1))
        s["slots"], s["pos"] = torch.empty(2, s["k"].shape[0], dtype=torch.int32, device="cuda").unbind()
    else:
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(case["heads"], s["q"].shape[0], device="cuda")
        if case["op"] == "attn_bwd":
            s.update({"d" + n: torch.empty_like(s[n]) for n in "qkv"})
            # what the forward pass saved
            o, s["lse"] = _forward(s, lambda b: _packed(s, b))
            s["o"] = o.to(s["q"].dtype)
    if own:  # the workspace that a program keeps
        import paper_2609_35593_gb300 as ress
        need = 256
        if case["op"] != "append":
            need = ress.attn_workspace_bytes(s["q"].shape[0], case["heads"], backward=case["op"] == "attn_bwd")
        s["ws"] = torch.zeros(need, dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2609_35593_gb300 as ress
    case = s["case"]
    if case["op"] == "append":
        ress.cache_tables(s["have"], s["add"], s["free"], s["taken"], s["table"], case["page"], s["lens"], s["q_start"],
                          s["slots"], s["pos"], s["taken_out"], s["ws"])
        ress.cache_write(s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"], s["ws"])
        return {n: s[n] for n in ("table", "lens", "q_start", "slots", "pos", "taken_out", "k_pages", "v_pages")}
    mask = {"causal": case["causal"], "prefix": s["prefix"], "cap": case["cap"], "slopes": s["slopes"]}
    if case["op"] == "attn":
        ress.attn(s["q"], s["k"], s["v"], s["o"], s["ws"], s["q_start"], s["k_start"], lse=s["lse"], **mask)
    elif case["op"] == "paged":
        ress.paged_attn(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["o"], s["ws"], s["q_start"],
                        lse=s["lse"], **mask)
    else:
        ress.attn_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["dq"], s["dk"], s["dv"], s["ws"], s["q_start"],
                      s["k_start"], **mask)
        return {n: s[n] for n in ("dq", "dk", "dv")}
    return {"o": s["o"], "lse": s["lse"]}


def _packed(s, b):
    """Heads of K and of V of sequence b in float32, [kv_heads, keys, 64]."""
    ks = _starts(_lengths(s["case"])[1])
    return [s[n][ks[b]:ks[b + 1]].float().transpose(0, 1) for n in "kv"]


def _gathered(s, b):
    """The same from the pages."""
    n = _lengths(s["case"])[1][b]
    ids = s["table"][b, :-(-n // s["case"]["page"])].long()
    return [s[c][ids].flatten(0, 1)[:n].float().transpose(0, 1) for c in ("k_pages", "v_pages")]


def _blocks(case):
    """Sequences and ranges of their rows, few enough for their scores to stay small, with what they see."""
    qs, ks = _lengths(case)
    starts = _starts(qs)
    for b, (q, k) in enumerate(zip(qs, ks)):
        step = max(1, (1 << 29) // (case["heads"] * k))
        for r in range(0, q, step):
            yield b, starts[b] + r, starts[b] + min(q, r + step), k - q + r


def _scores(s, b, q, k, at):
    """Scores [kv_heads, group, rows, keys] of rows q [rows, heads, 64] from position `at` on keys k
    [kv_heads, keys, 64], -inf where a row does not see a key, and the cap's slope (or 1)."""
    case = s["case"]
    hk, n = k.shape[:2]
    q = q.float().view(q.shape[0], hk, -1, 64).permute(1, 2, 0, 3)
    x = torch.matmul(q, k[:, None].transpose(2, 3)) * 0.125
    slope = 1.0
    if case["cap"]:
        t = torch.tanh(x / case["cap"])
        x, slope = case["cap"] * t, 1.0 - t * t
    row, key = at + torch.arange(q.shape[2], device="cuda")[:, None], torch.arange(n, device="cuda")
    if s["slopes"] is not None:
        x = x - s["slopes"].view(hk, -1, 1, 1) * (row - key).abs()
    if case["causal"]:
        seen = key <= row
        if s["prefix"] is not None:
            seen = seen | (key < s["prefix"][b])
        x = x.masked_fill(~seen, -math.inf)
    return q, x, slope


def _forward(s, keys):
    """Attention in float32 and the logarithm of each row's sum."""
    o, lse = torch.empty(s["q"].shape, device="cuda"), torch.empty(s["lse"].shape, device="cuda")
    last = None
    for b, r0, r1, at in _blocks(s["case"]):
        if b != last:
            (k, v), last = keys(b), b
        _, x, _ = _scores(s, b, s["q"][r0:r1], k, at)
        top = x.amax(3, keepdim=True)
        p = torch.exp(x - top)
        total = p.sum(3, keepdim=True)
        o[r0:r1] = torch.matmul(p / total, v[:, None]).permute(2, 0, 1, 3).flatten(1, 2)
        lse[:, r0:r1] = (top + torch.log(total)).flatten(0, 1)[..., 0]
    return o, lse


def _backward(s):
    grads = {n: torch.zeros(s[n].shape, device="cuda") for n in "qkv"}
    ks, last = _starts(_lengths(s["case"])[1]), None
    for b, r0, r1, at in _blocks(s["case"]):
        if b != last:
            (k, v), last = _packed(s, b), b
        q, x, slope = _scores(s, b, s["q"][r0:r1], k, at)
        p = torch.exp(x - s["lse"][:, r0:r1].view(*x.shape[:3], 1))
        do = s["do"][r0:r1].float().view(r1 - r0, k.shape[0], -1, 64).permute(1, 2, 0, 3)
        o = s["o"][r0:r1].float().view(r1 - r0, k.shape[0], -1, 64).permute(1, 2, 0, 3)
        ds = p * (torch.matmul(do, v[:, None].transpose(2, 3)) - (do * o).sum(3, keepdim=True)) * slope * 0.125
        grads["q"][r0:r1] = torch.matmul(ds, k[:, None]).permute(2, 0, 1, 3).flatten(1, 2)
        for n, w, y in (("k", ds, q), ("v", p, do)):
            grads[n][ks[b]:ks[b + 1]] += torch.matmul(w.transpose(2, 3), y).sum(1).transpose(0, 1)
    return grads


def _append(s):
    """The next tokens' pages, from the free ones in order, and their keys and values written there."""
    page, have, add = s["case"]["page"], s["have"].long(), s["add"].long()
    held, lens = (have + page - 1) // page, have + add
    new = (lens + page - 1) // page - held
    start, first = add.cumsum(0) - add, s["taken"] + new.cumsum(0) - new
    token = torch.arange(s["k"].shape[0], device="cuda")
    seq = torch.repeat_interleave(torch.arange(len(add), device="cuda"), add, output_size=len(token))
    pos = have[seq] + token - start[seq]
    col = pos // page
    fresh = col >= held[seq]
    ids = torch.where(fresh, s["free"][torch.where(fresh, first[seq] + col - held[seq], 0)], s["table"][seq, col])
    s["table"][seq, col] = ids
    slots = ids * page + pos % page
    for n in "kv":
        s[n + "_pages"].flatten(0, 1)[slots.long()] = s[n]
    q_start = torch.cat([start, start[-1:] + add[-1:]])
    return {"table": s["table"], "lens": lens.int(), "q_start": q_start.int(), "slots": slots.int(), "pos": pos.int(),
            "taken_out": s["taken"] + new.sum().int(), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain(s):
    op, kind = s["case"]["op"], TYPES[s["case"]["type"]]
    if op == "append":
        return _append(s)
    if op == "attn_bwd":
        return {"d" + n: g.to(kind) for n, g in _backward(s).items()}
    o, lse = _forward(s, (lambda b: _gathered(s, b)) if op == "paged" else (lambda b: _packed(s, b)))
    return {"o": o.to(kind), "lse": lse}


# ---- the same in float64 -------------------------------------------------------------------
def _exact_head(case, q, k, limit, slope):
    """Scores of one head in float64, rows [n, 64] on keys [m, 64], row i seeing keys below limit[i] and
    standing at position m - n + i; and the cap's slope."""
    x = torch.einsum("ic,jc->ij", q, k) / 8.0
    factor = torch.ones_like(x)
    if case["cap"]:
        x = case["cap"] * torch.tanh(x / case["cap"])
        factor = 1.0 - (x / case["cap"]) ** 2
    n, m = x.shape
    key = torch.arange(m, device="cuda", dtype=torch.float64)
    place = key[m - n:] if n <= m else torch.arange(m - n, m, device="cuda", dtype=torch.float64)
    if slope is not None:
        x -= slope.double() * (place[:, None] - key[None]).abs()
    x[key[None] >= limit[:, None]] = -math.inf
    return x, factor


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "append":
        return _exact_append(case, s)
    qs, ks = _lengths(case)
    bwd = case["op"] == "attn_bwd"
    if bwd:
        s = prepare(case, seed)  # with the output and the sums that it is given
    group = case["heads"] // case["kv_heads"]
    out = {"d" + n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in "qkv"} if bwd else {
        "o": torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"),
        "lse": torch.zeros(case["heads"], s["q"].shape[0], dtype=torch.float64, device="cuda")}
    q0 = k0 = 0
    for b, (nq, nk) in enumerate(zip(qs, ks)):
        rows, keys = slice(q0, q0 + nq), slice(k0, k0 + nk)
        q0, k0 = q0 + nq, k0 + nk
        limit = torch.full((nq,), float(nk), dtype=torch.float64, device="cuda")
        if case["causal"]:
            limit = torch.arange(nk - nq + 1, nk + 1, device="cuda", dtype=torch.float64)
            if s["prefix"] is not None:
                limit = limit.clamp(min=float(s["prefix"][b]))
        if case["op"] == "paged":
            where = torch.arange(nk, device="cuda")
            where = s["table"][b].long()[where // case["page"]], where % case["page"]
            kb, vb = s["k_pages"][where], s["v_pages"][where]
        else:
            kb, vb = s["k"][keys], s["v"][keys]
        for h in range(case["heads"]):
            q, k, v = (t.double() for t in (s["q"][rows, h], kb[:, h // group], vb[:, h // group]))
            x, factor = _exact_head(case, q, k, limit, None if s["slopes"] is None else s["slopes"][h])
            if not bwd:
                out["lse"][h, rows] = torch.logsumexp(x, 1)
                out["o"][rows, h] = torch.softmax(x, 1) @ v
                continue
            p = torch.exp(x - s["lse"][h, rows].double()[:, None])
            do, o = s["do"][rows, h].double(), s["o"][rows, h].double()
            ds = p * (do @ v.T - (do * o).sum(1)[:, None]) * factor / 8.0
            out["dq"][rows, h] = ds @ k
            out["dk"][keys, h // group] += ds.T @ q
            out["dv"][keys, h // group] += p.T @ do
    return out


def _exact_append(case, s):
    have, add = _counts(case)
    page, free = case["page"], s["free"].tolist()
    table, taken = s["table"].tolist(), int(s["taken"])
    slots, pos, q_start = [], [], [0]
    for row, h, a in zip(table, have, add):
        for p in range(h, h + a):
            if p % page == 0:
                row[p // page] = free[taken]
                taken += 1
            slots.append(row[p // page] * page + p % page)
            pos.append(p)
        q_start.append(len(slots))
    out = {"table": _int32(table), "lens": _int32([h + a for h, a in zip(have, add)]), "q_start": _int32(q_start),
           "slots": _int32(slots), "pos": _int32(pos), "taken_out": _int32([taken])}
    for n in ("k", "v"):
        cache = s[n + "_pages"].double().flatten(0, 1)
        cache[torch.tensor(slots, device="cuda")] = s[n].double()
        out[n + "_pages"] = cache.view(s[n + "_pages"].shape)
    return out

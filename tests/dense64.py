"""Dense attention of packed sequences and its gradient in float64, from the definition, with bounds on what
kernels that round where they say may be off by.

Bounds.  u: half a step of the tensors' 16-bit type, relative (bf16 2^-8, f16 2^-11).  A score is 64 exact products
summed in float32 (each addition off by at most 2^-23 of the terms' sizes, truncation included) and goes through
an fma and a base-2 exponential (2^-22): the exponent is off by at most
    d = 2^-17 sum|q k| / 8 + 2^-21 (1 + |s| + |lse|)
(with a cap, tanh adds 2^-20 cap) and a probability by 2 d of itself.  It is rounded to 16 bits (u; in f16 a
subnormal by 2^-25 of the row's largest), as is the result (u).  With A = sum p |v| a result is off by at most
    u |o| + (u + 2 d) A + 2^-25 sum|v| (f16)                      and lse by d + 2^-22 (1 + |lse|).
"""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def starts(lengths, device="cuda"):
    return torch.tensor([0] + list(lengths), device=device).cumsum(0).int()


def scores(q, k, causal, prefix, cap, slopes):
    """s [heads, nq, nk], what is seen, the slope of the cap, and the sizes sum|q k| / 8; q [nq, heads, 64] and k
    [nk, kv_heads, 64] in float64."""
    nq, nk = q.shape[0], k.shape[0]
    k = k.repeat_interleave(q.shape[1] // k.shape[1], 1)
    x = torch.einsum("ihc,jhc->hij", q, k) / 8
    size = torch.einsum("ihc,jhc->hij", q.abs(), k.abs()) / 8
    factor = torch.ones_like(x)
    if cap:
        t = torch.tanh(x / cap)
        x, factor = cap * t, 1 - t * t
    row = torch.arange(nk - nq, nk, device=q.device)[:, None]
    key = torch.arange(nk, device=q.device)[None]
    if slopes is not None:
        x = x - slopes.double()[:, None, None] * (row - key).abs()
    seen = torch.ones(nq, nk, dtype=torch.bool, device=q.device)
    if causal:
        seen = (key <= row) | (key < prefix)
    return x, seen, factor, size


def attention(q, k, v, q_lens, k_lens, causal=False, prefix=None, cap=0.0, slopes=None):
    """o, lse and their bounds; sequences one after another."""
    kind = q.dtype
    u = HALF_STEP[kind]
    q, k, v = q.double(), k.double(), v.double()
    o, lse = torch.zeros_like(q), torch.full((q.shape[1], q.shape[0]), -math.inf, dtype=torch.float64, device=q.device)
    o_off, lse_off = torch.zeros_like(o), torch.zeros_like(lse)
    a = b = 0
    for i, (nq, nk) in enumerate(zip(q_lens, k_lens)):
        if nq and nk:
            rows, vs = slice(a, a + nq), v[b:b + nk].repeat_interleave(q.shape[1] // k.shape[1], 1)
            s, seen, _, size = scores(q[rows], k[b:b + nk], causal, int(prefix[i]) if prefix is not None else 0, cap, slopes)
            x = s.masked_fill(~seen, -math.inf)
            z = torch.logsumexp(x, 2)
            p = torch.exp(x - z[..., None]).nan_to_num(0.0)
            o[rows] = torch.einsum("hij,jhc->ihc", p, vs)
            d = (2.0 ** -17 * size + 2.0 ** -21 * (1 + s.abs() + z.abs()[..., None].nan_to_num(0, 0, 0)) + 2.0 ** -20 * cap)
            d = d.masked_fill(~seen, 0).amax(2)
            big = torch.einsum("hij,jhc->ihc", p, vs.abs())
            o_off[rows] = u * o[rows].abs() + (u + 2 * d.T[..., None]) * big
            if kind == torch.float16:
                o_off[rows] += 2.0 ** -25 * vs.abs().sum(0) + 2.0 ** -25
            lse[:, rows] = z
            lse_off[:, rows] = d + 2.0 ** -22 * (1 + z.abs())
        a, b = a + nq, b + nk
    return o, lse, o_off, lse_off


def gradients(do, q, k, v, o, lse, q_lens, k_lens, causal=False, prefix=None, cap=0.0, slopes=None):
    """dq, dk, dv with the rows' o and lse as given, and their bounds.  A probability is off by 2 d of itself as above,
    dp - delta by e = 2^-17 (sum|do v| + sum|o do|); ds = p (dp - delta) c is rounded to 16 bits (u) like p.  (In f16 p is
    kept times 2^8 and ds times 1 / (its power of two, at least max|do| / 2): subnormals are off by 2^-33 and 2^-25 max|do|.)  Each sum
    is rounded once more."""
    kind = q.dtype
    u, f16 = HALF_STEP[kind], kind == torch.float16
    top = do.double().abs().max().item() if do.numel() else 0.0
    do, q, k, v, o, lse = (t.double() for t in (do, q, k, v, o, lse))
    n = q.shape[1] // k.shape[1]
    out = [torch.zeros_like(t) for t in (q, k, v)]
    off = [torch.zeros_like(t) for t in (q, k, v)]
    a = b = 0
    for i, (nq, nk) in enumerate(zip(q_lens, k_lens)):
        if nq and nk:
            rows, keys = slice(a, a + nq), slice(b, b + nk)
            ks, vs = k[keys].repeat_interleave(n, 1), v[keys].repeat_interleave(n, 1)
            s, seen, c, size = scores(q[rows], k[keys], causal, int(prefix[i]) if prefix is not None else 0, cap, slopes)
            z = lse[:, rows, None].nan_to_num(0, 0, 0)
            p = torch.exp(s - z).masked_fill(~seen, 0)
            d = 2.0 ** -17 * size + 2.0 ** -21 * (1 + s.abs() + z.abs()) + 2.0 ** -20 * cap
            dp = torch.einsum("ihc,jhc->hij", do[rows], vs)
            delta = (do[rows] * o[rows]).sum(2).T[..., None]
            e = 2.0 ** -17 * (torch.einsum("ihc,jhc->hij", do[rows].abs(), vs.abs())
                              + (do[rows] * o[rows]).abs().sum(2).T[..., None])
            ds = p * (dp - delta) * c
            # of the cap's slope: 2 t dt, dt at most 2^-20
            ds_off = (u + 2 * d) * ds.abs() + p * (e * c + (dp - delta).abs() * (2.0 ** -19 if cap else 0)) + (2.0 ** -25 * top if f16 else 0) * seen
            p_off = (u + 2 * d) * p + (2.0 ** -33 if f16 else 0) * seen
            out[0][rows] = torch.einsum("hij,jhc->ihc", ds, ks) / 8
            off[0][rows] = torch.einsum("hij,jhc->ihc", ds_off, ks.abs()) / 8
            fold = lambda t: t.unflatten(1, (-1, n)).sum(2)
            out[1][keys] = fold(torch.einsum("hij,ihc->jhc", ds, q[rows])) / 8
            off[1][keys] = fold(torch.einsum("hij,ihc->jhc", ds_off, q[rows].abs())) / 8
            out[2][keys] = fold(torch.einsum("hij,ihc->jhc", p, do[rows]))
            off[2][keys] = fold(torch.einsum("hij,ihc->jhc", p_off, do[rows].abs()))
        a, b = a + nq, b + nk
    # sums in float32, rounded to 16 bits
    off = [f + u * g.abs() + (2.0 ** -25 if f16 else 0) for f, g in zip(off, out)]
    return out, off


def close(got, want, off, what=""):
    """Within the bound everywhere; infinities in the same places.  Exponentials below float32's smallest normal number
    are 0 (2^-126 each); fewer than 2^13 of them times values below 2^13 are summed here: 2^-100."""
    got, off = got.double(), off + 2.0 ** -100
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), finite), what
    assert torch.equal(got[~finite], want[~finite]), what
    worst = ((got - want).abs()[finite] / off[finite]).max().item() if finite.any() else 0.0
    bad = (got - want).abs()[finite] > off[finite]
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} values, worst {worst:.3g} of the bound"

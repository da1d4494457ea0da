"""Gradients of dense attention in float64 with the bounds of dense64, but for two that are told from nearer:

Slope of the cap.  c = 1 - t^2, t = tanh(x / cap), is formed as 4 e r^2 with e = 2^(2 log2(e) x / cap), r = 1 / (1 + e), or
as 1 - t^2 where |t| is below 0.47 and nothing cancels.  x is off by at most 2^-17 sum|q k| / 8, which moves ln c by 2 / cap of
it; the exponent's rounding moves e by 2^-22 |x| / cap of itself, and the exponential, the addition, the reciprocal and three
products by less than 2^-20:   c is off by (2^-16 size / cap + 2^-20 (1 + |x| / cap)) c.

Steps of ds in f16.  |dp - delta| is at most B = 2 |dO| max|V| (norms over the 64 channels: o is a mean of rows of V), and the power
of two that ds is kept times brings B to 2^14..2^15: half a step of a subnormal, 2^-25, is 2^-39 B.  max|V| is that of the
sequence's keys; |dO| in dq that of the row, in dk the largest of the sequence's rows, both of the head of K.
"""
import torch

from dense64 import HALF_STEP, scores


def gradients(do, q, k, v, o, lse, q_lens, k_lens, causal=False, prefix=None, cap=0.0, slopes=None):
    kind = q.dtype
    u, f16 = HALF_STEP[kind], kind == torch.float16
    do, q, k, v, o, lse = (t.double() for t in (do, q, k, v, o, lse))
    n = q.shape[1] // k.shape[1]
    out = [torch.zeros_like(t) for t in (q, k, v)]
    off = [torch.zeros_like(t) for t in (q, k, v)]
    fold = lambda t: t.unflatten(1, (-1, n)).sum(2)
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
            c_off = 0.0
            if cap:
                x = torch.einsum("ihc,jhc->hij", q[rows], ks).abs() / 8
                c = 1 / torch.cosh(x / cap) ** 2  # (1 - tanh^2 of float64 cancels as well)
                c_off = 2.0 ** -16 * size / cap + 2.0 ** -20 * (1 + x / cap)
            ds = p * (dp - delta) * c
            ds_off = (u + 2 * d + c_off) * ds.abs() + p * e * c
            p_off = (u + 2 * d) * p + (2.0 ** -33 if f16 else 0) * seen
            # B of each row, [heads, rows, 1], and the largest of the heads that share one of K
            big = 2 * do[rows].norm(dim=2).T[..., None] * vs.norm(dim=2).amax(0)[:, None, None]
            most = big.amax(1, keepdim=True).unflatten(0, (-1, n)).amax(1).repeat_interleave(n, 0)
            row_step, key_step = (2.0 ** -39 * t * seen if f16 else 0 for t in (big, most))
            out[0][rows] = torch.einsum("hij,jhc->ihc", ds, ks) / 8
            off[0][rows] = torch.einsum("hij,jhc->ihc", ds_off + row_step, ks.abs()) / 8
            out[1][keys] = fold(torch.einsum("hij,ihc->jhc", ds, q[rows])) / 8
            off[1][keys] = fold(torch.einsum("hij,ihc->jhc", ds_off + key_step, q[rows].abs())) / 8
            out[2][keys] = fold(torch.einsum("hij,ihc->jhc", p, do[rows]))
            off[2][keys] = fold(torch.einsum("hij,ihc->jhc", p_off, do[rows].abs()))
        a, b = a + nq, b + nk
    return out, [f + u * g.abs() + (2.0 ** -25 if f16 else 0) for f, g in zip(off, out)]

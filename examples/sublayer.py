"""One global-attention sublayer of a 3D vision transformer, from the residual stream and back to it,
and head budgets calibrated from gradients.

    python examples/sublayer.py [--views 2] [--heads 4] [--sparsity 0.75]

Forward, all on this package's kernels:
    h = layer_norm(x)
    Q, K, V = projections of h; layer norm over the channels of each head of Q and K; rotary positions
              over the rows and columns of the patch grid (special tokens are not rotated)
    O = block-sparse attention, blocks selected by ReSS with the head budgets c_h
    y = x + O W_o^T
Calibration (the paper's Sec. 4.4 takes head budgets as given; Appendix D allots them by the Fisher
information of the heads' QKV projections, the squares of the gradients with respect to their outputs):
the gradient of a loss goes back through dense attention (attn, attn_bwd: O, its gradient and the
probabilities in bf16, as the sublayer itself holds them, sums in float32), then through the rotation and the
head norm (rope_bwd) to the projections' outputs, and on through the projections and layer_norm_bwd to the
residual stream, bf16 or float32, as a training step would take it.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_35593_gb300 as ress  # noqa: E402

PATCHES, SIDE, SPECIAL = 37 * 37, 37, 5  # tokens of one view


def positions(views, device="cuda"):
    """[tokens, 2] int32: row and column (from 1) of every patch, view after view, then the special tokens
    of all views at (0, 0), which turns nothing."""
    patch = torch.arange(PATCHES, device=device)
    grid = torch.stack([patch // SIDE + 1, patch % SIDE + 1], 1).repeat(views, 1)
    return torch.cat([grid, torch.zeros(views * SPECIAL, 2, dtype=grid.dtype, device=device)]).int().contiguous()


class Sublayer:
    """Weights and buffers of one sublayer on one scene size."""

    def __init__(self, views, heads, seed=0, eps=1e-5):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float32)
        self.views, self.H, self.N, self.eps = views, heads, views * (PATCHES + SPECIAL), eps
        dm = self.dm = 64 * heads
        self.norm = (1.0 + 0.1 * normal(dm), 0.1 * normal(dm))
        self.W = {n: (normal(dm, dm) / dm ** 0.5).bfloat16() for n in "qkv"}
        self.b = {n: (0.1 * normal(dm)).bfloat16() for n in "qkv"}
        self.head_norm = {n: (1.0 + 0.1 * normal(64), 0.1 * normal(64)) for n in "qk"}
        self.W_o = (0.02 * normal(dm, dm)).bfloat16()
        self.pos = positions(views)
        self.plan = ress.rope_plan((32, 32), base=100.0)
        self.d = ress.dims(self.N, heads, views * SPECIAL, dm)
        self.candidates = ress.num_candidates(self.d)
        empty = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="cuda")
        self.h, self.y = empty(self.N, dm), empty(self.N, dm)
        self.Q, self.K, self.V = (empty(self.N, heads, 64) for _ in range(3))
        self.raw = {n: empty(self.N, heads, 64) for n in "qkv"}
        self.mean, self.rstd = empty(self.N, dtype=torch.float32), empty(self.N, dtype=torch.float32)
        self.buf = None

    def inputs(self, x, ws):
        """Q, K and V of the residual stream x [N, d_model]; ws holds the projection's status afterwards."""
        W, b = self.W, self.b
        ress.layer_norm(x, *self.norm, self.h, eps=self.eps, mean=self.mean, rstd=self.rstd)
        ress.qkv_proj(self.d, self.h, W["q"], W["k"], W["v"], self.Q, self.K, self.V, ws, b_q=b["q"], b_k=b["k"],
                      b_v=b["v"], plan=self.plan, pos=self.pos, q_norm=self.head_norm["q"],
                      k_norm=self.head_norm["k"], eps=self.eps)

    def forward(self, x, c_h, rounds=3):
        """y = x + attention(x) with head budgets c_h (candidate key blocks kept per row)."""
        buf = self._buffers(c_h)
        self.inputs(x, buf.ws)
        ress.forward(self.d, self.Q, self.K, self.V, buf.F, list(c_h), rounds, 0.5, buf.ws, buf.row_ptr, buf.col_idx,
                     buf.O, buf.J_best)
        ress.out_proj(self.d, buf.O, self.W_o, x, self.y, buf.ws)
        ress.status(buf.ws)
        return self.y.clone()

    def _buffers(self, c_h):
        if self.buf is None or self.buf.c_h != list(c_h):
            self.buf = ress.Buffers(self.d, list(c_h))
            ress.prepare_wo(self.d, self.W_o, self.buf.F)
        return self.buf

    def gradients(self, x, dy):
        """Gradients of sum(dy y) for dense attention: of the residual stream, of the norms' parameters
        and of the outputs of the three projections."""
        W, ws = self.W, self._buffers([self.candidates] * self.H).ws
        self.inputs(x, ws)
        # the projections' outputs before norm and rotation, which the head norm's gradient reads
        ress.qkv_proj(self.d, self.h, W["q"], W["k"], W["v"], self.raw["q"], self.raw["k"], self.raw["v"], ws,
                      b_q=self.b["q"], b_k=self.b["k"], b_v=self.b["v"])
        ress.status(ws)
        O, dQ, dK, dV = (torch.empty_like(self.Q) for _ in range(4))
        lse = torch.empty(self.H, self.N, device="cuda", dtype=torch.float32)
        aws = torch.zeros(ress.attn_workspace_bytes(self.N, self.H, backward=True), dtype=torch.uint8, device="cuda")
        ress.attn(self.Q, self.K, self.V, O, aws, lse=lse)
        dO = (dy.float() @ self.W_o.float()).to(O.dtype).view(self.N, self.H, 64)
        ress.attn_bwd(dO, self.Q, self.K, self.V, O, lse, dQ, dK, dV, aws)
        ress.status(aws)
        dq, dk = torch.empty_like(dQ), torch.empty_like(dK)
        head = torch.empty(4, 64, device="cuda", dtype=torch.float32)
        rws = torch.empty(ress.rope_workspace_bytes(self.plan, self.N, self.H, self.H), dtype=torch.uint8, device="cuda")
        ress.rope_bwd(self.plan, self.pos, dQ, dq, dK, dk, q=self.raw["q"], k=self.raw["k"], q_norm=self.head_norm["q"],
                      k_norm=self.head_norm["k"], q_norm_grads=(head[0], head[1]), k_norm_grads=(head[2], head[3]),
                      eps=self.eps, ws=rws)
        dh = sum(d.reshape(self.N, self.dm) @ W[n] for d, n in ((dq, "q"), (dk, "k"), (dV, "v")))
        dx, dnorm = torch.empty_like(x), torch.empty(2, self.dm, device="cuda", dtype=torch.float32)
        nws = torch.empty(ress.layer_norm_workspace_bytes(self.N, self.dm), dtype=torch.uint8, device="cuda")
        ress.layer_norm_bwd(dh, x, self.norm[0], self.mean, self.rstd, dx, dweight=dnorm[0], dbias=dnorm[1], dres=dy,
                            ws=nws)
        return {"dx": dx, "norm": dnorm, "head_norm": head, "q": dq, "k": dk, "v": dV}


def head_budgets(grads, candidates, sparsity, low=0.25, high=2.0):
    """Candidate blocks kept by each head: shares by the trace of the Fisher information of the head's
    projections (squared gradients of their outputs), clipped to [low, high] of the mean."""
    trace = sum(grads[n].float().square().sum((0, 2)) for n in "qkv")
    share = trace / trace.mean()
    mean = (1.0 - sparsity) * candidates
    c = (share.clamp(low, high) * mean).round().clamp(2, candidates)
    return [int(v) for v in c.tolist()]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--views", type=int, default=2)
    ap.add_argument("--heads", type=int, default=4)
    ap.add_argument("--sparsity", type=float, default=0.75)
    a = ap.parse_args(argv)
    layer = Sublayer(a.views, a.heads)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(layer.N, layer.dm, generator=g, device="cuda", dtype=torch.float32).bfloat16()
    dy = (0.1 * torch.randn(layer.N, layer.dm, generator=g, device="cuda", dtype=torch.float32)).bfloat16()
    budgets = head_budgets(layer.gradients(x, dy), layer.candidates, a.sparsity)
    dense = layer.forward(x, [layer.candidates] * layer.H)
    sparse = layer.forward(x, budgets)
    change = (sparse.float() - dense.float()).norm() / (dense.float() - x.float()).norm()
    print(f"{layer.N} tokens, {layer.H} heads: {layer.candidates} candidate blocks, budgets {budgets}, "
          f"change of the sublayer's contribution {float(change):.3f}")
    return layer, budgets, float(change)


if __name__ == "__main__":
    main()

"""Performance cases of the operators that form Q, K and V out of the residual stream, and of their
gradients: what a user of this package calls before the attention of a layer, over the sizes it is
used at, each with its inputs, one pass of it, its work and its result in float64.

An operation is one of
  ln        layer norm of rows, with the statistics a backward pass needs
  ln_bwd    its gradients: of the input (with the residual branch's gradient added where there is
            one), of the weight and of the bias
  rope      rotary positions over several axes on the heads of Q and K, after a layer norm over each
            head's channels where the model has one
  rope_bwd  its gradients: of Q and K before the norm, of the norms' weights and biases
  qkv       the projection x W^T + b of a layer's input to Q, K and V with rope's norm and rotation

`own` False computes them from elementary torch operations in float32, rounded once at the end.

Sizes are those of 3D-ViT global attention: every view brings 37 x 37 patch tokens with a row and a
column and 5 special tokens without a position, the special tokens of all views last; heads have 64
channels; and generic ragged lengths.  Sequences of video have a time axis as well.
"""
import math

import numpy as np
import torch

own = False

PATCHES, SPECIAL, SIDE = 37 * 37, 5, 37  # tokens of one view
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5


def listed():
    rope = {"op": "rope", "type": "bf16", "heads": 16, "kv_heads": 16, "head_dim": 64, "axes": "32,32",
            "layout": "sections", "base": 100.0, "norm": True, "packed": False}
    return [
        # one camera token per view of a small scene, refined in a few small layers: latency
        {"op": "ln", "name": "ln_cameras", "rows": 8, "width": 1024, "type": "bf16", "out": "bf16", "params": "f32"},
        # a cropped sequence with a residual stream in float32 and a width that no vector divides
        {"op": "ln", "name": "ln_ragged_f32", "rows": 5003, "width": 1021, "type": "f32", "out": "bf16",
         "params": "f32"},
        # the residual stream of 32 images
        {"op": "ln", "name": "ln_v32", "rows": 32 * 1374, "width": 1024, "type": "bf16", "out": "bf16",
         "params": "bf16"},
        # fine-tuning a small model on a pair of images, in half precision
        {"op": "ln_bwd", "name": "ln_bwd_v2_f16", "rows": 2 * 1374, "width": 256, "type": "f16", "out": "f16",
         "params": "f32", "residual": False},
        # the gradient through the layer's first norm on 32 images, joined with the residual branch's
        {"op": "ln_bwd", "name": "ln_bwd_v32", "rows": 32 * 1374, "width": 1024, "type": "bf16", "out": "bf16",
         "params": "f32", "residual": True},
        # one token of each view: latency
        {**rope, "name": "rope_cameras", "tokens": 8, "special": 8},
        # Q and K of the 32-image layer: norm and positions on the patch grid
        {**rope, "name": "rope_v32", "tokens": 32 * 1374, "special": 32 * SPECIAL},
        # a video sequence in half precision: three axes, fewer heads for K, rows of a packed product
        {**rope, "name": "rope_video_packed", "type": "f16", "tokens": 20011, "special": 0, "heads": 12,
         "kv_heads": 4, "axes": "16,24,24", "layout": "halves", "base": 10000.0, "norm": False, "packed": True},
        # gradients of the 8-image layer (head budgets are calibrated with them)
        {**rope, "op": "rope_bwd", "name": "rope_bwd_v8", "tokens": 8 * 1374, "special": 8 * SPECIAL},
        # a cropped sequence in float32, neighbouring channels paired, half of them not rotated
        {**rope, "op": "rope_bwd", "name": "rope_bwd_ragged_f32", "type": "f32", "tokens": 5003, "special": 37,
         "heads": 3, "kv_heads": 3, "axes": "16,16", "layout": "interleaved"},
        # Q, K and V of one token per view
        {**rope, "op": "qkv", "name": "qkv_cameras", "tokens": 8, "special": 8, "d_model": 1024, "bias": True},
        # Q, K and V of the 32-image layer, the largest
        {**rope, "op": "qkv", "name": "qkv_v32", "tokens": 32 * 1374, "special": 32 * SPECIAL, "d_model": 1024,
         "bias": True},
    ]


def _log_int(rng, lo, hi):
    n = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    return n + (n == 3072)


def draw(rng):
    op = rng.choice(["ln", "ln", "ln_bwd", "ln_bwd", "rope", "rope", "rope_bwd", "rope_bwd", "qkv", "qkv"])
    kind = rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])
    if op in ("ln", "ln_bwd"):
        width = rng.choice([64, 192, 256, 768, 1024, 1024, 2048, _log_int(rng, 17, 5000)])
        case = {"op": op, "width": width, "type": kind, "out": rng.choice([kind, kind, "bf16"]),
                "params": rng.choice([kind, "f32"]), "rows": _log_int(rng, 1, 32 * 1374 * 1024 // width)}
        if case["out"] == "bf16" and kind == "f16":
            case["out"] = "f16"
        if op == "ln_bwd":
            case["residual"] = rng.choice([True, False])
        return case
    heads = rng.choice([3, 4, 8, 12, 16])
    case = {"op": op, "type": kind, "heads": heads, "kv_heads": heads, "head_dim": 64, "base": 100.0,
            "axes": "32,32", "layout": "sections", "norm": rng.choice([True, True, False]), "packed": False}
    if op != "qkv" and rng.random() < 0.4:  # other models' heads and positions
        case["head_dim"] = rng.choice([32, 64, 80, 128])
        case["axes"], case["layout"] = rng.choice(
            [("16,8,8", "sections"), ("8,12,12", "halves"), ("16,16", "halves"), ("8,12,12", "interleaved"),
             ("32", "halves"), ("10,6,14", "sections")])
        case["base"] = rng.choice([100.0, 10000.0])
        case["kv_heads"] = rng.choice([1, heads // 2, heads])
        case["packed"] = (heads + 2 * case["kv_heads"]) * case["head_dim"] != 3072 and rng.random() < 0.6
    row = (heads + case["kv_heads"]) * case["head_dim"]
    most = 32 * 1374 * 32 * 64 // row * 2 // BYTES[kind]
    if op == "qkv":
        case["type"], case["bias"] = "bf16", rng.choice([True, False])
        case["d_model"] = rng.choice([64 * heads, 64 * heads, 512, 768])
        most = min(200000, 32 * 1374 * 16 * 1024 // (heads * case["d_model"]))
    case["tokens"] = _log_int(rng, 1, most)
    case["special"] = rng.choice([0, case["tokens"] // 200, min(37, case["tokens"])])
    return case


# ---- sizes ---------------------------------------------------------------------------------
def _axes(case):
    return [int(a) for a in case["axes"].split(",")]


def work(case):
    op, t = case["op"], BYTES[case["type"]]
    if op in ("ln", "ln_bwd"):
        n, rows, width, o = case["rows"] * case["width"], case["rows"], case["width"], BYTES[case["out"]]
        if op == "ln":
            return {"bytes": n * (t + o) + 2 * width * BYTES[case["params"]] + 8 * rows, "flops": 8.0 * n}
        return {"bytes": n * (2 * t + o + (t if case["residual"] else 0)) + width * (BYTES[case["params"]] + 8) + 8 * rows,
                "flops": 14.0 * n}
    n, hd = case["tokens"], case["head_dim"]
    x = n * (case["heads"] + case["kv_heads"]) * hd
    positions, params = 4 * n * len(_axes(case)), 4 * 4 * hd if case["norm"] else 0
    if op == "rope":
        return {"bytes": 2 * x * t + positions + params, "flops": (11.0 if case["norm"] else 3.0) * x}
    if op == "rope_bwd":
        return {"bytes": (3 if case["norm"] else 2) * x * t + positions + (2 * params if case["norm"] else 0),
                "flops": (20.0 if case["norm"] else 3.0) * x}
    out, dm = 3 * 64 * case["heads"], case["d_model"]
    return {"bytes": 2 * (n * dm + out * dm + n * out + (out if case["bias"] else 0)) + positions + params,
            "flops": 2.0 * n * dm * out}


# ---- inputs --------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _positions(case, g):
    """[tokens, axes] int32: rows and columns (from 1) of the patches of one view after another, with
    a time step per view on the first of three axes; special tokens at the end, all zero."""
    n, axes = case["tokens"], len(_axes(case))
    patch = torch.arange(n - case["special"], device="cuda")
    view, at = patch // PATCHES, patch % PATCHES
    cols = [at // SIDE + 1, at % SIDE + 1]
    cols = [patch + 1] if axes == 1 else cols if axes == 2 else [view + 1, *cols]
    if axes == 1:  # a position in one long sequence, somewhere in it
        cols = [(patch + int(torch.randint(0, 64, (1,), generator=g, device="cuda"))) % 160]
    pos = torch.zeros(n, axes, dtype=torch.int32, device="cuda")
    pos[:n - case["special"]] = torch.stack(cols, 1).int()
    return pos


def _frequencies(case):
    """One per rotated pair, pairs of one axis after the other."""
    return [case["base"] ** (-2.0 * i / a) for a in _axes(case) for i in range(a // 2)]


def _pairs(case):
    """Axis, first and second channel of each rotated pair."""
    axis, lo, hi, start = [], [], [], 0
    for t, a in enumerate(_axes(case)):
        i = np.arange(a // 2)
        axis.append(np.full(a // 2, t))
        lo.append({"sections": start + i, "halves": start // 2 + i, "interleaved": start + 2 * i}[case["layout"]])
        hi.append({"sections": start + a // 2 + i, "halves": sum(_axes(case)) // 2 + start // 2 + i,
                   "interleaved": start + 2 * i + 1}[case["layout"]])
        start += a
    return [torch.from_numpy(np.concatenate(x)).cuda() for x in (axis, lo, hi)]


def _residual_stream(g, n, width):
    """Rows of the residual stream: an offset and a scale per channel, a few large channels."""
    scale = (0.5 * _normal(g, width)).exp()
    scale[torch.randint(0, width, (max(1, width // 128),), generator=g, device="cuda")] *= 8.0
    x = _normal(g, n, width)
    return x.mul_(scale).add_(0.5 * _normal(g, width))


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, kind = case["op"], TYPES[case["type"]]
    s = {}
    if op in ("ln", "ln_bwd"):
        n, w = case["rows"], case["width"]
        s["x"] = _residual_stream(g, n, w).to(kind)
        s["weight"] = (1.0 + 0.2 * _normal(g, w)).to(TYPES[case["params"]])
        s["bias"] = (0.1 * _normal(g, w)).to(TYPES[case["params"]])
        if op == "ln_bwd":
            s["dy"] = (0.1 * _normal(g, n, w)).to(TYPES[case["out"]])
            s["dres"] = (0.1 * _normal(g, n, w)).to(kind) if case["residual"] else None
            x = s["x"].float()  # what the forward pass saved
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + EPS)
        return s
    n, hq, hk, hd = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
    s["pos"] = _positions(case, g)
    for name in ("q", "k"):
        norm = case["norm"]
        s[name + "_weight"] = 1.0 + 0.2 * _normal(g, hd) if norm else None
        s[name + "_bias"] = 0.1 * _normal(g, hd) if norm else None
    if op == "qkv":
        dm = case["d_model"]
        s["x"] = _normal(g, n, dm).to(kind)
        for name in ("q", "k", "v"):
            s["W_" + name] = (_normal(g, hq * 64, dm) / math.sqrt(dm)).to(kind)
            s["b_" + name] = (0.1 * _normal(g, hq * 64)).to(kind) if case["bias"] else None
        return s
    if case["packed"]:  # rows of one product: the heads of Q, of K, of V
        rows = _normal(g, n, hq + 2 * hk, hd).to(kind)
        s["q"], s["k"] = rows[:, :hq], rows[:, hq:hq + hk]
    else:
        s["q"], s["k"] = _normal(g, n, hq, hd).to(kind), _normal(g, n, hk, hd).to(kind)
    if op == "rope_bwd":
        s["dq_out"], s["dk_out"] = (0.1 * _normal(g, n, h, hd).to(kind) for h in (hq, hk))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    s["case"] = case
    if op == "ln":
        s["y"] = torch.empty(s["x"].shape, dtype=TYPES[case["out"]], device="cuda")
        s["mean"], s["rstd"] = torch.empty(2, case["rows"], device="cuda").unbind()
    elif op == "ln_bwd":
        s["dx"] = torch.empty_like(s["x"])
        s["dweight"], s["dbias"] = torch.empty(2, case["width"], device="cuda").unbind()
    elif op == "qkv":
        s["Q"], s["K"], s["V"] = (torch.empty(case["tokens"], case["heads"], 64, dtype=torch.bfloat16, device="cuda")
                                  for _ in range(3))
    else:
        rows = {n: torch.empty(s[n].shape, dtype=s[n].dtype, device="cuda") for n in ("q", "k")}
        s["q_out"], s["k_out"] = rows["q"], rows["k"]  # or their gradients
        if op == "rope_bwd" and case["norm"]:
            s["grads"] = torch.empty(4, case["head_dim"], device="cuda").unbind()
    if op not in ("ln", "ln_bwd"):
        s["axis"], s["lo"], s["hi"] = _pairs(case)
        s["freq"] = torch.tensor(_frequencies(case), device="cuda", dtype=torch.float32)
    if own:  # the plan and the workspace that a program keeps
        import paper_2609_35593_gb300 as ress
        if op not in ("ln", "ln_bwd"):
            s["plan"] = ress.rope_plan(_axes(case), head_dim=case["head_dim"], base=case["base"], layout=case["layout"])
        need = 0
        if op == "ln_bwd":
            need = ress.layer_norm_workspace_bytes(case["rows"], case["width"])
        elif op == "rope_bwd":
            need = ress.rope_workspace_bytes(s["plan"], case["tokens"], case["heads"], case["kv_heads"])
        elif op == "qkv":
            s["dims"] = ress.dims(case["tokens"], case["heads"], 0, case["d_model"])
            need = ress.workspace_bytes(s["dims"])
        s["ws"] = torch.zeros(need, dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2609_35593_gb300 as ress
    case = s["case"]
    op = case["op"]
    if op == "ln":
        ress.layer_norm(s["x"], s["weight"], s["bias"], s["y"], eps=EPS, mean=s["mean"], rstd=s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "ln_bwd":
        ress.layer_norm_bwd(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], s["dx"], dweight=s["dweight"],
                            dbias=s["dbias"], dres=s["dres"], ws=s["ws"])
        return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    norms = {"q_norm": None, "k_norm": None}
    if case["norm"]:
        norms = {n + "_norm": (s[n + "_weight"], s[n + "_bias"]) for n in ("q", "k")}
    if op == "qkv":
        ress.qkv_proj(s["dims"], s["x"], s["W_q"], s["W_k"], s["W_v"], s["Q"], s["K"], s["V"], s["ws"], b_q=s["b_q"],
                      b_k=s["b_k"], b_v=s["b_v"], plan=s["plan"], pos=s["pos"], eps=EPS, **norms)
        return {"Q": s["Q"], "K": s["K"], "V": s["V"]}
    if op == "rope":
        ress.rope(s["plan"], s["pos"], s["q"], s["q_out"], s["k"], s["k_out"], eps=EPS, **norms)
        return {"q": s["q_out"], "k": s["k_out"]}
    out = {"dq": s["q_out"], "dk": s["k_out"]}
    grads = {}
    if case["norm"]:
        grads = {"q": s["q"], "k": s["k"], "q_norm_grads": s["grads"][:2], "k_norm_grads": s["grads"][2:]}
        out.update(zip(("dq_weight", "dq_bias", "dk_weight", "dk_bias"), s["grads"]))
    ress.rope_bwd(s["plan"], s["pos"], s["dq_out"], s["q_out"], s["dk_out"], s["k_out"], eps=EPS, ws=s["ws"], **norms,
                  **grads)
    return out


def _normalised(x):
    c = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(c.square().mean(-1, keepdim=True) + EPS)
    return c * r, r


def _rotated(s, x, sign):
    """The rotated pairs of x [tokens, heads, channels], other channels as they are."""
    angle = s["pos"].float()[:, s["axis"]] * s["freq"]
    cos, sin = angle.cos()[:, None], sign * angle.sin()[:, None]
    a, b = x[..., s["lo"]], x[..., s["hi"]]
    y = x.clone()
    y[..., s["lo"]] = a * cos - b * sin
    y[..., s["hi"]] = b * cos + a * sin
    return y


def _norm_grads(dy, xh, r, weight):
    """Gradients of xh weight + bias with respect to the input of the normalisation and to both."""
    g = dy * weight
    dx = r * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    other = tuple(range(dy.dim() - 1))
    return dx, (dy * xh).sum(other), dy.sum(other)


def _plain(s):
    case = s["case"]
    op, kind = case["op"], TYPES[case["type"]]
    if op == "ln":
        x = s["x"].float()
        mean = x.mean(1)
        c = x - mean[:, None]
        rstd = torch.rsqrt(c.square().mean(1) + EPS)
        y = c * rstd[:, None] * s["weight"].float() + s["bias"].float()
        return {"y": y.to(TYPES[case["out"]]), "mean": mean, "rstd": rstd}
    if op == "ln_bwd":
        r = s["rstd"][:, None]
        xh = (s["x"].float() - s["mean"][:, None]) * r
        dx, dw, db = _norm_grads(s["dy"].float(), xh, r, s["weight"].float())
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        return {"dx": dx.to(kind), "dweight": dw, "dbias": db}
    if op == "qkv":
        out, x = {}, s["x"].float()
        for n in ("q", "k", "v"):
            y = x @ s["W_" + n].float().T
            if case["bias"]:
                y = y + s["b_" + n].float()
            y = y.view(case["tokens"], case["heads"], 64)
            if n != "v":
                if case["norm"]:
                    y = _normalised(y)[0] * s[n + "_weight"] + s[n + "_bias"]
                y = _rotated(s, y, 1.0)
            out[n.upper()] = y.to(kind)
        return out
    out = {}
    for n in ("q", "k"):
        if op == "rope":
            x = s[n].float()
            if case["norm"]:
                x = _normalised(x)[0] * s[n + "_weight"] + s[n + "_bias"]
            out[n] = _rotated(s, x, 1.0).to(kind)
            continue
        dx = _rotated(s, s["d%s_out" % n].float(), -1.0)
        if case["norm"]:
            xh, r = _normalised(s[n].float())
            dx, out["d%s_weight" % n], out["d%s_bias" % n] = _norm_grads(dx, xh, r, s[n + "_weight"])
        out["d" + n] = dx.to(kind)
    return out


# ---- the same in float64 -------------------------------------------------------------------
def _rotations(case, pos):
    """Complex exp(i angle) of each token and pair, and the channels of each pair."""
    turns, first, second, start, axes = [], [], [], 0, _axes(case)
    for t, a in enumerate(axes):
        for i in range(a // 2):
            turns.append(pos[:, t].double() * case["base"] ** (-2.0 * i / a))
            if case["layout"] == "sections":
                pair = (start + i, start + a // 2 + i)
            elif case["layout"] == "halves":
                pair = (start // 2 + i, (sum(axes) + start) // 2 + i)
            else:
                pair = (start + 2 * i, start + 2 * i + 1)
            first.append(pair[0])
            second.append(pair[1])
        start += a
    angle = torch.stack(turns, 1)
    return torch.polar(torch.ones_like(angle), angle), first, second


def _turned(x, rot, first, second):
    """x with each pair of channels, as one complex number, times rot."""
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * rot[:, None]
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_norm(x, weight, bias):
    mean = x.mean(-1, keepdim=True)
    std = (x.var(-1, unbiased=False, keepdim=True) + EPS).sqrt()
    return (x - mean) / std * weight.double() + bias.double(), mean, std


def _exact_norm_back(x, dy, weight, mean, std):
    n = x.shape[-1]
    xh, g = (x - mean) / std, dy * weight.double()
    dx = (n * g - g.sum(-1, keepdim=True) - xh * (g * xh).sum(-1, keepdim=True)) / (n * std)
    return dx, (dy * xh).flatten(0, -2).sum(0), dy.flatten(0, -2).sum(0)


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "ln":
        y, mean, std = _exact_norm(s["x"].double(), s["weight"], s["bias"])
        return {"y": y, "mean": mean[:, 0], "rstd": 1.0 / std[:, 0]}
    if op == "ln_bwd":  # with the statistics that it is given
        dx, dw, db = _exact_norm_back(s["x"].double(), s["dy"].double(), s["weight"], s["mean"].double()[:, None],
                                      1.0 / s["rstd"].double()[:, None])
        return {"dx": dx if s["dres"] is None else dx + s["dres"].double(), "dweight": dw, "dbias": db}
    rot, first, second = _rotations(case, s["pos"])
    if op == "rope_bwd":
        out = {}
        for n in ("q", "k"):
            dx = _turned(s["d%s_out" % n].double(), rot.conj(), first, second)
            if case["norm"]:
                x = s[n].double()
                mean, std = _exact_norm(x, s[n + "_weight"], s[n + "_bias"])[1:]
                dx, out["d%s_weight" % n], out["d%s_bias" % n] = _exact_norm_back(x, dx, s[n + "_weight"], mean, std)
            out["d" + n] = dx
        return out
    out = {}
    for n in ("q", "k", "v") if op == "qkv" else ("q", "k"):
        if op == "qkv":
            x = s["x"].double() @ s["W_" + n].double().T
            x = (x + s["b_" + n].double() if case["bias"] else x).view(case["tokens"], case["heads"], 64)
        else:
            x = s[n].double()
        if n != "v":
            x = _exact_norm(x, s[n + "_weight"], s[n + "_bias"])[0] if case["norm"] else x
            x = _turned(x, rot, first, second)
        out[n.upper() if op == "qkv" else n] = x
    return out

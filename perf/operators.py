"""The operators of a gated feed-forward block in training and serving: what is timed, and their plain forms.

  glu_fwd    gated feed-forward: both projections, activation and product (bt_glu_fwd)
  glu_bwd    its gradients from the stored projections (bt_glu_bwd)
  norm_fwd   norm behind a block, gate, scaled residual sum and the norm before the next block (bt_block_norm_fwd)
  norm_bwd   its gradients (bt_block_norm_bwd)
  clip       gradient norm over many tensors, and clipping (bt_grad_clip_batch)

With `own` false, `run` computes them with elementary torch operations in 32 bits (sums over all gradients in 64); with
`own` true it makes the library's calls on buffers that a training program keeps.
"""
import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f64": torch.float64}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "f64": 8}

# the convolution weights of the VGG-16-shaped step and its linear head
VGG = [(64, 3, 3, 3), (64, 64, 3, 3), (128, 64, 3, 3), (128, 128, 3, 3), (256, 128, 3, 3), (256, 256, 3, 3), (256, 256, 3, 3),
       (512, 256, 3, 3), (512, 512, 3, 3), (512, 512, 3, 3), (512, 512, 3, 3), (512, 512, 3, 3), (512, 512, 3, 3), (1000, 512)]


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token through a feed-forward block: the weights are read once, launches count
        {"name": "glu_fwd_token_bf16", "kind": "glu_fwd", "dtype": "bf16", "rows": 1, "d": 2048, "ff": 8192, "act": "silu", "save": False},
        # a ragged batch in float16, sparse (ReLU) gate, projections kept for the backward pass
        {"name": "glu_fwd_ragged_f16", "kind": "glu_fwd", "dtype": "f16", "rows": 777, "d": 1000, "ff": 2728, "act": "relu", "save": True},
        # a training step's forward pass: the largest
        {"name": "glu_fwd_large_bf16", "kind": "glu_fwd", "dtype": "bf16", "rows": 8192, "d": 4096, "ff": 11264, "act": "silu", "save": True},
        # a small model in full precision
        {"name": "glu_fwd_small_f32", "kind": "glu_fwd", "dtype": "f32", "rows": 512, "d": 512, "ff": 1376, "act": "gelu", "save": True},
        # backward pass of a ragged batch, sparse gate
        {"name": "glu_bwd_ragged_f16", "kind": "glu_bwd", "dtype": "f16", "rows": 1021, "d": 1024, "ff": 2752, "act": "relu"},
        # backward pass of a training step
        {"name": "glu_bwd_large_bf16", "kind": "glu_bwd", "dtype": "bf16", "rows": 8192, "d": 2048, "ff": 8192, "act": "silu"},
        # one token between two blocks
        {"name": "norm_fwd_token_bf16", "kind": "norm_fwd", "dtype": "bf16", "rows": 1, "d": 2048, "groups": 0, "post": True},
        # a training step between two blocks, gate per channel
        {"name": "norm_fwd_large_bf16", "kind": "norm_fwd", "dtype": "bf16", "rows": 16384, "d": 4096, "groups": 1, "post": True},
        # six sequences with a gate of their own each, full precision, ragged width
        {"name": "norm_bwd_grouped_f32", "kind": "norm_bwd", "dtype": "f32", "rows": 6 * 333, "d": 1000, "groups": 6, "post": True},
        # backward pass of the training step's norms
        {"name": "norm_bwd_large_bf16", "kind": "norm_bwd", "dtype": "bf16", "rows": 16384, "d": 4096, "groups": 1, "post": True},
        # the gradients of the VGG-16-shaped step
        {"name": "clip_vgg_f32", "kind": "clip", "dtype": "f32", "shapes": "vgg", "layers": 0, "d": 0, "ff": 0},
        # the gradients of sixteen layers of a transformer with gated feed-forward blocks, and of its embedding
        {"name": "clip_blocks_bf16", "kind": "clip", "dtype": "bf16", "shapes": "blocks", "layers": 16, "d": 2048, "ff": 8192},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["glu_fwd", "glu_fwd", "glu_bwd", "norm_fwd", "norm_bwd", "clip"])
    if kind in ("glu_fwd", "glu_bwd"):
        d, ff = 8 * _log(rng, 32, 512), 8 * _log(rng, 64, 1408)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        # products at one order of magnitude less in full precision; a backward pass is two forward passes
        most = (4.0e11 if dtype != "f32" else 2.0e10) / (2 if kind == "glu_bwd" else 1)
        rows = _log(rng, 1 if kind == "glu_fwd" else 64, max(65, min(8192, int(most / (d * ff)))))
        case = {"kind": kind, "dtype": dtype, "rows": rows, "d": d, "ff": ff, "act": rng.choice(["relu", "silu", "gelu", "gelu_tanh"])}
        if kind == "glu_fwd":
            case["save"] = rng.random() < 0.7
        return case
    if kind in ("norm_fwd", "norm_bwd"):
        d = _log(rng, 64, 8192)
        if rng.random() < 0.7:
            d = (d + 7) // 8 * 8
        groups = rng.choice([0, 1, 1, 2, 5, 8])
        rows = _log(rng, 1, max(2, min(16384, (1 << 26) // d)))
        if groups > 1:
            rows = max(1, rows // groups) * groups
        return {"kind": kind, "dtype": rng.choice(["bf16", "f16", "f32"]), "rows": rows, "d": d, "groups": groups, "post": rng.random() < 0.8}
    return {"kind": "clip", "dtype": rng.choice(["bf16", "f32", "f16"]), "shapes": "blocks", "layers": rng.randrange(1, 13),
            "d": 8 * _log(rng, 8, 160) + rng.choice([0, 0, 4, 1]), "ff": 8 * _log(rng, 16, 512)}


def _shapes(case):
    if case["shapes"] == "vgg":
        return VGG
    d, ff = case["d"], case["ff"]
    layer = [(d, d)] * 4 + [(ff, d), (ff, d), (d, ff), (d,), (d,)]
    return [(32000, d)] + layer * case["layers"] + [(d,)]


def _elements(case):
    return sum(math.prod(s) for s in _shapes(case))


def work(case):
    kind, es = case["kind"], SIZE[case["dtype"]]
    if kind == "clip":
        n = _elements(case)
        # the norm and the product need every gradient once; it can be used for both only where it is still in the cache
        return {"bytes": 2 * n * es, "flops": 3 * n}
    rows, d = case["rows"], case["d"]
    if kind == "glu_fwd":
        ff = case["ff"]
        return {"bytes": es * (rows * d + 2 * ff * d + rows * ff * (3 if case["save"] else 1)), "flops": 4 * rows * d * ff}
    if kind == "glu_bwd":
        ff = case["ff"]
        return {"bytes": es * (3 * rows * ff + 2 * rows * d + 4 * ff * d), "flops": 8 * rows * d * ff}
    if kind == "norm_fwd":
        return {"bytes": es * (4 * rows * d + (1 + case["post"] + case["groups"]) * d), "flops": 12 * rows * d}
    return {"bytes": es * (6 * rows * d + 2 * (1 + case["post"] + case["groups"]) * d), "flops": 30 * rows * d}


# ---------------------------------------------------------------------------------------------- inputs
SCALE, EPS, MAX_NORM = 0.5, 1e-6, 1.0


def _normal(gen, shape, dtype, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * std + mean).to(DT[dtype])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 17)
    kind, dt = case["kind"], case["dtype"]
    s = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device="cuda"), "kept": {}}
    if kind == "clip":
        # gradients of layers differ in size by orders of magnitude
        shapes = _shapes(case)
        std = np.random.RandomState(int(seed) % (1 << 31)).uniform(-4, -2, len(shapes))
        s["grads"] = [_normal(gen, sh, dt, 10.0 ** v) for sh, v in zip(shapes, std)]
        # the clipped gradients lie one behind the other in the buffer that goes to the optimizer or to other ranks, each
        # from a 16-byte boundary on
        step = 16 // SIZE[dt]
        lengths = [g.numel() for g in s["grads"]]
        padded = [(n + step - 1) // step * step for n in lengths]
        s["clipped"] = torch.zeros(sum(padded), dtype=DT[dt], device="cuda")
        s["slots"] = [v[:n] for v, n in zip(s["clipped"].split(padded), lengths)]
        s["pads"] = [torch.zeros(p - n, dtype=DT[dt], device="cuda") for p, n in zip(padded, lengths)]
        s["norm"] = torch.empty(1, dtype=torch.float32, device="cuda")
        return s
    rows, d = case["rows"], case["d"]
    if kind in ("glu_fwd", "glu_bwd"):
        ff = case["ff"]
        s["x"] = _normal(gen, (rows, d), dt)
        s["w_gate"] = _normal(gen, (ff, d), dt, d ** -0.5)
        s["w_up"] = _normal(gen, (ff, d), dt, d ** -0.5)
        wide = lambda: torch.empty(rows, ff, dtype=DT[dt], device="cuda")  # noqa: E731
        if kind == "glu_fwd":
            s["out"] = [wide() for _ in range(3 if case["save"] else 1)]
        else:
            # as the forward pass stored them: a ReLU gate is zero where it is not positive
            g = _normal(gen, (rows, ff), dt)
            s["g"] = torch.clamp(g, min=0) if case["act"] == "relu" else g
            s["u"] = _normal(gen, (rows, ff), dt)
            s["grad_h"] = _normal(gen, (rows, ff), dt, 0.1)
            s["out"] = [torch.empty_like(s["x"]), torch.empty_like(s["w_gate"]), torch.empty_like(s["w_up"])]
        return s
    # hidden states with a common offset and a few channels that are much larger than the others
    wide = torch.ones(d, device="cuda")
    wide[::61] = 8.0
    s["x"] = (_normal(gen, (rows, d), "f32", 1.0, 0.1) * wide).to(DT[dt])
    s["f"] = (_normal(gen, (rows, d), "f32") * wide.flip(0)).to(DT[dt])
    s["w_pre"] = _normal(gen, (d,), dt, 0.1, 1.0)
    s["w_post"] = _normal(gen, (d,), dt, 0.1, 1.0) if case["post"] else None
    s["gate"] = _normal(gen, (case["groups"], d), dt, 0.3, 0.5) if case["groups"] else None
    if kind == "norm_fwd":
        s["out"] = [torch.empty_like(s["x"]), torch.empty_like(s["x"])]
    else:
        s["grad_n"] = _normal(gen, (rows, d), dt, 0.1)
        s["grad_x_out"] = _normal(gen, (rows, d), dt, 0.1)
        s["out"] = [torch.empty_like(s["x"]), torch.empty_like(s["f"])] + [
            None if s[k] is None else torch.empty_like(s[k]) for k in ("gate", "w_post", "w_pre")]
    return s


# ---------------------------------------------------------------------------------------------- the pass
def _act(g, act):
    """The activation and its derivative, in 32 bits."""
    if act == "relu":
        on = g > 0
        return g * on, on.to(g.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if act == "gelu":
        c = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * c, c + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    k, a = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(k * (g + a * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * a * g * g)


def _plain_glu_fwd(s):
    case, dt = s["case"], DT[s["case"]["dtype"]]
    x = s["x"].float()
    g, u = x @ s["w_gate"].float().T, x @ s["w_up"].float().T
    a, _ = _act(g, case["act"])
    h = (a * u).to(dt)
    if not case["save"]:
        return {"h": h}
    return {"h": h, "g": (a if case["act"] == "relu" else g).to(dt), "u": u.to(dt)}


def _plain_glu_bwd(s):
    case, dt = s["case"], DT[s["case"]["dtype"]]
    x, dh, u = s["x"].float(), s["grad_h"].float(), s["u"].float()
    a, da = _act(s["g"].float(), case["act"])
    dg, du = dh * u * da, dh * a
    dx = dg @ s["w_gate"].float() + du @ s["w_up"].float()
    return {"grad_x": dx.to(dt), "grad_w_gate": (dg.T @ x).to(dt), "grad_w_up": (du.T @ x).to(dt)}


def _rows_of(gate, rows):
    """The gate's rows, each repeated for the rows that share it."""
    return 1.0 if gate is None else gate.float().repeat_interleave(rows // gate.shape[0], dim=0)


def _rms(v):
    return torch.rsqrt((v * v).mean(dim=-1, keepdim=True) + EPS)


def _plain_norm_fwd(s):
    case, dt = s["case"], DT[s["case"]["dtype"]]
    x, f = s["x"].float(), s["f"].float()
    p = f if s["w_post"] is None else f * _rms(f) * s["w_post"].float()
    y = x + SCALE * (_rows_of(s["gate"], case["rows"]) * p)
    return {"x_out": y.to(dt), "n": (y * _rms(y) * s["w_pre"].float()).to(dt)}


def _plain_norm_bwd(s):
    case, dt = s["case"], DT[s["case"]["dtype"]]
    y, f, dn, dy = s["x"].float(), s["f"].float(), s["grad_n"].float(), s["grad_x_out"].float()
    r = _rms(y)
    yh, wn = y * r, dn * s["w_pre"].float()
    t = dy + r * (wn - yh * (wn * yh).mean(dim=-1, keepdim=True))
    out = {"grad_x": t.to(dt), "grad_w_pre": (dn * yh).sum(0).to(dt)}
    gate, e = _rows_of(s["gate"], case["rows"]), SCALE * t
    dp = e * gate
    if s["w_post"] is None:
        p, df = f, dp
    else:
        rf, w = _rms(f), s["w_post"].float()
        fh = f * rf
        p, wp = fh * w, dp * w
        df = rf * (wp - fh * (wp * fh).mean(dim=-1, keepdim=True))
        out["grad_w_post"] = (dp * fh).sum(0).to(dt)
    if s["gate"] is not None:
        out["grad_gate"] = (e * p).view(case["groups"], -1, case["d"]).sum(1).to(dt)
    out["grad_f"] = df.to(dt)
    return out


def _plain_clip(s):
    # 64 bits: gradients of very different sizes, a sum over all of them
    flat = torch.cat([v for g, pad in zip(s["grads"], s["pads"]) for v in (g.reshape(-1), pad)])
    norm = (flat.double() * flat.double()).sum().sqrt()
    c = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0).float()
    return {"norm": norm.float().view(1), "clipped": (flat.float() * c).to(flat.dtype)}


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"glu_fwd": _plain_glu_fwd, "glu_bwd": _plain_glu_bwd, "norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd,
                "clip": _plain_clip}[kind](s)
    return {"glu_fwd": _own_glu_fwd, "glu_bwd": _own_glu_bwd, "norm_fwd": _own_norm_fwd, "norm_bwd": _own_norm_bwd,
            "clip": _own_clip}[kind](s)


# ---- the library's calls; the workspace is made on the first pass and kept, as a training program keeps it
def _own_glu_fwd(s):
    from paper_2110_15362_b200 import binding as B
    case, ws = s["case"], s["kept"].get("ws")
    if ws is None:
        ws = s["kept"]["ws"] = B.new_glu_workspace(case["rows"], case["d"], case["ff"], DT[case["dtype"]])
    out = s["out"]
    h, g, u = out if case["save"] else (out[0], None, None)
    B.bt_glu_fwd(s["x"], s["w_gate"], s["w_up"], h, g, u, ws, s["status"], activation=case["act"])
    return {"h": h, "g": g, "u": u} if case["save"] else {"h": h}


def _own_glu_bwd(s):
    from paper_2110_15362_b200 import binding as B
    case, ws = s["case"], s["kept"].get("ws")
    if ws is None:
        ws = s["kept"]["ws"] = B.new_glu_workspace(case["rows"], case["d"], case["ff"], DT[case["dtype"]], backward=True)
    dx, dwg, dwu = s["out"]
    B.bt_glu_bwd(s["grad_h"], s["g"], s["u"], s["x"], s["w_gate"], s["w_up"], dx, dwg, dwu, ws, s["status"], activation=case["act"])
    return {"grad_x": dx, "grad_w_gate": dwg, "grad_w_up": dwu}


def _own_norm_fwd(s):
    from paper_2110_15362_b200 import binding as B
    y, n = s["out"]
    B.bt_block_norm_fwd(s["x"], s["f"], s["gate"], s["w_post"], s["w_pre"], y, n, scale=SCALE, eps=EPS)
    return {"x_out": y, "n": n}


def _own_norm_bwd(s):
    from paper_2110_15362_b200 import binding as B
    case, ws = s["case"], s["kept"].get("ws")
    if ws is None:
        ws = s["kept"]["ws"] = B.new_block_norm_workspace(case["rows"], case["d"], max(1, case["groups"]), DT[case["dtype"]])
    dx, df, dgate, dw_post, dw_pre = s["out"]
    B.bt_block_norm_bwd(s["x"], s["f"], s["gate"], s["w_post"], s["w_pre"], s["grad_n"], s["grad_x_out"], dx, df, dgate, dw_post,
                        dw_pre, ws, scale=SCALE, eps=EPS)
    out = {"grad_x": dx, "grad_w_pre": dw_pre}
    if dw_post is not None:
        out["grad_w_post"] = dw_post
    if dgate is not None:
        out["grad_gate"] = dgate
    out["grad_f"] = df
    return out


def _own_clip(s):
    from paper_2110_15362_b200 import binding as B
    items, ws = B.grad_items(s["grads"], s["slots"]), s["kept"].get("ws")
    if ws is None:
        ws = s["kept"]["ws"] = B.new_grad_workspace([g.numel() for g in s["grads"]])
    B.bt_grad_clip_batch(items, DT[s["case"]["dtype"]], MAX_NORM, s["norm"], ws)
    return {"norm": s["norm"], "clipped": s["clipped"]}


# ---------------------------------------------------------------------------------------------- 64 bits
_ACTS = {"relu": torch.nn.functional.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
         "gelu_tanh": lambda g: torch.nn.functional.gelu(g, approximate="tanh")}


def _normed(v, w):
    return v / torch.sqrt(torch.linalg.vecdot(v, v).unsqueeze(-1) / v.shape[-1] + EPS) * w


def _summed(x, f, gate, w_post):
    p = f if w_post is None else _normed(f, w_post)
    if gate is not None:
        p = (p.unflatten(0, (gate.shape[0], -1)) * gate.unsqueeze(1)).flatten(0, 1)
    return x + SCALE * p


def exact(case, seed):
    s = prepare(case, seed)
    d = lambda k: None if s[k] is None else s[k].double()  # noqa: E731
    kind = case["kind"]
    if kind == "glu_fwd":
        g, u = torch.nn.functional.linear(d("x"), d("w_gate")), torch.nn.functional.linear(d("x"), d("w_up"))
        h = _ACTS[case["act"]](g) * u
        return {"h": h, "g": torch.relu(g) if case["act"] == "relu" else g, "u": u} if case["save"] else {"h": h}
    if kind == "glu_bwd":
        g, u, x = d("g").requires_grad_(), d("u").requires_grad_(), d("x")
        dg, du = torch.autograd.grad(_ACTS[case["act"]](g) * u, (g, u), d("grad_h"))
        dx = torch.addmm(torch.mm(dg, d("w_gate")), du, d("w_up"))
        return {"grad_x": dx, "grad_w_gate": torch.einsum("rf,rd->fd", dg, x), "grad_w_up": torch.einsum("rf,rd->fd", du, x)}
    if kind == "norm_fwd":
        y = _summed(d("x"), d("f"), d("gate"), d("w_post"))
        return {"x_out": y, "n": _normed(y, d("w_pre"))}
    if kind == "norm_bwd":
        y, w = d("x").requires_grad_(), d("w_pre").requires_grad_()
        dy, dw_pre = torch.autograd.grad(_normed(y, w), (y, w), d("grad_n"))
        t = dy + d("grad_x_out")
        branch = {k: d(k).requires_grad_() for k in ("f", "gate", "w_post") if s[k] is not None}
        got = torch.autograd.grad(_summed(torch.zeros_like(t), branch["f"], branch.get("gate"), branch.get("w_post")), list(branch.values()), t)
        grads = dict(zip(branch, got))
        out = {"grad_x": t, "grad_w_pre": dw_pre}
        if "w_post" in grads:
            out["grad_w_post"] = grads["w_post"]
        if "gate" in grads:
            out["grad_gate"] = grads["gate"]
        out["grad_f"] = grads["f"]
        return out
    norm = torch.stack([torch.linalg.vector_norm(g, dtype=torch.float64) for g in s["grads"]]).square().sum().sqrt()
    c = min(1.0, MAX_NORM / (float(norm) + 1e-6))
    clipped = s["clipped"].double()
    at = 0
    for g, pad in zip(s["grads"], s["pads"]):
        clipped[at:at + g.numel()] = g.reshape(-1).double() * c
        at += g.numel() + pad.numel()
    return {"norm": norm.view(1), "clipped": clipped}

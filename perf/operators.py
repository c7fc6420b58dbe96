"""The operators of an attention block and a detector's head beside the normalization layers: a matrix product with bias,
residual and activation in its epilogue, the gated feed-forward block, and the per-head norm of queries and keys with the
rotation by position; forward and backward, float32 and bfloat16, from one token to long batches.

`listed()` names the cases, `draw(rng)` gives more of the same ranges, `prepare` makes what a program has in hand before the
call, `run` is one pass (the plain form, or the library's entry points where `own` is true), `exact` the same results from the
definitions in 64 bits and `work` the bytes and operations a pass cannot do without."""

import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6
TORCH_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}

# What a pass does ("op"):
#   linear_forward       z = x W^T + bias + residual, y = act(z); z is an output too where "save" is set
#   linear_backward      from dy and what the forward kept (y for ReLU, z for GELU and SiLU): dx, dW, dbias, dresidual
#   gated_forward        h = act(x Wg^T) * (x Wu^T); the two products are outputs too where "save" is set
#   gated_backward       from dh and the two products: dx, dWg, dWu
#   head_norm_forward    every head's row of q and k divided by its root mean square, times a weight, rotated by position
#   head_norm_backward   its gradients: dq, dk and those of the two weights


def _linear(name, op, dtype, m, n, k, act, bias=True, residual=False, save=False):
    return {"name": name, "op": op, "dtype": dtype, "M": m, "N": n, "K": k, "act": act, "bias": bias, "residual": residual, "save": save}


def _gated(name, op, dtype, m, f, k, act, save=False):
    return {"name": name, "op": op, "dtype": dtype, "M": m, "F": f, "K": k, "act": act, "save": save}


def _head_norm(name, op, dtype, t, hq, hk, d, r, style, table):
    return {"name": name, "op": op, "dtype": dtype, "T": t, "Hq": hq, "Hk": hk, "D": d, "R": r, "style": style, "table": table}


def listed():
    return [
        # one token through a small layer: latency is all there is to it
        _linear("one_token_bf16", "linear_forward", "bf16", 1, 1024, 1024, "gelu"),
        # a batch of sixteen sequences, one token each, through an output projection: the weights are read once
        _linear("proj_16_tokens_bf16", "linear_forward", "bf16", 16, 4096, 4096, "none", bias=False, residual=True),
        # the widening 1x1 convolution at the end of a fourth-stage bottleneck, 16 images of 50 x 84 pixels, channels last:
        # fixed statistics folded into weights and bias, shortcut and ReLU in the epilogue; memory counts as much as products
        _linear("res4_widen_bf16", "linear_forward", "bf16", 67200, 1024, 256, "relu", residual=True),
        # a feed-forward layer's first half under training, 16384 tokens, keeping what its backward needs
        _linear("ffn_up_16k_bf16", "linear_forward", "bf16", 16384, 8192, 2048, "gelu", save=True),
        # the region head's first layer in full precision: 512 crops of 7 x 7 pixels and 256 channels
        _linear("region_head_f32", "linear_forward", "f32", 512, 1024, 12544, "relu"),
        # the narrowing 1x1 convolution of a third-stage bottleneck on the way back, 64 images of 50 x 84 pixels: the gradient
        # of the weights is a small matrix summed over 268800 pixels
        _linear("res3_narrow_bwd_bf16", "linear_backward", "bf16", 268800, 128, 512, "relu"),
        # four sequences, one token each, through a gated block: serving's most expensive read of weights
        _gated("gated_4_tokens_bf16", "gated_forward", "bf16", 4, 11264, 4096, "silu"),
        # a gated block under training, keeping what its backward needs; the largest product
        _gated("gated_8k_bf16", "gated_forward", "bf16", 8192, 14336, 4096, "silu", save=True),
        # its backward where neither tokens nor width (two thirds of four times 2048) are round numbers
        _gated("gated_ragged_bwd_bf16", "gated_backward", "bf16", 5003, 5461, 2048, "gelu"),
        # eight sequences, one token each, at positions of their own
        _head_norm("norm_8_tokens_bf16", "head_norm_forward", "bf16", 8, 32, 8, 128, 128, "halves", 32768),
        # a prompt batch: q and k are slices of the joint projection's rows
        _head_norm("norm_32k_bf16", "head_norm_forward", "bf16", 32768, 32, 8, 128, 128, "halves", 32768),
        # training in full precision with heads of 80 values, of which 32 are rotated, pair by pair
        _head_norm("norm_8k_bwd_f32", "head_norm_backward", "f32", 8191, 20, 20, 80, 32, "interleaved", 2048),
    ]


def _spread(rng, lo, hi, multiple):
    """Log-uniform over [lo, hi]; three times in four a multiple of `multiple`, else as it falls."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(multiple, v // multiple * multiple) if rng.random() < 0.75 else v


def draw(rng):
    op = rng.choice(["linear_forward", "linear_backward", "gated_forward", "gated_backward", "head_norm_forward", "head_norm_backward"])
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    if op.startswith("head_norm"):
        d = rng.choice([32, 64, 80, 96, 128, 256, rng.randrange(33, 200)])
        r = rng.choice([d // 2 * 2, d // 4 * 2, 0])
        hk = rng.choice([1, 2, 4, 8, 16])
        hq = hk * rng.choice([1, 2, 4, 8])
        t = int(round(math.exp(rng.uniform(0, math.log(32768)))))
        t = max(1, min(t, 160_000_000 // ((hq + hk) * d)))
        return {"op": op, "dtype": dtype, "T": t, "Hq": hq, "Hk": hk, "D": d, "R": r, "style": rng.choice(["halves", "interleaved"]),
                "table": rng.choice([512, 4096, 32768])}
    m = _spread(rng, 1, 65536, 8) if rng.random() < 0.7 else rng.randrange(1, 65)
    n, k = _spread(rng, 64, 12288, 64), _spread(rng, 64, 8192, 64)
    # no more than about a quarter of the largest listed product; full precision, with a tenth of the rate, a tenth of that
    most = (2.4e11 if dtype == "bf16" else 2.4e10) / (2 if op.startswith("gated") else 1) / (2 if op.endswith("backward") else 1)
    m = max(1, min(m, int(most / (n * k))))
    act = rng.choice(["none", "relu", "gelu", "silu"])
    if op.startswith("gated"):
        return {"op": op, "dtype": dtype, "M": m, "F": n, "K": k, "act": act, "save": rng.random() < 0.5}
    return {"op": op, "dtype": dtype, "M": m, "N": n, "K": k, "act": act, "bias": rng.random() < 0.7, "residual": rng.random() < 0.5,
            "save": act in ("gelu", "silu") and rng.random() < 0.5}


# ---- inputs -----------------------------------------------------------------------------------------------------


def _act64(z, act):
    if act == "relu":
        return torch.nn.functional.relu(z)
    if act == "gelu":
        return torch.nn.functional.gelu(z)
    if act == "silu":
        return torch.nn.functional.silu(z)
    return z


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    dt = TORCH_DTYPE[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, device=DEVICE, generator=gen).mul_(scale)

    op = case["op"]
    if op.startswith("linear"):
        m, n, k = case["M"], case["N"], case["K"]
        a = {"x": normal(m, k).to(dt), "w": normal(n, k, scale=k ** -0.5).to(dt)}
        if op == "linear_forward":
            a["bias"] = normal(n, scale=0.1) if case["bias"] else None
            a["residual"] = normal(m, n).to(dt) if case["residual"] else None
        else:
            a["dy"] = normal(m, n, scale=1e-2).to(dt)
            # what the forward kept: its output for ReLU (half of it zero), z for GELU and SiLU, nothing for none
            a["saved"] = None if case["act"] == "none" else normal(m, n).to(dt)
            if case["act"] == "relu":
                a["saved"].clamp_(min=0)
        return a
    if op.startswith("gated"):
        m, f, k = case["M"], case["F"], case["K"]
        a = {"x": normal(m, k).to(dt), "wg": normal(f, k, scale=k ** -0.5).to(dt), "wu": normal(f, k, scale=k ** -0.5).to(dt)}
        if op == "gated_backward":
            a["dh"], a["gate"], a["up"] = normal(m, f, scale=1e-2).to(dt), normal(m, f).to(dt), normal(m, f).to(dt)
        return a
    t, hq, hk, d, r = case["T"], case["Hq"], case["Hk"], case["D"], case["R"]
    # the joint projection's rows: q, k, v side by side
    a = {"qkv": (normal(t, (hq + 2 * hk) * d) * (0.5 + torch.rand(t, 1, device=DEVICE, generator=gen))).to(dt)}
    a["wq"], a["wk"] = 0.5 + torch.rand(d, device=DEVICE, generator=gen), 0.5 + torch.rand(d, device=DEVICE, generator=gen)
    a["positions"] = torch.randint(0, case["table"], (t,), device=DEVICE, generator=gen, dtype=torch.int32)
    if r:
        angle = torch.arange(case["table"], device=DEVICE, dtype=torch.float64)[:, None] \
            * 10000.0 ** (-torch.arange(0, r, 2, device=DEVICE, dtype=torch.float64) / r)
        a["cos"], a["sin"] = angle.cos().float(), angle.sin().float()
    else:
        a["cos"] = a["sin"] = None
    if op == "head_norm_backward":
        a["dyq"], a["dyk"] = normal(t, hq * d, scale=1e-2).to(dt), normal(t, hk * d, scale=1e-2).to(dt)
    return a


def prepare(case, seed):
    a = _inputs(case, seed)
    dt, op = TORCH_DTYPE[case["dtype"]], case["op"]

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, device=DEVICE, dtype=dtype)

    # buffers that a program keeps from step to step
    if op == "linear_forward":
        out = {"y": empty(case["M"], case["N"]), "z": empty(case["M"], case["N"]) if case["save"] else None}
    elif op == "linear_backward":
        out = {"dx": torch.empty_like(a["x"]), "dw": torch.empty_like(a["w"]),
               "dbias": empty(case["N"], dtype=torch.float32) if case["bias"] else None,
               "dresidual": torch.empty_like(a["dy"]) if case["residual"] else None}
    elif op == "gated_forward":
        out = {"h": empty(case["M"], case["F"])}
        out["gate"], out["up"] = (torch.empty_like(out["h"]), torch.empty_like(out["h"])) if case["save"] else (None, None)
    elif op == "gated_backward":
        out = {"dx": torch.empty_like(a["x"]), "dwg": torch.empty_like(a["wg"]), "dwu": torch.empty_like(a["wu"])}
    else:
        nq, nk = case["Hq"] * case["D"], case["Hk"] * case["D"]
        a["q"], a["k"] = a["qkv"][:, :nq], a["qkv"][:, nq:nq + nk]
        if op == "head_norm_forward":
            out = {"yq": empty(case["T"], nq), "yk": empty(case["T"], nk)}
        else:
            out = {"dq": empty(case["T"], nq), "dk": empty(case["T"], nk), "dwq": empty(case["D"], dtype=torch.float32),
                   "dwk": empty(case["D"], dtype=torch.float32)}
    return {"case": case, "in": a, "out": out}


# ---- the plain form: elementary operations in 32 bits, rounded once at the end ------------------------------------


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return z * (0.5 * (1 + torch.erf(z * math.sqrt(0.5))))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _slope(z, act):
    """act'(z)"""
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _rotate(x, c, s, r, style):
    """x [T, H, D]; the first r of D values turned by the angles whose cosines and sines are c, s [T, 1, r / 2]."""
    if not r:
        return x
    if style == "halves":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., r:]], dim=-1)


def _angles(case, a):
    if not case["R"]:
        return None, None
    pos = a["positions"].long()
    return a["cos"][pos][:, None], a["sin"][pos][:, None]


def _norm_backward(case, x, dy, w, c, s):
    d = case["D"]
    x, dy = x.float().reshape(case["T"], -1, d), dy.float().reshape(case["T"], -1, d)
    e = _rotate(dy, c, None if s is None else -s, case["R"], case["style"])
    rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    n = x * rstd
    t = e * w
    dx = rstd * (t - n * (t * n).mean(-1, keepdim=True))
    return dx.reshape(case["T"], -1), (e * n).sum((0, 1))


def _plain(case, a):
    dt, op, act = TORCH_DTYPE[case["dtype"]], case["op"], case.get("act")
    if op == "linear_forward":
        z = a["x"].float() @ a["w"].float().t()
        if a["bias"] is not None:
            z = z + a["bias"]
        if a["residual"] is not None:
            z = z + a["residual"].float()
        return {"y": _act(z, act).to(dt), "z": z.to(dt) if case["save"] else None}
    if op == "linear_backward":
        dz = a["dy"].float()
        if act != "none":
            dz = dz * _slope(a["saved"].float(), act)
        return {"dx": (dz @ a["w"].float()).to(dt), "dw": (dz.t() @ a["x"].float()).to(dt), "dbias": dz.sum(0) if case["bias"] else None,
                "dresidual": dz.to(dt) if case["residual"] else None}
    if op == "gated_forward":
        x = a["x"].float()
        g, u = x @ a["wg"].float().t(), x @ a["wu"].float().t()
        return {"h": (_act(g, act) * u).to(dt), "gate": g.to(dt) if case["save"] else None, "up": u.to(dt) if case["save"] else None}
    if op == "gated_backward":
        x, dh, g, u = a["x"].float(), a["dh"].float(), a["gate"].float(), a["up"].float()
        dg, du = dh * u * _slope(g, act), dh * _act(g, act)
        dx = dg @ a["wg"].float() + du @ a["wu"].float()
        return {"dx": dx.to(dt), "dwg": (dg.t() @ x).to(dt), "dwu": (du.t() @ x).to(dt)}
    c, s = _angles(case, a)
    if op == "head_norm_forward":
        def one(x, w):
            x = x.float().reshape(case["T"], -1, case["D"])
            n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
            return _rotate(n, c, s, case["R"], case["style"]).reshape(case["T"], -1).to(dt)
        return {"yq": one(a["q"], a["wq"]), "yk": one(a["k"], a["wk"])}
    dq, dwq = _norm_backward(case, a["q"], a["dyq"], a["wq"], c, s)
    dk, dwk = _norm_backward(case, a["k"], a["dyk"], a["wk"], c, s)
    return {"dq": dq.to(dt), "dk": dk.to(dt), "dwq": dwq, "dwk": dwk}


# ---- the library's calls ------------------------------------------------------------------------------------------


def _workspace(state, need, *args):
    """The program's scratch, made at its first step and kept."""
    if "workspace" not in state:
        state["workspace"] = torch.empty(max(need(*args), 256), dtype=torch.uint8, device=DEVICE)
    return state["workspace"]


def _own(state):
    from paper_1711_07240_amd import cgbn
    case, a, o = state["case"], state["in"], state["out"]
    op, dtype = case["op"], case["dtype"]
    if op.startswith("linear"):
        size = (case["M"], case["N"], case["K"])
        ws = _workspace(state, cgbn.cgbn_linear_workspace_bytes, *size, dtype, op == "linear_backward")
        if op == "linear_forward":
            cgbn.cgbn_linear_forward(a["x"], a["w"], a["bias"], a["residual"], *size, case["act"], o["y"], o["z"], dtype, ws)
        else:
            cgbn.cgbn_linear_backward(a["dy"], a["x"], a["w"], a["saved"], *size, case["act"], o["dx"], o["dw"], o["dbias"],
                                      o["dresidual"], dtype, ws)
    elif op.startswith("gated"):
        size = (case["M"], case["F"], case["K"])
        ws = _workspace(state, cgbn.cgbn_gated_workspace_bytes, *size, dtype, op == "gated_backward")
        if op == "gated_forward":
            cgbn.cgbn_gated_forward(a["x"], a["wg"], a["wu"], *size, case["act"], o["h"], o["gate"], o["up"], dtype, ws)
        else:
            cgbn.cgbn_gated_backward(a["dh"], a["x"], a["wg"], a["wu"], a["gate"], a["up"], *size, case["act"], o["dx"], o["dwg"],
                                     o["dwu"], dtype, ws)
    else:
        heads = (case["T"], case["Hq"], case["Hk"], case["D"])
        turn = (case["R"], case["style"], a["positions"], a["cos"], a["sin"], case["table"])
        row = a["qkv"].shape[1]
        nq, nk = case["Hq"] * case["D"], case["Hk"] * case["D"]
        if op == "head_norm_forward":
            cgbn.cgbn_head_norm_forward(a["q"], row, a["k"], row, *heads, *turn, a["wq"], a["wk"], EPS, o["yq"], nq, o["yk"], nk, dtype)
        else:
            ws = _workspace(state, cgbn.cgbn_head_norm_workspace_bytes, *heads, dtype)
            cgbn.cgbn_head_norm_backward(a["dyq"], nq, a["dyk"], nk, a["q"], row, a["k"], row, *heads, *turn, a["wq"], a["wk"], EPS,
                                         o["dq"], nq, o["dk"], nk, o["dwq"], o["dwk"], dtype, ws)
    return o


def run(state):
    out = _own(state) if own else _plain(state["case"], state["in"])
    return {name: t for name, t in out.items() if t is not None}


# ---- the definitions in 64 bits: forward as defined, gradients by differentiating it ------------------------------


def _rotate64(case, x, positions, cos, sin):
    """The rotation as a complex product."""
    r = case["R"]
    if not r:
        return x
    turn = torch.complex(cos.double()[positions.long()], sin.double()[positions.long()])[:, None]
    head = x[..., :r]
    if case["style"] == "halves":
        z = torch.complex(head[..., :r // 2], head[..., r // 2:]) * turn
        head = torch.cat([z.real, z.imag], dim=-1)
    else:
        z = torch.view_as_complex(head.reshape(*head.shape[:-1], r // 2, 2).contiguous()) * turn
        head = torch.view_as_real(z).reshape(*head.shape)
    return torch.cat([head, x[..., r:]], dim=-1)


def exact(case, seed):
    a, op = _inputs(case, seed), case["op"]
    if op == "linear_forward":
        z = torch.matmul(a["x"].double(), a["w"].double().t())
        for extra in (a["bias"], a["residual"]):
            if extra is not None:
                z += extra.double()
        out = {"y": _act64(z, case["act"])}
        if case["save"]:
            out["z"] = z
        return out
    if op == "linear_backward":
        dz = a["dy"].double()
        if case["act"] != "none":
            z = a["saved"].double().requires_grad_()
            (dz,) = torch.autograd.grad(_act64(z, case["act"]), z, dz)
        out = {"dx": torch.matmul(dz, a["w"].double()), "dw": torch.matmul(dz.t(), a["x"].double())}
        if case["bias"]:
            out["dbias"] = dz.sum(0)
        if case["residual"]:
            out["dresidual"] = dz
        return out
    if op == "gated_forward":
        g, u = (torch.matmul(a["x"].double(), a[w].double().t()) for w in ("wg", "wu"))
        out = {"h": _act64(g, case["act"]) * u}
        if case["save"]:
            out["gate"], out["up"] = g, u
        return out
    if op == "gated_backward":
        g, u = a["gate"].double().requires_grad_(), a["up"].double().requires_grad_()
        dg, du = torch.autograd.grad(_act64(g, case["act"]) * u, (g, u), a["dh"].double())
        x = a["x"].double()
        return {"dx": torch.matmul(dg, a["wg"].double()) + torch.matmul(du, a["wu"].double()),
                "dwg": torch.matmul(dg.t(), x), "dwu": torch.matmul(du.t(), x)}
    t, d = case["T"], case["D"]
    nq, nk = case["Hq"] * d, case["Hk"] * d
    out = {}
    for which, lo, n in (("q", 0, nq), ("k", nq, nk)):
        x = a["qkv"][:, lo:lo + n].double().requires_grad_()
        w = a["w" + which].double().requires_grad_()
        rows = x.reshape(t, -1, d)
        y = _rotate64(case, rows / (rows.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w, a["positions"], a["cos"], a["sin"]).reshape(t, -1)
        if op == "head_norm_forward":
            out["y" + which] = y.detach()
        else:
            out["d" + which], out["dw" + which] = torch.autograd.grad(y, (x, w), a["dy" + which].double())
    if op == "head_norm_backward":
        out = {name: out[name] for name in ("dq", "dk", "dwq", "dwk")}
    return out


def work(case):
    """Every input read once, every output written once; two operations a multiply-add, and a handful an element beside them."""
    eb, op = (4 if case["dtype"] == "f32" else 2), case["op"]
    if op.startswith("linear"):
        m, n, k = case["M"], case["N"], case["K"]
        if op == "linear_forward":
            return {"bytes": eb * (m * k + n * k + m * n * (1 + case["residual"] + case["save"])) + 4 * n * case["bias"], "flops": 2 * m * n * k}
        return {"bytes": eb * (2 * m * k + 2 * n * k + m * n * (1 + (case["act"] != "none") + case["residual"])) + 4 * n * case["bias"],
                "flops": 4 * m * n * k}
    if op.startswith("gated"):
        m, f, k = case["M"], case["F"], case["K"]
        if op == "gated_forward":
            return {"bytes": eb * (m * k + 2 * f * k + m * f * (3 if case["save"] else 1)), "flops": 4 * m * f * k}
        return {"bytes": eb * (2 * m * k + 4 * f * k + 3 * m * f), "flops": 8 * m * f * k}
    t, d, r, rows = case["T"], case["D"], case["R"], case["T"] * (case["Hq"] + case["Hk"])
    table = 4 * min(t, case["table"]) * r + 4 * t
    if op == "head_norm_forward":
        return {"bytes": eb * 2 * rows * d + table + 8 * d, "flops": rows * (4 * d + 3 * r)}
    return {"bytes": eb * 3 * rows * d + table + 16 * d, "flops": rows * (12 * d + 3 * r)}

"""What a training step needs besides its layers in 8-bit integers: the calls that stand for its use, their inputs and work, plain forms and
64-bit results.

Matrices have a point of a region's sweep in each row.  A value in 8 bits is e4m3: one sign bit, three bits of fraction, the largest 448, steps of
2^-9 below 2^-6.  A block of values shares a scale 2^e, the smallest (e at least -126) with max|v| <= 448 * 2^e; its codes are v / 2^e rounded to
e4m3, ties to even.

``linear``    y = act(x W^T + b) of codes: blocks of x are 128 columns of a row, those of W are 128 x 128 values.  ``learn``: as a training step
              calls it, with weights that have changed since the last step, and x's codes by column (blocks of 128 rows of a column) put away for
              the backward pass, which are read back here.
``backward``  of the same layer, from x's codes by column: with dz = dy, 0 where the layer's ReLU gave y <= 0: dW = dz^T x with dz by column,
              dx = dz W with dz by row, db = the sum of dz's rows.
``clip``      the gradients' common norm (2: Euclidean, in 64 bits; inf: the largest magnitude), and each gradient times
              min(1, most / (norm + 1e-6)), rounded once to the type it is wanted in.
``norm``      group norm with an activation, channels last: for an image's points and a group's channels together, y = act(z),
              z = (x - mean) * (rstd * gamma) + beta, rstd = 1 / sqrt(variance + eps); mean and rstd are kept.
``unnorm``    its gradients: g = dy act'(z), dgamma = sum g (x - mean) rstd, dbeta = sum g, and, with the means over image and group,
              dx = rstd (g gamma - mean(g gamma) - (x - mean) rstd mean(g gamma (x - mean) rstd)).  A ReLU lets through where z > 0 for x - mean
              and rstd * gamma in 32 bits.
"""
import math

import torch

own = False

BLOCK = 128
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one point through a layer of the widest models: a surrogate asked from inside a serial loop
        dict(name="linear_one_point", op="linear", n=1, n_in=4096, n_out=4096, x="bf16", y="bf16", relu=True, bias=True, pad=0, learn=False),
        # a training batch of a stencil model's hidden layer
        dict(name="linear_learn", op="linear", n=65536, n_in=512, n_out=512, x="bf16", y="bf16", relu=True, bias=True, pad=0, learn=True),
        # the widest layer over one chunk of a large region
        dict(name="linear_wide", op="linear", n=131072, n_in=4096, n_out=4096, x="bf16", y="bf16", relu=True, bias=True, pad=0, learn=False),
        # a ragged fp32 batch of unequal odd widths, rows inside a wider record
        dict(name="backward_odd", op="backward", n=30011, n_in=201, n_out=50, dy="f32", relu=True, dx=True, pad=3),
        # a wide hidden layer over a large batch
        dict(name="backward_wide", op="backward", n=131072, n_in=2048, n_out=2048, dy="bf16", relu=True, dx=True, pad=0),
        # the gradients of a small fp32 model
        dict(name="clip_small", op="clip", dims="9,128,128,128,1", repeat=1, g="f32", out="f32", kind="2", most=0.5),
        # those of many middle-sized models that learn together
        dict(name="clip_many", op="clip", dims="36,256,256,256,4", repeat=64, g="f32", out="f32", kind="2", most=0.5),
        # those of a few of the widest layers, from bf16 to the optimizer's fp32
        dict(name="clip_wide", op="clip", dims="4096,4096,4096,4096,4096,4096,4096,4096,4096", repeat=1, g="bf16", out="f32", kind="2", most=0.5),
        # a hidden layer's activations: every point is an image of its own
        dict(name="norm_hidden", op="norm", images=65536, points=1, channels=512, groups=16, x="bf16", act="relu", pad=0),
        # a weather model's one image: few groups of a great many points
        dict(name="norm_grid", op="norm", images=1, points=2048 * 2048, channels=8, groups=2, x="f32", act="silu", pad=0),
        # frames of odd size and groups of odd width, rows inside a wider record
        dict(name="unnorm_odd", op="unnorm", images=37, points=13 * 17, channels=45, groups=9, x="f32", act="relu", pad=3),
        # a batch of frames behind a convolution
        dict(name="unnorm_frames", op="unnorm", images=1024, points=32 * 32, channels=128, groups=8, x="bf16", act="silu", pad=0),
    ]


def draw(rng):
    def log(lo, hi):  # odd sizes, multiples of 8 and powers of two
        v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
        near = [int(v - 1) | 1, max(1, int(v / 40)) * 40, 2 ** round(math.log2(v))]
        return int(round(v)) if v < 64 else min(hi, rng.choice(near))

    op = rng.choice(["linear", "backward", "clip", "norm", "unnorm"])
    kind, pad = rng.choice(["f32", "bf16", "bf16"]), rng.choice([0, 0, 0, 1, 8, 32])
    if op == "linear":
        return dict(op=op, n=log(1, 131072), n_in=log(5, 4096), n_out=log(1, 4096), x=kind, y=rng.choice(["f32", kind]), relu=rng.random() < 0.7,
                    bias=rng.random() < 0.8, pad=pad, learn=rng.random() < 0.3)
    if op == "backward":
        return dict(op=op, n=log(1, 131072), n_in=log(5, 2048), n_out=log(1, 2048), dy=kind, relu=rng.random() < 0.7, dx=rng.random() < 0.8, pad=pad)
    if op == "clip":
        width, depth = log(8, 2048), rng.randint(1, 6)
        dims = [rng.randint(1, 40)] + [width] * depth + [rng.randint(1, 9)]
        most = max(1, (1 << 26) // (width * width * depth))
        return dict(op=op, dims=",".join(map(str, dims)), repeat=min(log(1, 100), most), g=kind, out=rng.choice(["f32", kind]),
                    kind=rng.choice(["2", "2", "2", "inf"]), most=rng.choice([0.5, 0.01, 1e9]))
    groups = log(1, 64)
    channels = groups * log(1, max(1, 2048 // groups))
    points = rng.choice([1, log(2, 1 << 22)])
    points = max(1, min(points, (1 << 27) // channels))
    if points * channels == 2 * groups:  # normalising two values takes everything from their gradients: what is left is rounding
        channels *= 2
    return dict(op=op, images=max(1, min(log(1, 1 << 17), (1 << 27) // (points * channels))), points=points, channels=channels, groups=groups, x=kind,
                act=rng.choice(["none", "relu", "silu"]), pad=pad)


# ---- inputs ---------------------------------------------------------------------


def _rows(g, n, width, kind, pad, scale=1.0, offset=None):
    """Normal values with a magnitude of its own for each row (a few rows are zero), inside rows of width + pad."""
    t = torch.empty((n, width + pad), dtype=TYPES[kind], device="cuda")
    size = torch.exp2(torch.randn((n, 1), generator=g, device="cuda")) * scale
    size *= torch.rand((n, 1), generator=g, device="cuda") >= 1 / 64
    step = max(1, (1 << 26) // (width + pad))
    for i in range(0, n, step):
        m = min(step, n - i)
        v = torch.randn((m, width + pad), generator=g, device="cuda")
        t[i : i + m] = v * size[i : i + m] if offset is None else v * 2 + offset
    return t[:, :width]


def _dims(case):
    """(out, in) of every layer."""
    d = [int(v) for v in case["dims"].split(",")]
    return list(zip(d[1:], d)) * case["repeat"]


def _inputs(case, seed):
    """The tensors that both forms and the 64-bit results start from."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)
    new = dict(generator=g, device="cuda")
    if case["op"] == "clip":
        grads = []
        for o, i in _dims(case):
            grads.append((torch.randn((o, i), **new) * (0.02 / math.sqrt(i))).to(TYPES[case["g"]]))
            grads.append((torch.randn(o, **new) * 0.02).to(TYPES[case["g"]]))
        return grads
    if case["op"] in ("norm", "unnorm"):
        n, c = case["images"] * case["points"], case["channels"]
        x = _rows(g, n, c, case["x"], case["pad"], offset=torch.randn(c + case["pad"], **new))
        gamma, beta = 1 + torch.randn(c, **new) * 0.2, torch.randn(c, **new) * 0.2
        if case["op"] == "norm":
            return x, gamma, beta
        dy = _rows(g, n, c, case["x"], case["pad"], 1e-3)
        return (x, gamma, beta, *_moments(case, x), dy)
    n, n_in, n_out = case["n"], case["n_in"], case["n_out"]
    W = torch.randn((n_out, n_in), **new) * math.sqrt(2 / n_in)
    if case["op"] == "linear":
        b = (torch.rand(n_out, **new) - 0.5) * (2 / math.sqrt(n_in)) if case["bias"] else None
        return _rows(g, n, n_in, case["x"], case["pad"]), W, b
    x, dy = _rows(g, n, n_in, case["dy"], 0), _rows(g, n, n_out, case["dy"], case["pad"], 1e-3)
    y = torch.randn((n, n_out), **new).clamp_(min=0).to(TYPES[case["dy"]]) if case["relu"] else None
    return x, W, dy, y


def prepare(case, seed):
    ins = _inputs(case, seed)
    if own:
        return _prepare_own(case, ins)
    if case["op"] == "linear" and not case["learn"]:
        x, W, b = ins
        return {"case": case, "ins": (x, _square(W), b)}
    if case["op"] == "backward":
        x, W, dy, y = ins
        return {"case": case, "ins": (_by_column(x), _square(W), dy, y)}
    return {"case": case, "ins": ins}


def run(state):
    if own:
        return _run_own(state)
    return {"linear": _linear, "backward": _backward, "clip": _clip, "norm": _norm, "unnorm": _unnorm}[state["case"]["op"]](state["case"], state["ins"])


def _into(case):
    """The clipped gradients' tensors, in one buffer as an optimizer keeps them, each from a multiple of 64 on."""
    sizes = [s for o, i in _dims(case) for s in ((o, i), (o,))]
    ends, at = [], 0
    for s in sizes:
        ends.append(at)
        at += -(-math.prod(s) // 64) * 64
    flat = torch.zeros(at, dtype=TYPES[case["out"]], device="cuda")
    return flat, [flat[e : e + math.prod(s)].view(s) for e, s in zip(ends, sizes)]


def _prepare_own(case, ins):
    """What a program keeps: layers with their weights laid out, what was put away, outputs and scratch memory."""
    from paper_2407_18352_amd import _abi, api

    new, op = dict(device="cuda"), case["op"]
    state = {"case": case, "api": api}
    if op == "clip":
        flat, parts = _into(case)
        grads = api.GradientSet(ins, into=parts)
        return dict(state, grads=grads, flat=flat, norm=torch.empty(1, **new), kind=_abi.NORM_MAX if case["kind"] == "inf" else _abi.NORM_2,
                    scratch=torch.empty(grads.scratch_bytes(), dtype=torch.uint8, **new))
    if op in ("norm", "unnorm"):
        act = {"none": _abi.ACT_IDENTITY, "relu": _abi.ACT_RELU, "silu": _abi.ACT_SILU}[case["act"]]
        x = ins[0]
        y = torch.empty(x.shape, dtype=x.dtype, **new)
        need = api.group_norm_scratch_bytes(x, case["points"], case["groups"], backward=op == "unnorm")
        state |= dict(x=x, gamma=ins[1], beta=ins[2], y=y, act=act, scratch=torch.empty(need, dtype=torch.uint8, **new))
        if op == "norm":
            return dict(state, mean=torch.empty((case["images"], case["groups"]), **new), rstd=torch.empty((case["images"], case["groups"]), **new))
        return dict(state, mean=ins[3], rstd=ins[4], dy=ins[5], dgamma=torch.empty_like(ins[1]), dbeta=torch.empty_like(ins[2]))
    act = _abi.ACT_RELU if case["relu"] else _abi.ACT_IDENTITY
    kept = api.MatrixF8(case["n_in"], case["n"]) if op == "backward" or case["learn"] else None
    if op == "linear":
        x, W, b = ins
        layer = api.LinearF8(W, b, learn=case["learn"])
        y = torch.empty((case["n"], case["n_out"]), dtype=TYPES[case["y"]], **new)
        back = torch.empty((case["n_in"], case["n"]), dtype=torch.bfloat16, **new) if case["learn"] else None
        need = layer.scratch_bytes(case["n"])
        return dict(state, layer=layer, x=x, y=y, W=W, b=b, act=act, kept=kept, back=back, scratch=torch.empty(need, dtype=torch.uint8, **new))
    x, W, dy, y = ins
    api.quantizef8(x, by_column=kept)
    layer = api.LinearF8(W, learn=True)
    dw, db = torch.empty((case["n_out"], case["n_in"]), **new), torch.empty(case["n_out"], **new)
    dx = torch.empty((case["n"], case["n_in"]), dtype=dy.dtype, **new) if case["dx"] else None
    need = api.backwardf8_scratch_bytes(kept, dy, dx=case["dx"])
    return dict(state, layer=layer if case["dx"] else None, kept=kept, dy=dy, y=y, dw=dw, db=db, dx=dx, scratch=torch.empty(need, dtype=torch.uint8, **new))


def _run_own(s):
    api, op, case = s["api"], s["case"]["op"], s["case"]
    if op == "linear":
        if not case["learn"]:
            api.linearf8(s["layer"], s["x"], s["y"], s["act"], scratch=s["scratch"])
            return {"y": s["y"]}
        s["layer"].update(s["W"], s["b"])
        api.linearf8(s["layer"], s["x"], s["y"], s["act"], kept=s["kept"], scratch=s["scratch"])
        api.loadf8(s["kept"], s["back"])
        return {"y": s["y"], "kept": s["back"]}
    if op == "backward":
        api.backwardf8(s["kept"], s["dy"], s["dw"], s["db"], layer=s["layer"], dx=s["dx"], y=s["y"], scratch=s["scratch"])
        return {"dw": s["dw"], "db": s["db"]} | ({"dx": s["dx"]} if s["dx"] is not None else {})
    if op == "clip":
        api.clip_gradients(s["grads"], case["most"], s["norm"], s["kind"], scratch=s["scratch"])
        return {"norm": s["norm"], "grads": s["flat"]}
    if op == "norm":
        api.group_norm(s["x"], s["y"], case["points"], case["groups"], s["gamma"], s["beta"], EPS, s["act"], s["mean"], s["rstd"], scratch=s["scratch"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    api.group_norm_backward(s["x"], s["dy"], case["points"], case["groups"], s["mean"], s["rstd"], s["y"], s["dgamma"], s["dbeta"], s["gamma"], s["beta"],
                            s["act"], scratch=s["scratch"])
    return {"dx": s["y"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


# ---- plain forms, in 32 bits (sums over many points in 64) ----------------------------


def _times2(v, e):
    """v * 2^e (the power is exact, which torch.ldexp's is not everywhere)."""
    return v * torch.exp2(e.float())


def _e4m3(v):
    """The nearest e4m3 values of |v| <= 448."""
    step = torch.clamp(torch.frexp(v)[1] - 1, min=-6) - 3
    return _times2(torch.round(_times2(v, -step)), step)


def _blocks(v, dims):
    """What the codes of blocks, the whole of the dimensions `dims` of v, stand for."""
    part, power = torch.frexp(v.abs().amax(dim=dims, keepdim=True))
    e = torch.clamp(torch.where(part <= 0.875, power - 9, power - 8), min=-126)  # 448 = 0.875 * 2^9
    return _times2(_e4m3(_times2(v, -e)), e)


def _by_row(x):
    n, w = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -w % BLOCK)).unflatten(1, (-1, BLOCK))
    return _blocks(v, (2,)).flatten(1)[:, :w]


def _by_column(x):
    n, w = x.shape
    v = torch.nn.functional.pad(x.float(), (0, 0, 0, -n % BLOCK)).unflatten(0, (-1, BLOCK))
    return _blocks(v, (1,)).flatten(0, 1)[:n]


def _square(W):
    o, i = W.shape
    v = torch.nn.functional.pad(W.float(), (0, -i % BLOCK, 0, -o % BLOCK)).unflatten(1, (-1, BLOCK)).unflatten(0, (-1, BLOCK))
    return _blocks(v, (1, 3)).flatten(2).flatten(0, 1)[:o, :i]


def _linear(case, ins):
    x, W, b = ins
    y = _by_row(x) @ (_square(W) if case["learn"] else W).t()
    if b is not None:
        y = y + b
    if case["relu"]:
        y = torch.where(y < 0, torch.zeros_like(y), y)
    out = {"y": y.to(TYPES[case["y"]])}
    if case["learn"]:
        out["kept"] = _by_column(x).t().to(torch.bfloat16).contiguous()
    return out


def _backward(case, ins):
    x, W, dy, y = ins
    dz = dy.float()
    if y is not None:
        dz = torch.where(y <= 0, torch.zeros_like(dz), dz)
    out = {"dw": _by_column(dz).t().contiguous() @ x, "db": dz.sum(dim=0, dtype=torch.float64).float()}
    if case["dx"]:
        out["dx"] = (_by_row(dz) @ W).to(dy.dtype)
    return out


def _clip(case, grads):
    if case["kind"] == "inf":
        norm = torch.stack([t.abs().amax().double() for t in grads]).amax()
    else:
        norm = torch.stack([t.double().square().sum() for t in grads]).sum().sqrt()
    factor = torch.clamp(case["most"] / (norm + 1e-6), max=1.0).float()
    flat, parts = _into(case)
    for t, p in zip(grads, parts):
        p.copy_(t.float() * factor)
    return {"norm": norm.float().reshape(1), "grads": flat}


def _images(case, x):
    """x as [images][points][groups][channels of a group]."""
    return x.reshape(case["images"], case["points"], case["groups"], -1)


def _moments(case, x):
    """Mean and 1 / sqrt(variance + eps), [images][groups]."""
    v = _images(case, x).double()
    mean = v.mean(dim=(1, 3), keepdim=True)
    var = (v - mean).square_().mean(dim=(1, 3))
    return mean.float().reshape(var.shape), (1 / torch.sqrt(var + EPS)).float()


def _centred(case, x, gamma, mean, rstd):
    """x - mean and rstd * gamma, shaped as _images()."""
    d = _images(case, x.float()) - mean[:, None, :, None]
    return d, rstd[:, None, :, None] * gamma.reshape(1, 1, case["groups"], -1)


def _norm(case, ins):
    x, gamma, beta = ins
    mean, rstd = _moments(case, x)
    d, a = _centred(case, x, gamma, mean, rstd)
    z = d * a + beta.reshape(1, 1, case["groups"], -1)
    if case["act"] == "relu":
        z = torch.where(z < 0, torch.zeros_like(z), z)
    elif case["act"] == "silu":
        z = z / (1 + torch.exp(-z))
    return {"y": z.reshape(x.shape).to(x.dtype), "mean": mean, "rstd": rstd}


def _unnorm(case, ins):
    x, gamma, beta, mean, rstd, dy = ins
    d, a = _centred(case, x, gamma, mean, rstd)
    g, z = _images(case, dy.float()), (d.double() * a.double()).add_(beta.double().reshape(1, 1, case["groups"], -1))
    if case["act"] == "relu":
        g = torch.where(z <= 0, torch.zeros_like(g), g)
    elif case["act"] == "silu":
        z = z.float()
        s = 1 / (1 + torch.exp(-z))
        g = g * (s * (1 + z * (1 - s)))
    h = d * rstd[:, None, :, None]
    dgamma, dbeta = (g * h).sum(dim=(0, 1), dtype=torch.float64), g.sum(dim=(0, 1), dtype=torch.float64)
    g = g * gamma.reshape(1, 1, case["groups"], -1)
    m1, m2 = g.double().mean(dim=(1, 3), keepdim=True).float(), (g * h).double().mean(dim=(1, 3), keepdim=True).float()
    dx = rstd[:, None, :, None] * (g - m1 - h * m2)
    return {"dx": dx.reshape(x.shape).to(x.dtype), "dgamma": dgamma.float().flatten(), "dbeta": dbeta.float().flatten()}


# ---- work, and results in 64 bits ----------------------------------------------------


def work(case):
    """Each tensor read or written once; two operations for each product and sum of the matrix products, a few for each other value."""
    size, op = {"f32": 4, "bf16": 2}, case["op"]
    if op == "clip":
        v = sum(o * i + o for o, i in _dims(case))
        return {"bytes": v * (size[case["g"]] + size[case["out"]]) + 4, "flops": 3 * v}
    if op in ("norm", "unnorm"):
        v, c, s = case["images"] * case["points"] * case["channels"], case["channels"], 8 * case["images"] * case["groups"]
        tensors, each = (2, 8) if op == "norm" else (3, 20)
        return {"bytes": tensors * v * size[case["x"]] + s + 4 * c * (2 if op == "norm" else 4), "flops": each * v}
    n, i, o = case["n"], case["n_in"], case["n_out"]
    if op == "linear":
        bias, put = 4 * o if case["bias"] else 0, 2 * n * i + 4 * i * o if case["learn"] else i * o + -(-i // BLOCK) * -(-o // BLOCK)
        return {"bytes": n * i * size[case["x"]] + n * o * size[case["y"]] + bias + put, "flops": 2 * n * i * o}
    s = size[case["dy"]]
    more = (i * o + n * i * s, 2 * n * i * o) if case["dx"] else (0, 0)
    return {"bytes": n * (o * s * (2 if case["relu"] else 1) + i) + -(-n // BLOCK) * i + 4 * o * (i + 1) + more[0], "flops": 2 * n * i * o + n * o + more[1]}


def exact(case, seed):
    ins = _inputs(case, seed)

    def near(v, high, wide):
        """v in 64 bits with blocks of high x wide values rounded to e4m3 and a power of two."""
        out = v.to(torch.float64, copy=True)
        n, m = out.shape
        out = torch.nn.functional.pad(out, (0, -m % wide, 0, -n % high))
        t = out.view(out.shape[0] // high, high, out.shape[1] // wide, wide)
        top = t.abs().amax(3, keepdim=True).amax(1, keepdim=True)
        unit = torch.exp2(torch.ceil(torch.log2(top.masked_fill(top == 0, 1.0) / 448)).clamp(min=-126))
        t /= unit
        step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0**-6))) - 3)
        t.div_(step).round_().mul_(step).mul_(unit)
        return out[:n, :m]

    if case["op"] == "linear":
        x, W, b = ins
        y = torch.matmul(near(x, 1, BLOCK), near(W, BLOCK, BLOCK).T.contiguous())
        if b is not None:
            y += b.double()
        out = {"y": y.clamp_(min=0) if case["relu"] else y}
        if case["learn"]:
            out["kept"] = near(x, BLOCK, 1).T.contiguous()
        return out
    if case["op"] == "backward":
        x, W, dy, y = ins
        dz = dy.double()
        if y is not None:
            dz[y <= 0] = 0
        out = {"dw": torch.matmul(near(dz, BLOCK, 1).T.contiguous(), near(x, BLOCK, 1)), "db": dz.sum(0)}
        if case["dx"]:
            out["dx"] = torch.matmul(near(dz, 1, BLOCK), near(W, BLOCK, BLOCK))
        return out
    if case["op"] == "clip":
        top = max(t.double().abs().max().item() for t in ins)
        norm = top if case["kind"] == "inf" else math.sqrt(sum((t.double() ** 2).sum().item() for t in ins))
        flat, parts = _into(case)
        wide = flat.double()
        for t, p in zip(ins, parts):
            wide[p.storage_offset() : p.storage_offset() + p.numel()] = (t.double() * min(1.0, case["most"] / (norm + 1e-6))).flatten()
        return {"norm": torch.tensor([norm], dtype=torch.float64), "grads": wide}
    n, p, c, k = case["images"], case["points"], case["channels"], case["groups"]
    x, gamma, beta = (t.double() for t in ins[:3])
    x, shape = x.reshape(n, p, c), ins[0].shape
    wide = lambda v: v.double().repeat_interleave(c // k, dim=1)[:, None, :]  # noqa: E731
    if case["op"] == "norm":
        v = x.transpose(1, 2).reshape(n, k, -1)
        var, mean = torch.var_mean(v, dim=2, correction=0)
        rstd = (var + EPS).rsqrt()
        z = (x - wide(mean)) * wide(rstd) * gamma + beta
        z = z.clamp(min=0) if case["act"] == "relu" else z * torch.sigmoid(z) if case["act"] == "silu" else z
        return {"y": z.reshape(shape), "mean": mean, "rstd": rstd}
    mean, rstd, g = ins[3], ins[4], ins[5].double().reshape(n, p, c)
    h = (x - wide(mean)) * wide(rstd)
    if case["act"] == "relu":
        near0 = (x.float() - wide(mean).float()).double() * (wide(rstd).float() * ins[1]).double() + beta
        g = g * (near0 > 0)
    elif case["act"] == "silu":
        z = h * gamma + beta
        s = torch.sigmoid(z)
        g = g * (s + z * s * torch.sigmoid(-z))
    out = {"dgamma": (g * h).sum((0, 1)), "dbeta": g.sum((0, 1))}
    g = g * gamma
    group = lambda v: wide(v.reshape(n, p, k, -1).mean((1, 3)))  # noqa: E731
    out["dx"] = ((g - group(g) - h * group(g * h)) * wide(rstd)).reshape(shape)
    return out

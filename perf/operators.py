"""Dense layers in 8 bits: the calls that stand for their use, their inputs and work, their plain forms and 64-bit results.

Three operators on the rows of a layer's tensors (a row is a point of a region's sweep):

``linear``    y = act(x W^T + b) with x rounded to 8-bit codes by row and W by output: for a row x_i, s_i = max|x_i| / 127 and
              q = rint(x * (127 / max|x_i|)); y = act(s_i t_j sum_k q_ik w_jk + b_j), t_j and w_jk the same of row j of W.
``keep``      an activation put away in 8 bits for the backward pass, and brought back.  Blocks of 32 channels of a row share a
              power of two, 2^e: the smallest with max|a| < 2^(e+8) (after a ReLU: codes 0..255) or 2^(e+7) (no activation: codes
              -127..127, stored plus 128).  code = rint(a / 2^e), cut at the largest; a positive value keeps at least code 1 after
              a ReLU, so that the codes still say where the ReLU let values through.
``backward``  a linear layer's backward pass from its kept input a: dW = dY^T a, db = the sum of dY's rows, dX = dY W where the
              codes say that the ReLU let a through (everywhere without an activation).

Codes are formed in 32-bit arithmetic (a maximum, one division per row, one product and one rounding per value)."""
import math

import torch

own = False

BLOCK = 32
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one point through a layer of the widest models: a surrogate asked from inside a serial loop
        dict(name="linear_one_point", op="linear", n=1, n_in=4096, n_out=4096, x="bf16", y="bf16", relu=True, bias=True, pad=0),
        # a handful of points through a tapered model's hidden layer
        dict(name="linear_few_points", op="linear", n=24, n_in=1024, n_out=512, x="bf16", y="bf16", relu=True, bias=True, pad=0),
        # fp32 hidden layer of unequal odd widths, rows inside a wider record
        dict(name="linear_odd", op="linear", n=65521, n_in=201, n_out=50, x="f32", y="f32", relu=True, bias=True, pad=7),
        # a stencil model's hidden layer over one slab of its grid
        dict(name="linear_slab", op="linear", n=65536, n_in=512, n_out=512, x="bf16", y="bf16", relu=True, bias=True, pad=0),
        # the widest layer over one chunk of a large region
        dict(name="linear_wide", op="linear", n=131072, n_in=4096, n_out=4096, x="bf16", y="bf16", relu=True, bias=True, pad=0),
        # gathered inputs of a seven-point window of five fields, put away as they are
        dict(name="keep_inputs", op="keep", n=4099, width=35, z="f32", a="f32", relu=False, pad=0),
        # a hidden layer's activations of one training batch
        dict(name="keep_hidden", op="keep", n=65536, width=512, z="bf16", a="bf16", relu=True, pad=0),
        # the widest layer's activations of a large batch
        dict(name="keep_wide", op="keep", n=131072, width=4096, z="bf16", a="bf16", relu=True, pad=0),
        # a small batch of a small fp32 model
        dict(name="backward_small", op="backward", n=256, n_in=64, n_out=64, dy="f32", relu=True, dx=True, pad=0),
        # a ragged fp32 batch of unequal odd widths
        dict(name="backward_odd", op="backward", n=30011, n_in=201, n_out=50, dy="f32", relu=True, dx=True, pad=3),
        # a pose model's hidden layer over a large batch: a small gradient from many rows
        dict(name="backward_hidden", op="backward", n=262144, n_in=256, n_out=256, dy="bf16", relu=True, dx=True, pad=0),
        # a wide hidden layer over a large batch
        dict(name="backward_wide", op="backward", n=131072, n_in=2048, n_out=2048, dy="bf16", relu=True, dx=True, pad=0),
    ]


def draw(rng):
    def log(lo, hi):  # odd sizes, multiples of 8 and powers of two
        v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
        near = [int(v - 1) | 1, max(1, int(v / 40)) * 40, 2 ** round(math.log2(v))]
        return int(round(v)) if v < 64 else min(hi, rng.choice(near))

    op = rng.choice(["linear", "linear", "keep", "backward", "backward"])
    kind = rng.choice(["f32", "bf16", "bf16"])
    relu, pad = rng.random() < 0.7, rng.choice([0, 0, 0, 1, 8, 32])
    if op == "linear":
        return dict(op=op, n=log(1, 131072), n_in=log(5, 4096), n_out=log(16, 4096), x=kind, y=rng.choice(["f32", kind]), relu=relu,
                    bias=rng.random() < 0.8, pad=pad)
    if op == "keep":
        width = log(5, 4096)
        return dict(op=op, n=min(log(1, 1 << 20), (1 << (29 if kind == "bf16" else 28)) // width), width=width, z=kind, a=kind, relu=relu, pad=pad)
    n_in, n_out = log(5, 2048), log(1, 2048)
    return dict(op=op, n=log(1, 262144), n_in=n_in, n_out=n_out, dy=kind, relu=relu, dx=rng.random() < 0.8, pad=pad)


# ---- inputs ---------------------------------------------------------------------


def _rows(g, n, width, kind, pad, scale=1.0):
    """Normal values with a magnitude of its own for each row (a few rows are zero), inside rows of width + pad."""
    t = torch.empty((n, width + pad), dtype=TYPES[kind], device="cuda")
    size = torch.exp2(torch.randn((n, 1), generator=g, device="cuda")) * scale
    size *= torch.rand((n, 1), generator=g, device="cuda") >= 1 / 64
    step = max(1, (1 << 26) // (width + pad))
    for i in range(0, n, step):
        m = min(step, n - i)
        t[i : i + m] = torch.randn((m, width + pad), generator=g, device="cuda") * size[i : i + m]
    return t[:, :width]


def _inputs(case, seed):
    """The tensors that both forms and the 64-bit results start from."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)
    if case["op"] == "linear":
        x = _rows(g, case["n"], case["n_in"], case["x"], case["pad"])
        W = torch.randn((case["n_out"], case["n_in"]), generator=g, device="cuda") * math.sqrt(2 / case["n_in"])
        b = (torch.rand(case["n_out"], generator=g, device="cuda") - 0.5) * (2 / math.sqrt(case["n_in"])) if case["bias"] else None
        return x, W, b
    if case["op"] == "keep":
        return (_rows(g, case["n"], case["width"], case["z"], case["pad"]),)
    n, n_in, n_out = case["n"], case["n_in"], case["n_out"]
    blocks = -(-n_in // BLOCK)
    codes = torch.empty((n, blocks * BLOCK), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (blocks * BLOCK))
    for i in range(0, n, step):
        c = torch.randn((min(step, n - i), blocks * BLOCK), generator=g, device="cuda")
        c = (c * 80).clamp(0, 255) if case["relu"] else (c * 40).clamp(-127, 127) + 128
        codes[i : i + step] = c.round().to(torch.uint8)
    codes[:, n_in:] = 0 if case["relu"] else 128
    exps = (torch.randn((n, blocks), generator=g, device="cuda") * 1.5 + 120).round().clamp(100, 140).to(torch.uint8)
    dy = _rows(g, n, n_out, case["dy"], case["pad"], 1e-3)
    W = (torch.randn((n_out, n_in), generator=g, device="cuda") * math.sqrt(2 / n_in)).to(TYPES[case["dy"]])
    return dy, W, codes, exps


def prepare(case, seed):
    ins = _inputs(case, seed)
    if own:
        return _prepare_own(case, ins)
    if case["op"] != "linear":
        return {"case": case, "ins": ins}
    x, W, b = ins
    codes, scales = _codes_by_row(W)
    return {"case": case, "ins": (x, codes, scales, b)}


def run(state):
    if own:
        return _run_own(state)
    return {"linear": _linear, "keep": _keep, "backward": _backward}[state["case"]["op"]](state["case"], *state["ins"])


def _prepare_own(case, ins):
    """What a program keeps: the layer with its weights laid out, the kept activation's buffers, outputs and scratch memory."""
    from paper_2407_18352_amd import _abi, api

    act, new = _abi.ACT_RELU if case["relu"] else _abi.ACT_IDENTITY, dict(device="cuda")
    state = {"case": case, "api": api, "act": act}
    if case["op"] == "linear":
        x, W, b = ins
        layer = api.Linear8(W, b)
        y = torch.empty((case["n"], case["n_out"]), dtype=TYPES[case["y"]], **new)
        return dict(state, layer=layer, x=x, y=y, scratch=torch.empty(layer.scratch_bytes(case["n"]), dtype=torch.uint8, **new))
    if case["op"] == "keep":
        a, back = (torch.empty((case["n"], case["width"]), dtype=TYPES[case["a"]], **new) for _ in range(2))
        return dict(state, z=ins[0], a=a, back=back, kept=api.Checkpoint8(case["n"], case["width"], act))
    dy, W, codes, exps = ins
    kept = api.Checkpoint8(case["n"], case["n_in"], act, codes=codes, exps=exps)
    dw, db = torch.empty((case["n_out"], case["n_in"]), **new), torch.empty(case["n_out"], **new)
    dx = torch.empty((case["n"], case["n_in"]), dtype=dy.dtype, **new) if case["dx"] else None
    scratch = torch.empty(api.backward8_scratch_bytes(kept, dy, W if case["dx"] else None), dtype=torch.uint8, **new)
    return dict(state, kept=kept, dy=dy, W=W if case["dx"] else None, dw=dw, db=db, dx=dx, scratch=scratch)


def _run_own(s):
    api, op = s["api"], s["case"]["op"]
    if op == "linear":
        api.linear8(s["layer"], s["x"], s["y"], s["act"], scratch=s["scratch"])
        return {"y": s["y"]}
    if op == "keep":
        api.checkpoint8_save(s["kept"], s["z"], s["a"])
        api.checkpoint8_load(s["kept"], s["back"])
        return {"a": s["a"], "back": s["back"]}
    api.backward8(s["kept"], s["dy"], s["dw"], s["db"], W=s["W"], dx=s["dx"], scratch=s["scratch"])
    return {"dw": s["dw"], "db": s["db"]} | ({"dx": s["dx"]} if s["dx"] is not None else {})


# ---- plain forms, in 32 bits --------------------------------------------------------


def _codes_by_row(v):
    """Codes (whole numbers held in 32-bit floats) and the scale of each row."""
    v = v.float()
    most = v.abs().amax(dim=1, keepdim=True)
    live = most >= 2.0 ** -119  # below that a row counts as zeros
    inv = torch.where(live, torch.full_like(most, 127.0) / most, torch.zeros_like(most))
    scale = torch.where(live, most / torch.full_like(most, 127.0), torch.zeros_like(most))
    return torch.round(v * inv), scale


def _linear(case, x, w_codes, w_scales, b):
    codes, scales = _codes_by_row(x)
    y = (codes @ w_codes.t()) * scales * w_scales.t()
    if b is not None:
        y = y + b
    if case["relu"]:
        y = torch.where(y < 0, torch.zeros_like(y), y)
    return {"y": y.to(TYPES[case["y"]])}


def _value(codes, exps, relu, width):
    """What codes and exponents stand for."""
    c = codes.float().unflatten(1, (-1, BLOCK))
    if not relu:
        c = c - 128
    return torch.ldexp(c, exps.unsqueeze(2).to(torch.int32) - 127).flatten(1)[:, :width]


def _keep(case, z):
    a, relu = z.float(), case["relu"]
    if relu:
        a = torch.where(a < 0, torch.zeros_like(a), a)
    blocks = torch.nn.functional.pad(a, (0, -case["width"] % BLOCK)).unflatten(1, (-1, BLOCK))
    top = 255 if relu else 127
    e = torch.frexp(blocks.abs().amax(dim=2))[1] - (8 if relu else 7)
    e = torch.clamp(e, min=-126)
    c = torch.round(torch.ldexp(blocks, -e.unsqueeze(2))).clamp(-top, top)
    if relu:
        c = torch.where((blocks > 0) & (c < 1), torch.ones_like(c), c)
    codes = (c if relu else c + 128).to(torch.uint8).flatten(1)
    exps = (e + 127).to(torch.uint8)
    out = TYPES[case["a"]]
    return {"a": a.to(out), "back": _value(codes, exps, relu, case["width"]).to(out)}


def _backward(case, dy, W, codes, exps):
    a, g = _value(codes, exps, case["relu"], case["n_in"]), dy.float()
    out = {"dw": g.t().contiguous() @ a, "db": g.sum(dim=0)}
    if case["dx"]:
        dx = g @ W.float()
        if case["relu"]:
            dx = torch.where(codes[:, : case["n_in"]] != 0, dx, torch.zeros_like(dx))
        out["dx"] = dx.to(dy.dtype)
    return out


# ---- work, and results in 64 bits ----------------------------------------------------


def work(case):
    """Each tensor read or written once; two operations for each product and sum of the matrix products, a few for each value kept."""
    size, n = {"f32": 4, "bf16": 2}, case["n"]
    if case["op"] == "linear":
        i, o = case["n_in"], case["n_out"]
        return {"bytes": n * i * size[case["x"]] + n * o * size[case["y"]] + i * o + 4 * o * (2 if case["bias"] else 1), "flops": 2 * n * i * o}
    if case["op"] == "keep":
        v, e = n * case["width"], n * -(-case["width"] // BLOCK)
        return {"bytes": v * (size[case["z"]] + 2 * size[case["a"]] + 2) + 2 * e, "flops": 6 * v}
    i, o, s = case["n_in"], case["n_out"], size[case["dy"]]
    more = (o * i * s + n * i * s, 2 * n * i * o) if case["dx"] else (0, 0)
    return {"bytes": n * (o * s + i + -(-i // BLOCK)) + 4 * o * (i + 1) + more[0], "flops": 2 * n * i * o + n * o + more[1]}


def exact(case, seed):
    ins = _inputs(case, seed)
    if case["op"] == "linear":
        x, W, b = ins

        def halves(v):
            m = v.double().abs().max(1).values[:, None]
            m = m.masked_fill(m == 0, 1.0)
            return torch.round(127 * v.double() / m), m / 127

        (q, s), (w, t) = halves(x), halves(W)
        y = torch.matmul(q, w.T.contiguous()).mul_(s).mul_(t.T)
        if b is not None:
            y += b.double()
        return {"y": y.clamp_(min=0) if case["relu"] else y}
    if case["op"] == "keep":
        n, width = case["n"], case["width"]
        bits, back, full = (8 if case["relu"] else 7), [], []
        for rows in ins[0].split(max(1, (1 << 26) // width)):
            a = rows.double()
            if case["relu"]:
                a = a.clamp(min=0)
            kept = torch.empty_like(a)
            for k in range(0, width, BLOCK):
                part = a[:, k : k + BLOCK]
                m = part.abs().max(1).values
                step = torch.exp2(torch.floor(torch.log2(m.masked_fill(m == 0, 1.0))) + 1 - bits)[:, None]
                c = torch.round(part / step).clamp(-(2**bits - 1), 2**bits - 1)
                if case["relu"]:
                    c[(part > 0) & (c == 0)] = 1
                kept[:, k : k + BLOCK] = c * step
            full.append(a)
            back.append(kept)
        return {"a": torch.cat(full), "back": torch.cat(back)}
    dy, W, codes, exps = ins
    n_in, g = case["n_in"], dy.double()
    a = codes.double()
    if not case["relu"]:
        a -= 128
    a = (a * torch.exp2(exps.double() - 127).repeat_interleave(BLOCK, dim=1))[:, :n_in]
    out = {"dw": torch.matmul(g.T.contiguous(), a), "db": g.sum(0)}
    if case["dx"]:
        out["dx"] = torch.matmul(g, W.double())
        if case["relu"]:
            out["dx"][codes[:, :n_in] == 0] = 0
    return out

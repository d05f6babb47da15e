"""What a block's training step and its 8-bit serving add to its linear layers and
norms, with their plain forms.

A case is one pass of one operator as a program that trains or serves such a
block calls it: numbers cut to 8-bit floating point with a scale for each block
of 128, the linear layer of such operands, the two norms around a block fused
with its gate, its residual scale and the addition between them, their gradients,
and the clipping of all gradients by their common norm.  Inputs are synthetic and
made on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EIGHT = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
BLOCK = 128
TINY = 2.0 ** -126  # the smallest scale
EPS = 1e-5          # of the norms
CLIP_EPS = 1e-6     # added to the gradients' norm
MOST_FLOPS = 1.2e12  # of a drawn case: about the largest listed one's
MOST_BYTES = 1.7e9


# ------------------------------------------------------------------- the cases

def _quantize(name, rows, cols, dtype, block_rows, eight="e4m3", **more):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype,
            "block_rows": block_rows, "eight": eight, "transposed": False, "pitch": 0, **more}


def _linear(name, rows, inner, outer, dtype, act, **more):
    """rows x inner times outer x inner, both in 8 bits"""
    return {"name": name, "op": "linear", "rows": rows, "inner": inner, "outer": outer,
            "dtype": dtype, "act": act, "bias": True, "residual": False, "pre": False,
            "pitch": 0, "eight": "e4m3", "weight_rows": BLOCK, **more}


def _norm(name, rows, width, dtype, kind, **more):
    return {"name": name, "op": "norm", "rows": rows, "width": width, "dtype": dtype,
            "kind": kind, "weights": "f32", "bias": kind == "layer", "post": False, "groups": 0,
            "scale": 1.0, "pitch": 0, **more}


def _clip(name, layers, hidden, inner, dtype, **more):
    return {"name": name, "op": "clip", "layers": layers, "hidden": hidden, "inner": inner,
            "dtype": dtype, "kind": "2", "clipped": True, "pitch": 0, **more}


def listed():
    return [
        # a few tokens' activations before a decode step's product, odd sizes
        _quantize("quantize_few_odd", 29, 1021, "f16", 1, pitch=11),
        # a batch's activations for training: as rows for the layer, as columns
        # for the gradient of its weight
        _quantize("quantize_both", 8192, 4096, "bf16", 1, transposed=True),
        # one token of one sequence: the weight is read once and nothing else counts
        _linear("fp8_token", 1, 4096, 4096, "bf16", "none", residual=True),
        # a few sequences decoded together, odd sizes
        _linear("fp8_decode_odd", 29, 1021, 4099, "f16", "silu", pitch=11),
        # the first product of a block over a long prompt, its pre-activation kept
        _linear("fp8_prompt", 8192, 4096, 16384, "bf16", "gelu_tanh", pre=True),
        # the gradient of that product's weight: both operands scaled row by row
        _linear("fp8_weight_gradient", 16384, 8192, 4096, "bf16", "none", bias=False,
                eight="e5m2", weight_rows=1),
        # one token between two blocks
        _norm("residual_norm_token", 1, 4096, "bf16", "rms"),
        # a batch of prompts: the block's output normed, scaled by channel and added
        _norm("residual_norm_prompt", 32768, 4096, "bf16", "rms", post=True, groups=1, scale=0.5),
        # gradients in full precision at an odd width, a gate for each of 7 samples
        _norm("residual_norm_backward_odd", 5005, 1021, "f32", "layer", groups=7, op="norm_backward"),
        # gradients of the batch of prompts, a gate for each of 16 samples
        _norm("residual_norm_backward_prompt", 32768, 4096, "bf16", "rms", post=True, groups=16,
              op="norm_backward"),
        # the gradients of one small block
        _clip("clip_small", 1, 129, 515, "f32"),
        # the gradients of four wide blocks
        _clip("clip_layers", 4, 4096, 16384, "bf16"),
    ]


def _size(rng, lo, hi):
    """log-uniform; as often odd as it falls, as often a multiple of 64"""
    n = int(round(lo * (hi / lo) ** rng.random()))
    if rng.random() < 0.5 and n >= 64:
        n = n // 64 * 64
    return min(max(n, lo), hi)


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "norm", "norm_backward", "clip"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    eight = rng.choice(["e4m3", "e4m3", "e5m2"])
    while True:
        if op == "quantize":
            case = _quantize("", _size(rng, 1, 32768), _size(rng, 65, 16384), dtype,
                             rng.choice([1, 1, BLOCK]), eight, transposed=rng.random() < 0.5,
                             pitch=rng.choice([0, 0, 8, 5]))
        elif op == "linear":
            case = _linear("", _size(rng, 1, 16384), _size(rng, 65, 8192), _size(rng, 65, 16384),
                           rng.choice(["bf16", "f16"]),
                           rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                           bias=rng.random() < 0.7, residual=rng.random() < 0.5,
                           pre=rng.random() < 0.4, pitch=rng.choice([0, 0, 16, 5]), eight=eight,
                           weight_rows=rng.choice([BLOCK, BLOCK, 1]))
        elif op.startswith("norm"):
            groups = rng.choice([0, 1, 1, 3, 16])
            each = max(groups, 1)  # rows come as samples of one length
            case = _norm("", -(-_size(rng, 1, 65536) // each) * each, _size(rng, 65, 16384), dtype,
                         rng.choice(["rms", "layer"]), weights=rng.choice(["f32", dtype]),
                         post=rng.random() < 0.5, groups=groups, scale=rng.choice([1.0, 0.5]),
                         pitch=rng.choice([0, 0, 8, 5]), op=op)
        else:
            case = _clip("", rng.choice([1, 2, 4, 8]), _size(rng, 65, 4096), _size(rng, 65, 16384),
                         dtype, kind=rng.choice(["2", "2", "inf"]), clipped=rng.random() < 0.7,
                         pitch=rng.choice([0, 0, 5]))
        w = work(case)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            del case["name"]
            return case


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "quantize":
        m, n = case["rows"], case["cols"]
        scales = _blocks(n) * (m if case["block_rows"] == 1 else _blocks(m))
        scales_t = _blocks(m) * (n if case["block_rows"] == 1 else _blocks(n))
        both = 1 + case["transposed"]
        return {"bytes": (e + both) * m * n + 4 * (scales + scales_t * case["transposed"]),
                "flops": 2 * both * m * n}
    if case["op"] == "linear":
        m, k, n = case["rows"], case["inner"], case["outer"]
        scales = _blocks(k) * (m + (n if case["weight_rows"] == 1 else _blocks(n)))
        b = m * n * (1 + case["residual"] + case["pre"]) + n * case["bias"]
        return {"bytes": m * k + n * k + 4 * scales + e * b, "flops": 2 * m * n * k}
    if case["op"].startswith("norm"):
        m, n, we = case["rows"], case["width"], BYTES[case["weights"]]
        vectors = (1 + case["bias"]) * (1 + case["post"]) + case["groups"]
        stats = 4 * m * (1 + (case["kind"] == "layer")) * (1 + case["post"])
        if case["op"] == "norm":
            return {"bytes": e * 4 * m * n + we * vectors * n + stats, "flops": 16 * m * n}
        return {"bytes": e * 6 * m * n + we * 2 * vectors * n + stats, "flops": 30 * m * n}
    count = case["layers"] * (2 * case["hidden"] * case["inner"] + case["hidden"] + case["inner"])
    norms = case["layers"] * 2 * case["hidden"]
    return {"bytes": 2 * (e * count + 4 * norms), "flops": 3 * (count + norms)}


# ------------------------------------------------------------------ the inputs

def _normal(gen, shape, scale, dtype):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _activations(gen, rows, cols, pitch=0):
    """rows of different size with a few loud channels, `pitch` values of another
    tensor between them"""
    x = torch.randn((rows, cols + pitch), generator=gen, device="cuda")
    loud = torch.randint(0, cols, (max(1, cols // 256),), generator=gen, device="cuda")
    x[:, loud] *= 20.0
    x *= torch.rand((rows, 1), generator=gen, device="cuda") * 2 + 0.5
    return x


def _quantized(x, block_rows, eight):
    """x cut to 8 bits, and its scales"""
    rows, cols = x.shape
    wide = torch.zeros((-(-rows // block_rows) * block_rows, _blocks(cols) * BLOCK), device="cuda")
    wide[:rows, :cols] = x
    blocks = wide.view(-1, block_rows, _blocks(cols), BLOCK)
    scale = (blocks.abs().amax((1, 3)) / LARGEST[eight]).clamp(min=TINY)
    q = (blocks / scale[:, None, :, None]).clamp(-LARGEST[eight], LARGEST[eight]).to(EIGHT[eight])
    return q.view(wide.shape)[:rows, :cols], scale


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    if case["op"] == "quantize":
        x = _activations(gen, case["rows"], case["cols"], case["pitch"])
        return {"x": x.to(dt)[:, :case["cols"]]}
    if case["op"] == "linear":
        m, k, n = case["rows"], case["inner"], case["outer"]
        x, s = _quantized(_activations(gen, m, k), 1, case["eight"])
        wide = torch.empty((m, k + case["pitch"]), dtype=x.dtype, device="cuda")
        # (the bytes behind a row: NaN in both formats)
        wide.view(torch.uint8).fill_(0x7f)
        wide[:, :k] = x
        weight = torch.randn((n, k), generator=gen, device="cuda") / math.sqrt(k)
        w, ws = _quantized(weight, case["weight_rows"], "e4m3")
        return {"x": wide[:, :k], "x_scale": s, "weight": w.contiguous(), "weight_scale": ws,
                "bias": _normal(gen, (n,), 0.2, dt) if case["bias"] else None,
                "residual": _normal(gen, (m, n), 1.0, dt) if case["residual"] else None}
    if case["op"].startswith("norm"):
        m, n, wt = case["rows"], case["width"], DTYPES[case["weights"]]

        def vector(mean, shape=(n,)):
            return (mean + 0.2 * torch.randn(shape, generator=gen, device="cuda")).to(wt)

        # the residual stream, and a block's output
        h = (_activations(gen, m, n, case["pitch"]) + 0.3).to(dt)[:, :n]
        y = _normal(gen, (m, n), 1.5, dt)
        s = {"residual": h, "branch": y, "weight": vector(1.0),
             "bias": vector(0.0) if case["bias"] else None,
             "post_weight": vector(1.0) if case["post"] else None,
             "post_bias": vector(0.0) if case["post"] and case["bias"] else None,
             "gate": vector(0.5, (n,) if case["groups"] == 1 else (case["groups"], n))
             if case["groups"] else None}
        if case["op"] == "norm_backward":
            s["d_normed"] = _normal(gen, (m, n), 0.1, dt)
            s["d_residual"] = _normal(gen, (m, n), 0.1, dt)
            s["stats"] = (*_statistics(h.float(), case["kind"]),
                          *(_statistics(y.float(), case["kind"]) if case["post"] else (None, None)))
        return s
    h, n = case["hidden"], case["inner"]
    count = case["layers"] * (2 * h * n + h + n)
    norm = (10.0 if case["clipped"] else 0.5) if case["kind"] == "2" else (40.0 if case["clipped"] else 0.5)
    scale = norm / math.sqrt(count) if case["kind"] == "2" else norm / 8
    gradients = []
    for _ in range(case["layers"]):
        gradients += [_normal(gen, (n, h + case["pitch"]), scale, dt)[:, :h], _normal(gen, (n,), scale, dt),
                      _normal(gen, (h, n), scale, dt), _normal(gen, (h,), scale, dt),
                      _normal(gen, (h,), scale, torch.float32), _normal(gen, (h,), scale, torch.float32)]
    return {"gradients": gradients}


def _statistics(x, kind):
    """mean (none of an rms norm) and 1 / sqrt of each row"""
    mean = x.mean(1) if kind == "layer" else None
    centred = x if mean is None else x - mean[:, None]
    return mean, 1 / torch.sqrt((centred * centred).mean(1) + EPS)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        # the buffers that a training or serving loop keeps
        import paper_2512_08365_amd as mag
        s["mag"] = mag
        size = 0
        if case["op"] == "quantize":
            s["out"] = mag.quantize_fp8(s["x"], case["block_rows"], dtype=EIGHT[case["eight"]],
                                        transposed=case["transposed"])
        elif case["op"] == "linear":
            dt, shape = DTYPES[case["dtype"]], (case["rows"], case["outer"])
            s["out"] = torch.empty(shape, dtype=dt, device="cuda")
            s["pre_out"] = torch.empty(shape, dtype=dt, device="cuda") if case["pre"] else None
            size = mag.linear_fp8_workspace_size(s["x"], s["weight"])
        elif case["op"] == "norm":
            s["out"] = tuple(torch.empty((case["rows"], case["width"]), dtype=s["branch"].dtype,
                                         device="cuda") for _ in range(2))
            m = case["rows"]
            one = [torch.empty(m, device="cuda") if case["kind"] == "layer" else None,
                   torch.empty(m, device="cuda")]
            two = [torch.empty(m, device="cuda") if case["kind"] == "layer" else None,
                   torch.empty(m, device="cuda")] if case["post"] else [None, None]
            s["stats"] = (*one, *two)
        elif case["op"] == "norm_backward":
            s["out"] = tuple(None if x is None else torch.empty(x.shape, dtype=x.dtype, device="cuda")
                             for x in (s["residual"], s["branch"], s["gate"], s["weight"], s["bias"],
                                       s["post_weight"], s["post_bias"]))
            size = mag.residual_norm_backward_workspace_size(s["residual"], s["gate"])
        else:
            # clipped gradients lie behind one another, a buffer for each type
            s["flat"] = {ty: torch.empty(sum(g.numel() for g in s["gradients"] if g.dtype is ty),
                                         dtype=ty, device="cuda") for ty in {g.dtype for g in s["gradients"]}}
            at, outs = dict.fromkeys(s["flat"], 0), []
            for g in s["gradients"]:
                outs.append(s["flat"][g.dtype][at[g.dtype]:at[g.dtype] + g.numel()].view(g.shape))
                at[g.dtype] += g.numel()
            s["list"] = mag.TensorList(s["gradients"], out=outs)
            s["norm"] = torch.empty((), device="cuda")
            size = mag.clip_gradients_workspace_size(s["list"])
        s["workspace"] = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------- the calls

def run(state):
    case = state["case"]
    return (_run_own if own else _run_plain)(case["op"], case, state)


def _present(**outputs):
    return {k: v for k, v in outputs.items() if v is not None}


def _run_own(op, case, s):
    mag = s["mag"]
    if op == "quantize":
        return mag.quantize_fp8(s["x"], case["block_rows"], dtype=EIGHT[case["eight"]],
                                transposed=case["transposed"], out=s["out"])
    if op == "linear":
        return mag.linear_fp8(s["x"], s["x_scale"], s["weight"], s["weight_scale"], s["bias"],
                              s["residual"], activation=case["act"], pre=s["pre_out"],
                              out=s["out"], workspace=s["workspace"])
    if op == "norm":
        out, normed, stats = mag.residual_norm(
            s["residual"], s["branch"], s["weight"], s["bias"], kind=case["kind"], gate=s["gate"],
            scale=case["scale"], post=case["post"], post_weight=s["post_weight"],
            post_bias=s["post_bias"], eps=EPS, statistics=s["stats"], out=s["out"])
        return _present(residual=out, normed=normed, **dict(zip(("mean", "rstd", "post_mean", "post_rstd"), stats)))
    if op == "norm_backward":
        got = mag.residual_norm_backward(
            s["residual"], s["branch"], s["d_normed"], s["d_residual"], s["stats"], s["weight"], s["bias"],
            kind=case["kind"], gate=s["gate"], scale=case["scale"], post=case["post"],
            post_weight=s["post_weight"], post_bias=s["post_bias"], out=s["out"],
            workspace=s["workspace"])
        return _present(**dict(zip(("residual", "branch", "gate", "weight", "bias", "post_weight", "post_bias"), got)))
    mag.clip_gradients(s["list"], 1.0, kind=math.inf if case["kind"] == "inf" else 2, eps=CLIP_EPS,
                       norm=s["norm"], workspace=s["workspace"])
    return {"norm": s["norm"], **{str(ty): flat for ty, flat in s["flat"].items()}}


# -------------------------------------------------------------- the plain forms

def _act(z, kind):
    if kind == "relu":
        return torch.clamp(z, min=0.0)
    if kind == "gelu":
        return z * 0.5 * (1 + torch.erf(z / math.sqrt(2.0)))
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _values(q, scale):
    """what 8-bit numbers and their scales stand for"""
    rows, cols = q.shape
    if scale.shape[0] != rows:
        scale = scale.repeat_interleave(BLOCK, 0)[:rows]
    return q.float() * scale.repeat_interleave(BLOCK, 1)[:, :cols]


def _run_plain(op, case, s):
    if op == "quantize":
        q, scale = _quantized(s["x"].float(), case["block_rows"], case["eight"])
        if not case["transposed"]:
            return q, scale
        if case["block_rows"] != 1:
            return q, scale, q.t(), scale.t()
        return q, scale, *_quantized(s["x"].float().t(), 1, case["eight"])
    if op == "linear":
        dt = DTYPES[case["dtype"]]
        z = _values(s["x"], s["x_scale"]) @ _values(s["weight"], s["weight_scale"]).t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return (y.to(dt), z.to(dt)) if case["pre"] else y.to(dt)
    if op == "norm":
        return _plain_norm(case, s)
    if op == "norm_backward":
        return _plain_norm_backward(case, s)
    gradients = [g.float() for g in s["gradients"]]
    if case["kind"] == "inf":
        norm = torch.stack([g.abs().amax() for g in gradients]).amax()
    else:
        norm = torch.sqrt(torch.stack([(g * g).sum(dtype=torch.float64) for g in gradients]).sum()).float()
    by = torch.clamp(1.0 / (norm + CLIP_EPS), max=1.0)
    return {"norm": norm, **{str(ty): torch.cat([(g * by).to(ty).reshape(-1) for g, x in
                                                 zip(gradients, s["gradients"]) if x.dtype is ty])
                             for ty in {g.dtype for g in s["gradients"]}}}


def _normed(x, mean, rstd):
    return (x if mean is None else x - mean[:, None]) * rstd[:, None]


def _affine(x, weight, bias):
    x = x * weight.float()
    return x if bias is None else x + bias.float()


def _by_row(gate, rows):
    """the gate of each row (of one: itself)"""
    if gate is None:
        return 1.0
    gate = gate.float()
    return gate if gate.dim() == 1 else gate.repeat_interleave(rows // gate.shape[0], 0)


def _plain_norm(case, s):
    h, y = s["residual"].float(), s["branch"].float()
    post = (None, None)
    if case["post"]:
        post = _statistics(y, case["kind"])
        y = _affine(_normed(y, *post), s["post_weight"], s["post_bias"])
    out = (h + case["scale"] * _by_row(s["gate"], h.shape[0]) * y).to(s["branch"].dtype)
    stats = _statistics(out.float(), case["kind"])
    normed = _affine(_normed(out.float(), *stats), s["weight"], s["bias"]).to(out.dtype)
    return _present(residual=out, normed=normed,
                    **dict(zip(("mean", "rstd", "post_mean", "post_rstd"), (*stats, *post))))


def _norm_slope(h, x_hat, rstd, kind):
    """the gradient of a norm's input from that of its normed rows"""
    d = h - x_hat * (h * x_hat).mean(1, keepdim=True)
    if kind == "layer":
        d = d - h.mean(1, keepdim=True)
    return rstd[:, None] * d


def _plain_norm_backward(case, s):
    dt, wt, kind = s["branch"].dtype, s["weight"].dtype, case["kind"]
    mean, rstd, post_mean, post_rstd = s["stats"]
    dn, rows = s["d_normed"].float(), s["branch"].shape[0]
    x_hat = _normed(s["residual"].float(), mean, rstd)
    g = s["d_residual"].float() + _norm_slope(dn * s["weight"].float(), x_hat, rstd, kind)
    b = case["scale"] * _by_row(s["gate"], rows) * g
    y, y_hat, d_branch, d_post_weight, d_post_bias, d_gate = s["branch"].float(), None, b, None, None, None
    if case["post"]:
        y_hat = _normed(y, post_mean, post_rstd)
        y = _affine(y_hat, s["post_weight"], s["post_bias"])
        d_branch = _norm_slope(b * s["post_weight"].float(), y_hat, post_rstd, kind)
        d_post_weight = (b * y_hat).sum(0).to(wt)
        d_post_bias = None if s["post_bias"] is None else b.sum(0).to(wt)
    if s["gate"] is not None:
        d_gate = (case["scale"] * g * y).view(max(case["groups"], 1), -1, y.shape[1]).sum(1)
        d_gate = d_gate.view(s["gate"].shape).to(s["gate"].dtype)
    return _present(residual=g.to(dt), branch=d_branch.to(dt), gate=d_gate,
                    weight=(dn * x_hat).sum(0).to(wt),
                    bias=None if s["bias"] is None else dn.sum(0).to(wt),
                    post_weight=d_post_weight, post_bias=d_post_bias)


# --------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    return {"quantize": _exact_quantize, "linear": _exact_linear, "norm": _exact_norm,
            "norm_backward": _exact_norm_backward, "clip": _exact_clip}[case["op"]](case, s)


def _exact_eight(v, eight):
    """v rounded to the nearest number of the format, ties to even"""
    bits, least = (3, -6) if eight == "e4m3" else (2, -14)
    exponent = torch.frexp(v)[1].to(torch.float64) - 1
    step = torch.exp2(torch.clamp(exponent, min=least) - bits)
    return torch.clamp(torch.round(v / step) * step, -LARGEST[eight], LARGEST[eight])


def _exact_cut(x, rows_a_block, eight):
    m, n = x.shape
    row = torch.arange(m, device="cuda") // rows_a_block
    most = torch.zeros((int(row[-1]) + 1, n), dtype=torch.float64, device="cuda")
    most.scatter_reduce_(0, row[:, None].expand(m, n), x.abs(), "amax")
    most = torch.nn.functional.pad(most, (0, -n % BLOCK)).unflatten(1, (-1, BLOCK)).amax(2)
    scale = torch.clamp(most / LARGEST[eight], min=TINY)
    column = torch.arange(n, device="cuda") // BLOCK
    return _exact_eight(x / scale[row][:, column], eight), scale


def _exact_quantize(case, s):
    x = s["x"].double()
    got = _exact_cut(x, case["block_rows"], case["eight"])
    if not case["transposed"]:
        return got
    if case["block_rows"] == 1:
        return (*got, *_exact_cut(x.t().contiguous(), 1, case["eight"]))
    return (*got, got[0].t(), got[1].t())


def _exact_linear(case, s):
    k = torch.arange(case["inner"], device="cuda") // BLOCK
    n = torch.arange(case["outer"], device="cuda") // case["weight_rows"]
    x = s["x"].double().mul_(s["x_scale"].double()[:, k])
    w = s["weight"].double().mul_(s["weight_scale"].double()[n][:, k])
    z = torch.mm(x, w.t())
    if s["bias"] is not None:
        z += s["bias"].double()
    if case["act"] == "relu":
        y = torch.where(z > 0, z, torch.zeros_like(z))
    elif case["act"] == "gelu":
        y = z * torch.erfc(-z / math.sqrt(2)) / 2
    elif case["act"] == "gelu_tanh":
        y = z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    elif case["act"] == "silu":
        y = z * torch.sigmoid(z)
    else:
        y = z
    if s["residual"] is not None:
        y = y + s["residual"].double()
    return (y, z) if case["pre"] else y


def _exact_moments(x, kind):
    if kind == "rms":
        return None, torch.rsqrt(x.square().mean(1) + EPS)
    variance, mean = torch.var_mean(x, 1, correction=0)
    return mean, torch.rsqrt(variance + EPS)


def _exact_hat(x, mean, rstd):
    return (x if mean is None else x - mean.double()[:, None]) * rstd.double()[:, None]


def _exact_gated(case, s, rows):
    """scale times gate, a row of it for each row"""
    if s["gate"] is None:
        return torch.full((1, 1), case["scale"], dtype=torch.float64, device="cuda")
    gate = s["gate"].double().reshape(-1, case["width"]) * case["scale"]
    return gate[torch.arange(rows, device="cuda") * gate.shape[0] // rows]


def _exact_norm(case, s):
    h, y = s["residual"].double(), s["branch"].double()
    post = (None, None)
    if case["post"]:
        post = _exact_moments(y, case["kind"])
        y = _exact_hat(y, *post) * s["post_weight"].double()
        if s["post_bias"] is not None:
            y += s["post_bias"].double()
    # (the second norm reads the sum as it is stored: the nearest number of its type)
    out = h + _exact_gated(case, s, h.shape[0]) * y
    stored = out.to(s["branch"].dtype).double()
    moments = _exact_moments(stored, case["kind"])
    normed = _exact_hat(stored, *moments) * s["weight"].double()
    if s["bias"] is not None:
        normed += s["bias"].double()
    found = {"residual": out, "normed": normed, "mean": moments[0], "rstd": moments[1],
             "post_mean": post[0], "post_rstd": post[1]}
    return {k: v for k, v in found.items() if v is not None}


def _exact_norm_backward(case, s):
    mean, rstd, post_mean, post_rstd = s["stats"]
    rows, width = s["branch"].shape
    centre = case["kind"] == "layer"

    def through(d, hat, r):
        along = (d * hat).sum(1, keepdim=True) / width
        rest = d.sum(1, keepdim=True) / width if centre else 0.0
        return (d - rest - hat * along) * r.double()[:, None]

    hat = _exact_hat(s["residual"].double(), mean, rstd)
    dn = s["d_normed"].double()
    found = {"weight": torch.sum(dn * hat, 0), "bias": dn.sum(0) if s["bias"] is not None else None}
    g = through(dn * s["weight"].double(), hat, rstd) + s["d_residual"].double()
    del hat, dn
    d = _exact_gated(case, s, rows) * g
    y = s["branch"].double()
    if case["post"]:
        post_hat = _exact_hat(y, post_mean, post_rstd)
        found["post_weight"] = (d * post_hat).sum(0)
        found["post_bias"] = d.sum(0) if s["post_bias"] is not None else None
        y = post_hat * s["post_weight"].double()
        if s["post_bias"] is not None:
            y += s["post_bias"].double()
        d = through(d * s["post_weight"].double(), post_hat, post_rstd)
    if s["gate"] is not None:
        groups = s["gate"].numel() // width
        found["gate"] = torch.stack([(a * b).sum(0) * case["scale"] for a, b in
                                     zip(g.chunk(groups), y.chunk(groups))]).view(s["gate"].shape)
    found.update(residual=g, branch=d)
    return {k: v for k, v in found.items() if v is not None}


def _exact_clip(case, s):
    gradients = [g.double() for g in s["gradients"]]
    if case["kind"] == "inf":
        norm = max(g.abs().max().item() for g in gradients)
    else:
        norm = math.sqrt(math.fsum(torch.linalg.vector_norm(g).item() ** 2 for g in gradients))
    by = min(1.0, 1.0 / (norm + CLIP_EPS))
    found = {"norm": torch.tensor(norm, dtype=torch.float64)}
    for ty in {g.dtype for g in s["gradients"]}:
        found[str(ty)] = torch.cat([g.reshape(-1) * by for g, x in zip(gradients, s["gradients"])
                                    if x.dtype is ty])
    return found

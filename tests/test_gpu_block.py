"""The feed-forward block's operators against plain 64-bit forms of their
formulas, element by element, at the sizes, strides and values where they can
go wrong.

Tolerances (u: half a unit of the type's last place, relative; v = 2^-23).  A
product of two 8- or 11-bit numbers is exact in fp32; a sum of K of them is
taken 32 at a time by the matrix instruction and then added up, so it is off by
at most (K / 32 + 64) v of the sum of the magnitudes, and six times as many
additions in fp32, whose operands are cut in three with products below 2^-24
dropped twice.  An activation's slope is at most 1.13 and its evaluation costs
a few last places.  The gradients' products read dz rounded once: u of the sum
of magnitudes.  Every output is rounded once more: u of it."""
import math

import pytest

pytestmark = pytest.mark.gpu

V = 2.0 ** -23
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
TYPES = ["f32", "f16", "bf16"]


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    return torch


def _dt(name):
    torch = _torch()
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def _u(name):
    return {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[name]


def _tiny(name):
    """half the spacing of the subnormal numbers"""
    return {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -133}[name]


def _gen(seed):
    g = _torch().Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(gen, shape, scale, dt):
    return (_torch().randn(shape, generator=gen, device="cuda") * scale).to(dt)


def _layout(x, kind):
    """x's values in another layout: rows with a gap (odd, or keeping 16-byte
    rows), stored by columns, off the 16-byte grid, or every second element"""
    torch = _torch()
    r, c = x.shape
    if kind == "plain":
        return x
    if kind in ("gap", "gap8"):
        wide = torch.full((r, c + (5 if kind == "gap" else 8)), float("nan"), dtype=x.dtype,
                          device="cuda")
        wide[:, :c] = x
        return wide[:, :c]
    if kind == "columns":
        return x.t().contiguous().t()
    if kind == "shifted":
        flat = torch.full((r * c + 1,), float("nan"), dtype=x.dtype, device="cuda")
        flat[1:] = x.reshape(-1)
        return flat[1:].view(r, c)
    wide = torch.full((2 * r, 2 * c), float("nan"), dtype=x.dtype, device="cuda")
    wide[::2, ::2] = x
    return wide[::2, ::2]


def act64(z, kind):
    torch = _torch()
    if kind == "relu":
        return torch.clamp(z, min=0), (z > 0).double()
    if kind == "gelu":
        phi = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z ** 3))
        return (0.5 * z * (1 + t),
                0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z))
    if kind == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    return z, torch.ones_like(z)


def _close(got, want, bound, what):
    got, want = got.double(), want.double()
    assert got.shape == want.shape, what
    err = (got - want).abs()
    over = ~(err <= bound)
    assert not bool(over.any()), (
        f"{what}: {int(over.sum())} of {err.numel()} off, worst {float((err / bound).nan_to_num(float('inf')).max()):.3g} "
        f"times the bound, first {over.nonzero()[0].tolist()}")


def _sum_bound(k, ty):
    return ((6 if ty == "f32" else 1) * k / 32 + 64) * V + (2 * V if ty == "f32" else 0)


def check_linear(rows, inner, outer, ty, act="none", bias=True, residual=True, pre=True,
                 lx="plain", lw="plain", seed=1, wide_out=0):
    torch = _torch()
    import paper_2512_08365_amd as mag
    print(f"[case] linear {rows}x{inner}x{outer} {ty} {act} {lx} {lw}", flush=True)
    dt, g = _dt(ty), _gen(seed)
    x = _layout(_normal(g, (rows, inner), 1.0, dt), lx)
    w = _layout(_normal(g, (outer, inner), 1 / math.sqrt(max(inner, 1)), dt), lw)
    b = _normal(g, (outer,), 0.5, dt) if bias else None
    r = _normal(g, (rows, outer), 1.0, dt) if residual else None
    mark = 7.0
    out = torch.full((rows, outer + wide_out), mark, dtype=dt, device="cuda")
    keep = torch.full((rows, outer + wide_out), mark, dtype=dt, device="cuda")
    got = mag.linear(x, w, b, r, activation=act, out=out[:, :outer],
                     pre=keep[:, :outer] if pre else None)
    assert bool((out[:, outer:] == mark).all()) and bool((keep[:, outer:] == mark).all())
    y, z = got if pre else (got, None)
    x64, w64 = x.double(), w.double()
    z64 = torch.mm(x64, w64.t().contiguous())
    mag64 = torch.mm(x64.abs(), w64.abs().t().contiguous())
    if bias:
        z64 = z64 + b.double()
        mag64 = mag64 + b.double().abs()
    dz = _sum_bound(inner, ty) * mag64
    if pre:
        _close(z, z64, dz + _u(ty) * (z64.abs() + dz) + _tiny(ty), "pre")
    y64 = act64(z64, act)[0]
    dy = 1.13 * dz + 16 * V * (z64.abs() + y64.abs())
    if residual:
        y64 = y64 + r.double()
        dy = dy + V * y64.abs()
    _close(y, y64, dy + _u(ty) * (y64.abs() + dy) + _tiny(ty), "out")


SIZES = [(1, 1, 1), (1, 7, 5), (1, 64, 64), (1, 1000, 777), (2, 8, 16), (3, 4096, 40),
         (15, 33, 17), (16, 64, 256), (17, 65, 65), (31, 31, 500), (32, 512, 128), (33, 100, 129),
         (63, 63, 63), (64, 64, 64), (65, 200, 130), (100, 1024, 96), (127, 129, 255),
         (128, 128, 128), (129, 72, 257), (200, 328, 1000), (256, 256, 256), (257, 320, 511),
         (300, 1000, 16), (511, 16, 520), (1000, 96, 1000)]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_linear_sizes(size, ty):
    check_linear(*size, ty, act=ACTS[sum(size) % 5])


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [5, 150])
def test_linear_activations_and_epilogues(rows, act, ty):
    check_linear(rows, 136, 152, ty, act=act)
    check_linear(rows, 136, 152, ty, act=act, bias=False, residual=False, pre=False)
    check_linear(rows, 136, 151, ty, act=act, residual=False, wide_out=3)
    check_linear(rows, 136, 152, ty, act=act, bias=False, pre=False, wide_out=8)


LAYOUTS = ["plain", "gap", "gap8", "columns", "shifted", "every2"]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("lw", LAYOUTS)
@pytest.mark.parametrize("lx", LAYOUTS)
def test_linear_layouts(lx, lw, ty):
    check_linear(9, 200, 264, ty, act="silu", lx=lx, lw=lw)
    check_linear(136, 72, 80, ty, act="gelu", lx=lx, lw=lw)
    check_linear(130, 99, 133, ty, lx=lx, lw=lw)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("size", [(1, 8192, 8192), (4, 11008, 1032), (24, 4096, 4104),
                                  (48, 8200, 520), (96, 16384, 264), (700, 4096, 1111),
                                  (1536, 1536, 2048), (2050, 1030, 4100)],
                         ids=lambda s: "x".join(map(str, s)))
def test_linear_larger(size, ty):
    check_linear(*size, ty, act="gelu_tanh")


@pytest.mark.parametrize("ty", TYPES)
def test_linear_empty(ty):
    torch = _torch()
    import paper_2512_08365_amd as mag
    dt = _dt(ty)
    new = dict(dtype=dt, device="cuda")
    assert mag.linear(torch.empty(0, 16, **new), torch.ones(8, 16, **new)).shape == (0, 8)
    assert mag.linear(torch.ones(4, 16, **new), torch.empty(0, 16, **new)).shape == (4, 0)
    b = torch.arange(-4, 4, **new)
    y, z = mag.linear(torch.empty(3, 0, **new), torch.empty(8, 0, **new), b,
                      torch.ones(3, 8, **new), activation="relu", pre=True)
    assert torch.equal(z, b.expand(3, 8)) and torch.equal(y, b.clamp(min=0).expand(3, 8) + 1)
    dx, dw, db = mag.linear_backward(torch.empty(0, 16, **new), torch.ones(8, 16, **new),
                                     torch.empty(0, 8, **new))
    assert dx.shape == (0, 16) and not bool(dw.any()) and not bool(db.any())
    dx, dw, db = mag.linear_backward(torch.empty(3, 0, **new), torch.empty(8, 0, **new),
                                     torch.ones(3, 8, **new))
    assert dw.shape == (8, 0) and torch.equal(db, torch.full((8,), 3.0, **new))
    dx, dw, db = mag.linear_backward(torch.ones(3, 16, **new), torch.empty(0, 16, **new),
                                     torch.empty(3, 0, **new))
    assert not bool(dx.any()) and dx.shape == (3, 16) and dw.shape == (0, 16)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows", [3, 70])
def test_linear_broadcast_inputs_and_leading_dimensions(rows, ty):
    torch = _torch()
    import paper_2512_08365_amd as mag
    dt, g = _dt(ty), _gen(5)
    x = _normal(g, (1, 96), 1.0, dt)
    w = _normal(g, (104, 96), 0.1, dt)
    r = _normal(g, (104,), 1.0, dt).expand(rows, 104)
    one = mag.linear(x, w, None, r[:1].contiguous())
    many = mag.linear(x.expand(rows, 96), w, None, r)
    _close(many, one.expand(rows, 104), 2 * _u(ty) * one.double().abs() + 1e-5, "broadcast")
    y = mag.linear(_normal(g, (2, rows, 96), 1.0, dt), w)
    assert y.shape == (2, rows, 104)
    assert mag.linear(x[0], w).shape == (104,)
    # a gradient as sum() hands it back: one value for every element
    xs = _normal(g, (rows, 96), 1.0, dt)
    dy = torch.ones((), dtype=dt, device="cuda").expand(rows, 104)
    a = mag.linear_backward(xs, w, dy)
    b = mag.linear_backward(xs, w, dy.contiguous())
    for p, q, name in zip(a, b, ("dx", "dweight", "dbias")):
        _close(p, q, 4 * _u(ty) * q.double().abs() + 1e-4, name)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows", [2, 40, 300])
def test_linear_not_finite_values_stay_in_their_rows(rows, ty):
    torch = _torch()
    import paper_2512_08365_amd as mag
    dt, g = _dt(ty), _gen(6)
    x = _normal(g, (rows, 130), 1.0, dt)
    w = _normal(g, (70, 130), 0.1, dt)
    w[3, 7] = 0.0
    w[5] = 0.5  # (exact in one part)
    ref = mag.linear(x, w)
    bad = x.clone()
    bad[0, 7] = float("inf")
    bad[1, 9] = float("nan")
    y = mag.linear(bad, w)
    want = torch.mm(bad.double(), w.double().t().contiguous())
    assert torch.equal(y[2:], ref[2:])
    assert bool(torch.isnan(y[1]).all())
    assert torch.equal(torch.isnan(y[0]), torch.isnan(want[0]))  # inf times 0 alone
    assert torch.equal(y[0][torch.isinf(want[0])].double(), want[0][torch.isinf(want[0])])
    if ty == "f32":
        # the largest numbers keep their sign and size, sums that overflow are infinite
        big = torch.full((rows, 130), 0.0, device="cuda")
        big[:, 0] = 3.3e38
        ww = torch.zeros(70, 130, device="cuda")
        ww[:, 0] = 1.0
        ww[1, 0] = -1.0
        ww[2, 0] = 4.0
        y = mag.linear(big, ww)
        assert bool((y[:, 0] == 3.3e38).all()) and bool((y[:, 1] == -3.3e38).all())
        assert bool(torch.isposinf(y[:, 2]).all())


# fp32 products of many tiles, which are taken in parts: short and long reductions
FLOAT_SIZES = [(1000, 2050, 777), (2048, 1024, 4096), (512, 8192, 1024)]


@pytest.mark.parametrize("size", FLOAT_SIZES, ids=lambda s: "x".join(map(str, s)))
def test_linear_float_large_not_finite_values(size):
    torch = _torch()
    import paper_2512_08365_amd as mag
    rows, inner, outer = size
    g = _gen(16)
    x = _normal(g, (rows, inner), 1.0, torch.float32)
    w = _normal(g, (outer, inner), 0.1, torch.float32)
    w[3, 7] = 0.0
    w[5] = 0.5
    ref = mag.linear(x, w)
    bad = x.clone()
    bad[0, 7] = float("inf")
    bad[rows - 1, inner - 1] = float("nan")
    y = mag.linear(bad, w)
    want = torch.mm(bad[:1].double(), w.double().t().contiguous())
    assert torch.equal(y[1:rows - 1], ref[1:rows - 1])
    assert bool(torch.isnan(y[rows - 1]).all())
    assert torch.equal(torch.isnan(y[:1]), torch.isnan(want))
    assert torch.equal(y[:1][torch.isinf(want)].double(), want[torch.isinf(want)])
    x.zero_()
    x[:, 0] = 3.3e38
    w.zero_()
    w[:, 0] = 1.0
    w[outer - 1, 0] = -1.0
    w[2, 0] = 4.0
    y = mag.linear(x, w)
    assert bool((y[:, 0] == 3.3e38).all()) and bool((y[:, outer - 1] == -3.3e38).all())
    assert bool(torch.isposinf(y[:, 2]).all())


@pytest.mark.parametrize("layout", ["gap", "columns", "every2"])
@pytest.mark.parametrize("size", FLOAT_SIZES[:2], ids=lambda s: "x".join(map(str, s)))
def test_linear_float_large_layouts(size, layout):
    check_linear(*size, "f32", act="relu", lx=layout, lw=LAYOUTS[5 - LAYOUTS.index(layout)])
    check_linear_backward(*size, "f32", act="silu", lx=layout, lw="columns", ld=layout)


@pytest.mark.parametrize("ty", TYPES)
def test_linear_in_place_residual_another_stream_and_given_buffers(ty):
    torch = _torch()
    import paper_2512_08365_amd as mag
    dt, g = _dt(ty), _gen(7)
    for rows in (6, 200, 800):
        x = _normal(g, (rows, 520), 1.0, dt)
        w = _normal(g, (392, 520), 0.05, dt)
        r = _normal(g, (rows, 392), 1.0, dt)
        want = mag.linear(x, w, None, r, activation="silu")
        stream = r.clone()
        assert torch.equal(mag.linear(x, w, None, stream, activation="silu", out=stream), want)
        ws = torch.full((mag.linear_workspace_size(x, w) + 1,), 255, dtype=torch.uint8,
                        device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = mag.linear(x, w, None, r, activation="silu", workspace=ws)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)


def check_linear_backward(rows, inner, outer, ty, act="none", lx="plain", lw="plain", ld="plain",
                          bias=True, seed=2):
    torch = _torch()
    import paper_2512_08365_amd as mag
    print(f"[case] linear_backward {rows}x{inner}x{outer} {ty} {act} {lx} {lw} {ld}", flush=True)
    dt, g, u = _dt(ty), _gen(seed), _u(ty)
    x = _layout(_normal(g, (rows, inner), 1.0, dt), lx)
    w = _layout(_normal(g, (outer, inner), 1 / math.sqrt(inner), dt), lw)
    dy = _layout(_normal(g, (rows, outer), 0.25, dt), ld)
    pre = _layout(_normal(g, (rows, outer), 1.0, dt), ld) if act != "none" else None
    dx, dw, db = mag.linear_backward(x, w, dy, pre, activation=act, bias=bias)
    x64, w64, dz = x.double(), w.double(), dy.double()
    if pre is not None:
        dz = dz * act64(pre.double(), act)[1]
    rnd = (0 if ty == "f32" else u) + 24 * V  # of dz: the slope, and the rounding to the type
    tiny = _tiny(ty) if ty != "f32" else 0.0
    # (16 V of dy: a slope near its zero keeps the error of its terms)
    slack = 16 * V * dy.double().abs() + tiny
    for got, want, sums, n, name in (
            (dx, torch.mm(dz, w64.contiguous()),
             (dz.abs(), w64.abs().contiguous(), slack), outer, "dx"),
            (dw, torch.mm(dz.t().contiguous(), x64.contiguous()),
             (dz.abs().t().contiguous(), x64.abs().contiguous(), slack.t().contiguous()), rows, "dweight")):
        bound = (rnd + _sum_bound(n, ty)) * torch.mm(sums[0], sums[1]) + torch.mm(sums[2], sums[1])
        _close(got, want, bound + u * (want.abs() + bound) + _tiny(ty), name)
    if bias:
        want = dz.sum(0)
        bound = (rows + 32) * 2.0 ** -24 * dz.abs().sum(0) + 24 * V * dz.abs().sum(0) + slack.sum(0)
        _close(db, want, bound + u * (want.abs() + bound) + _tiny(ty), "dbias")
    else:
        assert db is None


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_linear_backward_sizes(size, ty):
    check_linear_backward(*size, ty, act=ACTS[sum(size) % 5])


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("act", ACTS)
def test_linear_backward_activations(act, ty):
    check_linear_backward(40, 88, 120, ty, act=act)
    check_linear_backward(264, 136, 152, ty, act=act, bias=False)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("ld", LAYOUTS)
@pytest.mark.parametrize("lw", LAYOUTS)
def test_linear_backward_layouts(lw, ld, ty):
    for lx in ("plain", "columns", "every2"):
        check_linear_backward(136, 72, 80, ty, act="gelu", lx=lx, lw=lw, ld=ld)
        check_linear_backward(131, 67, 99, ty, lx=lx, lw=lw, ld=ld)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("ld", LAYOUTS)
@pytest.mark.parametrize("lw", LAYOUTS)
def test_linear_backward_few_rows(lw, ld, ty):
    check_linear_backward(1, 65, 1100, ty, lw=lw, ld=ld)
    check_linear_backward(19, 272, 203, ty, act="silu", lx=ld, lw=lw, ld=ld)
    check_linear_backward(32, 1300, 72, ty, lx=lw, lw=lw, ld=ld)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("size", [(4100, 264, 520), (2048, 1024, 1536), (1001, 2049, 1111),
                                  (20000, 64, 72)], ids=lambda s: "x".join(map(str, s)))
def test_linear_backward_larger(size, ty):
    check_linear_backward(*size, ty, act="silu")


@pytest.mark.parametrize("act", ACTS)
def test_linear_gradients_against_differences(act):
    """In fp32, central differences of the forward pass itself along random
    directions: (f(t) - f(-t)) / 2t is off by t^2 / 6 of the third derivative and
    by the forward pass's rounding over t; at t = 2^-6 each is below 1e-3 of the
    scale here (activations with a kink: relu's pre-activations stay away from 0)."""
    torch = _torch()
    import paper_2512_08365_amd as mag
    g = _gen(11)
    x, w = (_normal(g, s, sc, torch.float32) for s, sc in (((24, 40), 1.0), ((32, 40), 0.15)))
    b = _normal(g, (32,), 0.2, torch.float32)
    if act == "relu":
        b = torch.where(torch.arange(32, device="cuda") % 2 == 0, 8.0, -8.0)
    dy = _normal(g, (24, 32), 1.0, torch.float32)
    _, pre = mag.linear(x, w, b, activation=act, pre=True)
    grads = mag.linear_backward(x, w, dy, pre, activation=act)

    def loss(x, w, b):
        return float((mag.linear(x, w, b, activation=act).double() * dy.double()).sum())

    t = 2.0 ** -6
    for i, grad in enumerate(grads):
        d = torch.randn(grad.shape, generator=g, device="cuda")
        hi = [v + t * d if i == j else v for j, v in enumerate((x, w, b))]
        lo = [v - t * d if i == j else v for j, v in enumerate((x, w, b))]
        got = (loss(*hi) - loss(*lo)) / (2 * t)
        want = float((grad.double() * d.double()).sum())
        scale = float(grad.double().norm() * d.double().norm())
        assert abs(got - want) <= 2e-3 * scale, (act, i, got, want, scale)


def test_linear_backward_wanted_outputs_alone():
    torch = _torch()
    import paper_2512_08365_amd as mag
    g = _gen(12)
    x, w, dy, pre = (_normal(g, s, 1.0, torch.bfloat16)
                     for s in ((130, 72), (80, 72), (130, 80), (130, 80)))
    full = mag.linear_backward(x, w, dy, pre, activation="gelu")
    for need, bias in (((True, False), False), ((False, True), False), ((False, False), True)):
        part = mag.linear_backward(x, w, dy, pre, activation="gelu", need=need, bias=bias)
        for p, f, n in zip(part, full, (*need, bias)):
            assert (p is None) if not n else torch.equal(p, f)


# ------------------------------------------------------------------ layer norm

def check_norm(rows, width, ty, wt, lx="plain", weight=True, bias=True, offset=0.5, wide_out=0):
    """Sums run over 64 lanes at least and a tree, so a mean is off by (width / 64
    + 32) 2^-24 of the mean magnitude; the variance is of squares about it."""
    torch = _torch()
    import paper_2512_08365_amd as mag
    print(f"[case] layer_norm {rows}x{width} {ty} {wt} {lx}", flush=True)
    dt, g, u, eps = _dt(ty), _gen(21), _u(ty), 1e-5
    x = _layout(_normal(g, (rows, width), 2.0, torch.float32).add_(offset).to(dt), lx)
    w = _normal(g, (width,), 1.0, _dt(wt)) if weight else None
    b = _normal(g, (width,), 1.0, _dt(wt)) if bias else None
    out = torch.full((rows, width + wide_out), 7.0, dtype=dt, device="cuda")
    y, mean, rstd = mag.layer_norm(x, w, b, eps, statistics=True, out=out[:, :width])
    assert bool((out[:, width:] == 7.0).all())
    x64 = x.double()
    m64 = x64.mean(1)
    d = x64 - m64[:, None]
    var = (d * d).mean(1)
    r64 = 1 / torch.sqrt(var + eps)
    dm = (width / 64 + 32) * 2.0 ** -24 * x64.abs().mean(1) + 2.0 ** -24 * m64.abs()
    _close(mean, m64, dm, "mean")
    # relative, of rstd: half the variance's error, which the mean's enters squared
    dr = 0.5 * ((width / 64 + 48) * V + dm * dm / (var + eps) + 2 * V) + 4 * V
    dr = dr + 0.5 * (4 * 2.0 ** -24 * x64.abs().amax(1) / torch.sqrt(var + eps))
    _close(rstd, r64, dr * r64, "rstd")
    xh = d * r64[:, None]
    y64 = xh * (w.double() if weight else 1.0)
    mag64 = y64.abs()
    bound = (dr[:, None] + 4 * V) * mag64
    bound = bound + ((dm + 2.0 ** -24 * x64.abs().amax(1)) * r64)[:, None] * (
        w.double().abs() if weight else 1.0)
    if bias:
        y64 = y64 + b.double()
        bound = bound + V * (mag64 + b.double().abs())
    _close(y, y64, bound + u * (y64.abs() + bound) + _tiny(ty), "out")


WIDTHS = [1, 2, 3, 7, 8, 31, 63, 64, 65, 100, 127, 128, 255, 256, 257, 511, 512, 513, 768, 1000,
          1021, 1024, 1025, 2047, 2048, 2056, 4096, 5000, 8192, 8200, 16384, 20000, 65536, 70001]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_layer_norm_widths(width, ty):
    check_norm(5, width, ty, "f32")
    check_norm(3, width, ty, ty, weight=width % 2 == 0, bias=width % 3 == 0)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("lx", LAYOUTS)
def test_layer_norm_layouts(lx, ty):
    check_norm(67, 200, ty, ty, lx=lx)
    check_norm(9, 1536, ty, "f32", lx=lx, wide_out=8)
    check_norm(4, 777, ty, "f32", lx=lx, wide_out=3)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("rows", [0, 1, 2, 300, 5000, 70000])
def test_layer_norm_rows(rows, ty):
    if rows:
        check_norm(rows, 264, ty, ty)
    else:
        torch = _torch()
        import paper_2512_08365_amd as mag
        x = torch.empty(0, 264, dtype=_dt(ty), device="cuda")
        assert mag.layer_norm(x).shape == (0, 264)
        w = torch.ones(264, device="cuda")
        dx, dw, db = mag.layer_norm_backward(x, x, w[:0], w[:0], w)
        assert dx.shape == (0, 264) and not bool(dw.any()) and not bool(db.any())


def test_layer_norm_large_mean_and_constant_rows():
    torch = _torch()
    import paper_2512_08365_amd as mag
    check_norm(16, 1024, "f32", "f32", offset=3000.0)
    x = torch.full((3, 1000), 1234.5, device="cuda")
    y, mean, rstd = mag.layer_norm(x, statistics=True)
    # a constant row: 1234.5 has 11 bits and its sums over 1,000 are exact
    assert bool((mean == 1234.5).all()) and not bool(y.any())
    x[1, 5] = float("nan")
    x[2, 6] = float("inf")
    y = mag.layer_norm(x)
    assert not bool(y[0].any()) and bool(torch.isnan(y[1]).all()) and bool(torch.isnan(y[2]).all())
    z = torch.randn(64, 300, device="cuda")
    want = mag.layer_norm(z)
    assert torch.equal(mag.layer_norm(z, out=z), want)


def check_norm_backward(rows, width, ty, wt, lx="plain", ld="plain", weight=True):
    torch = _torch()
    import paper_2512_08365_amd as mag
    print(f"[case] layer_norm_backward {rows}x{width} {ty} {wt} {lx} {ld}", flush=True)
    dt, g, u = _dt(ty), _gen(22), _u(ty)
    x = _layout(_normal(g, (rows, width), 2.0, torch.float32).add_(0.5).to(dt), lx)
    dy = _layout(_normal(g, (rows, width), 0.5, dt), ld)
    w = _normal(g, (width,), 1.0, _dt(wt)) if weight else None
    mean = x.float().mean(1)
    rstd = torch.rand(rows, generator=g, device="cuda") + 0.5
    dx, dw, db = mag.layer_norm_backward(x, dy, mean, rstd, w)
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    dy64 = dy.double()
    h = dy64 * (w.double() if weight else 1.0)
    s1, s2 = h.mean(1, keepdim=True), (h * xh).mean(1, keepdim=True)
    r = rstd.double()[:, None]
    want = r * (h - s1 - xh * s2)
    n = (width / 64 + 40) * 2.0 ** -24
    bound = r * (8 * V * (h.abs() + s1.abs() + (xh * s2).abs()) + n * h.abs().mean(1, keepdim=True)
                 + xh.abs() * n * (h * xh).abs().mean(1, keepdim=True))
    _close(dx, want, bound + u * (want.abs() + bound) + _tiny(ty), "dx")
    uw = _u(wt) if weight else 2.0 ** -24
    for got, terms, name in ((dw, dy64 * xh, "dweight"), (db, dy64, "dbias")):
        want = terms.sum(0)
        bound = ((rows + 8) * 2.0 ** -24 + 4 * V) * terms.abs().sum(0)
        _close(got, want, bound + uw * (want.abs() + bound) + _tiny(wt), name)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_layer_norm_backward_widths(width, ty):
    check_norm_backward(5, width, ty, "f32")
    check_norm_backward(70, width, ty, ty, weight=width % 2 == 0)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("lx", LAYOUTS)
def test_layer_norm_backward_layouts(lx, ty):
    for ld in ("plain", "gap", "every2"):
        check_norm_backward(67, 200, ty, ty, lx=lx, ld=ld)
        check_norm_backward(9, 1536, ty, "f32", lx=ld, ld=lx)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("size", [(1, 4096), (2, 64), (300, 1021), (5000, 264), (70000, 72),
                                  (3000, 4096), (1000, 10000)], ids=lambda s: "x".join(map(str, s)))
def test_layer_norm_backward_sizes(size, ty):
    check_norm_backward(*size, ty, ty)


def test_layer_norm_gradients_against_differences():
    torch = _torch()
    import paper_2512_08365_amd as mag
    g = _gen(23)
    x = _normal(g, (16, 96), 1.0, torch.float32)
    w, b = _normal(g, (96,), 1.0, torch.float32), _normal(g, (96,), 1.0, torch.float32)
    dy = _normal(g, (16, 96), 1.0, torch.float32)
    _, mean, rstd = mag.layer_norm(x, w, b, statistics=True)
    grads = mag.layer_norm_backward(x, dy, mean, rstd, w)
    t = 2.0 ** -6
    for i, grad in enumerate(grads):
        d = torch.randn(grad.shape, generator=g, device="cuda")
        f = [float((mag.layer_norm(*[v + s * t * d if i == j else v for j, v in
                                     enumerate((x, w, b))]).double() * dy.double()).sum())
             for s in (1, -1)]
        want = float((grad.double() * d.double()).sum())
        scale = float(grad.double().norm() * d.double().norm())
        assert abs((f[0] - f[1]) / (2 * t) - want) <= 2e-3 * scale, i


def test_layer_norm_backward_in_place_and_wanted_outputs_alone():
    torch = _torch()
    import paper_2512_08365_amd as mag
    g = _gen(24)
    x, dy = (_normal(g, (130, 520), 1.0, torch.bfloat16) for _ in range(2))
    w = _normal(g, (520,), 1.0, torch.float32)
    _, mean, rstd = mag.layer_norm(x, w, statistics=True)
    full = mag.layer_norm_backward(x, dy, mean, rstd, w)
    for need in ((True, False, False), (False, True, False), (False, False, True)):
        part = mag.layer_norm_backward(x, dy, mean, rstd, w, need=need)
        for p, f, n in zip(part, full, need):
            assert (p is None) if not n else torch.equal(p, f)
    for i in (0, 1):
        a = [x.clone(), dy.clone()]
        got = mag.layer_norm_backward(*a, mean, rstd, w,
                                      out=(a[i], torch.empty_like(w), torch.empty_like(w)))
        for p, f in zip(got, full):
            assert torch.equal(p, f)


# --------------------------------------------------------------- orthogonalize

COEFF = (3.4445, -4.7750, 2.0315)


def plain_orthogonalize(g, steps, coeff, eps, dtype):
    torch = _torch()
    x = g.to(dtype)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t().contiguous()
    x = x / (torch.sqrt((x * x).sum()) + eps)
    a, b, c = coeff
    for _ in range(steps):
        gram = x @ x.t().contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if tall else x


def check_orthogonalize(batch, rows, cols, ty, steps=5, coeff=COEFF, layout="plain", scale=0.02):
    """The kernels' operands keep 22 bits and their sums 24, as the plain
    iteration's in fp32 does, and both go through the same polynomial: the error
    is held against that iteration's own (16 times it, the operands being four
    times coarser and the order of the sums free), and u of the result."""
    torch = _torch()
    import paper_2512_08365_amd as mag
    print(f"[case] orthogonalize {batch}x{rows}x{cols} {ty} {steps} {layout}", flush=True)
    g = _gen(31)
    x = torch.stack([_layout(_normal(g, (rows, cols), scale, _dt(ty)), layout)
                     for _ in range(batch)]) if layout == "plain" else None
    if x is None:
        base = _layout(_normal(g, (batch * rows, cols), scale, _dt(ty)), layout)
        x = base.unflatten(0, (batch, rows)) if layout != "columns" else base.unflatten(
            0, (batch, rows))
    out = mag.orthogonalize(x, steps, coeff)
    assert out.shape == x.shape
    for i in range(batch):
        want = plain_orthogonalize(x[i], steps, coeff, 1e-7, torch.float64)
        own = plain_orthogonalize(x[i], steps, coeff, 1e-7, torch.float32)
        unit = float((own.double() - want).norm() / want.norm())
        got = float((out[i].double() - want).norm() / want.norm())
        bound = 16 * max(unit, 2.0 ** -22) + _u(ty)
        assert got <= bound, (i, got, unit, bound)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("size", [(1, 1, 1), (1, 1, 100), (2, 7, 3), (3, 16, 16), (1, 33, 65),
                                  (4, 64, 64), (2, 65, 200), (1, 128, 129), (3, 200, 130),
                                  (1, 256, 256), (2, 257, 300), (1, 500, 64), (1, 700, 1100),
                                  (1, 1024, 1024), (1, 2050, 300), (12, 96, 40)],
                         ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize_sizes(size, ty):
    check_orthogonalize(*size, ty)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_orthogonalize_layouts(layout, ty):
    check_orthogonalize(1, 72, 136, ty, layout=layout)
    check_orthogonalize(1, 139, 77, ty, layout=layout)


@pytest.mark.parametrize("steps", [0, 1, 2, 3, 8])
def test_orthogonalize_steps_and_polynomials(steps):
    check_orthogonalize(2, 100, 168, "f32", steps=steps)
    check_orthogonalize(1, 100, 168, "f32", steps=steps, coeff=(1.875, -1.25, 0.375))
    check_orthogonalize(1, 100, 168, "f32", steps=steps, coeff=(1.5, -0.5, 0.0))


# shapes much wider or taller than their short side, several steps of which may be
# taken at once, over spectra of full rank, of low rank and falling over six
# decades, by a steep polynomial and by a flat one: the bound of
# check_orthogonalize, and the quarter of a rounding that taking them at once may add
@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("coeff", [COEFF, (1.5, -0.5, 0.0), (2.0, -1.5, 0.5)])
@pytest.mark.parametrize("size,steps,spectrum", [((520, 4100), 2, "full"), ((520, 4100), 7, "falling"),
                                                 ((96, 6000), 4, "low"), ((2100, 700), 5, "falling"),
                                                 ((1030, 4104), 3, "low"), ((1030, 4104), 6, "full")])
def test_orthogonalize_long_sides(size, steps, spectrum, coeff, ty):
    torch = _torch()
    import paper_2512_08365_amd as mag
    print(f"[case] orthogonalize {size} {ty} {steps} {spectrum} {coeff}", flush=True)
    g = _gen(33)
    rows, cols = size
    x = torch.randn(rows, cols, generator=g, device="cuda")
    if spectrum != "full":
        m = min(size)
        side = torch.randn(m, m, generator=g, device="cuda") / math.sqrt(m)
        scale = torch.logspace(0, -6, m, device="cuda")
        if spectrum == "low":
            scale = (torch.arange(m, device="cuda") < m // 4).float()
        x = (side * scale) @ x if rows <= cols else x @ (side * scale)
    x = (x * 0.02).to(_dt(ty))
    want = plain_orthogonalize(x, steps, coeff, 1e-7, torch.float64)
    own = plain_orthogonalize(x, steps, coeff, 1e-7, torch.float32)
    unit = float((own.double() - want).norm() / want.norm())
    got = float((mag.orthogonalize(x, steps, coeff).double() - want).norm() / want.norm())
    bound = 16 * max(unit, 2.0 ** -22) + 1.25 * _u(ty)
    assert got <= bound, (got, unit, bound)


def test_orthogonalize_scales_zero_and_not_finite():
    torch = _torch()
    import paper_2512_08365_amd as mag
    check_orthogonalize(1, 64, 96, "f32", scale=1e25)
    check_orthogonalize(1, 64, 96, "f32", scale=1e-3)
    z = torch.zeros(3, 40, 64, device="cuda")
    z[1] = torch.randn(40, 64, generator=_gen(3), device="cuda")
    z[2, 0, 0] = float("nan")
    out = mag.orthogonalize(z)
    assert not bool(out[0].any()) and bool(torch.isfinite(out[1]).all())
    assert bool(torch.isnan(out[2]).all())
    assert torch.equal(out[1], mag.orthogonalize(z[1]))
    g = z[1].clone()
    assert torch.equal(mag.orthogonalize(g, out=g), out[1])


def test_orthogonalized_spectrum_through_invariants():
    """The singular values of the result are the polynomial's, iterated, of the
    input's over its norm (both spectra by the library's own invariants)."""
    torch = _torch()
    import paper_2512_08365_amd as mag
    g = _normal(_gen(32), (96, 160), 1.0, torch.float32)
    out = mag.orthogonalize(g)
    (s0, _), (s1, _) = mag.invariants([g]), mag.invariants([out])
    s = s0 / float(torch.sqrt((s0 * s0).sum()) + 1e-7)
    a, b, c = COEFF
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    want = torch.sort(s.abs(), descending=True).values
    # an fp32 iteration's error, amplified by slopes of up to 4 a step
    _close(s1, want, torch.full_like(want, 1e-3), "spectrum")


# --------------------------------------------------------- graphs and offsets

@pytest.mark.parametrize("ty", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [4, 600])
def test_calls_replay_in_a_graph(rows, ty):
    torch = _torch()
    import paper_2512_08365_amd as mag
    dt, g = _dt(ty), _gen(41)
    x = _normal(g, (rows, 264), 1.0, dt)
    w = _normal(g, (136, 264), 0.1, dt)
    b = _normal(g, (136,), 0.1, dt)
    dy = _normal(g, (rows, 136), 0.1, dt)
    nw = _normal(g, (264,), 1.0, torch.float32)

    def step():
        h, mean, rstd = mag.layer_norm(x, nw, statistics=True)
        y, pre = mag.linear(h, w, b, activation="gelu", pre=True)
        dh, dw, db = mag.linear_backward(h, w, dy, pre, activation="gelu")
        dx, dnw, dnb = mag.layer_norm_backward(x, dh, mean, rstd, nw)
        return [y, pre, dw, db, dx, dnw, dnb, mag.orthogonalize(dw)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for i in range(4):
        x.copy_(_normal(g, x.shape, 1.0 + i, dt))
        for o in outs:
            o.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for p, q in zip(got, step()):
            assert torch.equal(p, q), i
        torch.randn(1000, 1000, device="cuda").sum().item()


def test_offsets_beyond_32_bits():
    torch = _torch()
    import paper_2512_08365_amd as mag
    # 2.3e9 elements: more than 2^31, 4.6 GB
    rows, width = 70_000, 32_896
    x = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda")
    picks = [0, 1, 65_280, 65_281, rows - 2, rows - 1]
    x.zero_()
    for r in picks:
        x[r] = torch.randn(width, generator=_gen(r), device="cuda").bfloat16()
    y = mag.layer_norm(x)
    part = x[picks].contiguous()
    assert torch.equal(y[picks], mag.layer_norm(part))
    assert not bool(y[2:60_000:977].any())
    w = torch.randn(24, width, generator=_gen(9), device="cuda").mul_(0.01).bfloat16()
    z = mag.linear(x, w)
    want = torch.mm(part.double(), w.double().t().contiguous())
    bound = _sum_bound(width, "bf16") * torch.mm(part.double().abs(), w.double().abs().t().contiguous())
    _close(z[picks], want, bound + _u("bf16") * (want.abs() + bound), "linear")
    # as many outputs: [rows, 24] times [width, 24]^T
    v = torch.randn(width, 24, generator=_gen(10), device="cuda").bfloat16()
    mag.linear(z, v, out=y)
    want = torch.mm(z[picks].double(), v.double().t().contiguous())
    bound = _sum_bound(24, "bf16") * torch.mm(z[picks].double().abs(), v.double().abs().t().contiguous())
    _close(y[picks], want, bound + _u("bf16") * (want.abs() + bound) + 1e-30, "outputs")
    del y, x
    torch.cuda.empty_cache()


def test_results_are_the_same_every_time():
    torch = _torch()
    import paper_2512_08365_amd as mag
    g = _gen(51)
    x, w = _normal(g, (300, 1000), 1.0, torch.bfloat16), _normal(g, (264, 1000), 0.1, torch.bfloat16)
    dy, pre = (_normal(g, (300, 264), 1.0, torch.bfloat16) for _ in range(2))
    first = None
    for _ in range(5):
        now = [mag.linear(x, w), *mag.linear_backward(x, w, dy, pre, activation="silu"),
               *mag.layer_norm_backward(x, x, x.float().mean(1), x.float().mean(1)),
               mag.orthogonalize(w)]
        first = first or now
        for a, b in zip(now, first):
            assert torch.equal(a, b)


def test_refusals_on_the_device():
    torch = _torch()
    import paper_2512_08365_amd as mag
    from paper_2512_08365_amd import _native as N
    x, w = torch.ones(4, 16, device="cuda"), torch.ones(8, 16, device="cuda")

    def refused(code, call):
        with pytest.raises(mag.MagnetonError) as e:
            call()
        assert e.value.code == code, e.value

    refused(N.MAG_E_NULL, lambda: mag.linear(x.cpu(), w))
    refused(N.MAG_E_NULL, lambda: mag.linear(x, w.cpu()))
    refused(N.MAG_E_SIZE, lambda: mag.linear(x.double(), w.double()))
    refused(N.MAG_E_SIZE, lambda: mag.linear(x, w.half()))
    refused(N.MAG_E_SIZE, lambda: mag.linear(x, w[:, :8]))
    refused(N.MAG_E_SIZE, lambda: mag.linear(x, w, torch.ones(7, device="cuda")))
    refused(N.MAG_E_SIZE, lambda: mag.linear(x, w, torch.ones(16, device="cuda")[::2]))
    refused(N.MAG_E_SIZE, lambda: mag.linear(x, w, None, torch.ones(4, 7, device="cuda")))
    refused(N.MAG_E_SIZE, lambda: mag.linear(x, w, activation="tanh"))
    refused(N.MAG_E_SIZE, lambda: mag.linear(x, w, out=torch.ones(8, 4, device="cuda").t()))
    refused(N.MAG_E_SIZE, lambda: mag.linear(x, w, out=torch.ones(1, 8, device="cuda").expand(4, 8)))
    refused(N.MAG_E_SIZE, lambda: mag.linear(torch.ones(2, 3, 4, 16, device="cuda").transpose(0, 2), w))
    refused(N.MAG_E_NULL, lambda: mag.linear_backward(x, w, torch.ones(4, 8)))
    refused(N.MAG_E_SIZE, lambda: mag.linear_backward(x, w, torch.ones(4, 8, device="cuda"),
                                                      activation="silu"))
    refused(N.MAG_E_SIZE, lambda: mag.linear_backward(x, w, torch.ones(4, 9, device="cuda")))
    refused(N.MAG_E_SIZE, lambda: mag.layer_norm(x[:, :0]))
    refused(N.MAG_E_SIZE, lambda: mag.layer_norm(x, torch.ones(8, device="cuda")))
    refused(N.MAG_E_SIZE, lambda: mag.layer_norm(x, torch.ones(16, device="cuda").half()))
    refused(N.MAG_E_SIZE, lambda: mag.layer_norm(x, eps=-1.0))
    refused(N.MAG_E_SIZE, lambda: mag.layer_norm(x, eps=float("nan")))
    refused(N.MAG_E_SIZE, lambda: mag.orthogonalize(x, steps=65))
    refused(N.MAG_E_SIZE, lambda: mag.orthogonalize(x, coefficients=(float("inf"), 0, 0)))
    refused(N.MAG_E_SIZE, lambda: mag.orthogonalize(x, steps=64, coefficients=(1e9, 0, 0)))
    refused(N.MAG_E_SIZE, lambda: mag.orthogonalize(x[0]))
    big = torch.ones(300, 264, dtype=torch.bfloat16, device="cuda")
    need = mag.orthogonalize_workspace_size(big)
    refused(N.MAG_E_WORKSPACE, lambda: mag.orthogonalize(
        big, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda")))
    refused(N.MAG_E_WORKSPACE, lambda: mag.orthogonalize(
        big, workspace=torch.empty(need + 64, dtype=torch.uint8, device="cuda")[8:]))
    torch.cuda.synchronize()

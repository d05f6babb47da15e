"""The feed-forward block's operators at values at the ends of their range."""
import pytest

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    return torch


def _normal(seed, *shape):
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda")


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("size", [(40, 72), (96, 6000), (700, 100)], ids=lambda s: "x".join(map(str, s)))
def test_updates_by_polynomials_that_contract(size, dtype):
    """a X, again and again: exactly zero where the type's smallest number is larger,
    a^steps X otherwise, off by the operands' 22 bits a step and the result's rounding"""
    torch = _torch()
    import paper_2512_08365_amd as mag
    g = _normal(1, *size).to(getattr(torch, dtype))
    for coefficients, steps in (((0, 0, 0), 1), ((0, 0, 0), 2), ((0, 0, 0), 5), ((1e-200, 0, 0), 3),
                                ((0.1, 0, 0), 64), ((1e-20, 1e-20, 1e-20), 5)):
        out = mag.orthogonalize(g, steps, coefficients)
        assert not bool(out.any()), (coefficients, steps)
    x = g.double() / (g.double().norm() + 1e-7)
    unit = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}[dtype]
    tiny = {"float32": 2.0 ** -149, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -133}[dtype]
    for steps in (1, 4, 10, 20):
        out = mag.orthogonalize(g, steps, (0.5, 0.0, 0.0)).double()
        want = x * 0.5 ** steps
        # (two halves under a scale that takes 1 near 2^15: 22 bits, and 2^-39 below them)
        bound = steps * (2.0 ** -21 * want.abs() + 2.0 ** -39 * 0.5 ** steps) + unit * want.abs() + tiny
        assert bool(((out - want).abs() <= bound).all()), steps


ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("act", ACTS)
def test_activations_and_slopes_of_the_largest_numbers(act, dtype):
    """where an activation is z or 0 and its slope 1 or 0 in every type (silu of -40 is
    -1.7e-16 yet, and its slope there)"""
    torch = _torch()
    import paper_2512_08365_amd as mag
    from test_gpu_block import act64
    dt = getattr(torch, dtype)
    z = torch.tensor([v for v in (40.0, 1e3, 6e4, 1e10, 1.9e19, 1e30, 3.3e38) if v < torch.finfo(dt).max],
                     dtype=dt, device="cuda")
    z = torch.cat([z, -z])
    for rows in (1, 40):   # few rows, and a tile
        x, w = torch.zeros(rows, 1, dtype=dt, device="cuda"), torch.ones(len(z), 1, dtype=dt, device="cuda")
        on = (z > 0) | torch.tensor(act == "none", device="cuda")
        y = mag.linear(x, w, z, activation=act)
        far = z.abs() >= 1e3
        assert torch.equal(y[:, far], torch.where(on, z, torch.zeros_like(z))[far].expand(rows, -1)), act
        for got, want in zip(y[:, ~far].double().unbind(1), act64(z[~far].double(), act)[0]):
            assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -25).all())
        dy = torch.ones(rows, len(z), dtype=dt, device="cuda")
        dx, _, db = mag.linear_backward(x, w, dy, z.expand(rows, -1), activation=act)
        assert torch.equal(db[far], (rows * on).to(dt)[far]), act
        for got, want in zip(db[~far].double(), rows * act64(z[~far].double(), act)[1]):
            assert float((got - want).abs()) <= 2.0 ** -8 * float(want.abs()) + 2.0 ** -25
        assert bool((dx == on.sum()).all()), act


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_activations_keep_their_digits_in_the_tails(act, dtype):
    """Relative errors, down to where fp32 has its full digits.  fp32: an activation
    is some twelve operations that are off by a last place (2^-23) at most; a slope
    as many of each of its two terms.  Two bytes: 2^-15 for the six-term polynomial
    and the arguments' rounding, and the result's own rounding."""
    torch = _torch()
    import paper_2512_08365_amd as mag
    from test_gpu_block import act64
    dt = getattr(torch, dtype)
    z = torch.cat([torch.linspace(-20, 20, 160_001, device="cuda"), _normal(3, 40_000) * 4]).to(dt)
    z64 = z.double()
    off, tiny = {"float32": (12 * 2.0 ** -23, 2.0 ** -118), "float16": (2.0 ** -11 + 2.0 ** -15, 2.0 ** -25),
                 "bfloat16": (2.0 ** -8 + 2.0 ** -15, 2.0 ** -118)}[dtype]
    want, slope = act64(z64, act)
    if act != "gelu":
        # (the formulas' tails, which 1 + tanh and a sigmoid of z < -36 would cut off)
        e = torch.exp(-(z64 if act == "silu" else 2 * (2 / torch.pi) ** 0.5 * (z64 + 0.044715 * z64 ** 3)))
        s, c = 1 / (1 + e), e / (1 + e)
        k = 1 if act == "silu" else 2 * (2 / torch.pi) ** 0.5 * (1 + 3 * 0.044715 * z64 * z64)
        want, slope, terms = z64 * s, s + z64 * s * c * k, s + (z64 * s * c * k).abs()
    else:
        terms = 0.5 * torch.erfc(-z64 / 2 ** 0.5) + (z64 * torch.exp(-z64 * z64 / 2)).abs() / (2 * torch.pi) ** 0.5
    for rows in (1, 40):
        x, w = torch.zeros(rows, 1, dtype=dt, device="cuda"), torch.ones(len(z), 1, dtype=dt, device="cuda")
        y = mag.linear(x, w, z, activation=act).double()
        assert bool(((y - want).abs() <= off * want.abs() + tiny).all()), float(
            ((y - want).abs() / (off * want.abs() + tiny)).max())
    one = torch.ones(1, len(z), dtype=dt, device="cuda")
    _, _, db = mag.linear_backward(x[:1], w, one, z[None], activation=act, need=(False, False))
    rel = 12 * 2.0 ** -23 if dtype == "float32" else 2.0 ** -15
    bound = rel * terms + (0 if dtype == "float32" else off) * slope.abs() + tiny
    assert bool(((db.double() - slope).abs() <= bound).all()), float(((db.double() - slope).abs() / bound).max())


def _ms(call):
    torch = _torch()
    best = 1e9
    for _ in range(3):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


# fp32 products that are taken in parts: one tile of each size, a reduction that is
# split, and two gradients at once
@pytest.mark.parametrize("size", [(1000, 2050, 777), (2048, 1024, 4096), (512, 8192, 1024), (8192, 512, 2048),
                                  (2048, 1024, 1536)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("where", ["all", "last of each row", "one row of the weight", "half the rows"])
def test_nan_in_large_float_products(size, where):
    """NaN where an operand has one and nowhere else, and no call much longer for it:
    taking every such sum again is 200 to 500 times the time without"""
    torch = _torch()
    import paper_2512_08365_amd as mag
    rows, inner, outer = size
    x, w, dy = _normal(1, rows, inner), _normal(2, outer, inner) * 0.1, _normal(3, rows, outer)
    mag.linear(x, w)
    y0, grads0 = mag.linear(x, w), mag.linear_backward(x, w, dy)
    t0, b0 = _ms(lambda: mag.linear(x, w)), _ms(lambda: mag.linear_backward(x, w, dy))
    nan = float("nan")
    bad_rows, bad_cols = torch.zeros(rows, dtype=torch.bool), torch.zeros(outer, dtype=torch.bool)
    if where == "all":
        x[:] = nan
        dy[:] = nan
        bad_rows[:] = True
    elif where == "last of each row":
        x[:, -1] = nan
        dy[:, -1] = nan
        bad_rows[:] = True
    elif where == "half the rows":
        x[::2, 3] = nan
        dy[::2, 3] = nan
        bad_rows[::2] = True
    else:
        w[outer // 2, inner // 3] = nan
        bad_cols[outer // 2] = True
    y = mag.linear(x, w)
    bad = bad_rows[:, None].cuda() | bad_cols[None].cuda()
    assert torch.equal(torch.isnan(y), bad) and torch.equal(y[~bad], y0[~bad])
    dx, dw, db = mag.linear_backward(x, w, dy)
    # what has a NaN where: dx = dy w, dw = dy^T x, db = the sum of dy
    nx, nw, nd = (torch.isnan(v) for v in (x, w, dy))
    bad_dx = nd.any(1)[:, None] | nw.any(0)[None]
    bad_dw = nd.any(0)[:, None] | nx.any(0)[None]
    for got, want, bad in ((dx, grads0[0], bad_dx), (dw, grads0[1], bad_dw), (db, grads0[2], nd.any(0))):
        assert torch.equal(torch.isnan(got), bad) and torch.equal(got[~bad], want[~bad])
    t1, b1 = _ms(lambda: mag.linear(x, w)), _ms(lambda: mag.linear_backward(x, w, dy))
    print(f"[time] {size} {where}: {t0:.3f} -> {t1:.3f}, gradients {b0:.3f} -> {b1:.3f} ms", flush=True)
    assert t1 <= 40 * t0 and b1 <= 40 * b0


def test_results_carry_no_gradient():
    """as the docstrings say: the backward calls compute it"""
    torch = _torch()
    import paper_2512_08365_amd as mag
    x, w = _normal(1, 40, 64).requires_grad_(), _normal(2, 24, 64).requires_grad_()
    y, pre = mag.linear(x, w, pre=True)
    z, mean, rstd = mag.layer_norm(x, statistics=True)
    outs = [y, pre, z, mean, rstd, mag.orthogonalize(w), *mag.linear_backward(x, w, y),
            *mag.layer_norm_backward(x, z, mean, rstd)]
    assert not any(o.requires_grad for o in outs)
    for f in (mag.linear, mag.layer_norm, mag.orthogonalize):
        assert "no gradient" in " ".join(f.__doc__.split())


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_reductions_over_nothing(dtype):
    """no inputs, more rows than a decode step has: act(bias) + residual; no outputs: dx 0"""
    torch = _torch()
    import paper_2512_08365_amd as mag
    new = dict(dtype=getattr(torch, dtype), device="cuda")
    b, r = torch.arange(-40, 40, **new), torch.ones(100, 80, **new)
    y, z = mag.linear(torch.empty(100, 0, **new), torch.empty(80, 0, **new), b, r, activation="relu", pre=True)
    assert torch.equal(z, b.expand(100, 80)) and torch.equal(y, b.clamp(min=0).expand(100, 80) + 1)
    dx, dw, db = mag.linear_backward(torch.empty(100, 0, **new), torch.empty(80, 0, **new), r)
    assert dx.shape == (100, 0) and dw.shape == (80, 0) and bool((db == 100).all())
    dx, dw, db = mag.linear_backward(torch.ones(100, 72, **new), torch.empty(0, 72, **new),
                                     torch.empty(100, 0, **new))
    assert dx.shape == (100, 72) and not bool(dx.any()) and dw.shape == (0, 72) and db.shape == (0,)


def test_norm_weights_that_are_no_tensors_are_refused():
    torch = _torch()
    import paper_2512_08365_amd as mag
    from paper_2512_08365_amd import _native as N
    x, rows = torch.ones(4, 16, device="cuda"), torch.ones(4, device="cuda")
    for bad, code in ((2.0, N.MAG_E_NULL), ([1.0] * 16, N.MAG_E_NULL), (torch.ones(16), N.MAG_E_NULL),
                      (torch.ones(16, device="cuda", dtype=torch.float64), N.MAG_E_SIZE)):
        for call in (lambda: mag.layer_norm(x, bad), lambda: mag.layer_norm(x, None, bad),
                     lambda: mag.layer_norm_backward(x, x, rows, rows, bad)):
            with pytest.raises(mag.MagnetonError) as e:
                call()
            assert e.value.code == code, e.value

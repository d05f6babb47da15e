"""8-bit operands and their linear layer against plain 64-bit forms, element by
element, at the sizes, strides and values where they can go wrong.

Tolerances (u: half a unit of the type's last place, relative; v = 2^-23).  Products
of 8-bit numbers are exact in fp32.  The matrix instruction adds eight neighbours'
products as far as 2^-13 of their largest one's power of two: each of the other seven
loses less than that.  Blocks are multiplied by their scales' product (a rounding)
and added (a rounding each): (blocks + 4) v of the sum of magnitudes.  Where all
products are small whole numbers and the scales powers of two nothing is lost.  An
activation's slope is at most 1.13, its evaluation is within 2^-15 and the type's
rounding; every output is rounded once: u of it."""
import math

import pytest

from test_gpu_block import V, _close, _dt, _gen, _normal, _tiny, _torch, _u, act64

pytestmark = pytest.mark.gpu

BLOCK = 128
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
SMALL = {"e4m3": (3, -6), "e5m2": (2, -14)}   # bits behind the point, least exponent


def _eight(name):
    torch = _torch()
    return {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}[name]


def _blocks(n):
    return -(-n // BLOCK)


def _each(scale, rows, cols, block_rows=1):
    """a scale for every element"""
    s = scale.double().repeat_interleave(BLOCK, 1)[:, :cols]
    return s if block_rows == 1 else s.repeat_interleave(block_rows, 0)[:rows]


def _lay(x, kind):
    """x's bytes in another layout; what lies between them is NaN of both formats"""
    torch = _torch()
    r, c = x.shape
    b = x.view(torch.uint8) if x.is_contiguous() else x.contiguous().view(torch.uint8)
    if kind in ("plain", "columns"):
        y = b if kind == "plain" else b.t().contiguous().t()
    elif kind in ("gap", "gap16"):
        y = torch.full((r, c + 5 if kind == "gap" else -(-c // 16) * 16 + 16), 0x7f, dtype=torch.uint8,
                       device="cuda")
        y[:, :c] = b
        y = y[:, :c]
    else:
        y = torch.full((2 * r, 2 * c + 1), 0x7f, dtype=torch.uint8, device="cuda")
        y[::2, 1::2] = b
        y = y[::2, 1::2]
    return y.view(x.dtype) if y.stride(-1) == 1 else torch.as_strided(
        torch.empty(0, dtype=x.dtype, device="cuda").set_(y.untyped_storage()), y.shape, y.stride(),
        y.storage_offset())


# ------------------------------------------------------------------- quantization

def _check_cut(x, q, scale, block_rows, eight):
    """q and scale against their definition: the scale within a last place, q the nearest
    number to x / scale, but for quotients that fp32 cannot tell from a tie"""
    torch = _torch()
    rows, cols = x.shape
    x64 = x.double()
    wide = torch.zeros((-(-rows // block_rows) * block_rows, _blocks(cols) * BLOCK), dtype=torch.float64,
                       device="cuda")
    wide[:rows, :cols] = x64.abs()
    most = wide.view(-1, block_rows, _blocks(cols), BLOCK).amax((1, 3))
    exact = torch.clamp(most / LARGEST[eight], min=2.0 ** -126)
    assert scale.shape == exact.shape
    assert bool(((scale.double() - exact).abs() <= V / 2 * exact).all())
    # (x / scale by one rounding, so that a tie is one here too: a 64-bit quotient by
    # the rounded scale was off one by a last place)
    m = _each(most, rows, cols, block_rows)
    t = torch.where(m / LARGEST[eight] > 2.0 ** -126, x64 * LARGEST[eight] / m, x64 * 2.0 ** 126)
    bits, least = SMALL[eight]
    step = torch.exp2(torch.clamp(torch.frexp(t)[1].double() - 1, min=least) - bits)
    err = (q.double() - t).abs()
    # half a step, and of fp32 numbers what their quotient's rounding takes
    slack = (4 * V * t.abs() if x.dtype == torch.float32 else 0)
    assert bool((err <= step / 2 + slack).all()), float((err / step).max())
    if x.dtype != torch.float32:
        tie = err == step / 2
        even = torch.round(t / step) * step
        assert bool((q.double() == even)[tie].all())
    assert bool((q.double().abs() <= LARGEST[eight]).all())


@pytest.mark.parametrize("eight", ["e4m3", "e5m2"])
@pytest.mark.parametrize("ty", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", [(1, 1), (1, 127), (3, 129), (17, 1021), (130, 128), (257, 515), (16, 4096),
                                  (129, 7)])
def test_quantize(size, ty, eight):
    import paper_2512_08365_amd as mag
    torch = _torch()
    g = _gen(sum(size))
    x = _normal(g, size, 1.0, torch.float32) * torch.exp2(
        torch.randint(-12, 12, (size[0], 1), generator=g, device="cuda").float())
    x = x.to(_dt(ty))
    for lay in ("plain", "gap", "columns", "every"):
        if lay == "plain":
            y = x
        elif lay == "gap":
            y = torch.full((size[0], size[1] + 3), float("nan"), dtype=x.dtype, device="cuda")
            y[:, :size[1]] = x
            y = y[:, :size[1]]
        elif lay == "columns":
            y = x.t().contiguous().t()
        else:
            y = torch.full((2 * size[0], 3 * size[1]), float("nan"), dtype=x.dtype, device="cuda")
            y[::2, ::3] = x
            y = y[::2, ::3]
        for block_rows in (1, BLOCK):
            q, s = mag.quantize_fp8(y, block_rows, dtype=_eight(eight))
            _check_cut(x, q, s, block_rows, eight)
            both = mag.quantize_fp8(y, block_rows, dtype=_eight(eight), transposed=True)
            assert torch.equal(both[0].view(torch.uint8), q.view(torch.uint8)) and torch.equal(both[1], s)
            if block_rows == 1:
                _check_cut(x.t(), both[2], both[3], 1, eight)
            else:
                assert torch.equal(both[2].float(), q.float().t()) and torch.equal(both[3], s.t())


def test_quantize_ties_and_ends():
    """quotients that lie between two numbers, the smallest numbers, zeros"""
    import paper_2512_08365_amd as mag
    torch = _torch()
    for eight in ("e4m3", "e5m2"):
        for ty in ("bf16", "f16"):
            # the largest of each block times every number halfway between two
            bits, _ = SMALL[eight]
            m = torch.arange(2 ** (bits + 1), device="cuda").double() / 2 ** (bits + 1) + 1
            e = torch.arange(-20, 9 if eight == "e4m3" else 16, device="cuda").double()
            t = (m[:, None] * torch.exp2(e)).reshape(-1)
            t = t[t <= LARGEST[eight]]
            n = _blocks(t.numel()) * 127
            x = torch.zeros(n, dtype=torch.float64, device="cuda")
            x[:t.numel()] = t
            x = torch.cat([x.view(-1, 127), torch.full((n // 127, 1), LARGEST[eight], dtype=torch.float64,
                                                       device="cuda")], 1)
            for by in (1.0, 2.0 ** -7, 0.875, -0.8125):   # (in the range of half)
                y = (x * by).to(_dt(ty))
                q, s = mag.quantize_fp8(y, dtype=_eight(eight))
                _check_cut(y, q, s, 1, eight)
    # blocks of zeros and of numbers below the smallest scale
    x = torch.zeros((2, 256), device="cuda")
    x[1, 128:] = 2.0 ** -130
    x[0, 200] = 1e-30
    q, s = mag.quantize_fp8(x)
    assert bool((s[[0, 1], [0, 0]] == 2.0 ** -126).all()) and bool((q[:, :128].float() == 0).all())
    _check_cut(x, q, s, 1, "e4m3")
    # the largest numbers
    x = torch.full((1, 128), 3.3e38, device="cuda")
    x[0, ::2] = -3.4028234e38
    q, s = mag.quantize_fp8(x)
    _check_cut(x, q, s, 1, "e4m3")


@pytest.mark.parametrize("block_rows", [1, BLOCK])
def test_quantize_infinities_and_nan(block_rows):
    import paper_2512_08365_amd as mag
    torch = _torch()
    for eight in ("e4m3", "e5m2"):
        x = torch.randn((256, 300), generator=_gen(3), device="cuda")
        clean = x.clone()
        x[5, 7] = float("nan")
        x[140, 131] = float("inf")
        clean[5, 7] = 0
        got = mag.quantize_fp8(x, block_rows, dtype=_eight(eight), transposed=True)
        want = mag.quantize_fp8(clean, block_rows, dtype=_eight(eight), transposed=True)
        for k, (r, c) in enumerate(((5, 7), (7, 5))):
            q, s = got[2 * k].float(), got[2 * k + 1]
            i, j = (140, 131) if k == 0 else (131, 140)
            assert math.isnan(float(q[r, c])) and math.isnan(float(q[i, j]))
            ib = i if block_rows == 1 else i // BLOCK
            assert math.isinf(float(s[ib, j // BLOCK]))
            line = slice(i, i + 1) if block_rows == 1 else slice(ib * BLOCK, ib * BLOCK + BLOCK)
            block = q[line, j // BLOCK * BLOCK:j // BLOCK * BLOCK + BLOCK]
            assert int(block.isnan().sum()) == 1 and float(block.nan_to_num(0).abs().max()) == 0
            # the rest is as without them
            other = want[2 * k].float().clone()
            q, other = q.clone(), other
            for t in (q, other):
                t[r, c] = 0
                t[line, j // BLOCK * BLOCK:j // BLOCK * BLOCK + BLOCK] = 0
            assert torch.equal(q, other)


def test_quantize_writes_what_it_says():
    """given outputs, their gaps, and scales by rows and by columns"""
    import paper_2512_08365_amd as mag
    torch = _torch()
    x = torch.randn((200, 333), generator=_gen(4), device="cuda").to(torch.bfloat16)
    want = mag.quantize_fp8(x, transposed=True)
    for by in ("rows", "columns"):
        q = torch.full((200, 340), 0x55, dtype=torch.uint8, device="cuda")
        qt = torch.full((333, 209), 0x55, dtype=torch.uint8, device="cuda")
        if by == "rows":
            s, st = torch.full((200, 5), 7.0, device="cuda"), torch.full((333, 4), 7.0, device="cuda")
            out_s, out_st = s[:, :3], st[:, :2]
        else:
            s, st = torch.full((3, 201), 7.0, device="cuda"), torch.full((2, 334), 7.0, device="cuda")
            out_s, out_st = s.t()[:200], st.t()[:333]
        out = (q[:, :333].view(torch.float8_e4m3fn), out_s, qt[:, :200].view(torch.float8_e4m3fn), out_st)
        got = mag.quantize_fp8(x, transposed=True, out=out)
        for a, b in zip(got, want):
            assert torch.equal(a.float(), b.float())
        assert bool((q[:, 333:] == 0x55).all()) and bool((qt[:, 200:] == 0x55).all())
        gap, gap_t = (s[:, 3:], st[:, 2:]) if by == "rows" else (s[:, 200:], st[:, 333:])
        assert bool((gap == 7).all()) and bool((gap_t == 7).all())
    # rows only, a batch's leading dimensions as one, nothing at all
    got = mag.quantize_fp8(x.view(4, 50, 333))
    assert torch.equal(got[0].float(), want[0].float()) and torch.equal(got[1], want[1])
    assert mag.quantize_fp8(x[:0])[0].shape == (0, 333)
    assert mag.quantize_fp8(x[:, :0], transposed=True)[2].shape == (0, 200)


# ------------------------------------------------------------------------- linear

def _lost(x, w, sx, sw):
    """the most that eight neighbours' sums lose: 7 2^-13 of their largest product each"""
    torch = _torch()
    rows, inner = x.shape
    total = torch.zeros((rows, w.shape[0]), dtype=torch.float64, device="cuda")
    a = (x.double().abs() * sx).float()
    b = (w.double().abs() * sw).float()
    for k in range(0, inner, 8):
        total += (a[:, None, k:k + 8] * b[None, :, k:k + 8]).amax(2).double()
    return 7 * 2.0 ** -13 * total


def check_linear(rows, inner, outer, ty="bf16", act="none", bias=True, residual=True, pre=True, lx="plain",
                 lw="plain", formats=("e4m3", "e4m3"), by_row=False, whole=False, seed=1, scales="columns"):
    torch = _torch()
    import paper_2512_08365_amd as mag
    print(f"[case] linear_fp8 {rows}x{inner}x{outer} {ty} {act} {lx} {lw} {formats} {by_row} {whole}", flush=True)
    dt, g = _dt(ty), _gen(seed)

    def operand(n, eight, block_rows, lay):
        q = torch.randn((n, inner), generator=g, device="cuda") * 60
        if whole:
            q = torch.round(q / 40).clamp(-4, 4)
        q = q.clamp(-448, 448).to(_eight(eight))
        tall = n if block_rows == 1 else _blocks(n)
        s = torch.rand((tall, _blocks(inner)), generator=g, device="cuda") + 0.5
        s = torch.exp2(torch.floor(s * 6) - 6) if whole else s * 0.02
        if scales == "columns":
            s = s.t().contiguous().t()
        elif scales == "gap":
            s = torch.cat([s, torch.full_like(s, float("nan"))], 1)[:, :_blocks(inner)]
        return _lay(q, lay), s, _each(s, n, inner, block_rows), q

    x, sx, ex, qx = operand(rows, formats[0], 1, lx)
    w, sw, ew, qw = operand(outer, formats[1], 1 if by_row else BLOCK, lw)
    b = _normal(g, (outer,), 0.5, dt) if bias else None
    r = _normal(g, (rows, outer), 1.0, dt) if residual else None
    mark = 7.0
    out = torch.full((rows, outer + 3), mark, dtype=dt, device="cuda")
    keep = torch.full((rows, outer + 3), mark, dtype=dt, device="cuda")
    got = mag.linear_fp8(x, sx, w, sw, b, r, activation=act, out=out[:, :outer],
                         pre=keep[:, :outer] if pre else None)
    assert bool((out[:, outer:] == mark).all()) and bool((keep[:, outer:] == mark).all())
    y, z = got if pre else (got, None)
    a64, b64 = qx.double() * ex, qw.double() * ew
    z64 = torch.mm(a64, b64.t().contiguous())
    mag64 = torch.mm(a64.abs(), b64.abs().t().contiguous())
    if whole:
        dz = torch.zeros_like(z64)
    else:
        dz = (_blocks(inner) + 4) * V * mag64 + _lost(qx, qw, ex, ew)
    if bias:
        z64 = z64 + b.double()
        dz = dz + V * z64.abs()
    if pre:
        _close(z, z64, dz + _u(ty) * (z64.abs() + dz) + _tiny(ty), "pre")
    y64 = act64(z64, act)[0]
    dy = dz if act == "none" else 1.13 * dz + 2.0 ** -15 * (z64.abs() + y64.abs())
    if residual:
        y64 = y64 + r.double()
        dy = dy + V * y64.abs()
    _close(y, y64, dy + _u(ty) * (y64.abs() + dy) + _tiny(ty), "y")


ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
ROWS = [1, 2, 16, 17, 31, 32, 33, 64, 65, 130, 257]
INNER = [1, 15, 16, 17, 127, 128, 129, 144, 255, 256, 257, 1021]


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("whole", [True, False])
def test_linear_sizes(rows, whole):
    for i, inner in enumerate(INNER):
        check_linear(rows, inner, (1, 16, 65, 130, 257)[i % 5], ("bf16", "f16")[i % 2], ACTS[i % 5], whole=whole,
                     by_row=i % 3 == 0, seed=i)


@pytest.mark.parametrize("formats", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("by_row", [False, True])
@pytest.mark.parametrize("size", [(5, 300, 70), (24, 300, 70), (100, 400, 200), (300, 1000, 513)])
def test_linear_formats(size, by_row, formats):
    for whole in (True, False):
        check_linear(*size, formats=formats, by_row=by_row, whole=whole)


@pytest.mark.parametrize("lay", ["plain", "gap", "gap16", "columns", "every"])
@pytest.mark.parametrize("rows", [3, 70])
def test_linear_layouts(rows, lay):
    for other in ("plain", "gap", "gap16", "columns", "every"):
        for inner in (200, 256):
            check_linear(rows, inner, 77, lx=lay, lw=other, whole=True, scales=("columns", "gap", "rows")[inner % 3])


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("size", [(2050, 1024, 2050), (700, 4096, 1300), (3000, 640, 4100)])
def test_linear_large(size, whole):
    if not whole and size[0] * size[1] * size[2] > 4e9:
        size = (size[0], size[1], size[2] // 4)
    for by_row in (False, True):
        check_linear(*size, act="gelu_tanh", whole=whole, by_row=by_row)


def test_linear_nothing():
    import paper_2512_08365_amd as mag
    torch = _torch()
    q, s = mag.quantize_fp8(torch.randn((40, 200), device="cuda"))
    w, ws = mag.quantize_fp8(torch.randn((30, 200), device="cuda"), BLOCK)
    assert mag.linear_fp8(q[:0], s[:0], w, ws).shape == (0, 30)
    assert mag.linear_fp8(q, s, w[:0], ws[:0]).shape == (40, 0)
    # no inner width: the bias alone
    b = torch.randn(30, device="cuda").to(torch.bfloat16)
    for rows in (4, 40):
        y = mag.linear_fp8(q[:rows, :0], s[:rows, :0], w[:, :0], ws[:, :0], b)
        assert torch.equal(y, b.expand(rows, 30))


def test_linear_infinities_and_nan_stay_in_their_rows():
    import paper_2512_08365_amd as mag
    torch = _torch()
    for rows in (20, 200):
        x = torch.randn((rows, 300), generator=_gen(5), device="cuda")
        w = torch.randn((150, 300), generator=_gen(6), device="cuda")
        clean = mag.linear_fp8(*mag.quantize_fp8(x), *mag.quantize_fp8(w))
        x[3, 299] = float("nan")
        x[7, 0] = float("inf")
        w[140, 130] = float("nan")
        y = mag.linear_fp8(*mag.quantize_fp8(x), *mag.quantize_fp8(w))
        assert bool(y[3].isnan().all()) and bool(y[7].isnan().all()) and bool(y[:, 140].isnan().all())
        keep = torch.ones((rows, 150), dtype=torch.bool, device="cuda")
        keep[3] = keep[7] = False
        keep[:, 140] = False
        assert torch.equal(y[keep], clean[keep])


def test_gradients_of_a_layer():
    """the two gradients as such products, against differences of the layer's sum"""
    import paper_2512_08365_amd as mag
    torch = _torch()
    g = _gen(9)
    x = torch.randn((300, 260), generator=g, device="cuda")
    w = torch.randn((390, 260), generator=g, device="cuda") / 16
    dy = torch.randn((300, 390), generator=g, device="cuda")
    q, s, qt, st = mag.quantize_fp8(x, transposed=True)
    qw, sw, wt, swt = mag.quantize_fp8(w, BLOCK, transposed=True)
    d, ds, dt, dst = mag.quantize_fp8(dy, transposed=True)
    dx, dw = mag.linear_fp8(d, ds, wt, swt), mag.linear_fp8(dt, dst, qt, st)
    a, b = q.double() * _each(s, 300, 260), qw.double() * _each(sw, 390, 260, BLOCK)
    e = d.double() * _each(ds, 300, 390)
    f = dt.double() * _each(dst, 390, 300)
    c = qt.double() * _each(st, 260, 300)
    want = e @ b
    tol = (8 * V + 7 * 2.0 ** -13) * (e.abs() @ b.abs())
    _close(dx, want, tol + _u("bf16") * (want.abs() + tol), "dx")
    want = f @ c.t()
    tol = (8 * V + 7 * 2.0 ** -13) * (f.abs() @ c.abs().t())
    _close(dw, want, tol + _u("bf16") * (want.abs() + tol), "dweight")
    # the layer's sum with dy changes by dx along a step of x (linear: any step)
    step = torch.randn((300, 260), generator=g, device="cuda").double() * 0.1
    change = (((a + step) @ b.t() - a @ b.t()) * e).sum()
    along = (dx.double() * step).sum()
    bound = ((8 * V + 7 * 2.0 ** -13 + _u("bf16")) * (e.abs() @ b.abs()) * step.abs()).sum()
    assert abs(float(change - along)) <= float(bound)


@pytest.mark.parametrize("inner", [1, 100, 129, 1021, 2100])
def test_linear_of_many_tiles(inner):
    """more tiles than CUs, the last ones cut, reductions of one block and of odd lengths"""
    for i, by_row in enumerate((False, True)):
        check_linear(8200, inner, 4500, ("bf16", "f16")[i], ACTS[inner % 5], pre=not by_row, whole=True, by_row=by_row,
                     lx=("plain", "gap16")[i], formats=(("e4m3", "e4m3"), ("e5m2", "e4m3"))[i])


def test_linear_split_reductions():
    """few tiles and long reductions: partial sums and their sum"""
    for size in ((40, 20000, 70), (300, 30000, 300), (257, 16385, 130)):
        for by_row in (False, True):
            check_linear(*size, act="silu", whole=True, by_row=by_row)


@pytest.mark.parametrize("ty", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("cols", [8, 9, 15, 120, 127, 1016, 1023])
def test_quantize_ends_of_rows(cols, ty):
    """every place at which a row can end amid eight neighbours, what follows it NaN"""
    import paper_2512_08365_amd as mag
    torch = _torch()
    for pitch in (0, 1, 8):
        y = torch.full((140, cols + pitch), float("nan"), dtype=_dt(ty), device="cuda")
        y[:, :cols] = _normal(_gen(cols), (140, cols), 1.0, _dt(ty))
        x = y[:, :cols]
        for block_rows in (1, BLOCK):
            q, s, qt, st = mag.quantize_fp8(x, block_rows, transposed=True)
            _check_cut(x.contiguous(), q, s, block_rows, "e4m3")
            if block_rows == 1:
                _check_cut(x.t().contiguous(), qt, st, 1, "e4m3")
                rows = mag.quantize_fp8(x)
                assert torch.equal(rows[0].float(), q.float()) and torch.equal(rows[1], s)


@pytest.mark.parametrize("by_row", [False, True])
@pytest.mark.parametrize("size", [(5, 300, 70), (24, 300, 70), (100, 300, 200), (700, 300, 1300), (40, 20000, 70)])
def test_linear_scales_at_the_ends_of_their_range(size, by_row):
    """The two scales of a block are multiplied with each other first, whatever kernel a
    size takes: a tiny one and a huge one lose nothing, two tiny ones what their product's
    subnormal number lacks, two huge ones are infinite."""
    import paper_2512_08365_amd as mag
    torch = _torch()
    rows, inner, outer = size
    g, blocks = _gen(11), _blocks(inner)
    tall = outer if by_row else _blocks(outer)

    def numbers(n, most, unit):
        return (torch.randint(-most, most + 1, (n, inner), generator=g, device="cuda") * unit).to(_eight("e4m3"))

    def scales(n, unit):
        return (torch.randint(2, 4, (n, blocks), generator=g, device="cuda") / 2).float() * unit

    # sums of -9 to 9 in units of 2^-18, times 1, 1.5 or 2.25, are exact in fp32
    for a, b in ((2.0 ** 120, 2.0 ** -126), (2.0 ** -126, 2.0 ** 120), (2.0 ** 126, 2.0 ** -110)):
        x, w, sx, sw = numbers(rows, 3, 2.0 ** -9), numbers(outer, 3, 2.0 ** -9), scales(rows, a), scales(tall, b)
        want = torch.mm(x.double() * _each(sx, rows, inner),
                        (w.double() * _each(sw, outer, inner, 1 if by_row else BLOCK)).t().contiguous())
        assert torch.equal(mag.linear_fp8(x, sx, w, sw), want.bfloat16())
    # products of scales between 2^-141 and 2^-137, whole numbers times 32 (which lose nothing)
    x, w = numbers(rows, 14, 32.0), numbers(outer, 14, 32.0)
    sx, sw = ((1 + torch.rand((n, blocks), generator=g, device="cuda")) * 2.0 ** -by for n, by in ((rows, 70), (tall, 71)))
    want, mag64 = (torch.zeros((rows, outer), dtype=torch.float64, device="cuda") for _ in range(2))
    for k in range(blocks):
        each = sw[:, k] if by_row else sw[:, k].repeat_interleave(BLOCK)[:outer]
        by = (sx[:, None, k].cpu() * each[None].cpu()).cuda().double()   # (rounded once, in fp32)
        assert 2.0 ** -142 < float(by.min()) and float(by.max()) < 2.0 ** -138
        a, b = (v[:, k * BLOCK:(k + 1) * BLOCK].double() for v in (x, w))
        want += by * torch.mm(a, b.t().contiguous())
        mag64 += by * torch.mm(a.abs(), b.abs().t().contiguous())
    tol = (blocks + 4) * V * mag64
    _close(mag.linear_fp8(x, sx, w, sw), want, tol + _u("bf16") * (want.abs() + tol) + _tiny("bf16"), "subnormal products")
    # beyond fp32: infinite, and of a sum of zero NaN
    x, w = numbers(rows, 3, 1.0), numbers(outer, 3, 1.0)
    x[0] = 0
    got = mag.linear_fp8(x, scales(rows, 2.0 ** 100), w, scales(tall, 2.0 ** 100))
    assert bool(got[0].isnan().all()) and not bool(got.isfinite().any())

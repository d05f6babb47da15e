"""The norms around a block fused with gate, residual scale and addition, and their
gradients, against plain 64-bit forms, element by element.

Tolerances (u: half a unit of the type's last place, relative; v = 2^-23): as the layer
norms': sums over a row run over 64 lanes at least and a tree, (width / 64 + 32) 2^-24 of
the mean magnitude; each operation beside them rounds once.  The second norm is held
against the stream as it was returned: it reads what is stored.  Gradients: what the
row's sums are off by enters every element of the row, and with it the sums over rows."""
import math

import pytest

from test_gpu_block import TYPES, V, WIDTHS, _close, _dt, _gen, _layout, _normal, _tiny, _torch, _u

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _moments(x64, kind):
    """mean, rstd, and what they may be off by (rstd: relative)"""
    torch = _torch()
    width = x64.shape[1]
    if kind == "rms":
        r = 1 / torch.sqrt((x64 * x64).mean(1) + EPS)
        dr = 0.5 * ((width / 64 + 48) * V + 2 * V) + 4 * V
        return torch.zeros_like(r), r, torch.zeros_like(r), torch.full_like(r, dr)
    m = x64.mean(1)
    d = x64 - m[:, None]
    var = (d * d).mean(1)
    r = 1 / torch.sqrt(var + EPS)
    dm = (width / 64 + 32) * 2.0 ** -24 * x64.abs().mean(1) + 2.0 ** -24 * m.abs()
    dr = 0.5 * ((width / 64 + 48) * V + dm * dm / (var + EPS) + 2 * V) + 4 * V
    dr = dr + 0.5 * (4 * 2.0 ** -24 * x64.abs().amax(1) / torch.sqrt(var + EPS))
    return m, r, dm, dr


def _normed(x64, kind, w, b):
    """the norm's rows, their bound, and the statistics"""
    m, r, dm, dr = _moments(x64, kind)
    w64 = 1.0 if w is None else w.double()
    y = (x64 - m[:, None]) * r[:, None] * w64
    bound = (dr[:, None] + 4 * V) * y.abs()
    if kind == "layer":
        bound = bound + ((dm + 2.0 ** -24 * x64.abs().amax(1)) * r)[:, None] * (1.0 if w is None else w64.abs())
    if b is not None:
        bound = bound + V * (y.abs() + b.double().abs())
        y = y + b.double()
    return y, bound, (m, r, dm, dr)


def _gate(g, groups, rows, width, ty):
    if groups is None:
        return None
    if groups == "channel":
        return _normal(g, (width,), 1.0, _dt(ty))
    return _normal(g, (rows if groups == "row" else groups, width), 1.0, _dt(ty))


def _by_row(gate, rows):
    if gate is None:
        return 1.0
    gate = gate.double().reshape(-1, gate.shape[-1])
    return gate.repeat_interleave(rows // gate.shape[0], 0)


def check_forward(rows, width, ty="bf16", wt="f32", kind="rms", post=True, groups="channel", gt="f32", weight=True,
                  bias=True, lh="plain", ly="plain", scale=0.75, wide_out=0, in_place=False):
    torch = _torch()
    import paper_2512_08365_amd as mag
    print(f"[case] residual_norm {rows}x{width} {ty} {wt} {kind} {post} {groups} {gt} {lh} {ly}", flush=True)
    dt, g, u = _dt(ty), _gen(31), _u(ty)
    h = _layout(_normal(g, (rows, width), 2.0, torch.float32).add_(0.5).to(dt), lh)
    y = _layout(_normal(g, (rows, width), 1.5, torch.float32).add_(-0.25).to(dt), ly)
    w = _normal(g, (width,), 1.0, _dt(wt)) if weight else None
    b = _normal(g, (width,), 1.0, _dt(wt)) if bias else None
    pw = _normal(g, (width,), 1.0, _dt(wt)) if post and weight else None
    pb = _normal(g, (width,), 1.0, _dt(wt)) if post and bias else None
    gate = _gate(g, groups, rows, width, gt)
    h64, y64 = h.double(), y.double()
    if in_place:
        out = (h, y)
    else:
        keep = [torch.full((rows, width + wide_out), 7.0, dtype=dt, device="cuda") for _ in range(2)]
        out = tuple(k[:, :width] for k in keep)
    stream, normed, stats = mag.residual_norm(
        h, y, w, b, kind=kind, gate=gate, scale=scale, post=post, post_weight=pw, post_bias=pb, eps=EPS,
        statistics=True, out=out)
    assert stream is out[0] and normed is out[1]
    if not in_place:
        assert all(bool((k[:, width:] == 7.0).all()) for k in keep)
    a, da, post_stats = (y64, 0 * y64, None) if not post else _normed(y64, kind, pw, pb)
    by = scale * _by_row(gate, rows)
    branch = by * a
    want = h64 + branch
    bound = (by.abs() if groups else scale) * da + 4 * V * branch.abs() + V * want.abs()
    _close(stream, want, bound + u * (want.abs() + bound) + _tiny(ty), "stream")
    n64, dn, own = _normed(stream.double(), kind, w, b)
    _close(normed, n64, dn + u * (n64.abs() + dn) + _tiny(ty), "normed")
    for at, found in ((0, own), (2, post_stats)):
        if found is None or kind == "rms":
            assert stats[at] is None
        else:
            _close(stats[at], found[0], found[2], "mean")
        if found is None:
            assert stats[at + 1] is None
        else:
            _close(stats[at + 1], found[1], found[3] * found[1], "rstd")


def check_backward(rows, width, ty="bf16", wt="f32", kind="rms", post=True, groups="channel", gt="f32", weight=True,
                   bias=True, lays=("plain",) * 4, d_stream=True, scale=0.75, in_place=False):
    torch = _torch()
    import paper_2512_08365_amd as mag
    print(f"[case] residual_norm_backward {rows}x{width} {ty} {wt} {kind} {post} {groups} {gt} {lays}", flush=True)
    dt, g, u = _dt(ty), _gen(32), _u(ty)
    h = _layout(_normal(g, (rows, width), 2.0, torch.float32).add_(0.5).to(dt), lays[0])
    y = _layout(_normal(g, (rows, width), 1.5, torch.float32).add_(-0.25).to(dt), lays[1])
    dn = _layout(_normal(g, (rows, width), 0.5, dt), lays[2])
    dr = _layout(_normal(g, (rows, width), 0.5, dt), lays[3]) if d_stream else None
    w = _normal(g, (width,), 1.0, _dt(wt)) if weight else None
    b = _normal(g, (width,), 1.0, _dt(wt)) if bias else None
    pw = _normal(g, (width,), 1.0, _dt(wt)) if post and weight else None
    pb = _normal(g, (width,), 1.0, _dt(wt)) if post and bias else None
    gate = _gate(g, groups, rows, width, gt)

    def stats(on):
        return (torch.randn(rows, generator=g, device="cuda") if on and kind == "layer" else None,
                torch.rand(rows, generator=g, device="cuda") + 0.5 if on else None)

    s = (*stats(True), *stats(post))
    # (64-bit copies first: gradients may be written over what they are made of)
    h64, y64, n64 = h.double(), y.double(), dn.double()
    r64 = dr.double() if d_stream else torch.zeros_like(h64)
    out = None
    if in_place:
        like = [None if x is None else torch.empty_like(x) for x in (gate, w, b, pw, pb)]
        out = (dr if d_stream else torch.empty_like(h), dn if width % 2 else y, *like)
    got = mag.residual_norm_backward(h, y, dn, dr, s, w, b, kind=kind, gate=gate, scale=scale, post=post,
                                     post_weight=pw, post_bias=pb, out=out)
    n = (width / 64 + 40) * 2.0 ** -24
    centre = kind == "layer"

    def mean(x):
        return x.mean(1, keepdim=True)

    def through(d, dd, hat, r):
        """a norm's gradient of d, which is off by dd: (gradient, bound)"""
        m1, m2 = (mean(d) if centre else 0 * mean(d)), mean(d * hat)
        e1 = (mean(dd) + n * mean(d.abs())) if centre else 0
        e2 = mean(dd * hat.abs()) + n * mean((d * hat).abs())
        want = r * (d - m1 - hat * m2)
        return want, r * (dd + e1 + hat.abs() * e2 + 8 * V * (d.abs() + m1.abs() + (hat * m2).abs()))

    def hat(x, m, r):
        return (x - (0 if m is None else m.double()[:, None])) * r.double()[:, None]

    hh = hat(h64, s[0], s[1])
    t = n64 * (w.double() if weight else 1.0)
    g64, bg = through(t, V * t.abs(), hh, s[1].double()[:, None])
    g64 = g64 + r64
    bg = bg + 2 * V * (g64.abs() + r64.abs())
    by = scale * _by_row(gate, rows)
    abs_by = by.abs() if gate is not None else abs(by)
    d = by * g64
    bd = abs_by * (bg + 3 * V * g64.abs())
    a64, a_mag, yn = y64, y64.abs(), y64
    dy, bdy = d, bd
    if post:
        yn = hat(y64, s[2], s[3])
        p64 = pw.double() if weight else torch.ones(width, dtype=torch.float64, device="cuda")
        q64 = pb.double() if pb is not None else torch.zeros_like(p64)
        a64, a_mag = yn * p64 + q64, (yn * p64).abs() + q64.abs()
        dy, bdy = through(d * p64, (bd + V * d.abs()) * p64.abs(), yn, s[3].double()[:, None])
    _close(got[0], g64, bg + u * (g64.abs() + bg) + _tiny(ty), "d_residual")
    _close(got[1], dy, bdy + u * (dy.abs() + bdy) + _tiny(ty), "d_branch")

    def over_rows(x, terms, off, count, ty, name):
        """x: sums of `count` terms, each off by `off`, in (count + 8) additions"""
        assert x.shape == terms.sum(-2).reshape(x.shape).shape
        want = terms.sum(-2).reshape(x.shape)
        bound = (off.sum(-2) + ((count + 8) * 2.0 ** -24 + 6 * V) * terms.abs().sum(-2)).reshape(x.shape)
        _close(x, want, bound + _u(ty) * (want.abs() + bound) + _tiny(ty), name)

    if gate is None:
        assert got[2] is None
    else:
        many = gate.numel() // width
        split = (many, rows // many, width)
        want = (scale * g64 * a64).view(split)
        # (summed as post_weight (g yn) + post_bias g)
        mags = (abs(scale) * g64.abs() * a_mag).view(split)
        off = (abs(scale) * bg * a_mag).view(split) + ((rows // many + 8) * 2.0 ** -24 + 6 * V) * mags
        over_rows(got[2], want, off, rows // many, gt, "d_gate")
    if weight:
        over_rows(got[3], n64 * hh, 3 * V * (n64 * hh).abs(), rows, wt, "dweight")
    if bias:
        over_rows(got[4], n64, 0 * n64, rows, wt, "dbias")
    if post and weight:
        over_rows(got[5], d * yn, (bd + 4 * V * d.abs()) * yn.abs(), rows, wt, "dpost_weight")
    if post and bias:
        over_rows(got[6], d, bd, rows, wt, "dpost_bias")
    for x, on in zip(got[3:], (weight, bias, post and weight, post and bias)):
        assert (x is not None) == bool(on)


KINDS = ["rms", "layer"]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(width, ty):
    for i, kind in enumerate(KINDS):
        check_forward(5, width, ty, "f32", kind, post=bool((width + i) % 2), groups=("channel", None, "row")[width % 3])
        check_forward(6, width, ty, ty, kind, groups=3, gt=ty, weight=width % 2 == 0, bias=width % 3 == 0,
                      post=bool((width + i + 1) % 2))


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_backward_widths(width, ty):
    for i, kind in enumerate(KINDS):
        check_backward(5, width, ty, "f32", kind, post=bool((width + i) % 2), groups=("channel", None, "row")[width % 3])
        check_backward(66, width, ty, ty, kind, groups=3, gt=ty, weight=width % 2 == 0, bias=width % 3 == 0,
                       post=bool((width + i + 1) % 2), d_stream=width % 5 != 0)


LAYS = ["plain", "gap", "gap8", "columns", "shifted", "every2"]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("lay", LAYS)
def test_layouts(lay, ty):
    for k, width in enumerate((200, 777, 1536)):
        for other in ("plain", "gap", "every2"):
            check_forward(18, width, ty, "f32", KINDS[k % 2], lh=lay, ly=other, wide_out=(0, 3, 8)[k], groups=2)
            check_forward(18, width, ty, ty, KINDS[k % 2], lh=other, ly=lay, post=False)
        for at in range(4):
            lays = ["plain"] * 4
            lays[at] = lay
            check_backward(18, width, ty, "f32", KINDS[at % 2], lays=lays, groups=(None, "channel", 2, "row")[at])


@pytest.mark.parametrize("groups", [None, "channel", 2, 5, 300, 700, "row"])
@pytest.mark.parametrize("width", [72, 264, 1021, 2056])
def test_groups(width, groups):
    """gates of few samples (rows in chunks) and of many (whole samples a workgroup)"""
    for each in (1, 2, 3, 9):
        rows = each * (groups if isinstance(groups, int) else 350)
        kind = KINDS[each % 2]
        check_forward(rows, width, "bf16", kind=kind, groups=groups, post=each != 2)
        check_backward(rows, width, "bf16", kind=kind, groups=groups, post=each != 2)
        check_backward(rows, width, "f32", kind=kind, groups=groups, post=each == 2, d_stream=False)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("size", [(1, 4096), (2, 64), (300, 1021), (5000, 264), (40000, 72), (3000, 4096), (600, 10000),
                                  (100, 16392), (70, 20000)], ids=lambda s: "x".join(map(str, s)))
def test_sizes(size, ty):
    for kind in KINDS:
        check_forward(*size, ty, ty, kind, groups=2 if size[0] % 2 == 0 else None)
        check_backward(*size, ty, ty, kind, groups=2 if size[0] % 2 == 0 else "channel")


@pytest.mark.parametrize("width", [200, 777, 4096, 5000, 20000])
def test_in_place(width):
    for lay in ("plain", "gap"):
        check_forward(34, width, "bf16", groups=2, lh=lay, ly=lay, in_place=True)
        check_backward(34, width, "bf16", groups=2, lays=(lay,) * 4, in_place=True)


def test_scales_and_shared_gates():
    import paper_2512_08365_amd as mag
    torch = _torch()
    for scale in (0.0, -1.5, 1e-3):
        check_forward(12, 520, "f32", scale=scale, groups=3)
        check_backward(12, 520, "f32", scale=scale, groups=3)
    # a gate read again for every group, and one whose rows are apart
    g = _gen(5)
    h, y = (_normal(g, (12, 260), 1.0, torch.float32) for _ in range(2))
    one = _normal(g, (260,), 1.0, torch.float32)
    want = mag.residual_norm(h, y, gate=one)
    for gate in (one.expand(4, 260), torch.cat([one.repeat(3, 1)] * 2, 1)[:, :260]):
        for a, b in zip(mag.residual_norm(h, y, gate=gate), want):
            assert torch.equal(a, b)


def test_need_and_nothing():
    import paper_2512_08365_amd as mag
    torch = _torch()
    g = _gen(6)
    h, y, dn, dr = (_normal(g, (24, 300), 1.0, torch.bfloat16) for _ in range(4))
    w, gate = _normal(g, (300,), 1.0, torch.float32), _normal(g, (4, 300), 1.0, torch.float32)
    stream, normed, stats = mag.residual_norm(h, y, w, gate=gate, statistics=True)
    # without statistics, and leading dimensions
    for a, b in zip(mag.residual_norm(h.view(4, 6, 300), y.view(4, 6, 300), w, gate=gate), (stream, normed)):
        assert a.shape == (4, 6, 300) and torch.equal(a.view(24, 300), b)
    every = mag.residual_norm_backward(stream, y, dn, dr, stats, w, gate=gate)
    for need in ((True, False, False), (False, True, False), (False, False, True), (False, False, False)):
        got = mag.residual_norm_backward(stream, y, dn, dr, stats, w, gate=gate, need=need)
        on = (need[0], need[1], need[2], need[2], False, False, False)
        for a, b, wanted in zip(got, every, on):
            assert (a is None) if not wanted else torch.equal(a, b)
    # no rows: gradients of zero
    none = [x[:0] for x in (h, y, dn, dr)]
    assert mag.residual_norm(*none[:2], w, gate=gate)[1].shape == (0, 300)
    empty = torch.empty(0, device="cuda")
    got = mag.residual_norm_backward(*none, (None, empty, None, None), w, gate=gate)
    assert got[0].shape == (0, 300) and not bool(got[2].any()) and not bool(got[3].any())


def test_infinities_and_nan_stay_in_their_rows():
    import paper_2512_08365_amd as mag
    torch = _torch()
    for width in (264, 4096, 20000):
        g = _gen(7)
        h, y, dn, dr = (_normal(g, (40, width), 1.0, torch.float32) for _ in range(4))
        w = _normal(g, (width,), 1.0, torch.float32)
        clean = mag.residual_norm(h, y, w, post=True, statistics=True)
        grads = mag.residual_norm_backward(clean[0], y, dn, dr, clean[2], w, post=True)
        for bad in (float("nan"), float("inf"), -float("inf")):
            h2, dn2 = h.clone(), dn.clone()
            h2[7, 3] = dn2[20, width - 1] = bad
            got = mag.residual_norm(h2, y, w, post=True, statistics=True)
            keep = torch.arange(40, device="cuda") != 7
            assert torch.equal(got[0][keep], clean[0][keep]) and torch.equal(got[1][keep], clean[1][keep])
            assert bool(got[1][7].isnan().any())
            back = mag.residual_norm_backward(clean[0], y, dn2, dr, clean[2], w, post=True)
            keep = torch.arange(40, device="cuda") != 20
            assert torch.equal(back[0][keep], grads[0][keep]) and torch.equal(back[1][keep], grads[1][keep])
            assert bool(back[0][20].isnan().any())
            columns = torch.arange(width, device="cuda") != width - 1
            assert torch.equal(back[3][columns], grads[3][columns]) and not math.isfinite(float(back[3][-1]))


def test_gradients_against_differences():
    """the sum of both outputs with random weights, along random steps, in 64 bits"""
    import paper_2512_08365_amd as mag
    torch = _torch()
    for kind in KINDS:
        for post in (False, True):
            g = _gen(8)
            f64 = {"h": (12, 96), "y": (12, 96), "w": (96,), "b": (96,), "gate": (3, 96), "pw": (96,), "pb": (96,)}
            x = {k: _normal(g, s, 1.0, torch.float32) for k, s in f64.items()}
            if not post:
                x["pw"] = x["pb"] = None
            dn, dr = (_normal(g, (12, 96), 1.0, torch.float32) for _ in range(2))

            def value(x):
                y = x["y"]
                if post:
                    y = _normed(y, kind, x["pw"], x["pb"])[0]
                s = x["h"] + 0.7 * x["gate"].repeat_interleave(4, 0) * y
                return (_normed(s, kind, x["w"], x["b"])[0] * dn.double()).sum() + (s * dr.double()).sum()

            stream, _, stats = mag.residual_norm(x["h"], x["y"], x["w"], x["b"], kind=kind, gate=x["gate"], scale=0.7,
                                                 post=post, post_weight=x["pw"], post_bias=x["pb"], statistics=True)
            got = mag.residual_norm_backward(stream, x["y"], dn, dr, stats, x["w"], x["b"], kind=kind, gate=x["gate"],
                                             scale=0.7, post=post, post_weight=x["pw"], post_bias=x["pb"])
            d = {k: v.double() for k, v in x.items() if v is not None}
            for name, grad in zip(("h", "y", "gate", "w", "b", "pw", "pb"), got):
                if grad is None:
                    continue
                step = torch.randn(d[name].shape, generator=g, device="cuda").double()
                size = 1e-5
                up = value({**x, **d, name: d[name] + size * step})
                down = value({**x, **d, name: d[name] - size * step})
                slope = float((up - down) / (2 * size))
                along = float((grad.double() * step).sum())
                # differences: third derivatives times 1e-10 and roundings over 1e-5; fp32 gradients
                scale = float((grad.double() * step).abs().sum())
                assert abs(slope - along) <= 2e-5 * scale + 1e-6, (kind, post, name, slope, along)


def test_repeats_bit_for_bit_and_replays():
    """the same call twice, and both passes captured and replayed between eager work"""
    import paper_2512_08365_amd as mag
    torch = _torch()
    g = _gen(9)
    h, y, dn, dr = (_normal(g, (900, 1024), 1.0, torch.bfloat16) for _ in range(4))
    w, pw, gate = (_normal(g, s, 1.0, torch.float32) for s in ((1024,), (1024,), (3, 1024)))
    kw = dict(gate=gate, post=True, post_weight=pw)

    def step():
        s, n, stats = mag.residual_norm(h, y, w, statistics=True, **kw)
        return [s, n, stats[1], stats[3], *(x for x in mag.residual_norm_backward(
            s, y, dn, dr, stats, w, **kw) if x is not None)]

    first = step()
    for a, b in zip(first, step()):
        assert torch.equal(a, b)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for k in range(4):
        for x in (h, y, dn, dr):
            x.copy_(_normal(_gen(40 + k), x.shape, 1.0, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, step()):
            assert torch.equal(a, b)


def test_refusals():
    import paper_2512_08365_amd as mag
    torch = _torch()
    h = torch.zeros((12, 64), device="cuda")
    w = torch.ones(64, device="cuda")

    def refused(call, code):
        with pytest.raises(mag.MagnetonError) as e:
            call()
        assert e.value.code == code, e.value

    refused(lambda: mag.residual_norm(h, h.bfloat16()), -2)
    refused(lambda: mag.residual_norm(h, h[:, :63]), -2)
    refused(lambda: mag.residual_norm(h, h, w[:63]), -2)
    refused(lambda: mag.residual_norm(h, h, w, w.half()), -2)
    refused(lambda: mag.residual_norm(h, h, w, kind="group"), -2)
    refused(lambda: mag.residual_norm(h, h, w, gate=torch.ones((5, 64), device="cuda")), -2)
    refused(lambda: mag.residual_norm(h, h, w, gate=torch.ones((3, 63), device="cuda")), -2)
    refused(lambda: mag.residual_norm(h, h, w, gate=torch.ones((64, 3), device="cuda").t()), -2)
    refused(lambda: mag.residual_norm(h, h, w, gate=w.half()), -2)
    refused(lambda: mag.residual_norm(h, h, w, post_weight=w), -2)
    refused(lambda: mag.residual_norm(h, h, w, eps=-1.0), -2)
    refused(lambda: mag.residual_norm(h, h, w, scale=float("nan")), -2)
    refused(lambda: mag.residual_norm(h, h, w, out=(h.t().contiguous().t(), h)), -2)
    refused(lambda: mag.residual_norm(h.cpu(), h, w), -1)
    refused(lambda: mag.residual_norm(h, h, w.cpu()), -1)
    r = torch.ones(12, device="cuda")
    refused(lambda: mag.residual_norm_backward(h, h, h, h, (None, None, None, None), w), -1)
    refused(lambda: mag.residual_norm_backward(h, h, h, h, (None, r, None, None), w, kind="layer"), -1)
    refused(lambda: mag.residual_norm_backward(h, h, h, h, (None, r, None, None), w, post=True), -1)
    refused(lambda: mag.residual_norm_backward(h, h, h, h, (None, r[:11], None, None), w), -2)
    refused(lambda: mag.residual_norm_backward(h, h, h, h, (r, r), w), -2)
    refused(lambda: mag.residual_norm_backward(h, h, h, h, (None, r, None, None), w, workspace=torch.empty(
        8, dtype=torch.uint8, device="cuda")), -4)


@pytest.mark.parametrize("size", [(131080, 72), (65540, 700), (32776, 1100), (16392, 2056)],
                         ids=lambda s: "x".join(map(str, s)))
def test_groups_of_many_rows(size):
    """samples so long that workgroups go through them side by side"""
    for groups in (2, "channel"):
        check_forward(*size, "bf16", kind="layer", groups=groups)
        check_backward(*size, "bf16", kind="rms", groups=groups)


@pytest.mark.parametrize("width", [1, 3, 7, 8, 9, 15, 505, 513, 1023, 1025, 2041, 4089, 8191, 8193, 8199, 10241, 12295])
def test_ends_of_rows(width):
    """every place at which a row can end amid eight neighbours, around the widths where kernels
    change, rows at any element"""
    for ty in ("bf16", "f32"):
        for at, lay in enumerate(("plain", "gap", "shifted")):
            lays = ["plain"] * 4
            lays[at] = lay
            check_forward(9, width, ty, ty, KINDS[at % 2], lh=lay, ly="gap", groups=3, wide_out=at)
            check_backward(9, width, ty, "f32", KINDS[at % 2], lays=lays, groups=(3, "row", "channel")[at])


def test_more_refusals():
    import paper_2512_08365_amd as mag
    torch = _torch()
    h, r = torch.zeros((12, 64), device="cuda"), torch.ones(12, device="cuda")
    out = torch.full((12, 64), 7.0, device="cuda")
    for call in (lambda: mag.residual_norm(h, h, out=(out, out)), lambda: mag.residual_norm(h, h, out=(out,)),
                 lambda: mag.residual_norm_backward(h, h, h, h, (None, r, None, None),
                                                    out=(out, out, None, None, None, None, None))):
        with pytest.raises(mag.MagnetonError) as e:
            call()
        assert e.value.code == -2
    assert bool((out == 7).all())


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("width", [3, 72, 700, 1500, 2056, 3001, 4096, 5000, 8192, 8200, 16384, 20000])
def test_gradients_of_no_rows_are_zero(width, ty):
    """whatever the outputs and the workspace held before"""
    import paper_2512_08365_amd as mag
    torch = _torch()
    for groups in (None, 1, 3, 600):
        for wt in (ty, "f32"):
            x = torch.empty((0, width), dtype=_dt(ty), device="cuda")
            w, gate = torch.ones(width, dtype=_dt(wt), device="cuda"), None
            if groups:
                gate = torch.ones((groups, width), dtype=_dt(wt), device="cuda")
            stats = (torch.empty(0, device="cuda"),) * 4
            nan = float("nan")
            out = (x, x, None if gate is None else torch.full_like(gate, nan),
                   *(torch.full_like(w, nan) for _ in range(4)))
            ws = torch.full((mag.residual_norm_backward_workspace_size(x, gate) // 4 + 64,), nan, device="cuda")
            got = mag.residual_norm_backward(x, x, x, x, stats, w, w, kind="layer", gate=gate, post=True, post_weight=w,
                                             post_bias=w, out=out, workspace=ws)
            for grad in got[2:]:
                assert grad is None or bool((grad == 0).all()), (groups, wt)


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("width", [8200, 8207, 10240, 10241, 12289, 16384])
def test_wide_rows_in_place(width, ty):
    """rows that several workgroups share while they are written over, ends in a workgroup of
    their own among them"""
    for lay in ("plain", "gap"):
        for kind, groups in (("layer", 2), ("rms", "row")):
            check_forward(34, width, ty, kind=kind, groups=groups, lh=lay, ly=lay, in_place=True)
            check_backward(34, width, ty, kind=kind, groups=groups, lays=(lay,) * 4, in_place=True)
    check_backward(700, width, ty, groups="channel", post=False, in_place=True)

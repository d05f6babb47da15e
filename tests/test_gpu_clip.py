"""The common norm of many tensors, and tensors clipped by it, against 64-bit forms.

Tolerances: squares are exact to 2^-53 and added in 64 bits, the norm is rounded to fp32
once (2^-24), and so are the factor and its product; outputs are rounded once more."""
import math

import pytest

from test_gpu_block import V, _close, _dt, _gen, _normal, _tiny, _torch, _u

pytestmark = pytest.mark.gpu
TYPES = ["f32", "f16", "bf16"]


def _tensors(seed, shapes, scale=1.0):
    g = _gen(seed)
    return [_normal(g, s, scale, _dt(TYPES[i % 3])) for i, s in enumerate(shapes)]


def _norm64(tensors, kind):
    if kind == 2:
        return math.sqrt(math.fsum(float(t.double().square().sum()) for t in tensors))
    return max([float(t.double().abs().max()) for t in tensors if t.numel()], default=0.0)


def check_clip(tensors, most, kind=2, eps=1e-6, out=None, **kw):
    torch = _torch()
    import paper_2512_08365_amd as mag
    before = [t.double() for t in tensors]
    want = _norm64(tensors, kind)
    alone = mag.gradient_norm(tensors, kind=kind)
    assert abs(float(alone) - want) <= 2.0 ** -24 * 1.01 * want
    norm = mag.clip_gradients(tensors, most, kind=kind, eps=eps, out=out, **kw)
    assert torch.equal(norm, alone)
    by = min(1.0, most / (want + eps)) if want + eps > 0 else 1.0
    for t, b, o in zip(tensors, before, out or tensors):
        ty = {v: k for k, v in ((k, _dt(k)) for k in TYPES)}[t.dtype]
        _close(o, b * by, (2 * V + _u(ty) * (1 + V)) * (b * by).abs() + _tiny(ty), f"{tuple(t.shape)} {ty}")
        if out is not None:
            assert torch.equal(t.double(), b)
        if by == 1.0:
            assert torch.equal(o.double(), b)


SHAPES = {
    "one": [(1,)],
    "scalars": [(), (1,), (1, 1), ()],
    "odd": [(7,), (1021, 3), (5, 5, 5), (8191,), (8192,), (8193,), (0,), (16385,), (3, 0, 2)],
    "block": [(2304, 768), (2304,), (768, 2304), (768,), (768,), (768,)],
    "many": [(k % 97 + 1, k % 13 + 1) for k in range(200)],
    "exactly a launch": [(33,)] * 64,
    "one more": [(33,)] * 65,
    "large": [(4096, 4096), (3000, 5001), (17,)],
}


@pytest.mark.parametrize("kind", [2, math.inf])
@pytest.mark.parametrize("name", list(SHAPES))
def test_clip(name, kind):
    torch = _torch()
    for most in (0.0, 0.37, 1e9):
        print(f"[case] clip {name} {kind} {most}", flush=True)
        tensors = _tensors(3, SHAPES[name], 0.3)
        check_clip(tensors, most, kind)
        tensors = _tensors(4, SHAPES[name], 0.3)
        check_clip(tensors, most, kind, out=[torch.full_like(t, 7.0) for t in tensors])


def test_layouts():
    """transposed and permuted tensors, rows of a wider buffer, columns of one buffer,
    any element's alignment"""
    import paper_2512_08365_amd as mag
    torch = _torch()
    g = _gen(5)
    for ty in TYPES:
        wide = _normal(g, (300, 777), 1.0, _dt(ty))
        other = _normal(g, (40, 30, 20), 1.0, _dt(ty))
        flat = _normal(g, (100003,), 1.0, _dt(ty))
        keep = [t.clone() for t in (wide, other, flat)]
        tensors = [wide[:, :256], wide[:, 256:700], other.permute(2, 0, 1), flat[1:50002], flat[50002:],
                   _normal(g, (64, 33), 1.0, _dt(ty)).t()]
        check_clip(tensors, 1.0)
        # what lies between stays as it was
        assert torch.equal(wide[:, 700:], keep[0][:, 700:]) and torch.equal(flat[:1], keep[2][:1])
        # into rows of another width
        tensors = [_normal(g, (300, 77), 1.0, _dt(ty)), _normal(g, (9, 77), 1.0, _dt(ty))]
        buffer = torch.full((309, 80), 7.0, dtype=_dt(ty), device="cuda")
        check_clip(tensors, 1.0, out=[buffer[:300, :77], buffer[300:, 3:]])
        assert bool((buffer[:300, 77:] == 7).all()) and bool((buffer[300:, :3] == 7).all())
    # the norm alone takes tensors that overlap, each counted
    x = _normal(g, (500,), 1.0, torch.float32)
    assert abs(float(mag.gradient_norm([x, x, x[100:]])) - _norm64([x, x, x[100:]], 2)) <= 1e-5


def test_values():
    """infinities, NaN, the ends of the range, zeros"""
    import paper_2512_08365_amd as mag
    torch = _torch()

    def one(values, kind, most=1.0, ty=torch.float32):
        t = [torch.tensor(values, dtype=ty, device="cuda"), torch.ones(9000, dtype=ty, device="cuda")]
        return float(mag.clip_gradients(t, most, kind=kind)), t

    for kind in (2, math.inf):
        norm, t = one([3e38, -3e38, 1e30], kind)
        assert norm == (math.inf if kind == 2 else float(torch.tensor(3e38)))
        # (the norm passes fp32, the factor does not)
        want = 1.0 / math.sqrt(2 * 9e76 + 1e60 + 9000) if kind == 2 else 1 / 3e38
        assert abs(float(t[0][0]) / (3e38 * want) - 1) < 1e-6
        norm, t = one([math.inf, 1.0, -2.0], kind)
        assert norm == math.inf and math.isnan(float(t[0][0])) and not bool(t[1].any())
        assert t[0][1:].tolist() == [0.0, 0.0]
        norm, t = one([math.nan, 1.0, math.inf], kind)
        assert math.isnan(norm) and bool(t[0].isnan().all()) and bool(t[1].isnan().all())
    # squares below fp32's range count
    tiny = torch.full((10000,), 1e-30, device="cuda")
    assert abs(float(mag.gradient_norm([tiny])) / 1e-28 - 1) < 1e-6
    zeros = [torch.zeros(100, device="cuda")]
    assert float(mag.clip_gradients(zeros, 1.0)) == 0.0 and not bool(zeros[0].any())
    assert float(mag.clip_gradients(zeros, 0.0, eps=0.0)) == 0.0 and bool(zeros[0].isnan().all())


def test_lists():
    """a kept list sees new values; None is left out; a given norm and workspace"""
    import paper_2512_08365_amd as mag
    torch = _torch()
    tensors = _tensors(6, [(1000, 10), (77,), (5,)])
    kept = mag.TensorList([tensors[0], None, *tensors[1:]])
    assert len(kept) == 3
    norm = torch.empty((), device="cuda")
    ws = torch.empty(mag.clip_gradients_workspace_size(kept), dtype=torch.uint8, device="cuda")
    for k in range(3):
        for t in tensors:
            t.copy_(_normal(_gen(k), t.shape, 1.0, t.dtype))
        want = [t.clone() for t in tensors]
        other = mag.clip_gradients(want, 2.0)
        assert mag.clip_gradients(kept, 2.0, norm=norm, workspace=ws) is norm
        assert torch.equal(norm, other)
        for a, b in zip(tensors, want):
            assert torch.equal(a, b)


def test_repeats_and_replays():
    import paper_2512_08365_amd as mag
    torch = _torch()
    tensors = _tensors(7, [(3000, 700), (64, 3), (9999,)] * 30)
    out = [torch.empty_like(t) for t in tensors]
    first = mag.clip_gradients(tensors, 1.0, out=out)
    keep = [t.clone() for t in out]
    again = mag.clip_gradients(tensors, 1.0, out=out)
    assert torch.equal(first, again) and all(torch.equal(a, b) for a, b in zip(out, keep))
    kept = mag.TensorList(tensors, out=out)
    ws = torch.empty(mag.clip_gradients_workspace_size(kept), dtype=torch.uint8, device="cuda")
    norm = torch.empty((), device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        mag.clip_gradients(kept, 1.0, norm=norm, workspace=ws)
    for k in range(3):
        for t in tensors:
            t.copy_(_normal(_gen(k + 50), t.shape, 1.0, t.dtype))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        eager = [torch.empty_like(t) for t in tensors]
        assert torch.equal(mag.clip_gradients(tensors, 1.0, out=eager), norm)
        assert all(torch.equal(a, b) for a, b in zip(got, eager))


def test_refusals():
    import paper_2512_08365_amd as mag
    torch = _torch()
    x = torch.ones((20, 30), device="cuda")

    def refused(call, code=-2):
        with pytest.raises(mag.MagnetonError) as e:
            call()
        assert e.value.code == code, e.value

    refused(lambda: mag.clip_gradients([x.double()], 1.0))
    refused(lambda: mag.clip_gradients([x.cpu()], 1.0), -1)
    refused(lambda: mag.clip_gradients([], 1.0))
    refused(lambda: mag.clip_gradients([None], 1.0))
    refused(lambda: mag.clip_gradients([x], -1.0))
    refused(lambda: mag.clip_gradients([x], math.inf))
    refused(lambda: mag.clip_gradients([x], math.nan))
    refused(lambda: mag.clip_gradients([x], 1.0, kind=1))
    refused(lambda: mag.clip_gradients([x], 1.0, eps=-1.0))
    refused(lambda: mag.clip_gradients([x], 1.0, out=[x[:10]]))
    refused(lambda: mag.clip_gradients([x], 1.0, out=[x.half()]))
    refused(lambda: mag.clip_gradients([x], 1.0, out=[x, x]))
    refused(lambda: mag.clip_gradients(mag.TensorList([x]), 1.0, out=[x]))
    # the same tensor twice, tensors that overlap, an output on another tensor
    refused(lambda: mag.clip_gradients([x, x], 1.0))
    refused(lambda: mag.clip_gradients([x[:11], x[10:]], 1.0))
    refused(lambda: mag.clip_gradients([x[:, :11], x[:, 10:]], 1.0))
    y = torch.ones((20, 30), device="cuda")
    refused(lambda: mag.clip_gradients([x, y], 1.0, out=[y, x]))
    refused(lambda: mag.clip_gradients([x[:10], x[10:]], 1.0, out=[x[5:15], y[:10]]))
    refused(lambda: mag.clip_gradients([x[::2, ::2]], 1.0))
    refused(lambda: mag.clip_gradients([torch.ones(1, device="cuda").expand(5, 7)], 1.0))
    refused(lambda: mag.clip_gradients([x], 1.0, norm=torch.empty(2, device="cuda")))
    refused(lambda: mag.clip_gradients([x], 1.0, workspace=torch.empty(0, dtype=torch.uint8, device="cuda")), -1)
    assert bool((x == 1).all()) and bool((y == 1).all())


def test_clip_past_the_caches():
    """a list that no cache holds: other stores, and none where nothing is clipped in place"""
    torch = _torch()
    for kind in (2, math.inf):
        for most in (1.0, 1e9):
            tensors = _tensors(8, [(8192, 4099), (3,), (8192, 4100), (1021, 7)], 0.3)
            check_clip(tensors, most, kind, out=[torch.full_like(t, 7.0) for t in tensors])
            check_clip(tensors, most, kind)


def test_workspace_of_plain_tensors():
    import paper_2512_08365_amd as mag
    torch = _torch()
    for n in (1, 3, 70, 1000):
        tensors = [torch.ones(k % 50 + 1, device="cuda") for k in range(n)]
        assert mag.clip_gradients_workspace_size(tensors) == mag.clip_gradients_workspace_size(mag.TensorList(tensors))
        ws = torch.empty(mag.clip_gradients_workspace_size(tensors), dtype=torch.uint8, device="cuda")
        want = math.sqrt(sum(t.numel() for t in tensors))
        assert abs(float(mag.clip_gradients(tensors, 1.0, workspace=ws)) - want) <= 2.0 ** -23 * want


def test_slices_of_one_buffer():
    """slices that share no element: a single row's, every second row's, other columns'"""
    torch = _torch()
    for ty in TYPES:
        buffer = _normal(_gen(9), (41, 777), 1.0, _dt(ty))
        keep = buffer.clone()
        tensors = [buffer[0:1, :256], buffer[1:, :256], buffer[::2, 256:600], buffer[1::2, 256:700], buffer[4:5, 600:650],
                   buffer[6:20:2, 601:700]]
        check_clip(tensors, 1.0)
        left = torch.ones_like(buffer, dtype=torch.bool)
        for t in (left[:, :256], left[::2, 256:600], left[1::2, 256:700], left[4:5, 600:650], left[6:20:2, 601:700]):
            t[:] = False
        assert torch.equal(buffer[left], keep[left])
        check_clip([buffer[0:1, :256], buffer[:, 256:]], 0.5, out=[keep[7:8, 3:259], keep[8:, :].new_empty(41, 521)])


def test_factors_below_fp32():
    """a factor that is a subnormal number of fp32, or none of it any more, still counts for
    all its digits where its products are normal numbers"""
    import paper_2512_08365_amd as mag
    torch = _torch()
    for ty in ("f32", "bf16"):
        for kind in (2, math.inf):
            for most in (1e-5, 3e-7, 1e-2, 5e-30, 1e-36):
                g = _gen(12)
                x = torch.cat([_normal(g, (9001,), 5e37, torch.float32).clamp(-3e38, 3e38),
                               _normal(g, (300,), 1e36, torch.float32)]).to(_dt(ty))
                keep = x.double()
                norm = _norm64([x], kind)
                for out in (None, [torch.empty_like(x)]):
                    y = x.clone()
                    mag.clip_gradients([y], most, kind=kind, out=out)
                    want = keep * (most / (norm + 1e-6))
                    _close((out or [y])[0], want, (2 * V + _u(ty) * (1 + V)) * want.abs() + 2 * _tiny(ty), f"{ty} {kind} {most}")

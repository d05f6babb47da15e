"""A block's training step by the operators together: norms around the block, 8-bit
products and their gradients, clipping; eager, on a stream of its own and captured.

Tolerances.  Of the whole step: an 8-bit rounding is off by at most 2^-4 of a number, in
the root mean square of evenly spread numbers by 2^-4 / sqrt(3) = 0.036.  On the longest
path (normed rows, weight, hidden rows, second weight; the same for the gradients) lie
at most 12 of them, independent of one another: sqrt(12) 0.036 = 0.125 of a gradient's
2-norm; two-byte roundings, 2^-9 each, are below a tenth of that.  What does not pass
an 8-bit product is compared by the 64-bit formula on the step's own numbers."""
import math

import pytest

from test_gpu_block import V, _gen, _normal, _torch

pytestmark = pytest.mark.gpu

PATH = math.sqrt(12) * 2.0 ** -4 / math.sqrt(3) * 1.1


def _problem(rows, width, inner, seed):
    torch = _torch()
    g = _gen(seed)
    bf = torch.bfloat16
    return {"h": _normal(g, (rows, width), 1.0, bf), "y": _normal(g, (rows, width), 1.0, bf),
            "w": 1 + _normal(g, (width,), 0.2, torch.float32), "pw": 1 + _normal(g, (width,), 0.2, torch.float32),
            "gate": _normal(g, (2, width), 0.5, bf), "w1": _normal(g, (inner, width), width ** -0.5, bf),
            "b1": _normal(g, (inner,), 0.1, bf), "w2": _normal(g, (width, inner), inner ** -0.5, bf),
            "d_out": _normal(g, (rows, width), 1.0, bf), "d_stream": _normal(g, (rows, width), 0.5, bf)}


def _slope(z, dz):
    """dz times the slope of the tanh GELU, elementary operations"""
    torch = _torch()
    z, k = z.float(), math.sqrt(2 / math.pi)
    t = torch.tanh(k * (z + 0.044715 * z ** 3))
    return (dz.float() * (0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z))).to(dz.dtype)


def step(p):
    """(gradients, their norm, intermediate results)"""
    import paper_2512_08365_amd as mag
    norms = dict(kind="rms", gate=p["gate"], scale=0.5, post=True, post_weight=p["pw"])
    stream, normed, stats = mag.residual_norm(p["h"], p["y"], p["w"], statistics=True, **norms)
    q, s, qt, st = mag.quantize_fp8(normed, transposed=True)
    w1, s1, w1t, s1t = mag.quantize_fp8(p["w1"], 128, transposed=True)
    w2, s2, w2t, s2t = mag.quantize_fp8(p["w2"], 128, transposed=True)
    hidden, pre = mag.linear_fp8(q, s, w1, s1, p["b1"], activation="gelu_tanh", pre=True)
    u, su, ut, sut = mag.quantize_fp8(hidden, transposed=True)
    out = mag.linear_fp8(u, su, w2, s2, residual=stream)
    d, sd, dt, sdt = mag.quantize_fp8(p["d_out"], transposed=True)
    dz = _slope(pre, mag.linear_fp8(d, sd, w2t, s2t))
    e, se, et, set_ = mag.quantize_fp8(dz, transposed=True)
    d_normed = mag.linear_fp8(e, se, w1t, s1t)
    d_h, d_y, d_gate, d_w, _, d_pw, _ = mag.residual_norm_backward(
        stream, p["y"], d_normed, p["d_stream"], stats, p["w"], **norms)
    grads = {"h": d_h, "y": d_y, "gate": d_gate, "w": d_w, "pw": d_pw,
             "w1": mag.linear_fp8(et, set_, qt, st), "w2": mag.linear_fp8(dt, sdt, ut, sut)}
    clipped = {k: g.clone() for k, g in grads.items()}
    norm = mag.clip_gradients(list(clipped.values()), 1.0)
    return grads, clipped, norm, {"stream": stream, "normed": normed, "d_normed": d_normed, "out": out}


def _by_autograd(p):
    """the same step in 64 bits, without a rounding"""
    torch = _torch()
    t = {k: v.double().requires_grad_() for k, v in p.items() if k not in ("d_out", "d_stream")}

    def norm(x, w):
        return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5) * w

    rows = p["h"].shape[0]
    stream = t["h"] + 0.5 * t["gate"].repeat_interleave(rows // 2, 0) * norm(t["y"], t["pw"])
    z = torch.mm(norm(stream, t["w"]), t["w1"].t()) + t["b1"]
    k = math.sqrt(2 / math.pi)
    hidden = 0.5 * z * (1 + torch.tanh(k * (z + 0.044715 * z ** 3)))
    out = torch.mm(hidden, t["w2"].t())
    ((out * p["d_out"].double()).sum() + (stream * p["d_stream"].double()).sum()).backward()
    return {k: v.grad for k, v in t.items()}, out.detach() + stream.detach()


@pytest.mark.parametrize("size", [(64, 256, 512), (130, 264, 1021), (600, 1024, 2100)])
def test_step(size):
    torch = _torch()
    p = _problem(*size, seed=sum(size))
    grads, clipped, norm, mid = step(p)
    want, out = _by_autograd(p)
    for k, g in grads.items():
        off = float((g.double() - want[k]).norm() / want[k].norm())
        assert off <= PATH, (k, off)
    assert float((mid["out"].double() - out).norm() / out.norm()) <= PATH
    # clipping, on the step's own gradients
    n64 = math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads.values()))
    assert abs(float(norm) - n64) <= 2.0 ** -23 * n64
    for k, g in clipped.items():
        x = grads[k].double() * min(1.0, 1.0 / (n64 + 1e-6))
        u = torch.finfo(g.dtype).eps / 2
        assert bool(((g.double() - x).abs() <= (2 * V + u * (1 + V)) * x.abs() + torch.finfo(g.dtype).tiny * u * 2).all()), k


def test_step_on_a_stream_and_captured():
    torch = _torch()
    p = _problem(130, 264, 1021, 3)
    want = step(p)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        got = step(p)
    other.synchronize()

    def same(a, b):
        for x, y in zip((*a[0].values(), *a[1].values(), a[2], *a[3].values()),
                        (*b[0].values(), *b[1].values(), b[2], *b[3].values())):
            assert torch.equal(x, y)

    same(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step(p)
    for seed in (4, 5, 6):
        for k, v in _problem(130, 264, 1021, seed).items():
            p[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        same(kept, step(p))
        torch.cuda.synchronize()

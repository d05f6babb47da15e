"""A feed-forward block done two ways, compared as two systems.

A pre-norm block, y = x + W2 gelu(W1 norm(x) + b1) + b2: one training step of it
(forward, backward, orthogonalised updates of both weights) and a few single
tokens.  System A runs the library's operators, each one pass over its data;
system B the same formulas as one elementary operation after another.  Every
operator's run is an interval with a key; a power trace over these intervals is
attributed to them, the two systems' operators are ranked by relative energy, and
their outputs are matched by their tensor invariants.

    python examples/feed_forward_energy.py [--tokens 2048 --hidden 768 --inner 2304 --dtype bf16]

There is no meter here: the trace is synthetic, `idle` watts and `busy` ones while
an operator runs.  A measured one goes in its place as it is (seconds, watts).
"""

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2512_08365_amd as mag  # noqa: E402

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-5


class Intervals:
    """The operators' runs: events around each, read once all have run."""

    def __init__(self):
        self.names, self.runs = [], []
        self.begin = torch.cuda.Event(enable_timing=True)
        self.begin.record()

    def __call__(self, name, call, *args, **kwargs):
        if name not in self.names:
            self.names.append(name)
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        out = call(*args, **kwargs)
        b.record()
        self.runs.append((self.names.index(name), a, b))
        return out

    def arrays(self):
        torch.cuda.synchronize()
        dev = dict(device="cuda")
        start = torch.tensor([self.begin.elapsed_time(a) * 1e-3 for _, a, _ in self.runs],
                             dtype=torch.float64, **dev)
        end = torch.tensor([self.begin.elapsed_time(b) * 1e-3 for _, _, b in self.runs],
                           dtype=torch.float64, **dev)
        return start, end, torch.tensor([k for k, _, _ in self.runs], **dev)


def parameters(hidden, inner, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)

    return {"norm_w": 1 + normal(hidden, scale=0.1), "norm_b": normal(hidden, scale=0.1),
            "w1": normal(inner, hidden, scale=1 / math.sqrt(hidden)), "b1": normal(inner, scale=0.1),
            "w2": normal(hidden, inner, scale=1 / math.sqrt(inner)), "b2": normal(hidden, scale=0.1)}


def fused_forward(run, p, x, keep=False):
    h = run("norm", mag.layer_norm, x, p["norm_w"], p["norm_b"], EPS, statistics=keep or None)
    h, *stats = h if keep else (h,)
    u = run("up", mag.linear, h, p["w1"], p["b1"], activation="gelu_tanh", pre=keep or None)
    u, z = u if keep else (u, None)
    return run("down", mag.linear, u, p["w2"], p["b2"], x), (h, stats, u, z)


def fused_step(run, p, x, dy):
    y, (h, stats, u, z) = fused_forward(run, p, x, keep=True)
    du, dw2, db2 = run("down gradient", mag.linear_backward, u, p["w2"], dy)
    dh, dw1, db1 = run("up gradient", mag.linear_backward, h, p["w1"], du, z,
                       activation="gelu_tanh")
    dx, dnw, dnb = run("norm gradient", mag.layer_norm_backward, x, dh, *stats, p["norm_w"])
    updates = [run("update", mag.orthogonalize, w, STEPS, COEFFICIENTS) for w in (dw1, dw2)]
    return {"y": y, "dx": dx + dy, "dw1": dw1, "db1": db1, "dw2": dw2, "db2": db2, "dnorm_w": dnw,
            "dnorm_b": dnb, "update1": updates[0], "update2": updates[1]}


def _gelu(z):
    c = 2 * math.sqrt(2 / math.pi)
    s = 1 / (1 + torch.exp(-c * (z + 0.044715 * z * z * z)))
    return z * s, s + z * s * (1 - s) * c * (1 + 3 * 0.044715 * z * z)


def _norm(x, w, b):
    x = x.float()
    centred = x - x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt((centred * centred).mean(-1, keepdim=True) + EPS)
    xh = centred * rstd
    return (xh * w.float() + b.float()).to(w.dtype), xh, rstd


def _up(h, w, b):
    z = h.float() @ w.float().t() + b.float()
    return _gelu(z)[0].to(h.dtype), z.to(h.dtype)


def _down(u, w, b, x):
    return (u.float() @ w.float().t() + b.float() + x.float()).to(u.dtype)


def _linear_gradient(x, w, dz):
    dz = dz.float()
    return ((dz @ w.float()).to(x.dtype), (dz.t() @ x.float()).to(x.dtype), dz.sum(0).to(x.dtype))


def _up_gradient(h, w, du, z):
    return _linear_gradient(h, w, du.float() * _gelu(z.float())[1])


def _norm_gradient(dh, xh, rstd, w):
    d = dh.float()
    g = d * w.float()
    dx = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return dx.to(w.dtype), (d * xh).sum(0).to(w.dtype), d.sum(0).to(w.dtype)


def _update(g):
    a, b, c = COEFFICIENTS
    x = g.float()
    x = x / (torch.sqrt((x * x).sum()) + 1e-7)
    wide = x.shape[0] <= x.shape[1]
    x = x if wide else x.t()
    for _ in range(STEPS):
        s = x @ x.t()
        x = a * x + (b * s + c * (s @ s)) @ x
    return (x if wide else x.t()).to(g.dtype)


def plain_forward(run, p, x):
    h, xh, rstd = run("norm", _norm, x, p["norm_w"], p["norm_b"])
    u, z = run("up", _up, h, p["w1"], p["b1"])
    return run("down", _down, u, p["w2"], p["b2"], x), (h, xh, rstd, u, z)


def plain_step(run, p, x, dy):
    y, (h, xh, rstd, u, z) = plain_forward(run, p, x)
    du, dw2, db2 = run("down gradient", _linear_gradient, u, p["w2"], dy)
    dh, dw1, db1 = run("up gradient", _up_gradient, h, p["w1"], du, z)
    dx, dnw, dnb = run("norm gradient", _norm_gradient, dh, xh, rstd, p["norm_w"])
    updates = [run("update", _update, w) for w in (dw1, dw2)]
    return {"y": y, "dx": dx + dy, "dw1": dw1, "db1": db1, "dw2": dw2, "db2": db2, "dnorm_w": dnw,
            "dnorm_b": dnb, "update1": updates[0], "update2": updates[1]}


def synthetic_power(start, end, period=1e-6, idle=150.0, busy=900.0):
    """A trace over the intervals, one sample every `period` seconds."""
    t0, t1 = float(start.min()), float(end.max())
    t = t0 + period * torch.arange(int((t1 - t0) / period) + 2, dtype=torch.float64, device="cuda")
    running = (torch.searchsorted(start.sort().values, t, right=True)
               - torch.searchsorted(end.sort().values, t, right=True)) > 0
    return t, torch.where(running, busy, idle).float()


def energies(run):
    start, end, keys = run.arrays()
    t, power = synthetic_power(start, end)
    return mag.attribute(t, power, start, end, keys, latency=True)[1]


def compare(tokens=2048, hidden=768, inner=2304, dtype="bf16", single=4):
    """Both systems, warm: the operators' names, their ranking, which outputs match,
    and the outputs."""
    p = parameters(hidden, inner, DTYPES[dtype])
    x, dy = (parameters(hidden, tokens, DTYPES[dtype], seed)["w1"] for seed in (2, 3))
    tables, outputs = [], []
    for step, forward in ((fused_step, fused_forward), (plain_step, plain_forward)):
        for _ in range(2):  # (the first one warms up)
            run = Intervals()
            out = step(run, p, x, dy)
            out["tokens"] = torch.cat([
                forward(lambda name, call, *a, **k: run("token " + name, call, *a, **k), p,
                        x[i:i + 1])[0] for i in range(min(single, tokens))])
        tables.append(energies(run))
        outputs.append(out)
    ranking = mag.diff(*tables, len(run.names))
    eps = 1e-3 if dtype == "f32" else 2e-2
    tensors = [[o[k].float().contiguous() for k in outputs[0]] for o in outputs]
    spectra = [mag.invariants(t)[0] for t in tensors]
    same = mag.match(tensors[0], spectra[0], tensors[1], spectra[1], eps).diagonal()
    return run.names, ranking, dict(zip(outputs[0], same.bool().tolist())), outputs


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 2048), ("hidden", 768), ("inner", 2304)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dtype", choices=DTYPES, default="bf16")
    a = ap.parse_args()
    names, ranking, same, _ = compare(a.tokens, a.hidden, a.inner, a.dtype)
    print(f"{'operator':<20} {'A, mJ':>10} {'B, mJ':>10} {'(B - A) / A':>12}")
    for i in range(len(ranking["key"])):
        print(f"{names[int(ranking['key'][i])]:<20} {1e3 * float(ranking['energy_a'][i]):>10.3f} "
              f"{1e3 * float(ranking['energy_b'][i]):>10.3f} {float(ranking['ratio'][i]):>12.2f}")
    print("equivalent outputs:", ", ".join(k for k, v in same.items() if v))
    if not all(same.values()):
        sys.exit("not equivalent: " + ", ".join(k for k, v in same.items() if not v))


if __name__ == "__main__":
    main()

"""Every variant of the tile product (block_sizes.py; test_block_launches.py counts
them) against 64-bit products, with the bounds of test_gpu_block.py."""
import math

import block_sizes
import pytest
from test_gpu_block import (ACTS, COEFF, check_linear, check_linear_backward, check_orthogonalize,
                            plain_orthogonalize)

pytestmark = pytest.mark.gpu


def _cases(table):
    return [pytest.param(ty, size, id=f"{ty}-" + "x".join(map(str, size)))
            for ty, sizes in table.items() for size in sizes]


@pytest.mark.parametrize("lw", ["plain", "columns"])
@pytest.mark.parametrize("lx", ["plain", "columns"])
@pytest.mark.parametrize("ty,size", _cases(block_sizes.LINEAR))
def test_linear_tiles(ty, size, lx, lw):
    check_linear(*size, ty, act=ACTS[sum(size) % 5], lx=lx, lw=lw)


@pytest.mark.parametrize("layout", ["plain", "columns"])
@pytest.mark.parametrize("ty,size", _cases(block_sizes.LINEAR_BACKWARD))
def test_linear_backward_tiles(ty, size, layout):
    check_linear_backward(*size, ty, act=ACTS[sum(size) % 5], lx=layout, lw=layout, ld=layout)
    check_linear_backward(*size, ty, lx=layout, lw="plain", ld=layout)


@pytest.mark.parametrize("ty", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", block_sizes.UPDATES, ids=lambda s: "x".join(map(str, s)))
def test_update_tiles(size, ty):
    check_orthogonalize(*size, ty)


# shapes whose two-byte updates take several steps at once on the short side (the host
# tests see that they do), over full, low-rank and falling spectra
@pytest.mark.parametrize("ty,allowed", [("bf16", 2.0 ** -11), ("f16", 2.0 ** -14)])
@pytest.mark.parametrize("coeff", [COEFF, (1.5, -0.5, 0.0), (2.0, -1.5, 0.5)])
@pytest.mark.parametrize("size,steps,spectrum", block_sizes.GROUPED)
def test_steps_taken_at_once_add_a_quarter_of_a_rounding(size, steps, spectrum, coeff, ty, allowed):
    """Relative norms of the difference to the 64-bit iteration: the correctly rounded
    result's own, and beside it, at right angles to within a hundredth, what is let
    through before the rounding: `allowed`, a quarter of half a unit, and the
    operands' 22 bits (16 times what they cost an fp32 iteration, as elsewhere)."""
    import torch
    import paper_2512_08365_amd as mag
    print(f"[case] grouped update {size} {ty} {steps} {spectrum} {coeff}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(61)
    rows, cols = size
    x = torch.randn(rows, cols, generator=g, device="cuda")
    if spectrum != "full":
        m = min(size)
        side = torch.randn(m, m, generator=g, device="cuda") / math.sqrt(m)
        scale = torch.logspace(0, -6, m, device="cuda")
        if spectrum == "low":
            scale = (torch.arange(m, device="cuda") < m // 4).float()
        x = (side * scale) @ x if rows <= cols else x @ (side * scale)
    dt = torch.bfloat16 if ty == "bf16" else torch.float16
    x = (x * 0.02).to(dt)
    want = plain_orthogonalize(x, steps, coeff, 1e-7, torch.float64)
    own = plain_orthogonalize(x, steps, coeff, 1e-7, torch.float32)
    norm = float(want.norm())
    unit = float((own.double() - want).norm()) / norm
    rounding = float((want.to(dt).double() - want).norm()) / norm
    got = float((mag.orthogonalize(x, steps, coeff).double() - want).norm()) / norm
    bound = 1.01 * math.hypot(rounding, allowed) + 16 * max(unit, 2.0 ** -22)
    print(f"[error] {got:.3e} rounding {rounding:.3e} bound {bound:.3e} unit {unit:.1e}", flush=True)
    assert got <= bound

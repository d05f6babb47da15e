"""The feed-forward block's operators over many millions of rows: integers, whose
sums and products are exact in fp32, against the same integers summed by torch."""
import pytest

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    return torch


def _bits(shape, seed):
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, 2, shape, generator=g, device="cuda", dtype=torch.int8)


def test_many_rows_stored_by_columns():
    """17.1M rows of 64 features, each feature's rows neighbours in memory: 64 of
    them lie more than 31 bits of bytes apart.  Sums stay below 2^24."""
    torch = _torch()
    import paper_2512_08365_amd as mag
    rows, inner, outer = 17_100_000, 64, 16
    print(f"[case] {rows} x {inner} by columns, {outer} outputs", flush=True)
    x = _bits((inner, rows), 1).bfloat16().t()
    w = (_bits((outer, inner), 2) - _bits((outer, inner), 3)).bfloat16()
    y = mag.linear(x, w)
    step = 1 << 20
    for i in range(0, rows, step):
        want = x[i:i + step].float().contiguous() @ w.float().t().contiguous()
        assert torch.equal(y[i:i + step].float(), want), i
    del y
    dy = _bits((outer, rows), 4).bfloat16().t()
    _, dw, db = mag.linear_backward(x, w, dy, need=(False, True))
    want = torch.zeros(outer, inner, dtype=torch.float64, device="cuda")
    for i in range(0, rows, step):
        want += (dy[i:i + step].float().t().contiguous() @ x[i:i + step].float().contiguous()).double()
    assert float(want.max()) < 2.0 ** 24
    assert torch.equal(dw, want.bfloat16())
    assert torch.equal(db, dy.sum(0, dtype=torch.float64).bfloat16())
    del x, dy
    torch.cuda.empty_cache()


@pytest.mark.parametrize("ty,wt", [("bf16", "f32"), ("f32", "f32")])
def test_norms_of_many_rows_stored_by_columns(ty, wt):
    """4.3M rows: a workgroup of 1,024 threads for each would pass 2^32 threads"""
    torch = _torch()
    from test_gpu_block import check_norm, check_norm_backward
    check_norm(4_300_000, 8, ty, wt, lx="columns")
    torch.cuda.empty_cache()
    check_norm_backward(4_300_000, 8, ty, wt, lx="columns", ld="columns")
    torch.cuda.empty_cache()


def test_norms_of_one_column_with_any_stride():
    torch = _torch()
    import paper_2512_08365_amd as mag
    g = torch.Generator(device="cuda").manual_seed(5)
    rows = 4_300_000
    for n in (3, rows):
        x, dy = (torch.randn(n, generator=g, device="cuda") for _ in range(2))
        w, b = torch.tensor([2.0], device="cuda"), torch.tensor([0.75], device="cuda")
        for stride in (1, 5, 1 << 20):
            v, d = (t.as_strided((n, 1), (1, stride)) for t in (x, dy))
            y, mean, rstd = mag.layer_norm(v, w, b, statistics=True)
            assert bool((y == 0.75).all()) and torch.equal(mean, x)  # (x - mean is zero)
            dx, dw, db = mag.layer_norm_backward(v, d, mean, rstd, w)
            assert not bool(dx.any()) and not bool(dw.any())
            assert abs(float(db) - float(dy.double().sum())) <= (n + 8) * 2.0 ** -24 * float(dy.abs().sum())

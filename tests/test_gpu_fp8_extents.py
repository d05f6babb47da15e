"""The 8-bit operators over many millions of neighbours: whole numbers, whose sums are exact
in fp32, against the same numbers summed in 64 bits."""
import pytest

from test_gpu_block import _gen, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [(300, (1 << 23) + 65541, 70), (600, (1 << 23) - 100, 520), (70, 17_000_001, 300)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("by_row", [False, True])
def test_reductions_longer_than_a_tile_reaches_over(size, by_row):
    """A weight's gradient over millions of tokens, its operands stored so that they are
    packed.  Rows begin one or 16 bytes apart in one run of numbers: the memory of one row.
    Products are -1, 0 and 1 times scales of 1/4 to 1, their sums multiples of 1/4 far
    below 2^22: exact, and rounded to the result's type once."""
    torch = _torch()
    import paper_2512_08365_amd as mag
    rows, inner, outer = size
    g, blocks = _gen(7), -(-inner // 128)
    numbers = torch.randint(-1, 2, (2, inner + 16 * max(rows, outer)), generator=g, device="cuda", dtype=torch.int8)
    ex, ew = (2.0 ** -torch.randint(0, 2, (n, blocks), generator=g, device="cuda").float()
              for n in (rows, outer if by_row else -(-outer // 128)))
    for apart in ((1, 1), (16, 1), (1, 16)):
        print(f"[case] linear_fp8 {size} {by_row} {apart}", flush=True)
        x, w = (v.to(torch.float8_e4m3fn).as_strided((n, inner), (d, 1))
                for v, n, d in zip(numbers, (rows, outer), apart))
        y = mag.linear_fp8(x, ex, w, ew)
        want = torch.zeros((rows, outer), dtype=torch.float64, device="cuda")
        step = 1 << 19
        for k in range(0, inner, step):
            n = min(step, inner - k)
            a, b = (v[k:].as_strided((r, n), (d, 1)).double() for v, r, d in zip(numbers, (rows, outer), apart))
            at = slice(k // 128, -(-(k + n) // 128))
            a *= ex[:, at].repeat_interleave(128, 1)[:, :n]
            each = ew[:, at].repeat_interleave(128, 1)[:, :n]
            b *= each if by_row else each.repeat_interleave(128, 0)[:outer]
            want += torch.mm(a, b.t().contiguous())
        assert float(want.abs().max()) < 2.0 ** 20
        assert torch.equal(y, want.bfloat16())


def test_quantization_of_more_rows_than_a_launch_takes():
    """2^28 rows of one number: each is its block's largest"""
    torch = _torch()
    import paper_2512_08365_amd as mag
    rows = (1 << 28) + 1000
    print(f"[case] quantize_fp8 {rows} x 1", flush=True)
    x = torch.randn((rows, 1), generator=_gen(3), device="cuda").bfloat16()
    x[rows - 5] = x[7] = 0
    q = torch.full((rows, 1), 0x7f, dtype=torch.uint8, device="cuda")
    scale = torch.full((rows, 1), float("nan"), device="cuda")
    mag.quantize_fp8(x, out=(q.view(torch.float8_e4m3fn), scale))
    step = 1 << 26
    for at in range(0, rows, step):
        v, s, b = (t[at:at + step, 0] for t in (x, scale, q))
        most = v.double().abs()
        exact = torch.clamp(most / 448, min=2.0 ** -126)
        assert bool(((s.double() - exact).abs() <= 2.0 ** -24 * exact).all())
        want = torch.where(v == 0, 0, torch.where(v < 0, 0xfe, 0x7e))   # (-448 and 448)
        assert bool((b == want).all())

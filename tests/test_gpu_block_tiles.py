"""Every variant of the tile product (block_sizes.py; test_block_launches.py counts
them) against 64-bit products, with the bounds of test_gpu_block.py."""
import block_sizes
import pytest
from test_gpu_block import ACTS, check_linear, check_linear_backward, check_orthogonalize

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

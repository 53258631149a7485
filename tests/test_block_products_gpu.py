"""Forms of the e4m3 product that few sizes take: pairs that walk over several tiles, two or four pairs or several CTAs that
share a tile's K range, each with and without a residual, with rows that start on 16 bytes and rows that do not."""
import pytest
import torch

from tests import block_reference as ref
from tests.test_block_ops_gpu import B, check, operands, rand  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.mark.parametrize("path", [0, 2])
@pytest.mark.parametrize("M,N,K", [
    (777, 5003, 2064), (777, 5008, 1040),         # 80 tiles: more than half of 148 SMs makes pairs, so some take a second one
    (1300, 5000, 528),                            # 120 tiles
    (500, 4090, 2064), (512, 4096, 4096),         # 32 tiles: two pairs each
    (260, 505, 2064), (200, 1000, 4112),          # 4 tiles: four pairs each
])
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_pairs(B, M, N, K, dtype, path):  # noqa: F811
    a, sa, w, sw = operands(B, M, N, K, seed=M)
    check(B.es_op_linear_fp8(a, sa, w, sw, dtype=dtype, path=path, weights_ready=True), a, sa, w, sw)


@pytest.mark.parametrize("path,M,N,K", [
    (2, 777, 5003, 528), (2, 777, 5008, 528), (2, 500, 4090, 2064), (2, 512, 4096, 1040), (2, 260, 505, 2064), (2, 260, 512, 2064),
    (1, 3, 515, 4112), (1, 20, 512, 4096), (1, 50, 515, 4112), (1, 100, 515, 8208),         # few tiles: several CTAs share a K range
])
def test_the_residual_in_place(B, path, M, N, K):  # noqa: F811
    a, sa, w, sw = operands(B, M, N, K, seed=N)
    r = rand(M, N, seed=9)
    buffer = torch.full((M + 2, N), 3.0, device="cuda")
    out = buffer[1:-1]
    out.copy_(r)
    B.es_op_linear_fp8(a, sa, w, sw, residual=out, dtype=F32, path=path, out=out)
    check(out, a, sa, w, sw, r)
    assert bool((buffer[0] == 3).all()) and bool((buffer[-1] == 3).all())
    other = B.es_op_linear_fp8(a, sa, w, sw, residual=r, dtype=F32, path=path)
    assert torch.equal(out, other)

"""The attention block's calls refuse results on top of what they read: before anything is launched, so without a device.
Results right beside it are right: on a device."""
import pytest
import torch

from tests import block_reference as ref
from tests.test_block_refusals import B, _heads, _linear, _quant  # noqa: F401  (B is a fixture)

MiB = 1 << 20


@pytest.mark.parametrize("kw", [
    # x: 3 rows of 256 fp16, 1024 bytes apart; codes 3 x 256 bytes; scales [2, 3]: the first and the last byte of each
    {"codes": 64 * MiB}, {"codes": 64 * MiB + 2048 + 512 - 16}, {"codes": 64 * MiB - 752}, {"scale": 80 * MiB + 764}, {"scale": 80 * MiB - 20}, {"scale": 64 * MiB},
    {"scale": 64 * MiB + 2556}, {"scale": 64 * MiB - 20}, {"codes": 64 * MiB + 4096 + 1008, "dtype": 1, "stride": 512}, {"scale": 80 * MiB - 4, "rows": 128},
])
def test_quant(B, kw):  # noqa: F811
    a = dict(x=64 * MiB, stride=512, codes=80 * MiB, scale=96 * MiB)
    assert _quant(B, **dict(a, **kw)) == 1 and "lie apart" in B.es_last_error()


@pytest.mark.parametrize("kw", [
    # 3 x 5 x 256: a 768 bytes, its scales 24, w 1280, its scales 8, C and R 60 bytes
    {"R": 128 * MiB + 4}, {"R": 128 * MiB + 56}, {"R": 128 * MiB - 56}, {"C": 64 * MiB + 764}, {"C": 64 * MiB - 56}, {"C": 80 * MiB + 20}, {"C": 80 * MiB - 56},
    {"C": 96 * MiB + 1276}, {"C": 96 * MiB}, {"C": 112 * MiB + 4}, {"C": 112 * MiB - 56},
])
def test_linear(B, kw):  # noqa: F811
    a = dict(a=64 * MiB, sa=80 * MiB, w=96 * MiB, sw=112 * MiB, C=128 * MiB, out=1)
    assert _linear(B, **dict(a, **kw)) == 1 and "overlaps" in B.es_last_error()


@pytest.mark.parametrize("kw", [
    # q_out 3 x 4 x 128 fp16; pages 8 x 2 x 16 x 128, 65536 bytes each
    {"ko": 128 * MiB + 3056}, {"ko": 128 * MiB - 65520}, {"vo": 256 * MiB + 65520}, {"vo": 256 * MiB}, {"vo": 128 * MiB - 65520}, {"vo": 128 * MiB + 3056},
])
def test_heads(B, kw):  # noqa: F811
    a = dict(qo=128 * MiB, ko=256 * MiB, vo=512 * MiB)
    assert _heads(B, **dict(a, **kw)) == 1 and "two results" in B.es_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 128])
def test_codes_right_beside_the_values(B, rows):  # noqa: F811
    M, K = 130, 272
    memory = torch.zeros(M * K * 4, dtype=torch.uint8, device="cuda")
    x = memory[: M * K * 2].view(torch.float16).view(M, K)
    x.copy_(torch.randn(M, K, device="cuda"))
    scales = 3 * M if rows == 1 else 2 * 3
    codes = memory[M * K * 2: M * K * 3].view(torch.float8_e4m3fn).view(M, K)
    scale = memory[M * K * 3: M * K * 3 + 4 * scales].view(torch.float32).view((3, M) if rows == 1 else (2, 3))
    B.es_op_quant_e4m3(x, rows, out=(codes, scale))
    want, want_scale = ref.quant(x, rows)
    assert torch.equal(codes.view(torch.uint8), want.view(torch.uint8)) and torch.equal(scale.t() if rows == 1 else scale, want_scale)


@pytest.mark.gpu
def test_a_result_right_beside_the_residual(B):  # noqa: F811
    M, N, K = 20, 36, 256
    g = torch.Generator(device="cuda").manual_seed(0)
    a, sa = B.es_op_quant_e4m3(torch.randn(M, K, generator=g, device="cuda"))
    w, sw = B.es_op_quant_e4m3(torch.randn(N, K, generator=g, device="cuda"), 128)
    both = torch.randn(2 * M, N, generator=g, device="cuda")
    r = both[:M].clone()
    y = B.es_op_linear_fp8(a, sa, w, sw, residual=both[:M], dtype=torch.float32, out=both[M:])
    c, s = ref.linear(a, sa, w, sw, r)
    assert torch.equal(both[:M], r) and bool(((y.double() - c).abs() <= ref.linear_bound(c, s, K, torch.float32)).all())
    with pytest.raises(B.EsError) as e:
        B.es_op_linear_fp8(a, sa, w, sw, residual=both[:M], dtype=torch.float32, out=both[1:M + 1])
    assert e.value.status == 1

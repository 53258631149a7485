"""The e4m3 calls at the ends of their ranges."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2405_14371_b200 import binding
    torch.cuda.set_device(0)
    return binding


def test_the_most_columns(B):
    """K = 2^31 - 16: the columns of the last block, and blocks whose columns' numbers lie beside 2^31."""
    K = 2 ** 31 - 16
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("too little memory")
    blocks = 1 << 24
    x = torch.zeros(1, K, dtype=torch.float16, device="cuda")
    at = torch.tensor([0, 127, 128, 2 ** 30, K - 129, K - 113, K - 112, K - 1], device="cuda")
    x[0, at] = torch.tensor([3.0, -5.0, 7.0, 2.0, 1.5, 4.0, -6.0, 9.0], dtype=torch.float16, device="cuda")
    a, sa = B.es_op_quant_e4m3(x)
    w, sw = B.es_op_quant_e4m3(x, 128)
    assert sa.shape == (blocks, 1) and sw.shape == (1, blocks)
    assert torch.equal(a.view(torch.uint8), w.view(torch.uint8)) and torch.equal(sa[:, 0], sw[0])
    assert int((a.view(torch.uint8) != 0).sum()) == 8
    del x
    y = B.es_op_linear_fp8(a, sa, w, sw, dtype=torch.float32)
    want = float(((a[0, at].double() * sa[at // 128, 0].double()) ** 2).sum())
    assert abs(float(y) - want) <= 16 * 2.0 ** -24 * want           # 8 terms in 6 blocks: a scale's product, its own and an addition each

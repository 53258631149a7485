"""e4m3 codes and products, normalised heads: against plain forms in 64 bits, at the sizes where they can go wrong."""
import pytest
import torch

from tests import block_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2405_14371_b200 import binding
    torch.cuda.set_device(0)
    return binding


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(*shape, seed=0, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen(seed), device="cuda") * scale).to(dtype)


# ---- codes ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K", [(1, 16), (1, 4096), (3, 144), (5, 128), (129, 272), (256, 1024), (257, 1040)])
def test_codes(B, M, K, dtype, rows):
    x = rand(M, K, seed=M + K, dtype=dtype) * torch.exp2(torch.randint(-8, 8, (M, 1), generator=gen(1), device="cuda")).to(dtype)
    x[M // 2, : K // 2] = 0
    codes, scale = B.es_op_quant_e4m3(x, rows)
    want, want_scale = ref.quant(x, rows)
    assert torch.equal(scale if rows == 128 else scale.t(), want_scale)
    assert torch.equal(codes.view(torch.uint8), want.view(torch.uint8))


def test_codes_of_spaced_rows_into_given_memory(B):
    wide = rand(9, 512, seed=3, dtype=torch.bfloat16)
    x = wide[:, 64:320]
    codes = torch.full((9, 256), 7, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scale = torch.empty(2, 9, device="cuda")
    got = B.es_op_quant_e4m3(x, out=(codes, scale))
    want, want_scale = ref.quant(x, 1)
    assert got[0] is codes and torch.equal(codes.view(torch.uint8), want.view(torch.uint8)) and torch.equal(scale.t(), want_scale)


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_block_with_no_number_is_not_hidden(B, bad, rows):
    x = rand(130, 272, seed=5)
    x[129, 200] = bad
    codes, scale = B.es_op_quant_e4m3(x, rows)
    scale = scale if rows == 128 else scale.t()
    at = (129 // rows, 1)
    assert torch.isnan(scale[at]) and int(torch.isnan(scale).sum()) == 1
    assert bool(torch.isnan(codes[129, 128:256].float()).all()) and not bool(torch.isnan(codes[:128].float()).any())


def test_codes_of_tiny_values_and_zeros(B):
    x = torch.zeros(4, 256, device="cuda")
    x[1] = 1e-38
    x[2, 0] = 2.0 ** -140
    codes, scale = B.es_op_quant_e4m3(x)
    assert bool((scale == 2.0 ** -100).all()) and bool((codes.float() == 0).all())


# ---- products ------------------------------------------------------------------------------------------------------

def operands(B, M, N, K, seed=0, dtype=torch.bfloat16):
    x = rand(M, K, seed=seed, dtype=dtype) * torch.exp(rand(K, seed=seed + 1)).to(dtype)
    w = rand(N, K, seed=seed + 2, dtype=dtype, scale=0.02)
    return B.es_op_quant_e4m3(x) + B.es_op_quant_e4m3(w, 128)


def check(got, a, sa, w, sw, r=None):
    c, s = ref.linear(a, sa, w, sw, r)
    off = (got.double() - c).abs()
    bound = ref.linear_bound(c, s, a.shape[1], got.dtype)
    assert bool((off <= bound).all()), float((off / bound.clamp(min=1e-300)).max())


@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("M,N,K", [(1, 1, 16), (1, 128, 128), (16, 257, 1040), (17, 96, 144), (40, 640, 4096), (64, 129, 272), (65, 384, 512), (128, 256, 2048),
                                   (129, 200, 640), (300, 520, 1296), (513, 1000, 784)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
def test_products(B, M, N, K, dtype, path):
    a, sa, w, sw = operands(B, M, N, K, seed=M)
    check(B.es_op_linear_fp8(a, sa, w, sw, dtype=dtype, path=path), a, sa, w, sw)


@pytest.mark.parametrize("M,N,K", [(1, 12288, 4096), (16, 10240, 8192), (113, 5120, 13824), (1024, 4096, 4096), (2048, 2560, 1040)])
def test_products_of_model_sizes(B, M, N, K):
    a, sa, w, sw = operands(B, M, N, K)
    check(B.es_op_linear_fp8(a, sa, w, sw, dtype=torch.float32, weights_ready=True), a, sa, w, sw)


@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("M,N", [(5, 131), (130, 260), (260, 512)])
def test_product_added_to_the_residual_stream_in_place(B, M, N, path):
    a, sa, w, sw = operands(B, M, N, 528)
    r = rand(M, N, seed=9)
    buffer = torch.full((M + 2, N), 3.0, device="cuda")
    out = buffer[1:-1]
    out.copy_(r)
    B.es_op_linear_fp8(a, sa, w, sw, residual=out, dtype=torch.float32, path=path, out=out)
    check(out, a, sa, w, sw, r)
    assert bool((buffer[0] == 3).all()) and bool((buffer[-1] == 3).all())


@pytest.mark.parametrize("path", [1, 2])
def test_nothing_outside_the_result_is_written(B, path):
    a, sa, w, sw = operands(B, 70, 131, 400)
    buffer = torch.full((72, 131), 3.0, dtype=torch.float16, device="cuda")
    B.es_op_linear_fp8(a, sa, w, sw, path=path, out=buffer[1:-1])
    check(buffer[1:-1], a, sa, w, sw)
    assert bool((buffer[0] == 3).all()) and bool((buffer[-1] == 3).all())


@pytest.mark.parametrize("path", [1, 2])
def test_a_row_with_no_number_stays_alone(B, path):
    x = rand(33, 512, seed=1)
    x[7, 300] = float("nan")
    a, sa = B.es_op_quant_e4m3(x)
    w, sw = B.es_op_quant_e4m3(rand(200, 512, seed=2), 128)
    y = B.es_op_linear_fp8(a, sa, w, sw, path=path)
    bad = torch.isnan(y)
    assert bool(bad[7].all()) and int(bad.sum()) == 200


@pytest.mark.parametrize("path,M", [(1, 3), (1, 100), (2, 300)])
def test_same_inputs_same_bits(B, path, M):
    a, sa, w, sw = operands(B, M, 1100, 2064)
    first = B.es_op_linear_fp8(a, sa, w, sw, dtype=torch.float32, path=path)
    for _ in range(5):
        assert torch.equal(first, B.es_op_linear_fp8(a, sa, w, sw, dtype=torch.float32, path=path))


def test_no_rows(B):
    a, sa = B.es_op_quant_e4m3(torch.empty(0, 256, device="cuda"))
    w, sw = B.es_op_quant_e4m3(rand(10, 256), 128)
    assert B.es_op_linear_fp8(a, sa, w, sw).shape == (0, 10)


# ---- heads ---------------------------------------------------------------------------------------------------------

def tables(max_pos, rot):
    angle = torch.arange(max_pos, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, max(rot, 1), 2, dtype=torch.float64)[: rot // 2] / max(rot, 1))
    return angle.cos().float().cuda(), angle.sin().float().cuda()


def near(got, x, gain, eps, c, s, pos, halves):
    out, size = ref.heads(x, gain, eps, c, s, pos, halves)
    off = (got.double().view(out.shape) - out).abs()
    assert bool((off <= ref.heads_bound(out, size, x.shape[-1], got.dtype)).all()), float(off.max())


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("hd,rot", [(64, 64), (64, 32), (128, 128), (128, 64), (128, 16), (128, 96), (256, 256), (256, 48), (128, 0)])
@pytest.mark.parametrize("n,Hq,Hkv,dtype", [(1, 32, 32, torch.float16), (37, 7, 1, torch.bfloat16), (700, 64, 8, torch.bfloat16)])
def test_heads(B, n, Hq, Hkv, dtype, hd, rot, halves):
    qkv = (rand(n, Hq + 2 * Hkv, hd, seed=n) * torch.exp(2 * rand(Hq + 2 * Hkv, 1, seed=1))).to(dtype)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    qg, kg = 1 + 0.2 * rand(hd, seed=2), 1 + 0.2 * rand(hd, seed=3)
    c, s = tables(300, rot)
    pos = torch.randint(0, 300, (n,), generator=gen(4), device="cuda", dtype=torch.int32)
    qo, ko, vo = B.es_op_qk_norm_rope(q, k, qg, kg, 1e-6, c, s, pos, halves=halves, v=v)
    near(qo, q, qg, 1e-6, c, s, pos, halves)
    near(ko, k, kg, 1e-6, c, s, pos, halves)
    assert torch.equal(vo, v)


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_heads_into_the_cache(B, P, dtype):
    n, Hq, Hkv, hd, n_pages = 90, 8, 2, 128, 9
    q, k, v = rand(n, Hq, hd, seed=1, dtype=dtype), rand(n, Hkv, hd, seed=2, dtype=dtype), rand(n, Hkv, hd, seed=3, dtype=dtype)
    c, s = tables(50, hd)
    pos = torch.randint(0, 50, (n,), generator=gen(4), device="cuda", dtype=torch.int32)
    slots = torch.randperm(n_pages * P, generator=gen(5), device="cuda")[:n].to(torch.int32)
    pos[3], pos[10], slots[20], slots[21] = -1, 50, -1, n_pages * P           # padding and places that do not exist
    kp = torch.full((n_pages, Hkv, P, hd), 5.0, dtype=dtype, device="cuda")
    vp = kp.clone()
    qo = B.es_op_qk_norm_rope(q, k, None, None, 1e-6, c, s, pos, v=v, slot_map=slots, k_pages=kp, v_pages=vp)
    near(qo, q, None, 0, c, s, pos, False)
    assert bool((qo[3] == 0).all()) and bool((qo[10] == 0).all())
    want_k, want_v = torch.full_like(kp, 5.0), torch.full_like(vp, 5.0)
    _, ko, vo = B.es_op_qk_norm_rope(q, k, None, None, 1e-6, c, s, pos, v=v)
    for i in range(n):
        if i not in (3, 10, 20, 21):
            t = int(slots[i])
            want_k[t // P, :, t % P], want_v[t // P, :, t % P] = ko[i], vo[i]
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)


def test_heads_of_zeros_and_padding_without_eps(B):
    x = torch.zeros(2, 4, 64, dtype=torch.float16, device="cuda")
    x[1] = 1
    c, s = tables(4, 64)
    g = torch.ones(64, dtype=torch.float16, device="cuda")
    qo, ko = B.es_op_qk_norm_rope(x, x.clone(), g, g, 0.0, c, s, torch.tensor([-5, 0], dtype=torch.int32, device="cuda"))
    assert bool((qo[0] == 0).all()) and bool((ko[0] == 0).all()) and bool((qo[1] == 1).all())


def test_heads_refuse_a_result_on_top_of_the_input(B):
    x = rand(4, 2, 64, dtype=torch.float16)
    c, s = tables(4, 64)
    with pytest.raises(B.EsError) as e:
        B.es_op_qk_norm_rope(x, x, None, None, 0.0, c, s, torch.zeros(4, dtype=torch.int32, device="cuda"), out=x.view(4, 128))
    assert e.value.status == 1

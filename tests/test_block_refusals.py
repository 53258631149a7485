"""Refusals of the attention block's calls that need no device: they come before anything is launched."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2405_14371_b200 import build
    build.build()
    from paper_2405_14371_b200 import binding
    return binding


A = 1 << 20            # stands for an aligned device address that a refused call never touches
FAR = 1 << 40          # one far away from it


def _quant(b, **kw):
    a = dict(x=A, dtype=0, stride=256, M=3, K=256, rows=1, codes=A, scale=A)
    a.update(kw)
    return b.lib.es_op_quant_e4m3(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    ({"x": None}, 1), ({"codes": None}, 1), ({"scale": None}, 1), ({"dtype": 2}, 1), ({"dtype": 5}, 1), ({"M": -1}, 1), ({"K": 0}, 1), ({"K": 24}, 2), ({"rows": 2}, 1),
    ({"stride": 255}, 1), ({"stride": 260}, 1), ({"stride": 258, "dtype": 1}, 1), ({"x": A + 8}, 1), ({"codes": A + 4}, 1), ({"scale": A + 2}, 1), ({"M": 262141}, 3),
    ({"M": 8388481, "rows": 128}, 3), ({"M": 0}, 0), ({"M": 0, "x": None}, 0),
])
def test_quant(B, kw, status):
    assert _quant(B, **kw) == status


def _linear(b, **kw):
    a = dict(a=A, sa=A, w=A, sw=A, R=None, C=A, out=0, M=3, N=5, K=256, path=0, ready=0)
    a.update(kw)
    return b.lib.es_op_linear_fp8(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    ({"a": None}, 1), ({"sa": None}, 1), ({"w": None}, 1), ({"sw": None}, 1), ({"C": None}, 1), ({"out": 2}, 1), ({"out": 5}, 1), ({"R": A}, 1), ({"M": -1}, 1), ({"N": 0}, 1),
    ({"K": 0}, 1), ({"K": 40}, 2), ({"path": 3}, 1), ({"path": -1}, 1), ({"a": A + 8}, 1), ({"w": A + 8}, 1), ({"sa": A + 2}, 1), ({"C": A + 1}, 1), ({"C": A + 2, "out": 1}, 1),
    ({"M": 262141}, 3), ({"N": (1 << 24) + 1}, 3), ({"M": 0}, 0),
])
def test_linear(B, kw, status):
    assert _linear(B, **kw) == status


def _heads(b, **kw):
    a = dict(q=A, qs=512, k=A, ks=256, v=A, vs=256, dtype=0, qg=A, kg=A, gain=0, eps=1e-6, cos=A, sin=A, max_pos=64, rot=128, halves=0, pos=A, qo=FAR, ko=2 * FAR,
             vo=3 * FAR, n=3, Hq=4, Hkv=2, hd=128, slots=A, P=16, n_pages=8)
    a.update(kw)
    return b.lib.es_op_qk_norm_rope(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    ({"q": None}, 1), ({"k": None}, 1), ({"v": None}, 1), ({"vo": None}, 1), ({"qo": None}, 1), ({"ko": None}, 1), ({"pos": None}, 1), ({"cos": None}, 1), ({"sin": None}, 1),
    ({"dtype": 1}, 1), ({"gain": 4}, 1), ({"eps": -1.0}, 1), ({"eps": float("nan")}, 1), ({"n": -1}, 1), ({"Hq": 0}, 1), ({"Hkv": 0}, 1), ({"max_pos": 0}, 1), ({"hd": 96}, 2),
    ({"rot": 24}, 2), ({"rot": 144}, 2), ({"rot": -16}, 2), ({"qs": 504}, 1), ({"qs": 516}, 1), ({"ks": 250}, 1), ({"vs": 128}, 1), ({"q": A + 8}, 1), ({"qg": A + 2}, 1),
    ({"P": 8}, 2), ({"P": 24}, 2), ({"n_pages": 0}, 1), ({"n_pages": 1 << 28}, 3), ({"Hq": 65537}, 3), ({"qo": A}, 1), ({"ko": A + 16}, 1), ({"vo": A + 1024}, 1), ({"n": 0}, 0),
])
def test_heads(B, kw, status):
    assert _heads(B, **kw) == status


def _shared(b, **kw):
    a = dict(q=A, dtype=0, stride=512, k=A, v=A, pt=A, pl=A, gb=A, groups=2, pp=4, table=A, ctx=A, out=A, B=3, T=1, Hq=4, Hkv=2, hd=128, P=16, pps=4, n_pages=8,
             max_prefix=64, max_ctx=64, scratch=A, bytes=1 << 30)
    a.update(kw)
    return b.lib.es_op_decode_attention_prefix(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    ({"q": None}, 1), ({"k": None}, 1), ({"v": None}, 1), ({"pt": None}, 1), ({"pl": None}, 1), ({"gb": None}, 1), ({"table": None}, 1), ({"ctx": None}, 1), ({"out": None}, 1),
    ({"dtype": 1}, 1), ({"groups": -1}, 1), ({"B": 0}, 1), ({"T": 0}, 1), ({"Hq": 3}, 2), ({"Hq": 258, "stride": 1 << 20}, 2), ({"hd": 96}, 2), ({"P": 8}, 2), ({"P": 48}, 2),
    ({"pps": 0}, 1), ({"pp": 0}, 1), ({"n_pages": 0}, 1), ({"max_ctx": 0}, 1), ({"max_prefix": 0}, 1), ({"max_ctx": 65}, 3), ({"max_prefix": 65}, 3), ({"stride": 511}, 1),
    ({"stride": 504}, 1), ({"q": A + 8}, 1), ({"k": A + 2}, 1), ({"out": A + 4}, 1), ({"scratch": A + 8}, 1), ({"B": 8191}, 3), ({"n_pages": 1 << 26}, 3),
    ({"max_ctx": (1 << 30) + 1, "pps": 1 << 27}, 3), ({"B": 8000, "max_ctx": 1 << 23, "pps": 1 << 19}, 3), ({"T": 1 << 24}, 3), ({"bytes": 100}, 6), ({"scratch": None}, 6),
])
def test_shared(B, kw, status):
    assert _shared(B, **kw) == status


def test_shared_scratch(B):
    f = B.es_op_decode_attention_prefix_scratch_bytes
    assert f(1, 0, 1, 4, 2, 128) == 0 and f(1, 1, 1, 4, 3, 128) == 0 and f(1, 3, 1, 4, 2, 96) == 0
    assert f(0, 3, 1, 4, 2, 128) < f(1, 3, 1, 4, 2, 128)


def test_binding_refuses_host_tensors(B):
    h, i = torch.zeros(2, 2, 64, dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    f, t = torch.zeros(2, 128), torch.zeros(4, 32)
    c = torch.zeros(2, 128, dtype=torch.float8_e4m3fn)
    for call in (lambda: B.es_op_quant_e4m3(f), lambda: B.es_op_linear_fp8(c, f, c, f), lambda: B.es_op_qk_norm_rope(h, h, None, None, 0.0, t, t, i),
                 lambda: B.es_op_decode_attention_prefix(h, h, h, None, None, None, i.view(2, 1), i, 1, 1)):
        with pytest.raises(B.EsError) as e:
            call()
        assert e.value.status == 1

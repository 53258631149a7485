"""Refusals of the 8-bit cache and sampling calls that need no device: they come before anything is launched."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2405_14371_b200 import build
    build.build()
    from paper_2405_14371_b200 import binding
    return binding


A = 1 << 20            # stands for an aligned device address that a refused call never touches


def _plan(binding, **kw):
    a = dict(old=A, new=A, table=A, free=A, count=A, B=2, pps=4, P=16, n_pages=8, max_rows=8, ro=A, sm=A, pos=A, seq=A, runs=A, out=A)
    a.update(kw)
    return binding.lib.es_op_kv_plan(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    ({"old": None}, 1), ({"new": None}, 1), ({"table": None}, 1), ({"free": None}, 1), ({"count": None}, 1), ({"out": None}, 1), ({"runs": None}, 1),
    ({"B": 0}, 1), ({"pps": 0}, 1), ({"P": 0}, 1), ({"P": 8}, 2), ({"P": 48}, 2), ({"n_pages": 0}, 1), ({"max_rows": 0}, 1), ({"B": 8193}, 3),
    ({"pps": 1 << 27}, 3), ({"n_pages": 1 << 27}, 3), ({"max_rows": 2 ** 31 - 1}, 3),
    ({"max_rows": 2 ** 30 + 1}, 3), ({"B": 8192, "pps": 1 << 18}, 3),
])
def test_plan(B, kw, status):
    assert _plan(B, **kw) == status and B.es_last_error()


def _append(binding, **kw):
    a = dict(k=A, v=A, dtype=0, stride=256, n=3, slots=A, runs=None, n_runs=0, kp=A, vp=A, code=4, ks=A, vs=A, Hkv=2, hd=128, P=16, n_pages=8)
    a.update(kw)
    return binding.lib.es_op_kv8_append(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    ({"k": None}, 1), ({"slots": None}, 1), ({"kp": None}, 1), ({"vs": None}, 1), ({"dtype": 1}, 1), ({"dtype": 9}, 1), ({"code": 0}, 1), ({"stride": 255}, 1),
    ({"stride": 260}, 1), ({"n": -1}, 1), ({"n_runs": -1}, 1), ({"Hkv": 0}, 1), ({"hd": 96}, 2), ({"P": 12}, 2), ({"n_pages": 1 << 27}, 3), ({"k": A + 8}, 1), ({"vp": A + 1}, 1),
    ({"n": 2 ** 31 - 1, "Hkv": 2}, 3),
    ({"n": 0}, 0), ({"n": 0, "k": None}, 0), ({"runs": A, "n_runs": 0}, 0),
])
def test_append(B, kw, status):
    assert _append(B, **kw) == status


def _gather(binding, **kw):
    a = dict(slots=A, n=3, kp=A, vp=A, code=5, ks=A, vs=A, Hkv=2, hd=64, P=16, n_pages=8, k=A, v=A, dtype=3)
    a.update(kw)
    return binding.lib.es_op_kv8_gather(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    ({"slots": None}, 1), ({"k": None}, 1), ({"code": 1}, 1), ({"dtype": 2}, 1), ({"n": -2}, 1), ({"hd": 32}, 2), ({"P": 1}, 2), ({"v": A + 4}, 1), ({"n": 0}, 0),
])
def test_gather(B, kw, status):
    assert _gather(B, **kw) == status


def _attn(binding, **kw):
    a = dict(q=A, dtype=0, stride=512, kp=A, vp=A, code=4, ks=A, vs=A, table=A, ctx=A, out=A, B=1, T=1, Hq=4, Hkv=2, hd=128, P=16, pps=4, n_pages=8, max_ctx=64, scratch=A, bytes=1 << 30)
    a.update(kw)
    return binding.lib.es_op_decode_attention_kv8(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    ({"q": None}, 1), ({"ks": None}, 1), ({"table": None}, 1), ({"out": None}, 1), ({"dtype": 1}, 1), ({"code": 3}, 1), ({"B": 0}, 1), ({"T": 0}, 1), ({"Hq": 3}, 2),
    ({"hd": 80}, 2), ({"P": 20}, 2), ({"pps": 0}, 1), ({"max_ctx": 65}, 3), ({"max_ctx": 0}, 1), ({"max_ctx": (1 << 30) + 1, "pps": 1 << 27}, 3), ({"stride": 511}, 1),
    ({"stride": 516}, 1), ({"q": A + 2}, 1), ({"scratch": A + 8}, 1), ({"B": 65536}, 3), ({"T": 65535}, 3), ({"n_pages": 0}, 1),
])
def test_attention(B, kw, status):
    assert _attn(B, **kw) == status


def test_attention_scratch(B):
    f = B.es_op_decode_attention_kv8_scratch_bytes
    assert f(0, 1, 4, 2, 128, 16, 64) == 0 and f(1, 1, 4, 3, 128, 16, 64) == 0
    assert f(1, 1, 4, 2, 128, 16, 32) == 0              # one tile of keys needs none


def _sample(binding, **kw):
    a = dict(x=A, dtype=1, stride=100, u=A, T=None, k=None, p=None, m=None, tok=A, lp=None, B=1, V=100)
    a.update(kw)
    return binding.lib.es_op_sample(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    ({"x": None}, 1), ({"u": None}, 1), ({"tok": None}, 1), ({"dtype": 2}, 1), ({"B": 0}, 1), ({"V": 0}, 1), ({"stride": 99}, 1), ({"V": 262145, "stride": 1 << 20}, 3), ({"B": 1 << 25}, 3),
])
def test_sample(B, kw, status):
    assert _sample(B, **kw) == status


def test_binding_refuses_host_tensors(B):
    i, f = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2, 16, 64, dtype=torch.int8)
    h = torch.zeros(2, 2, 64, dtype=torch.float16)
    s = torch.zeros(2, 2)
    for call in (lambda: B.es_op_kv_plan(i, i, i.view(2, 1), 16, 4), lambda: B.es_op_kv8_append(h, h, i, f, f, s, s),
                 lambda: B.es_op_kv8_gather(i, f, f, s, s), lambda: B.es_op_decode_attention_kv8(h, f, f, s, s, i.view(2, 1), i, 16),
                 lambda: B.es_op_sample(s, s[0])):
        with pytest.raises(B.EsError) as e:
            call()
        assert e.value.status == 1


def test_max_runs(B):
    assert B.es_op_kv_plan_max_runs(0, 5, 16) == 0
    assert B.es_op_kv_plan_max_runs(4, 5, 16) == 5
    assert B.es_op_kv_plan_max_runs(1, 1600, 16) == 102

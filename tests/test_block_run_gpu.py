"""The operators of the attention block one after another, as a step uses them: captured and replayed, on other streams, as a
process's first call, at the largest sizes."""
import os
import subprocess
import sys

import pytest
import torch

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    from paper_2405_14371_b200 import binding
    torch.cuda.set_device(0)
    return binding


def rand(*shape, seed=0, dtype=BF16, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale).to(dtype)


def block(b, seed=0, n=6, d=512, Hq=8, Hkv=2, hd=64, P=16, prefix=100):
    """A batch of n sequences behind one prefix; the state of one step."""
    own = [5, 16, 17, 1, 40, 30][:n]
    pages = -(-prefix // P) + sum(-(-c // P) for c in own)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    pt, rest = order[: -(-prefix // P)], order[-(-prefix // P):]
    table = torch.full((n, 3), -1, dtype=torch.int32)
    slots, at = [], 0
    for i, c in enumerate(own):
        m = -(-c // P)
        table[i, :m] = torch.tensor(rest[at:at + m])
        slots.append(rest[at + (c - 1) // P] * P + (c - 1) % P)
        at += m
    angle = torch.arange(256, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, hd, 2, dtype=torch.float64) / hd)
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    wide = (Hq + 2 * Hkv) * hd
    s = dict(x=rand(n, d, seed=seed + 1), stream=rand(n, d, seed=seed + 2, dtype=torch.float32), wqkv=b.es_op_quant_e4m3(rand(wide, d, seed=3, scale=0.05), 128),
             wo=b.es_op_quant_e4m3(rand(d, Hq * hd, seed=4, scale=0.05), 128), qg=1 + rand(hd, seed=5, scale=0.1), kg=1 + rand(hd, seed=6, scale=0.1),
             cos=angle.cos().float().cuda(), sin=angle.sin().float().cuda(), pos=i32([prefix + c - 1 for c in own]), slots=i32(slots), pt=i32([pt]), pl=i32([prefix]),
             begin=i32([0, n]), table=table.cuda(), ctx=i32(own), k=rand(pages, Hkv, P, hd, seed=7), v=rand(pages, Hkv, P, hd, seed=8), Hq=Hq, Hkv=Hkv, hd=hd)
    return s


def step(b, s):
    n, Hq, Hkv, hd = len(s["x"]), s["Hq"], s["Hkv"], s["hd"]
    a = b.es_op_quant_e4m3(s["x"])
    qkv = b.es_op_linear_fp8(*a, *s["wqkv"], dtype=BF16, weights_ready=True)
    heads = qkv.view(n, Hq + 2 * Hkv, hd)
    q = b.es_op_qk_norm_rope(heads[:, :Hq], heads[:, Hq:Hq + Hkv], s["qg"], s["kg"], 1e-5, s["cos"], s["sin"], s["pos"], v=heads[:, Hq + Hkv:], slot_map=s["slots"],
                             k_pages=s["k"], v_pages=s["v"])
    o = b.es_op_decode_attention_prefix(q.view(n, Hq, hd), s["k"], s["v"], s["pt"], s["pl"], s["begin"], s["table"], s["ctx"], 112, 48)
    c = b.es_op_quant_e4m3(o)
    y = b.es_op_linear_fp8(*c, *s["wo"], residual=s["stream"], dtype=torch.float32, weights_ready=True)
    return dict(a=a, qkv=qkv, q=q, o=o, c=c, y=y)


def check(s, r):
    """Every stage against its plain form of what it was given."""
    n, Hq, Hkv, hd = len(s["x"]), s["Hq"], s["Hkv"], s["hd"]
    codes, scale = ref.quant(s["x"], 1)
    assert torch.equal(r["a"][0].view(torch.uint8), codes.view(torch.uint8)) and torch.equal(r["a"][1].t(), scale)
    c, m = ref.linear(*r["a"], *s["wqkv"])
    assert bool(((r["qkv"].double() - c).abs() <= ref.linear_bound(c, m, s["x"].shape[1], BF16)).all())
    heads = r["qkv"].view(n, Hq + 2 * Hkv, hd)
    q, m = ref.heads(heads[:, :Hq], s["qg"], 1e-5, s["cos"], s["sin"], s["pos"], False)
    assert bool(((r["q"].double().view(q.shape) - q).abs() <= ref.heads_bound(q, m, hd, BF16)).all())
    P = s["k"].shape[2]
    slot = s["slots"].long()
    k, m = ref.heads(heads[:, Hq:Hq + Hkv], s["kg"], 1e-5, s["cos"], s["sin"], s["pos"], False)
    assert bool(((s["k"][slot // P, :, slot % P].double() - k).abs() <= ref.heads_bound(k, m, hd, BF16)).all())
    assert torch.equal(s["v"][slot // P, :, slot % P], heads[:, Hq + Hkv:])
    rows = r["q"].view(n, 1, Hq, hd)
    o, m = ref.shared(rows, s["k"], s["v"], s["pt"], s["pl"], s["begin"], s["table"], s["ctx"])
    assert bool(((r["o"].double().view(o.shape) - o).abs() <= ref.shared_bound(rows, s["k"], o, m)).all())
    c, m = ref.linear(*r["c"], *s["wo"], s["stream"])
    assert bool(((r["y"].double() - c).abs() <= ref.linear_bound(c, m, Hq * hd, torch.float32)).all())


def test_a_step(B):
    s = block(B)
    check(s, step(B, s))


def test_a_step_as_a_replayed_graph(B):
    s, fresh = block(B), block(B, seed=50)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        step(B, s)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            r = step(B, s)
    graph.replay()
    torch.cuda.synchronize()
    check(s, r)
    for name in ("x", "stream", "k", "v", "pos", "ctx", "table", "slots", "pt"):       # another step's inputs in the same places
        s[name].copy_(fresh[name])
    graph.replay()
    torch.cuda.synchronize()
    check(s, r)


def test_two_streams_at_once(B):
    a, b = block(B, seed=1), block(B, seed=2)
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(10):
        for s, st in ((a, one), (b, two)):
            with torch.cuda.stream(st):
                got.append((s, step(B, s)))
    torch.cuda.synchronize()
    for s, r in got[-2:]:
        check(s, r)
    for s, r in got[:-2]:
        assert torch.equal(r["y"], got[-2][1]["y"] if s is a else got[-1][1]["y"])


def test_inputs_still_being_made_on_the_stream(B):
    s = block(B, seed=3)
    want = step(B, s)["y"].clone()
    x = s["x"].clone()
    for _ in range(5):
        s["x"].zero_()
        big = torch.randn(4096, 4096, device="cuda")
        big = big @ big
        s["x"].copy_(x)
        assert torch.equal(step(B, s)["y"], want)


def test_weights_made_just_before_their_use(B):
    """Without the promise that the weights are complete, their codes may come from the kernel in front."""
    for seed in range(4):
        x, w = rand(4, 2048, seed=seed), rand(1024, 2048, seed=seed + 9, scale=0.02)
        a = B.es_op_quant_e4m3(x)
        codes = B.es_op_quant_e4m3(w, 128)
        y = B.es_op_linear_fp8(*a, *codes, dtype=torch.float32)
        c, m = ref.linear(*a, *codes)
        assert bool(((y.double() - c).abs() <= ref.linear_bound(c, m, 2048, torch.float32)).all())


def test_first_call_of_a_process_may_be_a_captured_one(B):
    code = """
import torch
from tests import test_block_run_gpu as t
from paper_2405_14371_b200 import binding as b
g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
s = t.block(b)                                  # the weights' codes come from another kernel than the step's
torch.cuda.synchronize()
with torch.cuda.graph(g, stream=st):
    r = t.step(b, s)
g.replay()
torch.cuda.synchronize()
t.check(s, r)
print('captured')
"""
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "captured" in out.stdout, out.stderr[-2000:]


def test_a_cache_beyond_32_bit_offsets(B):
    n_pages, Hkv, P, hd = 36000, 8, 64, 128                   # 2.4e9 values a pool
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("too little memory")
    k = torch.empty(n_pages, Hkv, P, hd, dtype=BF16, device="cuda")
    v = torch.empty_like(k)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    own, front = [n_pages - 1, n_pages - 3], [n_pages - 2, 1]
    k[own + front], v[own + front] = rand(4, Hkv, P, hd, seed=1), rand(4, Hkv, P, hd, seed=2)
    x = rand(2, Hkv, hd, seed=3)
    slots = i32([own[0] * P + 40, own[1] * P + 63])
    cos, sin = torch.ones(4, hd // 2, device="cuda"), torch.zeros(4, hd // 2, device="cuda")
    q = B.es_op_qk_norm_rope(x, x, None, None, 0.0, cos, sin, i32([0, 1]), v=x, slot_map=slots, k_pages=k, v_pages=v).view(2, 1, Hkv, hd)
    assert torch.equal(k[own[0], :, 40], x[0]) and torch.equal(v[own[1], :, 63], x[1])
    pt, pl, begin, table, ctx = i32([front]), i32([100]), i32([0, 2]), i32([[own[0]], [own[1]]]), i32([41, 64])
    got = B.es_op_decode_attention_prefix(q, k, v, pt, pl, begin, table, ctx, 128, 64)
    o, m = ref.shared(q, k, v, pt, pl, begin, table, ctx)
    used = torch.stack([k[i] for i in own + front])
    assert bool(((got.double().view(o.shape) - o).abs() <= ref.shared_bound(q, used, o, m)).all())


@pytest.mark.parametrize("B_,groups", [(700, 90), (7000, 1000)])
def test_many_segments(B, B_, groups):
    """More segments than a block has threads, and so many that a CTA has an SM to itself: as calls of parts of the batch."""
    P, Hkv, hd, T = 16, 1, 64, 1
    g = torch.Generator().manual_seed(B_)
    ctx = torch.randint(0, 40, (B_,), generator=g)
    lens = torch.randint(0, 100, (groups,), generator=g)
    begin = torch.sort(torch.randint(0, B_ + 1, (groups + 1,), generator=g))[0]
    n_pages = 500
    i32 = lambda x: x.to(torch.int32).cuda()  # noqa: E731
    table, pt = i32(torch.randint(0, n_pages, (B_, 3), generator=g)), i32(torch.randint(0, n_pages, (groups, 7), generator=g))
    q, k, v = rand(B_, T, 4, hd, seed=1), rand(n_pages, Hkv, P, hd, seed=2), rand(n_pages, Hkv, P, hd, seed=3)
    whole = B.es_op_decode_attention_prefix(q, k, v, pt, i32(lens), i32(begin), table, i32(ctx), 112, 48)
    for at in range(0, B_, max(350, B_ // 4)):
        to = min(B_, at + max(350, B_ // 4))
        part = B.es_op_decode_attention_prefix(q[at:to], k, v, pt, i32(lens), i32((begin - at).clamp(0, to - at)), table[at:to].contiguous(), i32(ctx[at:to]), 112, 48)
        # the same rows with their keys cut differently: a rounding each, and the weights' own, of values below 5
        assert float((whole[at:to].float() - part.float()).abs().max()) <= 5 * 3 * 2.0 ** -8
    some = [0, B_ // 3, B_ - 1]
    for b in some:
        o, m = ref.shared(q[b:b + 1], k, v, pt, i32(lens), i32(begin - b), table[b:b + 1], i32(ctx[b:b + 1]))
        assert bool(((whole[b:b + 1].double().view(o.shape) - o).abs() <= ref.shared_bound(q, k, o, m)).all())

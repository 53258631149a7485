"""The operations over the 8-bit cache at the edges of their definitions: codes that are no numbers, queries of very different
magnitudes, waits that run out, exact ties, pages whose scale another program chose.  References in 64 bits or exact fractions."""
import math
import os
import subprocess
import sys
from fractions import Fraction

import pytest
import torch

from tests import kv8_reference as R
from tests.test_kv8_ops_gpu import _attn_case, _check_sample, _gen, _i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2405_14371_b200 import binding
    return binding


def _attend(B, case):
    return B.es_op_decode_attention_kv8(*[t.cuda() for t in case[:7]], case[7]).cpu().double()


def _inside(got, want, bound):
    assert torch.equal(got.isnan(), want.isnan()), (got.isnan().nonzero()[:8].tolist(), want.isnan().nonzero()[:8].tolist())
    ok = ~want.isnan()
    over = ((got - want).abs() / bound)[ok]
    assert float(over.max()) <= 1.0, float(over.max())


# ---- attention: codes that are no numbers ------------------------------------------------------------------------

@pytest.mark.parametrize("Bn,T,Hq,Hkv,hd,P,ctxs", [
    (1, 3, 2, 2, 64, 16, [40]), (2, 3, 4, 2, 128, 32, [37, 3]), (1, 4, 16, 2, 128, 64, [70]), (2, 17, 1, 1, 64, 16, [60, 20]), (20, 3, 8, 8, 128, 64, [30 + 7 * i for i in range(20)]),
    (20, 4, 32, 8, 64, 16, [30 + 7 * i for i in range(20)]), (20, 2, 8, 8, 128, 16, [600 + 3 * i for i in range(20)]), (20, 6, 16, 8, 128, 32, [90 + 7 * i for i in range(20)]),
])
def test_attention_a_value_that_is_no_number_shows_only_where_it_is_seen(B, Bn, T, Hq, Hkv, hd, P, ctxs):
    """e4m3 NaN codes in V at draft tokens: the queries before such a token do not see it, the others are NaN in its dimension
    alone (a sum with it has no other value)."""
    case = _attn_case(Bn, T, Hq, Hkv, hd, P, ctxs, "e4m3", "fp16", 101)
    vc, table = case[2].view(torch.int8), case[5]
    for b, n in enumerate(ctxs):
        for back, dim, code in ((1, 5, 0x7f), (2, hd - 1, -1), (T - 1, 17, 0x7f)):
            pos = n - max(back, 1)
            if b % 3 != 2 and pos >= 0:
                vc[int(table[b, pos // P]), (b + back) % Hkv, pos % P, dim] = code
    q, kc, _, ks, vs, table, ctx, max_ctx = case
    want, bound = R.attend(q, kc, case[2], ks, vs, table, ctx, P, max_ctx)
    assert bool(want.isnan().any())
    _inside(_attend(B, case).reshape(want.shape), want, bound)


# ---- attention: queries of very different magnitudes -------------------------------------------------------------

@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("big", [2.0 ** 15, 2.0 ** 20, 2.0 ** 23, -2.0 ** 23])
@pytest.mark.parametrize("f", [1.0, 2.0 ** -60, 2.0 ** 90])
def test_attention_keeps_the_small_elements_of_a_bf16_query(B, code, big, f):
    """One element of the query is large and the keys are zero there, so the result is that of the others alone: nothing of
    them may be lost beside it.  Tolerance: that of the reference for the query without the large element, to which the
    products with zero add nothing; elements down to 2^-30 of the largest are held exactly."""
    case = list(_attn_case(2, 2, 8, 2, 128, 16, [33, 150], code, "bf16", 103))
    q, kc = case[0], case[1]
    kc[..., 9] = 0
    q[..., 9] = 0
    q.copy_(torch.where(q.abs() < 2.0 ** -6, torch.zeros_like(q), q))         # 2^-6 / 2^23: within 2^-30 of the largest
    case[0], case[3] = (q.float() * f).bfloat16(), case[3] / f
    want, bound = R.attend(case[0], *case[1:6], case[6], 16, case[7])
    case[0][..., 9] = big * f
    _inside(_attend(B, case).reshape(want.shape), want, bound)


# ---- attention: a wait that runs out -----------------------------------------------------------------------------

_RUN_OUT = """
import torch
from paper_2405_14371_b200 import binding as B
from tests.test_kv8_ops_gpu import _attn_case

def rows(*a, **kw):
    case = _attn_case(*a, **kw)
    out = B.es_op_decode_attention_kv8(*[t.cuda() for t in case[:7]], case[7])
    torch.cuda.synchronize()
    return out

for code, dtype in (("int8", "fp16"), ("e4m3", "bf16")):
    for args in ((1, 1, 8, 8, 128, 64, [2000]), (1, 1, 40, 40, 64, 16, [70]), (3, 1, 8, 1, 128, 16, [0, 1, 40]), (2, 5, 8, 2, 128, 32, [90, 300]),
                 (20, 1, 8, 8, 128, 64, [1 + 150 * i for i in range(20)]), (20, 3, 32, 8, 128, 64, [1 + 150 * i for i in range(20)]),
                 (40, 1, 16, 8, 64, 16, [1 + i % 16 for i in range(40)]), (20, 1, 8, 8, 128, 16, [9000] + [0] * 19)):
        got = rows(*args, code, dtype, 5)
        assert bool(got.isnan().all()), (args, code, int((~got.isnan()).sum()))
tok, _ = B.es_op_sample(torch.zeros(2, 50, device="cuda"), torch.full((2,), 0.5, device="cuda"))
assert tok.tolist() == [25, 25]
print("all rows without a result")
"""


def test_attention_a_wait_that_runs_out_leaves_no_result():
    """ES_KV8_GIVE_UP (read once per process, hence a child process): every first wait counts as run out.  The copies under way
    still land before a CTA ends, the rows become NaN in both ways of sharing the tiles, and the device goes on working."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _RUN_OUT], cwd=root, env=dict(os.environ, ES_KV8_GIVE_UP="1"), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "all rows without a result" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]


# ---- append: rounding at ties, scales that another program chose ---------------------------------------------------

def _e4m3_numbers():
    c = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    return sorted({Fraction(float(x)) for x in c[c.isfinite()]})


E4M3 = _e4m3_numbers()


def _nearest(x, int8):
    """The code's number nearest to the fraction x, ties to even."""
    if int8:
        return round(x)
    if abs(x) >= 448:
        return Fraction(448) if x > 0 else Fraction(-448)
    best = min(E4M3, key=lambda n: abs(n - x))
    two = [n for n in E4M3 if abs(n - x) == abs(best - x)]
    if len(two) == 1:
        return best
    # of two neighbours the one whose code is even
    code = lambda n: int(torch.tensor(float(n)).to(torch.float8_e4m3fn).view(torch.uint8))  # noqa: E731
    return next(n for n in two if code(n) % 2 == 0)


def _append_into(B, held, s_old, new, dtype, code):
    """One page, one head: `held` [n, 64] codes at scale s_old in front, rows `new` [m, 64] behind; (numbers, scale) after."""
    P = 32
    ct = torch.int8 if code == "int8" else torch.float8_e4m3fn
    page = torch.zeros(1, 1, P, 64)
    page[0, 0, :len(held)] = held
    kp = page.to(ct).cuda()
    vp, s = kp.clone(), torch.full((1, 1), s_old).cuda()
    vs = s.clone()
    x = new.to(dtype).view(-1, 1, 64).cuda()
    B.es_op_kv8_append(x, x, _i32([len(held) + i for i in range(len(new))]).cuda(), kp, vp, s, vs)
    assert torch.equal(kp.view(torch.int8), vp.view(torch.int8)) and torch.equal(s, vs)
    return kp.cpu().float()[0, 0], float(s)


@pytest.mark.parametrize("first,second", [(444.5, 635.0), (349.25, 635.0), (889.0, 635.0 * 2), (2.0 * 127, 7.0 * 127), (3.0 * 127, 11.0 * 127), (1.25 * 127, 13.0 * 127)])
def test_append_brings_int8_codes_in_front_to_the_new_scale_with_ties_to_even(B, first, second):
    """Scales that are small whole numbers (largest magnitude 127 times them), so that many codes fall in the middle of two."""
    held = torch.zeros(2, 64)
    held[0], held[1] = torch.arange(1, 65), -torch.arange(64, 128)
    new = torch.zeros(1, 64)
    new[0, 3] = second
    old = first / 127
    assert float(torch.tensor(first).half()) == first and float(torch.tensor(second).half()) == second
    got, s = _append_into(B, held, old, new, torch.float16, "int8")
    assert s == second / 127
    want = [[int(_nearest(Fraction(float(c)) * Fraction(old) / Fraction(s), True)) for c in row] for row in held]
    assert got[:2].long().tolist() == want


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("s_old", [3.0, 5.0, 7.0, 13.0, 0.40625, 41.0, 49.0, 61.0, 0.1, 1.0 / 3.0, 47.0 / 127.0])
def test_append_rounds_to_e4m3_exactly_at_a_kept_scale_that_is_no_power_of_two(B, s_old, dtype):
    """Values at and next to the middle between two codes, at scales that only another program can have left."""
    s = Fraction(float(torch.tensor(s_old)))
    mids = [(a + b) / 2 for a, b in zip(E4M3, E4M3[1:]) if abs(a) <= 240 and abs(b) <= 240]
    x = torch.tensor([float(m * s) for m in mids]).to(dtype)
    near = [torch.nextafter(x, torch.full_like(x, e)) for e in (math.inf, -math.inf)]
    x = torch.cat([x, *near])
    x = torch.cat([x, torch.zeros(-len(x) % 64, dtype=dtype)]).view(-1, 64)
    for i in range(0, len(x), 24):
        new = x[i:i + 24]
        got, kept = _append_into(B, torch.ones(1, 64), s_old, new, dtype, "e4m3")
        assert kept == float(s)
        want = [[float(_nearest(Fraction(float(v)) / s, False)) for v in row] for row in new]
        assert got[1:1 + len(new)].tolist() == want


@pytest.mark.parametrize("number", [1.0, 1.125, 3.25, 15.0, 0.4375])
def test_append_brings_e4m3_codes_to_the_new_scale_from_one_that_is_no_power_of_two(B, number):
    """code * old / new next to the middle between two numbers: the product has more bits than 32-bit floats hold."""
    new = torch.zeros(1, 64)
    new[0, 0] = 448.0 * 64                                # a scale of 64
    for mid in (1.0625, 1.1875, 5.25, 2.0 ** -8 * 3 / 2):
        base = torch.tensor(mid * 64 / number)
        for old in (base, *[torch.nextafter(base, torch.tensor(e)) for e in (math.inf, -math.inf)]):
            if float(old) >= 64:
                continue
            held = torch.full((1, 64), number)
            held[0, 1::2] *= -1
            got, s = _append_into(B, held, float(old), new, torch.float16, "e4m3")
            assert s == 64.0
            want = [float(_nearest(Fraction(float(c)) * Fraction(float(old)) / 64, False)) for c in held[0]]
            assert got[0].tolist() == want


# ---- sampling ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n,V", [(3, 40000), (40, 9000), (400, 20000)])
def test_sampling_both_thresholds_in_one_list(B, n, V):
    """700 logits so close together that the borders of top-k and of top-p lie in one bin, whose elements are collected once
    and searched twice: right, and the same tokens every time."""
    g = _gen(n)
    x = -10 - 10 * torch.rand(n, V, generator=g)
    for r in range(n):
        x[r, torch.randperm(V, generator=g)[:700]] = 0.001 * torch.rand(700, generator=g)
    u = torch.rand(n, generator=g).tolist()
    k = [300 + 7 * r % 350 for r in range(n)]
    p = [(0.2, 0.5, 0.9, 0.97)[r % 4] for r in range(n)]
    tokens, _ = _check_sample(B, x, u, k=k, p=p)
    dev = [x.cuda(), torch.tensor(u).cuda(), None, torch.tensor(k, dtype=torch.int32).cuda(), torch.tensor(p).cuda()]
    for _ in range(30):
        assert B.es_op_sample(*dev)[0].tolist() == tokens


# ---- launches ----------------------------------------------------------------------------------------------------

_EDGES = """
import torch
from cuda.bindings import runtime as R
from paper_2405_14371_b200 import binding as B
from tests.test_kv8_ops_gpu import _attn_case, _gen, _i32

long, short = [[t.cuda() if torch.is_tensor(t) else t for t in _attn_case(n, 1, 16, 8, 64, 16, [400] * n, "int8", "fp16", 3)] for n in (40, 1)]
x, u = torch.randn(300, 9000, generator=_gen(5)).cuda(), torch.rand(300, generator=_gen(6)).cuda()
lens, table = _i32([5, 6]).cuda(), _i32([[0, 1], [2, 3]]).cuda()
slots, wide = _i32(list(range(16))).cuda(), _i32([[i] for i in range(2)]).repeat(1, 400).cuda()

def calls():
    out = [B.es_op_decode_attention_kv8(*c) for c in (long, short)]
    out += [*B.es_op_kv_plan(lens, lens + 3, table, 16, 8, n_pages=4), *B.es_op_kv_plan(lens, lens + 3, wide, 16, 5000, n_pages=2)]
    return out + [*B.es_op_kv8_gather(slots, *long[1:5]), *B.es_op_sample(x, u), *B.es_op_sample(x[:2], u[:2])]

want = calls()
graph = torch.cuda.CUDAGraph(keep_graph=True)
with torch.cuda.graph(graph):
    got = calls()
raw = R.cudaGraph_t(graph.raw_cuda_graph())
err, *_, n = R.cudaGraphGetEdges_v2(raw, 0)
err, _, _, data, n = R.cudaGraphGetEdges_v2(raw, n)
assert int(err) == 0
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, want))
print("early", sum(int(e.type) == int(R.cudaGraphDependencyType.cudaGraphDependencyTypeProgrammatic) for e in data), "of", n)
print("sums", [float(t.double().nan_to_num().sum()) for t in want])
"""


def test_launches_follow_the_knob_for_dependent_launch():
    """ES_PDL (read once per process, hence child processes): with 0 no launch of these calls begins before the one in front has
    ended, and the results are the same."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = {}
    for pdl in ("0", "1"):
        r = subprocess.run([sys.executable, "-c", _EDGES], cwd=root, env=dict(os.environ, ES_PDL=pdl), capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
        out[pdl] = [line.split(" ", 1) for line in r.stdout.splitlines() if line.startswith(("early", "sums"))]
    early = {pdl: lines[0][1].split(" of ") for pdl, lines in out.items()}
    assert early["0"][0] == "0" and int(early["1"][0]) > 0, early
    assert early["0"][1] == early["1"][1] and out["0"][1] == out["1"][1]


_FIRST = """
import sys
import torch
from paper_2405_14371_b200 import binding as B
from tests.test_kv8_ops_gpu import _attn_case, _gen, _i32

long, short = [[t.cuda() if torch.is_tensor(t) else t for t in _attn_case(n, 1, 16, 8, 64, 16, [400] * n, "int8", "fp16", 3)] for n in (40, 1)]
x, u = torch.randn(300, 9000, generator=_gen(5)).cuda(), torch.rand(300, generator=_gen(6)).cuda()
n = 4000
lens, more, table = _i32([0] * n).cuda(), _i32([5] * n).cuda(), _i32([[i] for i in range(n)]).cuda()
rows, slots = torch.randn(32, 8, 64, generator=_gen(7)).half().cuda(), _i32(list(range(32))).cuda()
pages, scales = [torch.zeros(2, 8, 16, 64, dtype=torch.int8, device="cuda") for _ in range(2)], [torch.zeros(2, 8, device="cuda") for _ in range(2)]
calls = dict(attend=lambda: (B.es_op_decode_attention_kv8(*long),), joined=lambda: (B.es_op_decode_attention_kv8(*short),),
             plan=lambda: B.es_op_kv_plan(lens, more, table, 16, 20000, n_pages=n), few=lambda: B.es_op_kv_plan(lens[:9], more[:9], table[:9], 16, 45, n_pages=n),
             append=lambda: (B.es_op_kv8_append(rows, rows, slots, *pages, *scales),), gather=lambda: B.es_op_kv8_gather(slots, *pages, *scales),
             sample=lambda: B.es_op_sample(x, u), sample_one=lambda: B.es_op_sample(x[:1], u[:1]))
got = {}
for name, call in calls.items():
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got[name] = graph, call()
for name, call in calls.items():
    graph, out = got[name]
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(out, call()):
        assert a is None or torch.equal(a, b), name
print("captured first")
"""


def test_the_first_call_of_a_process_may_be_a_captured_one():
    """What a call sets up once (shared-memory limits, the cluster size of large plans) it may set up while capturing."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _FIRST], cwd=root, env=dict(os.environ), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured first" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]

"""The operations over the paged 8-bit cache and sampling, against plain 64-bit forms, at the sizes and contents where they
can go wrong; refusals that need a device; graphs, streams and a run of all of them together."""
import math
import random

import pytest
import torch

from tests import kv8_reference as R

pytestmark = pytest.mark.gpu
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
HALF = {"fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def B():
    from paper_2405_14371_b200 import binding
    return binding


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _i32(x):
    return torch.as_tensor(x, dtype=torch.int32)


def _codes(shape, code, g):
    x = torch.randn(shape, generator=g)
    return (x * 32).round().clamp(-127, 127).to(torch.int8) if code == "int8" else (x * 100).clamp(-448, 448).to(torch.float8_e4m3fn)


# ---- plan --------------------------------------------------------------------------------------------------------

def _plan_case(Bn, P, pps, spare, seed, wild=False):
    """Sound random state: lengths, a table with distinct pages, the others on the stack."""
    rng = random.Random(seed)
    cap = P * pps
    old = [rng.choice([0, 1, P - 1, P, P + 1, rng.randrange(cap + 1)]) for _ in range(Bn)]
    old = [min(o, cap) for o in old]
    kind = [rng.randrange(5) for _ in range(Bn)]
    new = [0 if k == 0 else o if k == 1 else rng.randrange(o + 1) if k == 2 else min(cap, o + 1) if k == 3 else rng.randrange(o, cap + 1)
           for o, k in zip(old, kind)]
    held = sum(-(-o // P) for o in old)
    n_pages = held + spare
    pages = list(range(n_pages))
    rng.shuffle(pages)
    table = [[-1] * pps for _ in range(Bn)]
    for b in range(Bn):
        for j in range(-(-old[b] // P)):
            table[b][j] = pages.pop()
    free = pages + [-7] * (n_pages - len(pages))
    if wild:
        for b in range(0, Bn, 3):
            new[b] = rng.choice([-1, cap + 1, 2 ** 31 - 1, -2 ** 31])
    return old, new, table, free, len(pages)


def _run_plan(B, old, new, table, free, n_free, P, max_rows, alloc=True, **kw):
    """Library against simulator; returns the library's plan and state."""
    tb = [r[:] for r in table]
    fr = free[:] if alloc else None
    want = R.plan(old, new, tb, fr, n_free if alloc else 0, P, max_rows, n_pages=len(free))
    dt, df, dc = _i32(table).cuda(), _i32(free).cuda(), _i32([n_free]).cuda()
    got = B.es_op_kv_plan(_i32(old).cuda(), _i32(new).cuda(), dt, P, max_rows, df if alloc else None, dc if alloc else None,
                          n_pages=len(free), **kw)
    for name in B.KvPlan._fields:
        assert getattr(got, name).tolist() == want[name], name
    assert dt.tolist() == tb
    if alloc:
        assert int(dc) == want["free_count"]
        assert df.tolist() == fr, "the stack, left-over entries above its top included"
    return got, dt, df, dc


@pytest.mark.parametrize("Bn,P,pps,spare,max_rows", [
    (1, 16, 1, 1, 1), (1, 16, 3, 5, 7), (2, 16, 4, 3, 64), (7, 16, 5, 11, 33), (64, 64, 6, 100, 4000), (33, 32, 9, 4, 200),
    (300, 16, 8, 900, 9000), (1025, 16, 3, 2000, 20000), (1500, 128, 2, 10, 5000),
])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_plan_matches_the_simulator(B, Bn, P, pps, spare, max_rows, seed):
    """Served and refused requests (too few pages, too few rows), pages returned and taken in one call, one CTA and a
    cluster (max_rows above 4096), several chunks of 1024 requests."""
    old, new, table, free, n_free = _plan_case(Bn, P, pps, spare, seed * 1000 + Bn)
    _plan_stack(B, old, new, table, free, n_free, P, max_rows)


def _plan_stack(B, old, new, table, free, n_free, P, max_rows):
    # the simulator pushes and pops one entry at a time, so its entries above the final top differ: compare what counts
    tb, fr = [r[:] for r in table], free[:]
    want = R.plan(old, new, tb, fr, n_free, P, max_rows)
    dt, df, dc = _i32(table).cuda(), _i32(free).cuda(), _i32([n_free]).cuda()
    got = B.es_op_kv_plan(_i32(old).cuda(), _i32(new).cuda(), dt, P, max_rows, df, dc)
    for name in B.KvPlan._fields:
        assert getattr(got, name).tolist() == want[name], name
    assert dt.tolist() == tb
    left = want["free_count"]
    assert int(dc) == left
    assert df.tolist()[:left] == fr[:left]
    # no page is lost or given twice
    held = [p for b, row in enumerate(tb) for p in row[: -(-want["len_out"][b] // P)]]
    assert sorted(held + fr[:left]) == list(range(len(free)))
    return got, dt, df, dc


def test_plan_refuses_single_requests_with_lengths_out_of_range(B):
    old, new, table, free, n_free = _plan_case(40, 16, 4, 60, 5, wild=True)
    _plan_stack(B, old, new, table, free, n_free, 16, 700)
    old[1], old[4] = -5, 10 ** 9                      # lengths held that cannot be
    table[1], table[4] = [-1] * 4, [-1] * 4
    tb, fr = [r[:] for r in table], free[:]
    want = R.plan(old, new, tb, fr, n_free, 16, 700)
    got = B.es_op_kv_plan(_i32(old).cuda(), _i32(new).cuda(), _i32(table).cuda(), 16, 700, _i32(free).cuda(), _i32([n_free]).cuda())
    for name in B.KvPlan._fields:
        assert getattr(got, name).tolist() == want[name], name


def test_plan_stays_in_bounds_with_unsound_state(B):
    """A stack count beyond its room, table entries that are no pages: nothing is read or written outside, and slots are
    only ever inside the pool."""
    Bn, P, pps = 20, 16, 4
    old = [P * (b % 5) for b in range(Bn)]
    new = [P * ((b * 3) % 5) for b in range(Bn)]
    pad = 64
    for count in (-3, 0, 10 ** 9):
        room = torch.full((pad + 30 + pad,), 77, dtype=torch.int32, device="cuda")
        table = torch.full((pad + Bn * pps + pad,), 10 ** 9, dtype=torch.int32, device="cuda")
        dt, df = table[pad:-pad].view(Bn, pps), room[pad:-pad]
        dt[::2] = -1
        got = B.es_op_kv_plan(_i32(old).cuda(), _i32(new).cuda(), dt, P, 300, df, _i32([count]).cuda())
        s = got.slot_map
        assert bool(((s == -1) | ((s >= 0) & (s < 30 * P))).all())
        for t, v in ((room, 77), (table, 10 ** 9)):
            assert bool((t[:pad] == v).all()) and bool((t[-pad:] == v).all())


def test_plan_without_allocation_maps_ranges_of_an_existing_table(B):
    P = 16
    table = [[5, 2, 9, -1], [7, 0, 1, 3], [30, 4, 6, 8]]
    for max_rows in (40, 200, 6000):
        _run_plan(B, [3, 0, 17], [40, 64, 20], table, [0] * 12, 0, P, max_rows, alloc=False)
        _run_plan(B, [0, 10, 60], [64, 0, 64], table, [0] * 12, 0, P, max_rows, alloc=False)


def test_plan_writes_into_given_outputs_and_lengths_in_place(B):
    old, new, table, free, n_free = _plan_case(50, 16, 6, 300, 9)
    first, _, _, _ = _plan_stack(B, old, new, table, free, n_free, 16, 3000)
    do = _i32(old).cuda()
    out = B.KvPlan(*[torch.full_like(t, 123) for t in first[:-1]], do)
    got = B.es_op_kv_plan(do, _i32(new).cuda(), _i32(table).cuda(), 16, 3000, _i32(free).cuda(), _i32([n_free]).cuda(), out=out)
    assert got.len_out.data_ptr() == do.data_ptr()
    for a, b in zip(got, first):
        assert torch.equal(a, b)


# ---- append and gather -------------------------------------------------------------------------------------------

def _append_case(lens, P, Hkv, hd, code, dtype, seed, spread=1.0):
    """Sequences of (held, new) tokens over scattered pages; returns everything on the CPU."""
    g = _gen(seed)
    pps = max(1, max(-(-(h + n) // P) for h, n in lens))
    n_pages = sum(-(-(h + n) // P) for h, n in lens) + 3
    perm = torch.randperm(n_pages, generator=g)
    table, at = torch.full((len(lens), pps), -1, dtype=torch.long), 0
    for b, (h, n) in enumerate(lens):
        u = -(-(h + n) // P)
        table[b, :u] = perm[at:at + u]
        at += u
    slots = [int(table[b, i // P]) * P + i % P for b, (h, n) in enumerate(lens) for i in range(h, h + n)]
    codes = [_codes((n_pages, Hkv, P, hd), code, g) for _ in range(2)]
    e = torch.randn(2, n_pages, Hkv, generator=g) - 5
    scales = torch.exp2(e if code == "int8" else e.round())
    x = (torch.randn(len(slots), 2 * Hkv, hd, generator=g) * torch.exp(spread * torch.randn(len(slots), 2 * Hkv, 1, generator=g))).to(HALF[dtype])
    return table, slots, codes, scales, x


def _check_append(B, lens, P, Hkv, hd, code, dtype, seed, mode, change=None, slots_of=None):
    table, slots, codes, scales, x = _append_case(lens, P, Hkv, hd, code, dtype, seed)
    if change is not None:
        change(x)
    if slots_of is not None:
        slots = slots_of(slots)
    d = [c.cuda() for c in codes]
    s = [t.contiguous().cuda() for t in scales]
    fused = x.cuda()
    k, v = fused[:, :Hkv], fused[:, Hkv:]
    runs = None
    if mode == "runs":
        first = [i for i in range(len(slots)) if i == 0 or slots[i] != slots[i - 1] + 1 or slots[i] % P == 0]
        runs = _i32(first + [-1] * 5).cuda()
    elif mode == "dense":
        k, v = k.contiguous(), v.contiguous()
    B.es_op_kv8_append(k, v, _i32(slots + [-1] * 4).cuda(), d[0], d[1], s[0], s[1], runs=runs)
    for i in range(2):
        want, sc = codes[i].clone(), scales[i].clone()
        R.append(x[:, i * Hkv:(i + 1) * Hkv], slots, want, sc, P)
        assert torch.equal(s[i].cpu().nan_to_num(-1.0), sc.nan_to_num(-1.0))
        assert torch.equal(d[i].cpu().view(torch.int8), want.view(torch.int8))     # pages that no row went to included
    every = [int(table[b, i // P]) * P + i % P for b, (h, n) in enumerate(lens) for i in range(h + n)] + [-1, 10 ** 9, -10 ** 9]
    for out in (torch.float16, torch.bfloat16, torch.float32):
        gk, gv = B.es_op_kv8_gather(_i32(every).cuda(), d[0], d[1], s[0], s[1], dtype=out)
        for got, i in ((gk, 0), (gv, 1)):
            want = R.gather(every, d[i].cpu(), s[i].cpu(), P, out)
            assert torch.equal(got.cpu().float().nan_to_num(-1.0), want.float().nan_to_num(-1.0))


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("lens,P,Hkv,hd,mode", [
    ([(0, 1)], 16, 1, 64, "rows"), ([(5, 1), (0, 1), (15, 1), (16, 1), (31, 1)], 16, 2, 128, "rows"),
    ([(0, 16), (3, 13), (3, 14), (0, 33), (40, 1)], 16, 3, 64, "runs"), ([(0, 1), (63, 2), (64, 130), (7, 200)], 64, 2, 128, "runs"),
    ([(0, 300), (1, 299)], 128, 1, 128, "rows"), ([(9, 70), (0, 5)], 32, 5, 128, "dense"), ([(200, 100)], 256, 1, 64, "runs"),
])
def test_append_and_gather_are_exact(B, lens, P, Hkv, hd, mode, code, dtype):
    _check_append(B, lens, P, Hkv, hd, code, dtype, 17, mode)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("mode", ["rows", "runs"])
def test_append_borders_zeros_and_values_without_a_number(B, code, dtype, mode):
    """Ties between two codes, all-zero rows, the type's largest and smallest numbers, infinities and NaN (a NaN scale for
    that page and head alone)."""
    def change(x):
        x[0] = 0.0
        x[1, 0] = 0.0
        x[1, 0, :8] = torch.tensor([127.0, 2.5, -2.5, 3.5, 0.5, -0.5, 1.5, 126.5], dtype=x.dtype)
        x[2, 0] = torch.finfo(x.dtype).max
        x[2, 1] = torch.finfo(x.dtype).tiny
        x[3, 0, 3] = math.inf
        x[4, 1, 5] = -math.inf
        x[5, 2, 7] = math.nan
        x[6] = 448.0
        x[6, 0, 0] = 449.0 if x.dtype == torch.bfloat16 else 448.25
        x[7, 0] = 6e-8 if x.dtype == torch.float16 else 1e-40
    _check_append(B, [(0, 1), (0, 1), (3, 1), (5, 1), (0, 1), (9, 1), (0, 1), (0, 1), (2, 20)], 16, 2, 64, code, dtype, 23, mode, change)


@pytest.mark.parametrize("mode", ["rows", "runs"])
def test_append_leaves_out_rows_without_a_place(B, mode):
    def slots_of(s):
        s = s[:]
        s[0], s[5], s[-1] = -1, 10 ** 9, -(2 ** 31)
        return s
    _check_append(B, [(0, 4), (14, 20), (3, 9)], 16, 2, 128, "int8", "fp16", 29, mode, slots_of=slots_of)


def test_append_one_by_one_keeps_every_value_within_the_scale_steps(B):
    """A page filled token by token with growing values: each growth rounds the codes in front once more, by half a step of
    the scale of that time, so the stored value is off by at most the sum of half steps since it was written."""
    P, Hkv, hd = 16, 1, 64
    g = _gen(3)
    x = torch.randn(P, Hkv, hd, generator=g).half()
    x[:] = (x.float() * torch.linspace(0.1, 3, P)[:, None, None]).half()
    kp, vp = (torch.zeros(1, Hkv, P, hd, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(1, Hkv, device="cuda") for _ in range(2))
    allowed = torch.zeros(P, dtype=torch.float64)
    last = None
    for i in range(P):
        B.es_op_kv8_append(x[i:i + 1].cuda(), x[i:i + 1].cuda(), _i32([i]).cuda(), kp, vp, ks, vs)
        s = float(ks)
        allowed[i] = s / 2
        if last is not None and s != last:
            allowed[:i] += s / 2
        last = s
    k, _ = B.es_op_kv8_gather(_i32(list(range(P))).cuda(), kp, vp, ks, vs, dtype=torch.float32)
    off = (k.cpu().double() - x.double()).abs().amax((1, 2))
    assert bool((off <= allowed * (1 + 2 ** -20)).all())


# ---- attention ---------------------------------------------------------------------------------------------------

def _attn_case(Bn, T, Hq, Hkv, hd, P, ctxs, code, dtype, seed, max_ctx=None, extra_pages=2):
    g = _gen(seed)
    max_ctx = max_ctx or max(1, max(ctxs))
    pps = -(-max_ctx // P)
    n_pages = sum(-(-c // P) for c in ctxs) + extra_pages
    perm, at = torch.randperm(n_pages, generator=g), 0
    table = torch.full((Bn, pps), -1, dtype=torch.int32)
    for b, c in enumerate(ctxs):
        u = -(-c // P)
        table[b, :u] = perm[at:at + u].int()
        at += u
    kc, vc = (_codes((n_pages, Hkv, P, hd), code, g) for _ in range(2))
    ks, vs = (torch.exp2(torch.randn(n_pages, Hkv, generator=g) - 5) for _ in range(2))
    q = torch.randn(Bn, T, Hq, hd, generator=g).to(HALF[dtype])
    return q, kc, vc, ks, vs, table, _i32(ctxs), max_ctx


def _check_attn(B, case, got=None, P=None):
    q, kc, vc, ks, vs, table, ctx, max_ctx = case
    P = kc.shape[2]
    if got is None:
        got = B.es_op_decode_attention_kv8(*[t.cuda() for t in (q, kc, vc, ks, vs, table, ctx)], max_ctx)
    want, bound = R.attend(q, kc, vc, ks, vs, table, ctx, P, max_ctx)
    got = got.cpu().double().reshape(want.shape)
    over = (got - want).abs() / bound
    worst = float(over.max())
    where = [int(i) for i in torch.unravel_index(over.argmax(), over.shape)]
    assert worst <= 1.0, f"{worst} of what is allowed at [b, t, head, dim] {where}, {int((over > 1).sum())} places"
    return got


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("Bn,T,Hq,Hkv,hd,P,ctxs", [
    (1, 1, 1, 1, 64, 16, [1]), (2, 1, 4, 4, 128, 16, [0, 17]), (3, 1, 8, 1, 128, 64, [5, 64, 200]), (2, 1, 10, 2, 64, 32, [300, 31]),
    (1, 1, 8, 8, 128, 64, [2000]), (4, 1, 16, 1, 128, 16, [16, 15, 100, 1]), (2, 3, 6, 2, 64, 16, [2, 50]), (2, 4, 12, 2, 128, 32, [1, 130]),
    (2, 2, 16, 2, 128, 128, [700, 3]), (1, 5, 40, 2, 64, 16, [90]), (1, 17, 2, 1, 128, 16, [40]), (9, 1, 2, 2, 64, 16, [0, 1, 15, 16, 17, 63, 64, 65, 129]),
])
def test_attention(B, Bn, T, Hq, Hkv, hd, P, ctxs, code, dtype):
    _check_attn(B, _attn_case(Bn, T, Hq, Hkv, hd, P, ctxs, code, dtype, 31))


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("P,hd,Hq,T", [(16, 64, 8, 1), (32, 128, 16, 1), (64, 128, 8, 3), (128, 64, 24, 2), (16, 128, 24, 4), (64, 128, 40, 3)])
@pytest.mark.parametrize("longest", [400, 3000])
def test_attention_many_items_share_the_machine(B, P, hd, Hq, T, longest, code):
    """More (sequence, head) items than SMs: stretches of tiles that begin and end inside items, tiles of both sizes, one and
    two row blocks, several row tiles, sequences without keys among them."""
    rng = random.Random(P * T + Hq)
    ctxs = [rng.choice([0, 1, 15, 31, 32, 33, 63, 64, 65, 130, 200]) for _ in range(20)]
    ctxs[7], ctxs[13] = longest, longest // 2
    case = _attn_case(20, T, Hq, 8, hd, P, ctxs, code, "bf16" if T == 3 else "fp16", 71)
    assert B.es_op_decode_attention_kv8_scratch_bytes(20, T, Hq, 8, hd, P, longest) > 0
    _check_attn(B, case)


def test_attention_short_sequences_in_a_long_table(B):
    """Every sequence lies in one tile, so nothing is left to merge; what follows on the stream still finds the outputs."""
    case = _attn_case(40, 1, 16, 8, 128, 16, [1 + i % 16 for i in range(40)], "int8", "fp16", 73, max_ctx=8000)
    dev = [t.cuda() for t in case[:7]]
    out = torch.zeros(40, 1, 16 * 128, dtype=torch.float16, device="cuda")
    for _ in range(20):
        out.fill_(math.nan)
        B.es_op_decode_attention_kv8(*dev, 8000, out=out)
        last = out.clone()
        assert not bool(last.isnan().any())
    _check_attn(B, case, got=last)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_attention_never_meets_what_lies_behind_the_context(B, code):
    """Garbage codes (NaN among them) behind the last token, in pages of nobody and NaN scales on pages out of sight do not
    reach a result, and lengths beyond max_ctx or the table are cut."""
    case = list(_attn_case(3, 2, 8, 2, 128, 16, [37, 1, 64], code, "fp16", 37, max_ctx=64))
    q, kc, vc, ks, vs, table, ctx, max_ctx = case
    used = {int(p) for p in table.flatten() if p >= 0}
    for p in range(kc.shape[0]):
        if p not in used:
            ks[p], vs[p] = math.nan, math.inf
            kc[p].view(torch.int8).fill_(0x7f)
            vc[p].view(torch.int8).fill_(0x7f)
    last = int(table[0, 2])
    for c in (kc, vc):
        c[last].view(torch.int8)[:, 5:] = 0x7f
        c[int(table[1, 0])].view(torch.int8)[:, 1:] = -1
    _check_attn(B, case)
    case[6] = _i32([37, 1, 10 ** 9])
    _check_attn(B, case)
    case[6] = _i32([37, -5, 64])
    got = _check_attn(B, case)
    assert bool((got[1] == 0).all())


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_attention_passes_over_table_entries_that_are_no_pages(B, dtype):
    case = _attn_case(2, 1, 4, 2, 64, 16, [100, 40], "int8", dtype, 41)
    case[5][0, 1], case[5][0, 6], case[5][1, 0], case[5][1, 1], case[5][1, 2] = -1, 10 ** 6, -9, 2 ** 31 - 1, -1
    got = _check_attn(B, case)
    assert bool((got[1] == 0).all())                   # a row that the table leaves nothing


def test_attention_pages_of_very_different_scales(B):
    """V's scales 2^60 apart and a score gap that makes the large page's weight 2^-30: its share must not be lost.  One
    query, two pages: want = sum of p v by the definition."""
    P, hd = 16, 64
    q = torch.zeros(1, 1, 1, hd, dtype=torch.bfloat16)
    q[..., 0] = 1.0
    kc = torch.zeros(2, 1, P, hd, dtype=torch.int8)
    kc[0, 0, :, 0], kc[1, 0, :, 0] = 100, -66            # scores 166 s / 8 apart: about 20.75 = ln 2^30
    vc = torch.randint(-127, 128, (2, 1, P, hd), generator=_gen(2)).to(torch.int8)
    ks = torch.ones(2, 1)
    vs = torch.tensor([[2.0 ** -40], [2.0 ** 20]])
    for ctx in (32, 20):
        _check_attn(B, (q, kc, vc, ks, vs, _i32([[0, 1]]), _i32([ctx]), 32))
        _check_attn(B, (q, kc, vc, ks, vs.flip(0), _i32([[1, 0]]), _i32([ctx]), 32))


def test_attention_bf16_queries_beyond_the_range_of_fp16(B):
    for f in (2.0 ** 40, 2.0 ** -60):
        case = list(_attn_case(2, 1, 4, 2, 128, 16, [33, 50], "e4m3", "bf16", 43))
        case[0] = (case[0].float() * f).bfloat16()
        case[3] = case[3] / f
        _check_attn(B, case)


def test_attention_shows_a_page_without_a_number_to_the_rows_that_see_it(B):
    q, kc, vc, ks, vs, table, ctx, max_ctx = _attn_case(2, 2, 4, 2, 64, 16, [17, 40], "int8", "fp16", 47)
    page = int(table[0, 1])                             # holds token 16 only, which the first of the two queries does not see
    for scale in (ks, vs):
        scale[page, 1] = math.nan
        got = B.es_op_decode_attention_kv8(*[t.cuda() for t in (q, kc, vc, ks, vs, table, ctx)], max_ctx).cpu().reshape(2, 2, 4, 64)
        assert bool(got[0, 1, 2:].isnan().all())
        got[0, 1, 2:] = 0
        assert bool(got.isfinite().all())
        scale[page, 1] = 1.0
    q[0, 0, 0, 3] = math.inf
    q[1, 1, 3, 0] = math.nan
    got = B.es_op_decode_attention_kv8(*[t.cuda() for t in (q, kc, vc, ks, vs, table, ctx)], max_ctx).cpu().reshape(2, 2, 4, 64)
    bad = got.isnan().all(-1)
    assert bad.nonzero().tolist() == [[0, 0, 0], [1, 1, 3]]


def test_attention_long_context_many_splits_and_sliced_queries(B):
    """One sequence cut into many splits, q a slice of a fused projection's rows, both result layouts, the same bits from a
    caller's scratch full of garbage and from run to run."""
    case = _attn_case(1, 1, 8, 2, 128, 64, [20001], "int8", "fp16", 53)
    q, kc, vc, ks, vs, table, ctx, max_ctx = case
    dev = [t.cuda() for t in (kc, vc, ks, vs, table, ctx)]
    fused = torch.full((1, 12, 128), math.nan, dtype=torch.float16, device="cuda")
    fused[:, :8] = q[:, 0].cuda()
    a = B.es_op_decode_attention_kv8(fused[:, :8], *dev, max_ctx)
    assert a.shape == (1, 1024)
    _check_attn(B, case, got=a)
    n = B.es_op_decode_attention_kv8_scratch_bytes(1, 1, 8, 2, 128, 64, max_ctx)
    assert n > 0
    scratch = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.empty(1, 1, 1024, dtype=torch.float16, device="cuda")
    for _ in range(3):
        b = B.es_op_decode_attention_kv8(q.cuda(), *dev, max_ctx, scratch=scratch, out=out)
        assert b.data_ptr() == out.data_ptr() and torch.equal(a, b[:, 0])
    with pytest.raises(B.EsError) as e:
        B.es_op_decode_attention_kv8(q.cuda(), *dev, max_ctx, scratch=scratch[: n - 16])
    assert e.value.status == 6


def test_attention_agrees_with_the_fp16_cache(B):
    """The same values in both caches: codes times a power of two are fp16 numbers, so es_op_decode_attention sees the same
    keys and values; both are within their own rounding of the same result."""
    case = list(_attn_case(4, 1, 16, 4, 128, 64, [700, 64, 1, 333], "int8", "fp16", 59))
    for i in (3, 4):
        case[i] = torch.exp2(case[i].log2().round())
    q, kc, vc, ks, vs, table, ctx, max_ctx = [t.cuda() if torch.is_tensor(t) else t for t in case]
    got = B.es_op_decode_attention_kv8(q, kc, vc, ks, vs, table, ctx, max_ctx)[:, 0].double()
    kf, vf = (c.half() * s[..., None, None].half() for c, s in ((kc, ks), (vc, vs)))
    other = B.es_op_decode_attention(q[:, 0].contiguous(), kf, vf, table.clamp(min=0), ctx, max_ctx).double()
    # the fp16 kernel rounds its probabilities to fp16 and its result to fp16: 2^-11 each of what it sums
    _, bound = R.attend(case[0], case[1], case[2], case[3], case[4], case[5], case[6], 64, max_ctx)
    scale = vf.double().abs().max()
    assert bool(((got - other).abs().cpu() <= bound.reshape(4, -1) + 2.0 ** -10 * float(scale)).all())


# ---- sampling ----------------------------------------------------------------------------------------------------

def _check_sample(B, x, u, T=None, k=None, p=None, m=None, same=True):
    n = x.shape[0]
    dev = lambda t, d: None if t is None else torch.tensor(t, dtype=d).cuda()  # noqa: E731
    f = torch.float32
    tok, lp = B.es_op_sample(x.cuda(), dev(u, f), dev(T, f), dev(k, torch.int32), dev(p, f), dev(m, f))
    tok, lp = tok.tolist(), lp.tolist()
    for r in range(n):
        at = lambda t, d: d if t is None else float(torch.tensor(t[r], dtype=f))  # noqa: E731
        want, logp = R.sample(x[r], at(u, 0.0), at(T, 1.0), 0 if k is None else k[r], at(p, 1.0), at(m, 0.0))
        assert tok[r] == want, (r, tok[r], want)
        # the sum of weights is within 2^-45 a token of the whole, the logarithm is rounded to 32 bits once
        assert lp[r] == logp or abs(lp[r] - logp) <= 2.0 ** -24 * abs(logp) + 2.0 ** -26, (r, lp[r], logp)
    return tok, lp


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,V", [(1, 1), (3, 2), (2, 127), (5, 128), (4, 129), (3, 1000), (9, 4099), (2, 32000), (40, 5000), (1, 50257), (200, 300)])
def test_sampling_matches_the_definition(B, n, V, dtype):
    """One CTA and clusters of 2 to 8 per row; every setting alone and together, low precision logits with many ties."""
    g, rng = _gen(n * 7 + V), random.Random(n + V)
    x = (torch.randn(n, V, generator=g) * (0.5 + 4 * torch.rand(n, 1, generator=g))).to(dtype)
    u = torch.rand(n, generator=g).tolist()
    T = [rng.choice([0.0, 0.3, 0.7, 1.0, 1.7]) for _ in range(n)]
    k = [rng.choice([0, 1, 2, 5, 50, V - 1, V, V + 3, -1]) for _ in range(n)]
    p = [rng.choice([0.0, 0.1, 0.5, 0.9, 0.99, 1.0, 2.0]) for _ in range(n)]
    m = [rng.choice([0.0, 0.01, 0.2, 1.0]) for _ in range(n)]
    _check_sample(B, x, u)
    _check_sample(B, x, u, T=T)
    _check_sample(B, x, u, k=k)
    _check_sample(B, x, u, p=p)
    _check_sample(B, x, u, m=m)
    _check_sample(B, x, u, T, k, p, m)


@pytest.mark.parametrize("dtype,n,V", [(torch.float32, 700, 1100), (torch.bfloat16, 310, 20001), (torch.float16, 160, 30000), (torch.float32, 80, 60001),
                                        (torch.bfloat16, 40, 130003), (torch.float32, 300, 17000)])
def test_sampling_many_rows(B, n, V, dtype):
    """More CTAs than run at once, so slices are read again from L2: clusters of 1 to 8 and the larger slices of large calls; rows
    of ties among them (plateaus longer than any list, across the borders of top-k and top-p)."""
    g, rng = _gen(n + V), random.Random(n * V)
    x = torch.randn(n, V, generator=g) * (0.5 + 4 * torch.rand(n, 1, generator=g))
    x[::7] = (x[::7] * 2).round() / 2
    x[3::11] = (torch.arange(V) % 3).float()
    x[5::13] = 0.0
    x[8::17, V // 3:] = -math.inf
    x = x.to(dtype)
    u = torch.rand(n, generator=g).tolist()
    T = [rng.choice([0.0, 0.3, 0.7, 1.0, 1.7]) for _ in range(n)]
    k = [rng.choice([0, 1, 2, 50, 190, 300, 5000, V - 1, V + 3]) for _ in range(n)]
    p = [rng.choice([0.1, 0.5, 0.9, 0.99, 1.0]) for _ in range(n)]
    m = [rng.choice([0.0, 0.01, 0.2]) for _ in range(n)]
    _check_sample(B, x, u, k=k)
    _check_sample(B, x, u, p=p)
    _check_sample(B, x, u, T, k, p, m)


@pytest.mark.parametrize("V", [7, 1000, 40000])
def test_sampling_ties_go_to_the_lowest_index(B, V):
    """All logits equal, two values, a plateau across the border of top-k and of top-p."""
    x = torch.zeros(6, V)
    x[1] = -3.0
    x[2, ::2] = 1.0
    x[3, V // 2:] = 2.0
    x[4, : V // 3] = -0.0
    x[5] = torch.arange(V) % 3
    for u in (0.0, 0.25, 0.5, 0.999999):
        for kk in (0, 1, 3, V // 2, V - 1):
            for pp in (1.0, 0.3, 0.77):
                _check_sample(B, x, [u] * 6, k=[kk] * 6, p=[pp] * 6)


def test_sampling_masks_infinities_and_rows_with_nothing_left(B):
    V = 600
    g = _gen(5)
    x = torch.randn(12, V, generator=g)
    x[0] = -math.inf
    x[1] = math.nan
    x[2, ::2] = math.nan
    x[3, 1:] = -math.inf
    x[4, 10:] = torch.finfo(torch.float32).min
    x[5] = torch.finfo(torch.float32).min
    x[6, 77] = math.inf
    x[7, [30, 500]] = math.inf
    x[8] = torch.finfo(torch.float32).max
    x[8, 4] = torch.finfo(torch.float32).min
    x[9, :300] = -math.inf
    x[10, 5] = 3e38
    x[11] = -1e-40
    for u in (0.0, 0.4, 0.99):
        for kw in ({}, {"k": [300] * 12}, {"p": [0.6] * 12}, {"m": [0.3] * 12}, {"T": [0.0] * 12}, {"T": [1e-30] * 12}, {"T": [3e38] * 12, "k": [10] * 12}):
            tok, lp = _check_sample(B, x, [u] * 12, **kw)
            assert tok[0] == tok[1] == -1 and lp[0] == -math.inf


def test_sampling_random_numbers_at_and_beyond_the_ends(B):
    x = torch.tensor([[0.0, 1.0, -math.inf, 0.5, -math.inf]]).repeat(5, 1)
    tok, _ = _check_sample(B, x, [0.0, 1.0, -3.0, 7.0, 0.9999999])
    assert tok == [0, 3, 0, 3, 3]
    tok, _ = B.es_op_sample(x.cuda(), torch.full((5,), math.nan, device="cuda"))
    assert tok.tolist() == [0] * 5                      # no number counts as 0


def test_sampling_follows_the_distribution(B):
    """20000 draws with evenly spaced u from one row: every token's share is its probability to within one draw at each end
    of its interval."""
    n, V = 20000, 50
    x = torch.randn(1, V, generator=_gen(8)).repeat(n, 1)
    u = (torch.arange(n) + 0.5) / n
    tok, _ = B.es_op_sample(x.cuda(), u.cuda())
    share = torch.bincount(tok.cpu().long(), minlength=V).double() / n
    p = torch.softmax(x[0].double(), 0)
    # u is held in 32 bits: its own rounding moves a border by at most 2^-25
    assert bool(((share - p).abs() <= (1.0 + 1e-2) / n).all())


def test_sampling_takes_padded_rows_and_given_outputs(B):
    wide = torch.full((4, 1100), 50.0)
    wide[:, :1000] = torch.randn(4, 1000, generator=_gen(9))
    d = wide.cuda()
    out = (torch.full((4,), -9, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda"))
    u = torch.tensor([0.1, 0.3, 0.6, 0.95]).cuda()
    got = B.es_op_sample(d[:, :1000], u, out=out)
    assert got[0].data_ptr() == out[0].data_ptr()
    assert got[0].tolist() == [R.sample(wide[r, :1000], float(u[r]))[0] for r in range(4)]


# ---- refusals that need a device ---------------------------------------------------------------------------------

def test_calls_refuse_what_they_cannot_take(B):
    q, kc, vc, ks, vs, table, ctx, max_ctx = [t.cuda() if torch.is_tensor(t) else t for t in _attn_case(2, 1, 4, 2, 64, 16, [20, 30], "int8", "fp16", 61)]
    slots = _i32([0, 1]).cuda()
    k = torch.zeros(2, 2, 64, dtype=torch.float16, device="cuda")

    def refused(f, *a, status=1, **kw):
        with pytest.raises(B.EsError) as e:
            f(*a, **kw)
        assert e.value.status == status and e.value.message

    at = B.es_op_decode_attention_kv8
    refused(at, q.float(), kc, vc, ks, vs, table, ctx, max_ctx)
    refused(at, q, kc.half(), vc.half(), ks, vs, table, ctx, max_ctx)
    refused(at, q, kc, vc.view(torch.float8_e4m3fn), ks, vs, table, ctx, max_ctx)
    refused(at, q, kc, vc, ks.double(), vs, table, ctx, max_ctx)
    refused(at, q, kc, vc, ks, vs, table.long(), ctx, max_ctx)
    refused(at, q, kc, vc, ks, vs, table, ctx[:1], max_ctx)
    refused(at, q, kc, vc, ks, vs, table, ctx, 1000, status=3)
    refused(at, q, kc, vc, ks, vs, table, ctx, 0)
    refused(at, q[..., :3, :], kc, vc, ks, vs, table, ctx, max_ctx, status=2)
    refused(at, q.transpose(1, 2).contiguous().transpose(1, 2)[..., ::2], kc, vc, ks, vs, table, ctx, max_ctx)
    refused(at, q.cpu(), kc, vc, ks, vs, table, ctx, max_ctx)
    refused(at, torch.zeros(2 * 4 * 64 + 1, dtype=torch.float16, device="cuda")[1:].view(2, 1, 4, 64), kc, vc, ks, vs, table, ctx, max_ctx)
    ap = B.es_op_kv8_append
    refused(ap, k, k.bfloat16(), slots, kc, vc, ks, vs)
    refused(ap, k.float(), k.float(), slots, kc, vc, ks, vs)
    refused(ap, k, k, slots[:1], kc, vc, ks, vs)
    refused(ap, k, k, slots.long(), kc, vc, ks, vs)
    refused(ap, k.transpose(0, 1), k.transpose(0, 1), slots, kc, vc, ks, vs)
    refused(ap, k, k, slots, kc[:, :, :8].contiguous(), vc[:, :, :8].contiguous(), ks, vs, status=2)
    refused(B.es_op_kv8_gather, slots, kc, vc, ks, vs, dtype=torch.float64)
    x, u = torch.zeros(2, 10, device="cuda"), torch.zeros(2, device="cuda")
    refused(B.es_op_sample, x.double(), u)
    refused(B.es_op_sample, x, u.double())
    refused(B.es_op_sample, x, u[:1])
    refused(B.es_op_sample, x, u, top_k=u)
    refused(B.es_op_sample, x.t(), u)
    refused(B.es_op_sample, x[:1].expand(2, 10), u)
    refused(B.es_op_sample, torch.zeros(1, 262145, device="cuda"), u[:1], status=3)
    lens, t2 = _i32([1, 2]).cuda(), _i32([[0], [1]]).cuda()
    refused(B.es_op_kv_plan, lens, lens, t2, 16, 0)
    refused(B.es_op_kv_plan, lens, lens, t2, 24, 4, status=2)
    refused(B.es_op_kv_plan, lens, lens, t2, 16, 4, lens)
    refused(B.es_op_kv_plan, lens.long(), lens, t2, 16, 4)
    refused(B.es_op_kv_plan, _i32([0] * 8193).cuda(), _i32([0] * 8193).cuda(), _i32([[0]] * 8193).cuda(), 16, 4, status=3)


def test_calls_refuse_expanded_rows(B):
    """Rows that all lie in one place have no row stride: taken for dense they would be read beyond the tensor's end."""
    q, kc, vc, ks, vs, table, ctx, max_ctx = [t.cuda() if torch.is_tensor(t) else t for t in _attn_case(2, 3, 4, 2, 64, 16, [20, 30], "int8", "fp16", 61)]
    slots = _i32([0, 1, 2]).cuda()
    k = torch.zeros(3, 2, 64, dtype=torch.float16, device="cuda")
    for bad in (q[:1].expand(2, 3, 4, 64), q[:, :1].expand(2, 3, 4, 64), q[:1, :1].expand(2, 3, 4, 64), q[:1, 0].expand(2, 4, 64)):
        with pytest.raises(B.EsError):
            B.es_op_decode_attention_kv8(bad, kc, vc, ks, vs, table, ctx, max_ctx)
    for a, b in ((k[:1].expand(3, 2, 64), k[:1].expand(3, 2, 64)), (k, k[:1].expand(3, 2, 64)), (k[:, :1].expand(3, 2, 64), k)):
        with pytest.raises(B.EsError):
            B.es_op_kv8_append(a, b, slots, kc, vc, ks, vs)
    B.es_op_decode_attention_kv8(q[:1].expand(1, 3, 4, 64), kc, vc, ks, vs, table[:1], ctx[:1], max_ctx)      # one of them is no expansion


def test_pools_beyond_32_bit_offsets(B):
    """4.6 GB of codes each: pages on both sides of 2^31 and 2^32 bytes."""
    n_pages, Hkv, P, hd = 70000, 8, 64, 128
    pages = [69999, 2, 65536, 32768, 65535, 32767]
    g = _gen(83)
    kp, vp = (torch.empty(n_pages, Hkv, P, hd, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(n_pages, Hkv, device="cuda") for _ in range(2))
    n = 6 * P - 7
    k, v = (torch.randn(n, Hkv, hd, generator=g).half() for _ in range(2))
    place = [(pages[i // P], i % P) for i in range(n)]
    slots = _i32([p * P + o for p, o in place])
    B.es_op_kv8_append(k.cuda(), v.cuda(), slots.cuda(), kp, vp, ks, vs)
    small = [(torch.zeros(6, Hkv, P, hd, dtype=torch.int8), torch.zeros(6, Hkv)) for _ in range(2)]
    local = list(range(n))
    back = B.es_op_kv8_gather(slots.cuda(), kp, vp, ks, vs, dtype=torch.float32)
    for x, (c, s), dc, ds, got in zip((k, v), small, (kp, vp), (ks, vs), back):
        R.append(x, local, c, s, P)
        at = torch.tensor(pages, device="cuda")
        rows = lambda t: t.transpose(1, 2).reshape(6 * P, Hkv, hd)[:n]
        assert torch.equal(rows(dc[at].cpu()), rows(c)) and torch.equal(ds[at].cpu(), s)
        assert torch.equal(got.cpu(), rows(c.float() * s[:, :, None, None]))
    q = torch.randn(1, 1, 16, hd, generator=g).half()
    got = B.es_op_decode_attention_kv8(q.cuda(), kp, vp, ks, vs, _i32([pages]).cuda(), _i32([n]).cuda(), 6 * P)
    _check_attn(B, (q, small[0][0], small[1][0], small[0][1], small[1][1], _i32([list(range(6))]), _i32([n]), 6 * P), got=got)


def test_calls_of_two_streams_at_once(B):
    """Attention with and without a second kernel and sampling, under way on two streams at a time: the results of one at a time."""
    cases = [_attn_case(40, 1, 8, 8, 64, 16, [100 + 13 * i for i in range(40)], "int8", "fp16", 85), _attn_case(1, 1, 8, 2, 128, 64, [5000], "e4m3", "fp16", 86)]
    dev = [[t.cuda() for t in c[:7]] + [c[7]] for c in cases]
    x = [torch.randn(n, 33000, generator=_gen(87 + n)).cuda() for n in (3, 200)]
    u = [torch.rand(t.shape[0], generator=_gen(89)).cuda() for t in x]
    top = [torch.full((t.shape[0],), 0.9, device="cuda") for t in x]
    want = [(B.es_op_decode_attention_kv8(*d), B.es_op_sample(y, r, top_p=p)) for d, y, r, p in zip(dev, x, u, top)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append((B.es_op_decode_attention_kv8(*dev[i]), B.es_op_sample(x[i], u[i], top_p=top[i])))
    torch.cuda.synchronize()
    for w, all_got in zip(want, got):
        for a, (t, lp) in all_got:
            assert torch.equal(a, w[0]) and torch.equal(t, w[1][0]) and torch.equal(lp, w[1][1])


@pytest.mark.parametrize("captured", [False, True])
def test_calls_wait_for_what_another_stream_made(B, captured):
    """Every call follows one of its own kind on its stream and an event of another stream, on which its input is still being
    made: called one by one and as a captured fork and join."""
    case = _attn_case(3, 1, 8, 2, 128, 64, [900, 40, 3000], "int8", "fp16", 93)
    dev = [t.cuda() for t in case[:7]]
    n = 3000
    fresh = [t.clone() for t in dev]
    rows = torch.randn(64, 2, 128, generator=_gen(94)).half().cuda()
    logits, u = torch.randn(5, 40000, generator=_gen(95)).cuda(), torch.rand(5, generator=_gen(96)).cuda()
    slots, lens, table = _i32(list(range(64, 128))).cuda(), _i32([5, 6]).cuda(), _i32([[0], [1]]).cuda()
    slow, pages = torch.zeros(64 << 20, device="cuda"), [torch.zeros_like(dev[1][:3]) for _ in range(2)]
    scales = [torch.zeros_like(dev[3][:3]) for _ in range(2)]
    made = [torch.zeros_like(t) for t in (dev[0], rows, logits, lens)]

    def work():
        main, side = torch.cuda.current_stream(), torch.cuda.Stream()
        out = []
        for i, call in enumerate((lambda x: B.es_op_decode_attention_kv8(x, *dev[1:], n), lambda x: B.es_op_kv8_append(x, x, slots, *pages, *scales),
                                  lambda x: B.es_op_sample(x, u), lambda x: B.es_op_kv_plan(x, x + 3, table, 16, 8, n_pages=2))):
            source = (fresh[0], rows, logits, lens)[i]
            side.wait_stream(main)
            with torch.cuda.stream(side):
                for _ in range(8):
                    slow.add_(1.0)
                made[i].copy_(source)
            call(source)
            main.wait_stream(side)
            out.append(call(made[i]))
        out.append(B.es_op_kv8_gather(slots, *pages, *scales))
        for _ in range(4):
            slow.add_(1.0)
        return out

    flat = lambda out: [t for o in out if o is not None for t in ((o,) if torch.is_tensor(o) else o)]  # noqa: E731
    for t in made:
        t.zero_()
    want = flat(work())                                 # warm; every call here is made on equal inputs, so its result is what counts
    torch.cuda.synchronize()
    want = [t.clone() for t in want]
    assert torch.equal(want[0], B.es_op_decode_attention_kv8(*dev, n)) and torch.equal(want[1], B.es_op_sample(logits, u)[0])
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = flat(work())
    for _ in range(5):
        for t in made:
            t.zero_()
        if captured:
            graph.replay()
        else:
            got = flat(work())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---- a run of them together --------------------------------------------------------------------------------------

class _Loop:
    """A small server over the operations: Bn requests, one layer of Hkv heads, token rows out of an embedding."""

    def __init__(self, B, code, Bn=5, Hq=4, Hkv=2, hd=64, P=16, pps=8, V=700, seed=3, device="cuda"):
        g = _gen(seed)
        self.B, self.Hq, self.Hkv, self.hd, self.P, self.pps, self.V, self.Bn = B, Hq, Hkv, hd, P, pps, V, Bn
        self.n_pages = Bn * pps - 3
        self.table = torch.full((Bn, pps), -1, dtype=torch.int32, device=device)
        self.free = torch.randperm(self.n_pages, generator=g).int().to(device)
        self.count = _i32([self.n_pages]).to(device)
        self.length = torch.zeros(Bn, dtype=torch.int32, device=device)
        shape = (self.n_pages, Hkv, P, hd)
        self.kp, self.vp = (torch.full(shape, 0x55, dtype=torch.int8, device=device).view(CODES[code]) for _ in range(2))
        self.ks, self.vs = (torch.full(shape[:2], math.nan, device=device) for _ in range(2))
        self.embed = torch.randn(V, (Hq + 2 * Hkv) * hd, generator=g).half().to(device)
        self.head = (torch.randn(V, Hq * hd, generator=g) * 0.3).half().to(device)
        self.u = torch.rand(64, Bn, generator=g).to(device)
        self.settings = [t.to(device) for t in (torch.full((Bn,), 0.8), torch.full((Bn,), 40, dtype=torch.int32), torch.full((Bn,), 0.9), torch.full((Bn,), 0.01))]

    def step(self, tokens, new, max_rows, u, T=None):
        """Tokens (packed rows) enter the cache; with T their rows are queries, T a sequence, and the last ones are sampled."""
        qkv = self.embed[tokens.long()].view(-1, self.Hq + 2 * self.Hkv, self.hd)
        plan = self.B.es_op_kv_plan(self.length, new, self.table, self.P, max_rows, self.free, self.count)
        self.length.copy_(plan.len_out)
        k, v = qkv[:, self.Hq:self.Hq + self.Hkv], qkv[:, self.Hq + self.Hkv:]
        self.B.es_op_kv8_append(k, v, plan.slot_map, self.kp, self.vp, self.ks, self.vs, runs=plan.runs)
        if T is None:
            return plan, None, None
        q = qkv[:, :self.Hq].view(self.Bn, T, self.Hq, self.hd)
        att = self.B.es_op_decode_attention_kv8(q, self.kp, self.vp, self.ks, self.vs, self.table, self.length, self.P * self.pps)
        logits = self.B.es_op_linear(att[:, -1].contiguous(), self.head)
        tok, lp = self.B.es_op_sample(logits, u, *self.settings)
        return plan, att, tok


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_decode_loop_of_all_operations(B, code):
    """Prompts, decode steps, draft tokens of which some are rejected, a request that ends and one that takes its place: at
    every attention the whole cache is held against a simulation, and the tokens against the definition."""
    L = _Loop(B, code)
    P = L.P
    sim = [(c.cpu().clone(), s.cpu().clone()) for c, s in ((L.kp, L.ks), (L.vp, L.vs))]
    lens = [5, 17, 1, 40, 32]
    rng = random.Random(1)
    tokens = torch.tensor([rng.randrange(L.V) for _ in range(sum(lens))], device="cuda")
    plan, _, _ = L.step(tokens, _i32(lens).cuda(), sum(lens), None)

    def follow(plan, tokens):
        n = tokens.numel()
        slots = plan.slot_map.tolist()[:n]
        x = L.embed[tokens.long()].cpu().view(-1, L.Hq + 2 * L.Hkv, L.hd)
        for (c, s), at in zip(sim, (L.Hq, L.Hq + L.Hkv)):
            R.append(x[:, at:at + L.Hkv], slots, c, s, P)

    follow(plan, tokens)
    ids = torch.zeros(L.Bn, dtype=torch.int32, device="cuda")
    for step in range(8):
        T = 3 if step % 3 == 2 else 1
        if step == 5:                                   # request 1 ends, a new one of 20 tokens takes its place
            L.length.copy_(B.es_op_kv_plan(L.length, _i32([int(n) * (b != 1) for b, n in enumerate(L.length)]).cuda(), L.table, P, 1, L.free, L.count).len_out)
            t = torch.tensor([rng.randrange(L.V) for _ in range(20)], device="cuda")
            plan, _, _ = L.step(t, _i32([20 if b == 1 else int(n) for b, n in enumerate(L.length)]).cuda(), 20, None)
            follow(plan, t)
        tokens = ids.repeat_interleave(T) if T > 1 else ids
        plan, att, tok = L.step(tokens, L.length + T, L.Bn * T, L.u[step], T)
        follow(plan, tokens)
        for (c, s), (dc, ds) in zip(sim, ((L.kp, L.ks), (L.vp, L.vs))):
            assert torch.equal(c.view(torch.int8), dc.cpu().view(torch.int8))
            assert torch.equal(s.nan_to_num(-1.0), ds.cpu().nan_to_num(-1.0))
        q = L.embed[tokens.long()].view(-1, L.Hq + 2 * L.Hkv, L.hd)[:, :L.Hq].view(L.Bn, T, L.Hq, L.hd).cpu()
        _check_attn(B, (q, sim[0][0], sim[1][0], sim[0][1], sim[1][1], L.table.cpu(), L.length.cpu(), P * L.pps), got=att)
        logits = B.es_op_linear(att[:, -1].contiguous(), L.head).cpu()
        want = [R.sample(logits[b], float(L.u[step, b]), float(torch.tensor(0.8)), 40, float(torch.tensor(0.9)), float(torch.tensor(0.01)))[0] for b in range(L.Bn)]
        assert tok.tolist() == want
        ids = tok
        if T > 1:                                       # the last two draft tokens are rejected
            L.length.copy_(B.es_op_kv_plan(L.length, L.length - 2, L.table, P, 1, L.free, L.count).len_out)
    assert int(L.count) == L.n_pages - sum(-(-int(n) // P) for n in L.length)


def test_decode_loop_as_a_replayed_graph(B):
    """One step captured on a side stream and replayed, against the same steps called one by one: the same bits."""
    plain, graphed = _Loop(B, "int8", pps=16), _Loop(B, "int8", pps=16)
    prompt = torch.arange(5 * 7, device="cuda") % plain.V
    ids = []
    for L in (plain, graphed):
        L.step(prompt, _i32([7] * 5).cuda(), 35, None)
    tok = torch.zeros(5, dtype=torch.int32, device="cuda")
    for i in range(12):
        _, att, tok = plain.step(tok, plain.length + 1, 5, plain.u[i], 1)
        ids.append((tok.tolist(), att.clone()))
    L = graphed
    tok, u = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(5, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    state = [t.clone() for t in (L.table, L.free, L.count, L.length, L.kp.view(torch.int8), L.vp.view(torch.int8), L.ks, L.vs)]
    with torch.cuda.stream(side):
        L.step(tok, L.length + 1, 5, u, 1)
    torch.cuda.current_stream().wait_stream(side)
    for t, s in zip((L.table, L.free, L.count, L.length, L.kp.view(torch.int8), L.vp.view(torch.int8), L.ks, L.vs), state):
        t.copy_(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, att, out = L.step(tok, L.length + 1, 5, u, 1)
        tok.copy_(out)
    for i in range(12):
        u.copy_(L.u[i])
        graph.replay()
        assert tok.tolist() == ids[i][0]
        assert torch.equal(att, ids[i][1])


def test_calls_on_another_stream(B):
    """Inputs made on a stream of the caller's, calls given that stream, memory of the results and the scratch from it."""
    case = _attn_case(1, 1, 8, 2, 128, 64, [5000], "int8", "fp16", 67)
    dev = [t.cuda() for t in case[:7]]
    want = B.es_op_decode_attention_kv8(*dev, case[7])
    tokens = B.es_op_sample(want.float()[:, 0], torch.tensor([0.5], device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        with torch.cuda.stream(side):
            q = dev[0] * 1.0
        got = B.es_op_decode_attention_kv8(q, *dev[1:], case[7], stream=side)
        with torch.cuda.stream(side):
            x = got.float()[:, 0]
            u = torch.full((1,), 0.5, device="cuda")
        t = B.es_op_sample(x, u, stream=side)
        side.synchronize()
        assert torch.equal(got, want) and torch.equal(t[0], tokens[0])
        torch.empty(1 << 20, device="cuda").fill_(math.nan)     # what the default stream's allocations write must not be theirs

"""Decode attention over shared prefixes: against a plain form in 64 bits, at the sizes and masks where it can go wrong."""
import pytest
import torch

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def B():
    from paper_2405_14371_b200 import binding
    torch.cuda.set_device(0)
    return binding


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def setup(prefixes, begin, ctx, T=1, Hq=8, Hkv=2, hd=128, P=64, dtype=F16, seed=0, spare=2):
    """Random pages in a random order for prefixes and sequences of these lengths; what no key lies in is not a number."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    used = [-(-n // P) for n in list(prefixes) + list(ctx)]
    n_pages = sum(used) + spare
    order = torch.randperm(n_pages, generator=g, device="cuda").tolist()
    k = torch.randn(n_pages, Hkv, P, hd, generator=g, device="cuda").to(dtype)
    v = torch.randn(n_pages, Hkv, P, hd, generator=g, device="cuda").to(dtype)
    free = torch.ones(n_pages, P, dtype=torch.bool, device="cuda")
    rows, at = [], 0
    for n, m in zip(list(prefixes) + list(ctx), used):
        row = order[at:at + m]
        at += m
        for j, page in enumerate(row):
            free[page, : max(0, min(P, n - j * P))] = False
        rows.append(row)
    for t in (k, v):
        t.transpose(1, 2)[free] = float("nan")
    np_ = len(prefixes)

    def table(rs):
        w = max([1] + [len(r) for r in rs])
        return i32([r + [-1] * (w - len(r)) for r in rs])

    q = (torch.randn(len(ctx), T, Hq, hd, generator=g, device="cuda") * 1.5).to(dtype)
    s = dict(q=q, k=k, v=v, pt=table(rows[:np_]) if np_ else None, pl=i32(list(prefixes)) if np_ else None, begin=i32(begin) if np_ else None,
             table=table(rows[np_:]), ctx=i32(list(ctx)), max_prefix=max([1] + list(prefixes)), max_ctx=max([1] + list(ctx)))
    return s


def call(B, s, **kw):
    return B.es_op_decode_attention_prefix(s["q"], s["k"], s["v"], s["pt"], s["pl"], s["begin"], s["table"], s["ctx"], s["max_prefix"], s["max_ctx"], **kw)


def check(B, s, got=None):
    got = call(B, s) if got is None else got
    out, size = ref.shared(s["q"], s["k"], s["v"], s["pt"], s["pl"], s["begin"], s["table"], s["ctx"])
    off = (got.double().view(out.shape) - out).abs()
    bound = ref.shared_bound(s["q"], s["k"], out, size)
    assert bool((off <= bound).all()), (float(off.max()), float((off / bound.clamp(min=1e-300)).max()))


@pytest.mark.parametrize("dtype,hd", [(F16, 128), (BF16, 128), (F16, 64), (BF16, 64)])
@pytest.mark.parametrize("prefix,ctx", [(1, [1]), (63, [1, 64]), (64, [65, 5]), (65, [128, 1, 63]), (200, [7] * 5), (1000, [1, 300, 64, 129])])
def test_one_prefix(B, prefix, ctx, dtype, hd):
    check(B, setup([prefix], [0, len(ctx)], ctx, dtype=dtype, hd=hd, seed=prefix))


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 7), (10, 2), (64, 8), (40, 40), (48, 1), (128, 1)])
def test_heads_and_pages(B, Hq, Hkv, P):
    check(B, setup([333, 50, 129], [0, 3, 4, 9], [3, 64, 200, 1, 17, 80, 33, 65, 2, 130], Hq=Hq, Hkv=Hkv, P=P, seed=Hq))


@pytest.mark.parametrize("T,Hq,Hkv", [(2, 8, 2), (5, 40, 8), (4, 6, 6), (70, 4, 2), (33, 16, 2)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_several_tokens(B, T, Hq, Hkv, dtype):
    check(B, setup([100, 257], [1, 4, 6], [T, T + 1, T + 63, T + 64, 200 + T, T, T + 5], T=T, Hq=Hq, Hkv=Hkv, dtype=dtype, P=32, seed=T))


def test_no_prefixes(B):
    check(B, setup([], None, [1, 500, 64, 3], Hq=16, Hkv=4))


def test_many_sequences(B):
    check(B, setup([700, 1, 64], [0, 100, 101, 150], [1 + 7 * i % 90 for i in range(160)], Hq=8, Hkv=1, P=16, seed=2))


def test_long_prefix(B):
    check(B, setup([20000], [0, 40], [1 + i for i in range(40)], Hq=16, Hkv=2, dtype=BF16, seed=3))


def test_rows_that_see_nothing_or_only_one_side(B):
    s = setup([100, 64], [0, 2, 4], [5, 1, 1, 70, 9], T=3, seed=4)
    s["ctx"] = i32([5, 0, -7, 70, 0])                  # fewer own keys than tokens; none; a length that is none
    s["pl"] = i32([100, 0])
    got = call(B, s)
    s["ctx"] = i32([5, 0, 0, 70, 0])
    check(B, s, got)
    assert bool((got[2] == 0).all()) and bool((got[4] == 0).all()) and not bool((got[1] == 0).all())


def test_lengths_above_the_caps_and_groups_out_of_order(B):
    s = setup([90, 90, 90], [0, 2, 4, 6], [40] * 6, seed=5)
    s["max_prefix"], s["max_ctx"] = 70, 30
    s["pl"], s["ctx"] = i32([2 ** 31 - 1, 90, 71]), i32([40, 2 ** 31 - 1, 31, 30, 29, 40])
    s["begin"] = i32([1, 4, 2, 2 ** 31 - 1])           # sequences 1-3, none, 4-5
    got = call(B, s)
    s["pl"], s["ctx"], s["begin"] = i32([70, 70, 70]), i32([30, 30, 30, 30, 29, 30]), i32([1, 4, 4, 6])
    check(B, s, got)
    s["begin"] = i32([-3, -1, 7, 2])                   # nobody, everybody, nobody
    got = call(B, s)
    s["begin"] = i32([0, 0, 6, 6])
    check(B, s, got)


def test_pages_that_do_not_exist(B):
    s = setup([200], [0, 2], [150, 40, 100], P=16, seed=6)
    s["pt"][0, 3], s["pt"][0, 0], s["table"][0, 5], s["table"][2, 0], s["table"][1] = -1, 10 ** 6, 2 ** 31 - 1, -5, -1
    check(B, s)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_later_draft_tokens_do_not_reach_earlier_queries(B, dtype):
    s = setup([70], [0, 3], [3, 66, 130], T=3, Hq=4, Hkv=2, dtype=dtype, P=64, seed=7)
    clean = call(B, s)
    for b, key in ((0, 2), (1, 65), (2, 129)):         # each sequence's newest token: no number in V, or in K
        page, off = int(s["table"][b, key // 64]), key % 64
        s["v" if b < 2 else "k"][page, 1, off, 5 + b] = float("inf") if b == 0 else float("nan")
    got = call(B, s)
    assert torch.equal(got[:, :2], clean[:, :2])
    new, old = got[:, 2].view(3, 4, 128), clean[:, 2].view(3, 4, 128)
    assert torch.equal(new[:, :2], old[:, :2])         # the other KV head's queries
    assert bool(torch.isinf(new[0, 2:, 5]).all()) and bool(torch.isnan(new[1, 2:, 6]).all()) and bool(torch.isnan(new[2, 2:]).all())
    rest = torch.ones(128, dtype=torch.bool, device="cuda")
    rest[5] = rest[6] = False
    assert torch.equal(new[:2, 2:][..., rest], old[:2, 2:][..., rest])


def test_a_value_that_is_no_number_in_the_prefix_reaches_its_group_alone(B):
    s = setup([70, 70], [0, 2, 4], [5] * 4, seed=8)
    clean = call(B, s)
    s["v"][int(s["pt"][0, 0]), 0, 3, 9] = float("nan")
    got = call(B, s)
    bad = torch.isnan(got.view(4, 8, 128))
    assert bool(bad[:2, :4, 9].all()) and int(bad.sum()) == 8 and torch.equal(got[2:], clean[2:])


def test_large_scores_and_far_apart_maxima(B):
    s = setup([300], [0, 3], [90, 1, 64], seed=9)
    s["q"] *= 12
    s["k"].nan_to_num_(0.0)
    s["k"][int(s["table"][0, 0]), :, 10] *= 4
    check(B, s)


def test_spaced_queries_given_memory_and_no_write_beside_it(B):
    s = setup([130], [0, 3], [9, 70, 4], T=2, Hq=8, Hkv=2, seed=10)
    wide = torch.zeros(3, 2, 20, 128, dtype=F16, device="cuda")
    wide[:, :, 4:12] = s["q"]
    s["q"] = wide[:, :, 4:12]
    out = torch.full((5, 2, 1024), 3.0, dtype=F16, device="cuda")
    scratch = torch.full((B.es_op_decode_attention_prefix_scratch_bytes(1, 3, 2, 8, 2, 128) + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    got = call(B, s, out=out[1:4], scratch=scratch[:-512])
    check(B, s, got)
    assert bool((out[0] == 3).all()) and bool((out[4] == 3).all()) and bool((scratch[-512:] == 0xFF).all())


def test_three_dimensions_and_same_bits(B):
    s = setup([900], [0, 8], [100] * 8, Hq=64, Hkv=8, seed=11)
    s["q"] = s["q"][:, 0]
    first = call(B, s)
    assert first.shape == (8, 64 * 128)
    for _ in range(5):
        assert torch.equal(first, call(B, s))


def test_agrees_with_the_attention_without_prefixes(B):
    """The same keys as one sequence's own: the framework's decode attention of the whole context."""
    s = setup([128], [0, 2], [40, 70], Hq=8, Hkv=2, seed=12)
    whole = torch.cat([s["pt"].expand(2, 2), s["table"]], dim=1).contiguous()
    s["k"].nan_to_num_(0.0)
    s["v"].nan_to_num_(0.0)
    one = B.es_op_decode_attention(s["q"][:, 0].contiguous(), s["k"], s["v"], whole.clamp(min=0), s["ctx"] + 128, 256)
    two = call(B, s)[:, 0]
    assert float((one.float() - two.float()).abs().max()) <= 4 * 2.0 ** -11 * 4      # two roundings each of values below 4

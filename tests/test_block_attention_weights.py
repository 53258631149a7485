"""Decode attention over shared prefixes: the weights that meet V hold more bits than q's type, however the row's sums come out.

The keys of these cases come in pairs with opposite V, under scores that are nearly equal: what a row adds up to is small
against its terms, so that a weight rounded to 8 or 11 bits shows far above the rounding of the result."""
import math

import pytest
import torch

from tests import block_reference as ref

F16, BF16 = torch.float16, torch.bfloat16


def bound(q, k, v, n, out, size):
    """n keys.  A score is a sum of hd products in fp32, scaled and brought to its exponent with a rounding each, by a function
    good to 2^-22; a weight is the sum of two numbers of q's type, each rounded (half a step of half a step), and below their
    normal range good to 2^-32 of the row's largest; sums are fp32, two products of 16 keys a step, each a unit in the last place.
    A weight's error counts twice, in its product and in the sum that it is divided by.  One rounding of the result."""
    dtype, hd = q.dtype, q.shape[-1]
    largest = q.double().norm(dim=-1).max() * k.double().norm(dim=-1).max() / math.sqrt(hd)
    score = float(largest) * (hd * 2.0 ** -24 + 2.0 ** -23)
    weight = 2 * (score + 2.0 ** -20 + ref.HALF_STEP[dtype] ** 2 + (2 * (n / 16) + 16) * 2.0 ** -23)
    return size * weight + n * 2.0 ** -32 * float(v.double().abs().max()) + out.abs() * ref.HALF_STEP[dtype] + ref.SMALLEST[dtype]


def pairs(n, rows, hd, dtype, seed, device, spread=0.02):
    """q [rows, 1, 1, hd], and n keys with values that cancel in pairs."""
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(rows, 1, 1, hd, generator=g) * spread
    k = torch.randn(n, hd, generator=g)
    v = 1 + torch.rand(n, hd, generator=g)
    v[1::2] = -v[: n - 1: 2]
    return [t.to(dtype).to(device) for t in (q, k, v)]


def plain(q, k, v, round_to=None):
    """(result, sum of the terms' magnitudes) in 64 bits, the weights rounded on the way if asked for."""
    s = torch.einsum("bthd,nd->bthn", q.double(), k.double()) / math.sqrt(q.shape[-1])
    w = torch.exp(s - s.amax(-1, keepdim=True))
    if round_to:
        w = w.to(round_to).double()
    w = w / w.sum(-1, keepdim=True)
    return torch.einsum("bthn,nd->bthd", w, v.double()), torch.einsum("bthn,nd->bthd", w, v.double().abs())


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_the_bound_tells_rounded_weights(dtype):
    """Weights rounded to q's type, planted in the plain form, are outside of what is allowed."""
    q, k, v = pairs(40, 30, 64, dtype, 1, "cpu")
    out, size = plain(q, k, v)
    wrong, _ = plain(q, k, v, dtype)
    assert bool(((wrong - out).abs() > bound(q, k, v, 40, out, size)).any())
    assert bool((out.to(dtype).double() - out).abs().le(bound(q, k, v, 40, out, size)).all())


def paged(k, v, prefix, P=16):
    """The first `prefix` keys as a shared prefix, the others as every sequence's own."""
    n, hd = k.shape
    parts = [(0, prefix), (prefix, n)]
    used = [-(-(b - a) // P) for a, b in parts]
    kp, vp = (torch.zeros(sum(used), 1, P, hd, dtype=k.dtype, device=k.device) for _ in range(2))
    at, rows = 0, []
    for (a, b), m in zip(parts, used):
        kp[at:at + m].view(-1, hd)[: b - a], vp[at:at + m].view(-1, hd)[: b - a] = k[a:b], v[a:b]
        rows.append(torch.arange(at, at + m, dtype=torch.int32, device=k.device))
        at += m
    return kp, vp, rows


def attend(q, k, v, prefix):
    from paper_2405_14371_b200 import binding as B
    torch.cuda.set_device(0)
    kp, vp, (front, own) = paged(k, v, prefix)
    n, rows = len(k), len(q)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    groups = (front[None], i32([prefix]), i32([0, rows])) if prefix else (None, None, None)
    got = B.es_op_decode_attention_prefix(q, kp, vp, *groups, own.expand(rows, -1).contiguous(), i32([n - prefix] * rows), max(1, prefix), n - prefix)
    return got.double().view(q.shape)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,prefix", [(2, 0), (7, 0), (40, 24), (40, 39), (200, 128), (200, 70)])
def test_weights_keep_their_bits(n, prefix, hd, dtype):
    q, k, v = pairs(n, 150, hd, dtype, n + hd, "cuda")
    out, size = plain(q, k, v)
    off = (attend(q, k, v, prefix) - out).abs()
    limit = bound(q, k, v, n, out, size)
    assert bool((off <= limit).all()), float((off / limit).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("prefix", [0, 64, 3000])
def test_many_small_weights_beside_a_large_one(prefix, dtype):
    """One key takes nearly all of the weight and has a value near zero; each of the others weighs less than 2^-25 of it."""
    n, hd = 4000, 64
    g = torch.Generator().manual_seed(3)
    q = torch.zeros(20, 1, 1, hd)
    q[..., 0] = 8.0
    k = torch.zeros(n, hd)
    k[:, 0] = -17.5 + 0.25 * torch.rand(n, generator=g)          # exponents of about -25.3 (base 2)
    k[5, 0] = 0.0
    v = 1000 * (0.5 + torch.rand(n, hd, generator=g))
    v[5] = 0.001
    q, k, v = [t.to(dtype).cuda() for t in (q, k, v)]
    out, size = plain(q, k, v)
    off = (attend(q, k, v, prefix) - out).abs()
    limit = bound(q, k, v, n, out, size)
    assert bool((limit < 0.1 * out).all())
    assert bool((off <= limit).all()), float((off / limit).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("prefix", [0, 100])
def test_infinities_that_a_row_sees_reach_it_as_infinities(prefix, dtype):
    """Whatever their weights are: also where a weight is a number of q's type exactly, or so small (2^-60) that it has none."""
    n, hd = 164, 64
    q, k, v = pairs(n, 30, hd, dtype, 4, "cuda", spread=1.5)
    clean = attend(q, k, v, prefix)
    for key, col, value in ((3, 1, math.inf), (70, 2, -math.inf), (99, 3, math.inf), (101, 4, math.nan), (163, 5, -math.inf), (3, 6, math.inf), (160, 6, -math.inf)):
        v[key, col] = value
    k[70] = -2.2 * q[0, 0, 0]                                     # about 2^-60 of row 0
    got = attend(q, k, v, prefix).view(30, hd)
    for col, value in ((1, math.inf), (2, -math.inf), (3, math.inf), (5, -math.inf)):
        assert bool((got[:, col] == value).all()), col
    assert bool(torch.isnan(got[:, [4, 6]]).all())
    rest = [c for c in range(hd) if c not in range(1, 7)]
    assert bool(torch.isfinite(got[:, rest]).all()) and bool(torch.isfinite(clean).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("prefix", [0, 70])
@pytest.mark.parametrize("large", [2.0 ** 9, 2.0 ** 12, 2.0 ** 14, 2.0 ** 15])
def test_scores_whose_own_steps_are_large(prefix, large, dtype):
    """Scores of 2^21 to 2^33, which fp32 holds in steps of 1/4 to 2^10: no weight is larger than the largest key's by more than
    such a step makes it, so every result is finite and lies among the values."""
    n, hd = 200, 64
    g = torch.Generator().manual_seed(5)
    q = large * (1 + 0.01 * torch.rand(40, 1, 1, hd, generator=g))
    k = large * (1 + 0.001 * torch.rand(n, hd, generator=g))
    v = 1 + torch.rand(n, hd, generator=g)
    q, k, v = [t.to(dtype).cuda() for t in (q, k, v)]
    got = attend(q, k, v, prefix)
    assert bool(torch.isfinite(got).all()) and float(got.min()) >= 1 - 2 * ref.HALF_STEP[dtype] and float(got.max()) <= 2 + 4 * ref.HALF_STEP[dtype]

"""Decode attention over shared prefixes: draft tokens with values that are no numbers, in one short item after another."""
import pytest
import torch

from tests.test_block_attention_gpu import B, call, i32, setup  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prefixes", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (32, 4)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_every_item_has_a_broken_draft_token(B, dtype, Hq, Hkv, prefixes):  # noqa: F811
    """About twenty items follow one another in a stretch, and the newest tokens of every one hold an infinity and, of every
    third, a NaN, in all KV heads: each reaches the rows that see it, of its own sequence, and no others."""
    n, T, hd = 1500, 3, 64
    ctx = [3 + b % 38 for b in range(n)]
    s = setup([30, 70] if prefixes else [], [100, 600, 900] if prefixes else None, ctx, T=T, Hq=Hq, Hkv=Hkv, hd=hd, P=16, dtype=dtype, seed=1)
    clean = call(B, s).view(n, T, Hq, hd)
    assert bool(torch.isfinite(clean).all())
    b = torch.arange(n, device="cuda")
    inf, nan = b % hd, (b * 7 + 1) % hd                  # never the same column: 6 b + 1 is odd
    where = i32(ctx).long()
    third = b[b % 3 == 0]
    for seq, back, col, value in ((b, 1, inf, float("inf")), (third, 2, nan[third], float("nan"))):
        key = where[seq] - back
        s["v"][s["table"][seq, key // 16].long(), :, key % 16, col] = value
    want = clean.clone()
    want[b, T - 1, :, inf] = float("inf")
    for t in (T - 2, T - 1):
        want[third, t, :, nan[third]] = float("nan")
    for _ in range(20):
        got = call(B, s).view(n, T, Hq, hd)
        same = (got == want) | (torch.isnan(got) & torch.isnan(want))
        assert bool(same.all()), int((~same).sum())

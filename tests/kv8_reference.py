"""Plain 64-bit forms of the operations over the paged 8-bit cache, request by request, for the tests only."""
from __future__ import annotations

import math

import torch

FLOOR = 2.0 ** -100
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}       # half the smallest step


def plan(old, new, table, free, n_free, P, max_rows, n_pages=None):
    """Lists in, a dict of lists out; table, free are changed in place.  free None: the table is taken as it is."""
    B, pps = len(old), len(table[0])
    cap = pps * P
    alloc = free is not None
    n_pages = len(free) if alloc else n_pages
    up = lambda n: -(-n // P)  # noqa: E731
    ok = [0 <= o <= cap and 0 <= n <= cap for o, n in zip(old, new)]
    if alloc:
        for b in range(B):
            if ok[b]:
                for j in range(up(new[b]), up(old[b])):
                    free[n_free] = table[b][j]
                    n_free += 1
                    table[b][j] = -1
    rows_sum = need_sum = 0
    avail = n_free
    out = {k: [] for k in ("slot_map", "positions", "row_seq", "runs", "len_out")}
    out["row_offsets"] = [0]
    for b in range(B):
        o, n = old[b], new[b]
        gain = max(0, n - o) if ok[b] else 0
        need = max(0, up(n) - up(o)) if ok[b] else 0
        rows_sum += gain
        need_sum += need
        served = gain == 0 or (rows_sum <= max_rows and (not alloc or need == 0 or need_sum <= avail))
        if gain and served and alloc:
            for j in range(up(o), up(n)):
                n_free -= 1
                table[b][j] = free[n_free]
        for pos in range(o, o + gain):
            if len(out["slot_map"]) == max_rows:
                break
            page = table[b][pos // P]
            there = served and 0 <= page < n_pages
            if served and (pos == o or pos % P == 0):
                out["runs"].append(len(out["slot_map"]) if there else -1)
            out["slot_map"].append(page * P + pos % P if there else -1)
            out["positions"].append(pos)
            out["row_seq"].append(b)
        out["row_offsets"].append(min(rows_sum, max_rows))
        out["len_out"].append(n if ok[b] and served else o)
    for k in ("slot_map", "positions", "row_seq"):
        out[k] += [-1] * (max_rows - len(out[k]))
    out["runs"] += [-1] * (min(max_rows, max_rows // P + 2 * B) - len(out["runs"]))
    out["free_count"] = n_free
    return out


def round_e4m3(x):
    """Nearest e4m3 number, ties to even, saturating; x in fp64."""
    a = x.abs()
    step = torch.ldexp(torch.ones_like(a), (torch.frexp(a)[1] - 1).clamp(min=-6) - 3)
    return torch.sign(x) * torch.clamp(torch.round(a / step) * step, max=448.0)


def wanted_scale(big, int8):
    """fp64 tensor of largest magnitudes -> scales (fp32 numbers in fp64)."""
    if int8:
        return torch.clamp(big.float() / 127, min=FLOOR).double()
    e = torch.full_like(big, -100.0)
    for i in range(big.numel()):
        m = float(big.flatten()[i])
        k = -100
        while 448.0 * 2.0 ** k < m:
            k += 1
        e.view(-1)[i] = k
    return torch.exp2(e)


def append(x, slots, codes, scale, P):
    """x [n, Hkv, hd] fp16/bf16, slots list, codes [n_pages, Hkv, P, hd] (int8 or e4m3) and scale [n_pages, Hkv], all on the
    CPU; codes and scale are changed in place."""
    int8 = codes.dtype == torch.int8
    n_pages = codes.shape[0]
    value = codes.double() if int8 else codes.float().double()
    sc = scale.double()
    i, n = 0, x.shape[0]
    touched = set()
    while i < n:
        if not 0 <= slots[i] < n_pages * P:
            i += 1
            continue
        page, off = divmod(slots[i], P)
        j = i + 1
        while j < n and slots[j] == slots[i] + j - i and slots[j] // P == page:
            j += 1
        rows = x[i:j].double().transpose(0, 1)
        big = rows.abs().amax((1, 2))
        for h in range(x.shape[1]):
            if not math.isfinite(float(big[h])):
                s = float("nan")
            else:
                s = float(wanted_scale(big[h:h + 1], int8)[0])
                if off > 0 and (float(sc[page, h]) >= s or math.isnan(float(sc[page, h]))):
                    s = float(sc[page, h])
            if math.isnan(s):
                value[page, h, off:off + j - i] = 0
            else:
                rnd = torch.round if int8 else round_e4m3
                if off > 0 and s != float(sc[page, h]):
                    value[page, h, :off] = rnd(value[page, h, :off] * (float(sc[page, h]) / s))
                value[page, h, off:off + j - i] = rnd(rows[h] / s)
            sc[page, h] = s
        touched.add(page)
        i = j
    codes.copy_(value.to(torch.int8) if int8 else value.float().to(codes.dtype))
    scale.copy_(sc.float())
    return touched


def gather(slots, codes, scale, P, dtype):
    n_pages, Hkv, _, hd = codes.shape
    out = torch.zeros(len(slots), Hkv, hd, dtype=dtype)
    for r, s in enumerate(slots):
        if 0 <= s < n_pages * P:
            out[r] = (codes[s // P, :, s % P].float() * scale[s // P][:, None]).to(dtype)
    return out


def attend(q, kc, vc, ks, vs, table, ctx, P, max_ctx):
    """(want, bound) fp64 [B, T, Hq, hd] of q [B, T, Hq, hd] (CPU): the result and how far fp32 arithmetic and one rounding
    to q's type may take a kernel from it.

    A score is a sum of hd products in fp32, in steps of 16 (the tensor cores), each step within 2^-22 of the sum of
    magnitudes (they may cut off instead of rounding): its error is at most (hd / 16 + 4) 2^-22 A with
    A = sum |q k| / sqrt(hd), the 4 for the factors and the exponent's multiplication.  bf16 queries scaled to fp16
    lose at most 2^-24 of the row's largest an element.  exp turns an error d of a score into a factor 1 + d, it shifts
    numerator and denominator, and is itself within 2^-21: 2 (d + 2^-20) sum(p |v|) in all, with the two fp16 halves of
    a probability (2^-22) and the sums in it.  A half has no bits below 2^-24, and the probabilities of up to 64 tokens
    (a stretch of positions 64 i .. 64 i + 63 at most) are scaled so that the largest lies in (2^14, 2^15]: what is lost
    of each is below 2^-25 / 2^14 = 2^-39 of the largest.  Then the result is rounded once."""
    B, T, Hq, hd = q.shape
    Hkv, n_pages = kc.shape[1], kc.shape[0]
    G = Hq // Hkv
    want, bound = torch.zeros(B, T, Hq, hd, dtype=torch.float64), torch.zeros(B, T, Hq, hd, dtype=torch.float64)
    for b in range(B):
        n = max(0, min(int(ctx[b]), max_ctx))
        pos = [i for i in range(n) if 0 <= int(table[b, i // P]) < n_pages]
        pages = torch.tensor([int(table[b, i // P]) for i in pos], dtype=torch.long)
        offs = torch.tensor([i % P for i in pos], dtype=torch.long)
        for t in range(T):
            m = sum(1 for i in pos if i < n - T + t + 1)
            if m == 0:
                continue
            pg, of = pages[:m], offs[:m]
            for h in range(Hkv):
                k = kc[pg, h, of].float().double() * ks[pg, h].double()[:, None]
                v = vc[pg, h, of].float().double() * vs[pg, h].double()[:, None]
                qq = q[b, t, h * G:(h + 1) * G].double()
                s = qq @ k.T / math.sqrt(hd)
                p = torch.softmax(s, -1)
                want[b, t, h * G:(h + 1) * G] = p @ v
                A = (qq.abs() @ k.abs().T).amax(-1) / math.sqrt(hd)
                d = (hd / 16 + 4) * 2.0 ** -22 * A
                if q.dtype == torch.bfloat16:
                    d = d + 2.0 ** -24 * qq.abs().amax(-1) * float(k.abs().sum(-1).max()) / math.sqrt(hd)
                bound[b, t, h * G:(h + 1) * G] = 2 * (d[:, None] + 2.0 ** -20) * (p @ v.abs())
                group = torch.tensor([i // 64 for i in pos[:m]])
                for i in group.unique().tolist():
                    at = group == i
                    bound[b, t, h * G:(h + 1) * G] += 2.0 ** -39 * p[:, at].amax(-1, keepdim=True) * v[at].abs().sum(0)
    eps = torch.finfo(q.dtype).eps / 2
    return want, bound * (1 + eps) + eps * want.abs() + TINY[q.dtype]


def sample(x, u, T=1.0, k=0, p=1.0, m=0.0):
    """(token, log probability) of one row x (any float type, CPU)."""
    x = x.double()
    x = torch.where(torch.isnan(x), torch.tensor(-math.inf, dtype=torch.float64), x)
    V = x.numel()
    if float(x.max()) == -math.inf:
        return -1, -math.inf
    order = torch.argsort(x, descending=True, stable=True)
    if not T > 0:
        return int(order[0]), 0.0
    top = x[order[0]]
    w = torch.where(x == top, torch.ones_like(x), torch.exp((x - top) / T))[order]
    if 0 < k < V:
        order, w = order[:k], w[:k]
    if p < 1:
        n = 1
        total = float(w.sum())
        run = w.cumsum(0)
        while n < len(order) and float(run[n - 1]) < p * total:
            n += 1
        order, w = order[:n], w[:n]
    if m > 0:
        n = max(1, int((w >= min(m, 1.0)).sum()))
        order, w = order[:n], w[:n]
    order, by = torch.sort(order)
    w = w[by]
    run = w.cumsum(0)
    over = (run > min(max(u, 0.0), 1.0) * float(run[-1])).nonzero()
    i = int(over[0]) if len(over) else int((w > 0).nonzero()[-1])
    return int(order[i]), math.log(float(w[i]) / float(run[-1]))

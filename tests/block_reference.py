"""Plain forms in 64 bits of the operators of an attention block: e4m3 codes and products, heads, attention over a shared prefix."""
import math

import torch

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # of a rounding, relative
SMALLEST = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0, torch.float32: 0.0}                       # of a rounding below the normal range


def blocks_of(x, rows):
    """x [M, K] in blocks [row blocks, rows, column blocks, 128], zeros behind its ends."""
    M, K = x.shape
    m, k = -(-M // rows), -(-K // 128)
    return torch.nn.functional.pad(x, (0, k * 128 - K, 0, m * rows - M)).view(m, rows, k, 128)


def quant(x, rows):
    """(codes, scale [row blocks, column blocks]): the scale in fp32 arithmetic, the codes of the exact quotient."""
    b = blocks_of(x.float(), rows)
    top = b.abs().amax(dim=(1, 3))
    scale = (top * torch.tensor(1.0 / 448.0, dtype=torch.float32, device=x.device)).clamp(min=2.0 ** -100)
    scale = torch.where(torch.isfinite(top), scale, math.nan)
    q = (b.double() / scale.double()[:, None, :, None]).float()
    return q.reshape(b.shape[0] * rows, -1)[: x.shape[0], : x.shape[1]].to(torch.float8_e4m3fn), scale


def spread(scale, rows, M, K):
    """A scale for every element."""
    return scale.double().repeat_interleave(rows, 0)[:M].repeat_interleave(128, 1)[:, :K]


def linear(a, a_scale, w, w_scale, r=None):
    """(product, sum of the terms' magnitudes); a_scale [K blocks, M]."""
    x = a.double() * spread(a_scale.t(), 1, *a.shape)
    y = w.double() * spread(w_scale, 128, *w.shape)
    c, s = x @ y.t(), x.abs() @ y.abs().t()
    return (c, s) if r is None else (c + r.double(), s + r.double().abs())


def linear_bound(c, s, K, dtype):
    """Products of codes are exact; a block's sum is 4 additions in the tensor cores to fp32 (a unit in the last place of the
    sum of magnitudes each, at most), its scale a product (half a unit), its way into the result one more addition; up to
    8 ranges and a residual are added; one rounding of the result."""
    n = -(-K // 128)
    return s * (4 + n + 2 + 9) * 2.0 ** -23 + c.abs() * HALF_STEP[dtype] + SMALLEST[dtype]


def heads(x, gain, eps, cosines, sines, positions, halves):
    """(rotated heads, magnitudes that met in each value)."""
    y = x.double()
    if gain is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * gain.double()
    half = cosines.shape[1]
    first = torch.arange(half, device=x.device) * (1 if halves else 2)
    second = first + (half if halves else 1)
    ok = (positions >= 0) & (positions < len(cosines))
    at = torch.where(ok, positions, 0).long()
    c, s = cosines.double()[at][:, None], sines.double()[at][:, None]
    out, size = y.clone(), y.abs()
    out[..., first] = y[..., first] * c - y[..., second] * s
    out[..., second] = y[..., second] * c + y[..., first] * s
    size[..., first] = size[..., second] = y[..., first].abs() + y[..., second].abs()
    return torch.where(ok[:, None, None], out, 0.0), size


def heads_bound(out, size, hd, dtype):
    """Squares: hd / 8 + 5 additions, a root (2 units), 3 products and the rotation's 3 roundings, all fp32; one rounding."""
    return size * (hd / 8 + 5 + 2 + 6) * 2.0 ** -24 + out.abs() * HALF_STEP[dtype] + SMALLEST[dtype]


def shared(q, k_pages, v_pages, prefix_table, prefix_len, begin, table, ctx):
    """(attention [B, T, Hq, hd], sum over the keys of weight times |v|): query t of a sequence sees its prefix and own keys
    0 .. ctx - T + t; pages that do not exist hold nothing.  `begin` is taken as it is given (in order)."""
    B, T, Hq, hd = q.shape
    n_pages, Hkv, P, _ = k_pages.shape
    out = torch.zeros(B, T, Hq, hd, dtype=torch.float64, device=q.device)
    size = torch.zeros_like(out)

    def keys(row, n):
        """Pages and offsets of the first n keys of a table's row that lie in pages that exist."""
        at = torch.arange(n, device=q.device)
        page = row.long()[at // P]
        ok = (page >= 0) & (page < n_pages)
        return page[ok], at[ok] % P, at[ok]

    for b in range(B):
        group = next((g for g in range(len(prefix_len)) if int(begin[g]) <= b < int(begin[g + 1])), None) if prefix_len is not None else None
        mine = keys(table[b], int(ctx[b]))
        front = (torch.empty(0, dtype=torch.long, device=q.device),) * 2 if group is None else keys(prefix_table[group], int(prefix_len[group]))[:2]
        for t in range(T):
            see = mine[2] <= int(ctx[b]) - T + t
            page, off = torch.cat([front[0], mine[0][see]]), torch.cat([front[1], mine[1][see]])
            if len(page) == 0:
                continue
            k, v = k_pages[page, :, off].double(), v_pages[page, :, off].double()
            w = torch.softmax(torch.einsum("hgd,nhd->hgn", q[b, t].double().view(Hkv, -1, hd), k) / math.sqrt(hd), -1)
            out[b, t] = torch.einsum("hgn,nhd->hgd", w, v).reshape(Hq, hd)
            size[b, t] = torch.einsum("hgn,nhd->hgd", w, v.abs()).reshape(Hq, hd)
    return out, size


def shared_bound(q, k_pages, out, size):
    """A score is a sum of hd products of magnitude |q||k| in fp32, its exponent in units of log2(e) / sqrt(hd) rounded once and
    taken by a function good to 2^-22; a weight is rounded to q's type in the product (half a step of it) and joins with at most
    a few fp32 roundings per tile; one rounding of the result.  The weights' common factor cancels against their sum's, so an
    error of a weight counts at most twice."""
    dtype, hd = q.dtype, q.shape[-1]
    largest = q.double().norm(dim=-1).max() * torch.nan_to_num(k_pages.double(), 0.0, 0.0, 0.0).norm(dim=-1).max() / math.sqrt(hd)
    score = float(largest) * (hd * 2.0 ** -24 + 2.0 ** -23)
    weight = 2 * (score + 2.0 ** -20) + 2 * HALF_STEP[dtype]
    return size * weight + out.abs() * HALF_STEP[dtype] + SMALLEST[dtype]

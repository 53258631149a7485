"""Cases for measuring the operators of an attention block with 8-bit weights, normalised heads and a shared prefix,
and their plain forms.

  linear  activations brought to e4m3, product with block-scaled e4m3 weights   es_op_quant_e4m3, es_op_linear_fp8
  heads   norm of every query and key head, rotation, into the cache            es_op_qk_norm_rope
  shared  attention of the newest tokens over a shared prefix and own keys      es_op_decode_attention_prefix

`own` chooses between the library's entry points and the plain form of the same definition in elementary torch
operations.  Head shapes 32/32, 40/40 and 64/8 of 128 dimensions, pages of 64 tokens and the matrices' sizes of the
7B, 13B and 70B layers are those of the benchmark's configurations; the others are generic.
"""
import math

import torch

own = False

BLOCK = 128                                        # side of a block that shares a scale
LARGEST = 448.0                                    # of e4m3
FLOOR = 2.0 ** -100                                # no scale is below it
TYPE = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # one user's token through a 7B layer's fused QKV matrix
        dict(name="linear one", op="linear", M=1, N=12288, K=4096, dtype="fp16", out="fp16", residual=False),
        # a decode batch through a 70B layer's QKV matrix (64 query and 8 KV heads)
        dict(name="linear decode 16", op="linear", M=16, N=10240, K=8192, dtype="bf16", out="bf16", residual=False),
        # a short ragged chunk of prompts through a 13B layer's down projection, added to the fp32 residual stream
        dict(name="linear chunk 113", op="linear", M=113, N=5120, K=13824, dtype="fp16", out="fp32", residual=True),
        # a prompt through a projection whose sizes fill no tile
        dict(name="linear odd 777", op="linear", M=777, N=5003, K=2064, dtype="bf16", out="bf16", residual=False),
        # eight 1024-token prompts through a 70B layer's gate matrix
        dict(name="linear prompts 8192", op="linear", M=8192, N=28672, K=8192, dtype="bf16", out="bf16", residual=False),
        # one user's token: 32 heads
        dict(name="heads one", op="heads", n=1, Hq=32, Hkv=32, hd=128, rot=128, P=64, longest=4096, dtype="fp16", halves=False),
        # a decode batch with grouped heads, rotation of the first half of a head
        dict(name="heads decode 200", op="heads", n=200, Hq=64, Hkv=8, hd=128, rot=64, P=16, longest=8192, dtype="bf16", halves=True),
        # packed prompts
        dict(name="heads prompts 16000", op="heads", n=16000, Hq=64, Hkv=8, hd=128, rot=128, P=64, longest=8192, dtype="bf16", halves=True),
        # four samples of one prompt
        dict(name="shared 4 samples", op="shared", B=4, T=1, Hq=32, Hkv=32, hd=128, P=64, groups=1, alone=0, prefix=1000, shortest=1, longest=90, dtype="fp16"),
        # a system prompt in front of 64 chats, grouped heads
        dict(name="shared 64 chats", op="shared", B=64, T=1, Hq=64, Hkv=8, hd=128, P=64, groups=1, alone=0, prefix=4100, shortest=16, longest=600, dtype="bf16"),
        # several prefixes, four draft tokens each, some requests with no prefix
        dict(name="shared drafts", op="shared", B=40, T=4, Hq=40, Hkv=40, hd=128, P=16, groups=5, alone=3, prefix=1500, shortest=4, longest=301, dtype="fp16"),
        # many requests about one long document
        dict(name="shared 256 long", op="shared", B=256, T=1, Hq=64, Hkv=8, hd=128, P=64, groups=1, alone=0, prefix=16000, shortest=1, longest=1000, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "heads", "shared"])
    dtype = rng.choice(["fp16", "bf16"])
    if op == "linear":
        N, K = _log(rng, 60, 28000), 16 * _log(rng, 8, 800)
        M = _log(rng, 1, max(1, min(8192, int(1.8e12 / (2 * N * K)))))
        if rng.random() < 0.5:
            N = (N + 127) // 128 * 128
        out = rng.choice(["fp32", dtype])
        return dict(op=op, M=M, N=N, K=K, dtype=dtype, out=out, residual=out == "fp32" and rng.random() < 0.5)
    if op == "heads":
        Hkv, hd = rng.choice([1, 2, 5, 8, 32, 40]), rng.choice([64, 128, 128, 256])
        Hq = Hkv * rng.choice([1, 2, 4, 7, 8])
        n = _log(rng, 1, max(1, min(16000, 16000 * 80 * 128 // (hd * (Hq + 2 * Hkv)))))
        return dict(op=op, n=n, Hq=Hq, Hkv=Hkv, hd=hd, rot=rng.choice([hd, hd, hd // 2]), P=rng.choice([16, 32, 64, 128]),
                    longest=_log(rng, 64, 8192), dtype=dtype, halves=rng.random() < 0.5)
    Hkv, G, hd, T = rng.choice([1, 2, 4, 8, 32, 40]), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 128]), rng.choice([1, 1, 2, 5])
    prefix, longest = _log(rng, 16, 16000), _log(rng, T, 1000)
    cost = Hkv * G * T * (prefix + longest) + Hkv * 8 * longest
    B = _log(rng, 1, max(1, min(256, 1.2e8 / cost)))
    groups = rng.randrange(1, min(B, 8) + 1)
    return dict(op=op, B=B, T=T, Hq=Hkv * G, Hkv=Hkv, hd=hd, P=rng.choice([16, 32, 64, 128]), groups=groups, alone=rng.randrange(0, (B - groups) // 4 + 1),
                prefix=prefix, shortest=rng.randrange(T, longest + 1), longest=longest, dtype=dtype)


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed), torch.Generator().manual_seed(seed)


def _spread(n, lo, hi, hg):
    """n lengths from lo to hi in a random order, with the same sum every time."""
    return (torch.linspace(lo, hi, n) if n > 1 else torch.full((n,), float(hi))).round().long()[torch.randperm(n, generator=hg)]


def _i32(t):
    return t.to(torch.int32).cuda()


def _table(lens, P, order):
    """Block table of sequences of these lengths out of the pages in `order`; -1 where none is needed."""
    used = (lens + P - 1) // P
    table = torch.full((len(lens), max(1, int(used.max()))), -1)
    table[torch.arange(table.shape[1])[None, :] < used[:, None]] = order[: int(used.sum())]
    return table


def _shared_lens(c, hg):
    """Lengths of the prefixes, first members, lengths of the sequences' own tokens."""
    lens = _spread(c["groups"], max(1, c["prefix"] // 2), c["prefix"], hg)
    member = c["B"] - c["alone"]
    begin = torch.linspace(0, member, c["groups"] + 1).round().long()
    return lens, begin, _spread(c["B"], c["shortest"], c["longest"], hg)


def prepare(case, seed):
    c = case
    g, hg = _gen(seed)
    s = dict(c)
    dt = TYPE[c["dtype"]]
    if c["op"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        # activations behind a norm: some channels are far larger than others
        x = torch.randn(M, K, generator=g, device="cuda") * torch.exp(0.7 * torch.randn(K, generator=g, device="cuda"))
        w = torch.randn(N, K, generator=g, device="cuda") * 0.02
        nb, kb = (N + BLOCK - 1) // BLOCK, (K + BLOCK - 1) // BLOCK
        big = torch.nn.functional.pad(w, (0, kb * BLOCK - K, 0, nb * BLOCK - N)).view(nb, BLOCK, kb, BLOCK)
        scale = (big.abs().amax(dim=(1, 3)) / LARGEST).clamp(min=FLOOR)
        codes = (big / scale[:, None, :, None]).view(nb * BLOCK, kb * BLOCK)[:N, :K].to(torch.float8_e4m3fn).contiguous()
        s.update(x=x.to(dt), w=codes, ws=scale, r=torch.randn(M, N, generator=g, device="cuda") if c["residual"] else None)
    elif c["op"] == "heads":
        n, Hq, Hkv, hd, P = c["n"], c["Hq"], c["Hkv"], c["hd"], c["P"]
        qkv = torch.randn(n, Hq + 2 * Hkv, hd, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(Hq + 2 * Hkv, hd, generator=g, device="cuda"))
        qkv = qkv.to(dt)
        n_pages = (n + P - 1) // P + 3
        slots = torch.randperm(n_pages, generator=hg)[:, None] * P + torch.arange(P)
        freq = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])
        angle = torch.arange(c["longest"], dtype=torch.float64)[:, None] * freq
        pool = (n_pages, Hkv, P, hd)
        # prompts of about a thousand tokens, or the newest tokens of as many sequences
        start = torch.randint(0, c["longest"], ((n + 999) // 1000 if n > 999 else n,), generator=hg)
        step = n // len(start) if n > 999 else 1
        pos = (start.repeat_interleave(step + 1)[:n] + torch.arange(n) % max(1, step)) % c["longest"] if n > 999 else start
        s.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], slots=_i32(slots.flatten()[:n]), pos=_i32(torch.nn.functional.pad(pos, (0, n - len(pos)))),
                 qg=(1 + 0.1 * torch.randn(hd, generator=g, device="cuda")).to(dt), kg=(1 + 0.1 * torch.randn(hd, generator=g, device="cuda")).to(dt),
                 cos=angle.cos().float().cuda(), sin=angle.sin().float().cuda(), eps=1e-6,
                 kp=torch.randn(pool, generator=g, device="cuda", dtype=dt), vp=torch.randn(pool, generator=g, device="cuda", dtype=dt))
    else:
        B, P, Hkv, hd = c["B"], c["P"], c["Hkv"], c["hd"]
        lens, begin, ctx = _shared_lens(c, hg)
        both = torch.cat([lens, ctx])
        n_pages = int(((both + P - 1) // P).sum()) + 3
        order = torch.randperm(n_pages, generator=hg)
        used = int(((lens + P - 1) // P).sum())
        shape = (n_pages, Hkv, P, hd)
        q = torch.randn(B, c["T"], c["Hq"], hd, generator=g, device="cuda") * 1.5
        s.update(q=q.to(dt), kp=torch.randn(shape, generator=g, device="cuda", dtype=dt), vp=torch.randn(shape, generator=g, device="cuda", dtype=dt),
                 prefix_table=_i32(_table(lens, P, order)), prefix_len=_i32(lens), begin=_i32(begin), table=_i32(_table(ctx, P, order[used:])), ctx=_i32(ctx),
                 members=int((begin[1:] - begin[:-1]).max()))
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(state):
    return _RUN[state["op"]](state)


def _run_linear(s):
    if own:
        from paper_2405_14371_b200 import binding as b
        codes, scale = b.es_op_quant_e4m3(s["x"])
        return b.es_op_linear_fp8(codes, scale, s["w"], s["ws"], residual=s["r"], dtype=TYPE[s["out"]], weights_ready=True)
    return _linear(s["x"], s["w"], s["ws"], s["r"], TYPE[s["out"]])


def _run_heads(s):
    if own:
        from paper_2405_14371_b200 import binding as b
        q = b.es_op_qk_norm_rope(s["q"], s["k"], s["qg"], s["kg"], s["eps"], s["cos"], s["sin"], s["pos"], halves=s["halves"], v=s["v"], slot_map=s["slots"],
                                 k_pages=s["kp"], v_pages=s["vp"])
        return [q, s["kp"], s["vp"]]
    slot = s["slots"].long()
    page, at = slot // s["P"], slot % s["P"]
    s["kp"][page, :, at] = _heads(s["k"], s["kg"], s)
    s["vp"][page, :, at] = s["v"]
    return [_heads(s["q"], s["qg"], s).flatten(1), s["kp"], s["vp"]]


def _run_shared(s):
    if own:
        from paper_2405_14371_b200 import binding as b
        return b.es_op_decode_attention_prefix(s["q"], s["kp"], s["vp"], s["prefix_table"], s["prefix_len"], s["begin"], s["table"], s["ctx"], s["prefix"], s["longest"])
    return _shared(s)


_RUN = {"linear": _run_linear, "heads": _run_heads, "shared": _run_shared}


# ---- plain forms -------------------------------------------------------------------------------------------------

def _linear(x, w, ws, r, dtype):
    """Activations to codes with a scale per row and 128 columns, and the product of what the codes of both stand for."""
    M, K = x.shape
    kb = ws.shape[1]
    blocks = torch.nn.functional.pad(x.float(), (0, kb * BLOCK - K)).view(M, kb, BLOCK)
    scale = (blocks.abs().amax(dim=2, keepdim=True) / LARGEST).clamp(min=FLOOR)
    a = ((blocks / scale).to(torch.float8_e4m3fn).float() * scale).view(M, kb * BLOCK)[:, :K]
    b = w.float() * ws.repeat_interleave(BLOCK, 0)[: len(w)].repeat_interleave(BLOCK, 1)[:, :K]
    y = a @ b.t()
    return (y if r is None else y + r).to(dtype)


def _heads(x, gain, s):
    """Every head divided by its root mean square, times the gain, its first dimensions rotated by the position."""
    y = x.float()
    y = y * torch.rsqrt(y.square().mean(dim=-1, keepdim=True) + s["eps"]) * gain.float()
    pos, rot = s["pos"].long(), s["rot"]
    c, d = s["cos"][pos][:, None], s["sin"][pos][:, None]
    if s["halves"]:
        a, b = y[..., : rot // 2], y[..., rot // 2: rot]
        turned = torch.cat([a * c - b * d, b * c + a * d], dim=-1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * c - b * d, b * c + a * d], dim=-1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], dim=-1).to(x.dtype)


def _pages(pool, table, P):
    """[n, Hkv, pages * P, hd] of every row of a block table, in 32 bits."""
    n, pps = table.shape
    return pool[table.long().clamp(min=0)].transpose(1, 2).reshape(n, pool.shape[1], pps * P, pool.shape[3]).float()


def _part(q, k, v, seen):
    """Of rows q [n, Hkv, R, hd]: largest score, sum of the exponentials, their sum times v; masked keys take no part."""
    score = (q @ k.transpose(2, 3)) * (1.0 / math.sqrt(q.shape[-1]))
    score = torch.where(seen, score, -math.inf)
    top = score.amax(dim=-1, keepdim=True)
    e = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    return top, e.sum(dim=-1, keepdim=True), e @ v


def _shared(s):
    q, P, Hkv = s["q"], s["P"], s["Hkv"]
    B, T, Hq, hd = q.shape
    G = Hq // Hkv
    rows = q.float().view(B, T, Hkv, G, hd).transpose(1, 2).reshape(B, Hkv, T * G, hd)
    dev = q.device
    # the prefixes, each for the rows of all its sequences at once
    begin, end = s["begin"][:-1].long(), s["begin"][1:].long()
    who = begin[:, None] + torch.arange(s["members"], device=dev)
    who = torch.where(who < end[:, None], who, B)
    n = len(begin)
    some = torch.nn.functional.pad(rows, (0, 0, 0, 0, 0, 0, 0, 1))[who].transpose(1, 2).reshape(n, Hkv, -1, hd)
    k, v = _pages(s["kp"], s["prefix_table"], P), _pages(s["vp"], s["prefix_table"], P)
    seen = torch.arange(k.shape[2], device=dev)[None, None, None, :] < s["prefix_len"].long()[:, None, None, None]
    parts = _part(some, k, v, seen)

    def back(t, fill):
        t = t.reshape(n, Hkv, s["members"], T * G, t.shape[-1]).transpose(1, 2)
        full = torch.full((B + 1,) + t.shape[2:], fill, device=dev)
        full[who] = t
        return full[:B]

    top0, sum0, out0 = back(parts[0], -math.inf), back(parts[1], 0.0), back(parts[2], 0.0)
    # the sequences' own keys
    k, v = _pages(s["kp"], s["table"], P), _pages(s["vp"], s["table"], P)
    t = torch.arange(T, device=dev).repeat_interleave(G)
    seen = torch.arange(k.shape[2], device=dev)[None, None, None, :] <= (s["ctx"].long()[:, None] - T + t)[:, None, :, None]
    top1, sum1, out1 = _part(rows, k, v, seen)
    top = torch.maximum(top0, top1)
    top = torch.where(top == -math.inf, 0.0, top)
    f0, f1 = torch.exp(top0 - top), torch.exp(top1 - top)
    total = sum0 * f0 + sum1 * f1
    out = torch.where(total > 0, (out0 * f0 + out1 * f1) / torch.where(total > 0, total, 1.0), 0.0)
    return out.view(B, Hkv, T, G, hd).transpose(1, 2).reshape(B, T, Hq * hd).to(q.dtype)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "heads": _exact_heads, "shared": _exact_shared}[case["op"]](s)


def _exact_linear(s):
    x, w = s["x"].double(), s["w"].double()
    M, K = x.shape
    y = torch.zeros(M, len(w), dtype=torch.float64, device="cuda") if s["r"] is None else s["r"].double()
    tall = s["ws"].double().repeat_interleave(BLOCK, 0)[: len(w)]
    for i, at in enumerate(range(0, K, BLOCK)):
        piece = x[:, at:at + BLOCK]
        scale = (piece.abs().amax(dim=1, keepdim=True).float() / LARGEST).clamp(min=FLOOR).double()     # held in 32 bits
        codes = (piece / scale).float().to(torch.float8_e4m3fn).double()
        y += (codes * scale) @ (w[:, at:at + BLOCK] * tall[:, i:i + 1]).t()
    return y


def _exact_heads(s):
    def turn(x, gain):
        x = x.double()
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]).sqrt() * gain.double()
        half = s["rot"] // 2
        first = torch.arange(half, device="cuda") * (1 if s["halves"] else 2)
        second = first + (half if s["halves"] else 1)
        z = torch.complex(x[..., first], x[..., second]) * torch.complex(s["cos"].double(), s["sin"].double())[s["pos"].long()].unsqueeze(1)
        x[..., first], x[..., second] = z.real, z.imag
        return x

    kp, vp = s["kp"].double(), s["vp"].double()
    slot = s["slots"].long()
    kp[slot // s["P"], :, slot % s["P"]] = turn(s["k"], s["kg"])
    vp[slot // s["P"], :, slot % s["P"]] = s["v"].double()
    return [turn(s["q"], s["qg"]).flatten(1), kp, vp]


def _exact_shared(s):
    B, T, Hq, hd = s["q"].shape
    Hkv, P = s["Hkv"], s["P"]
    out = torch.zeros(B, T, Hq, hd, dtype=torch.float64, device="cuda")
    begin, plen, ctx = s["begin"].tolist(), s["prefix_len"].tolist(), s["ctx"].tolist()

    def rows(pool, table, n):
        return pool[table[: (n + P - 1) // P].long()].double().transpose(1, 2).reshape(-1, Hkv, hd)[:n]

    for b in range(B):
        group = next((i for i in range(len(plen)) if begin[i] <= b < begin[i + 1]), None)
        pools = []
        for pool in (s["kp"], s["vp"]):
            mine = rows(pool, s["table"][b], ctx[b])
            pools.append(mine if group is None else torch.cat([rows(pool, s["prefix_table"][group], plen[group]), mine]))
        k, v = pools
        front = len(k) - ctx[b]
        for t in range(T):
            n = front + max(0, ctx[b] - T + t + 1)
            if n:
                q = s["q"][b, t].double().view(Hkv, Hq // Hkv, hd)
                p = torch.softmax(torch.einsum("hgd,nhd->hgn", q, k[:n]) / math.sqrt(hd), -1)
                out[b, t] = torch.einsum("hgn,nhd->hgd", p, v[:n]).reshape(Hq, hd)
    return out.view(B, T, Hq * hd)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    c = case
    size = {"fp16": 2, "bf16": 2, "fp32": 4}
    if c["op"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        kb, nb = (K + BLOCK - 1) // BLOCK, (N + BLOCK - 1) // BLOCK
        out = M * N * size[c["out"]] + (M * N * 4 if c["residual"] else 0)
        return {"bytes": M * K * 2 + N * K + nb * kb * 4 + out, "flops": 2 * M * N * K}
    if c["op"] == "heads":
        row = (c["Hq"] + 2 * c["Hkv"]) * c["hd"]
        return {"bytes": c["n"] * (2 * row * 2 + c["rot"] * 4 + 8), "flops": c["n"] * row * 8}
    mean = lambda n, lo, hi: (lo + hi) / 2 if n > 1 else hi  # noqa: E731
    prefixes = c["groups"] * mean(c["groups"], max(1, c["prefix"] // 2), c["prefix"])
    own_keys = c["B"] * mean(c["B"], c["shortest"], c["longest"])
    row = c["Hkv"] * c["hd"] * 2 * 2
    seen = (c["B"] - c["alone"]) * prefixes / c["groups"] + own_keys
    return {"bytes": (prefixes + own_keys) * row + 2 * c["B"] * c["T"] * c["Hq"] * c["hd"] * 2, "flops": 4 * seen * c["T"] * c["Hq"] * c["hd"]}

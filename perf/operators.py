"""Cases for measuring the operators of a decode loop over a paged 8-bit key/value cache, and their plain forms.

  plan    block tables and slot maps from the lengths of the requests        es_op_kv_plan
  cache   new K/V rows written into the 8-bit pages, sequences read back     es_op_kv8_append, es_op_kv8_gather
  attend  attention of the newest tokens over the 8-bit pages                es_op_decode_attention_kv8
  sample  the next token from the logits and given random numbers            es_op_sample

`own` chooses between the library's entry points and the plain form of the same definition in elementary torch
operations.  Sizes: head shapes 32/32, 40/40 and 64/8 of 128 dimensions, pages of 64 tokens and a vocabulary of 32000
are those of the benchmark's configurations; the others are generic.
"""
import math

import torch

own = False

FLOOR_EXP = -100                                   # a block's scale is never below 2^-100
HALF = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def listed():
    return [
        # one step of a server: 64 running requests take one token each and give it back (a rejected draft token)
        dict(name="plan decode 64", op="plan", B=64, P=64, longest=4096, prompts=0, prompt=0, finish=0, draft=1),
        # a busy scheduler: 1024 requests, a tenth new prompts, a tenth finished, the others a few draft tokens each
        dict(name="plan mixed 1024", op="plan", B=1024, P=16, longest=8192, prompts=100, prompt=1500, finish=100, draft=4),
        # the newest token of 64 short sequences enters the cache (grouped heads)
        dict(name="cache decode 64 int8", op="cache", B=64, Hkv=8, hd=128, P=64, held=120, new=1, code="int8", dtype="fp16"),
        # prompts of different lengths, 8 KV heads, small pages
        dict(name="cache prompts e4m3", op="cache", B=12, Hkv=8, hd=128, P=16, held=0, new=700, code="e4m3", dtype="bf16"),
        # long prompts joining sequences that hold tokens already, 32 KV heads
        dict(name="cache long prompts int8", op="cache", B=8, Hkv=32, hd=128, P=64, held=300, new=2600, code="int8", dtype="fp16"),
        # one user, 32 heads, about a thousand tokens
        dict(name="attend one int8", op="attend", B=1, T=1, Hq=32, Hkv=32, hd=128, P=64, shortest=1000, longest=1000, code="int8", dtype="fp16"),
        # 16 sequences of a 64/8-head model at the benchmark's lengths
        dict(name="attend 16 grouped e4m3", op="attend", B=16, T=1, Hq=64, Hkv=8, hd=128, P=64, shortest=1025, longest=1152, code="e4m3", dtype="fp16"),
        # draft tokens checked four at a time, 40 heads, ragged
        dict(name="attend drafts int8", op="attend", B=8, T=4, Hq=40, Hkv=40, hd=128, P=32, shortest=3, longest=2500, code="int8", dtype="bf16"),
        # long ragged contexts, grouped heads
        dict(name="attend long ragged int8", op="attend", B=32, T=1, Hq=64, Hkv=8, hd=128, P=64, shortest=500, longest=8191, code="int8", dtype="bf16"),
        # one user's token
        dict(name="sample one", op="sample", B=1, V=32000, mode="all", dtype="fp32"),
        # 64 requests with settings of their own
        dict(name="sample 64 mixed", op="sample", B=64, V=32000, mode="mixed", dtype="fp32"),
        # many requests over a large vocabulary, half of them unrestricted
        dict(name="sample 256 large", op="sample", B=256, V=128001, mode="mixed", dtype="fp32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "cache", "attend", "sample"])
    if op == "plan":
        B = _log(rng, 1, 1000)
        return dict(op=op, B=B, P=rng.choice([16, 32, 64, 128]), longest=_log(rng, 64, 8000), prompts=rng.randrange(0, B // 4 + 1),
                    prompt=_log(rng, 2, 500), finish=rng.randrange(0, B // 10 + 1), draft=rng.randrange(1, 9))
    if op == "cache":
        Hkv, hd, new = rng.choice([1, 2, 4, 5, 8, 32, 40]), rng.choice([64, 128]), _log(rng, 1, 2000)
        B = _log(rng, 1, max(1, min(128, 16000 * 32 // (Hkv * (new + 64)))))
        return dict(op=op, B=B, Hkv=Hkv, hd=hd, P=rng.choice([16, 32, 64, 128]), held=_log(rng, 1, 300), new=new,
                    code=rng.choice(["int8", "e4m3"]), dtype=rng.choice(["fp16", "bf16"]))
    if op == "attend":
        Hkv, G, hd, T = rng.choice([1, 2, 4, 8, 32, 40]), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128]), rng.choice([1, 1, 2, 5])
        longest = _log(rng, 1, 8000)
        B = _log(rng, 1, max(1, min(64, 1000000 * 8 // (longest * Hkv * max(8, T * G)))))
        return dict(op=op, B=B, T=T, Hq=Hkv * G, Hkv=Hkv, hd=hd, P=rng.choice([16, 32, 64, 128]),
                    shortest=rng.randrange(0, longest + 1), longest=longest, code=rng.choice(["int8", "e4m3"]), dtype=rng.choice(["fp16", "bf16"]))
    V = _log(rng, 100, 128000)
    return dict(op=op, B=_log(rng, 1, 250), V=V, mode=rng.choice(["mixed", "all", "off"]), dtype=rng.choice(["fp32", "fp32", "fp16", "bf16"]))


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed), torch.Generator().manual_seed(seed)


def _spread(n, lo, hi, hg):
    """n lengths from lo to hi in a random order, with the same sum every time."""
    return (torch.linspace(lo, hi, n) if n > 1 else torch.full((n,), float(hi))).round().long()[torch.randperm(n, generator=hg)]


def _mean(n, lo, hi):
    return (lo + hi) / 2 if n > 1 else hi


def _plan_lens(c, hg):
    """Host lengths of a plan case: what each request holds, and what it is to hold."""
    fresh, done = c["prompts"], c["finish"]
    going = c["B"] - fresh - done
    held = _spread(going, 1, c["longest"], hg)
    old = torch.cat([held, torch.zeros(fresh, dtype=torch.long), _spread(done, 1, c["longest"], hg)])
    new = torch.cat([held + _spread(going, 1, c["draft"], hg), _spread(fresh, 1, c["prompt"], hg), torch.zeros(done, dtype=torch.long)])
    who = torch.randperm(c["B"], generator=hg)
    return old[who], new[who]


def _cache_lens(c, hg):
    return _spread(c["B"], 0, c["held"], hg), _spread(c["B"], 1, c["new"], hg)


def _codes(shape, code, g):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float16)
    return (x * 32).round().clamp(-127, 127).to(torch.int8) if code == "int8" else (x * 100).float().clamp(-448, 448).to(torch.float8_e4m3fn)


def _scales(shape, code, g):
    e = torch.randn(shape, generator=g, device="cuda") * 0.7 - 5
    return torch.exp2(e) if code == "int8" else torch.exp2(e.round() - 1)


def _slots(table, begin, end, P):
    """Slots of positions [begin, end) of every sequence, one after the other (host tensors)."""
    return torch.cat([table[b, torch.arange(int(i), int(j)) // P] * P + torch.arange(int(i), int(j)) % P for b, (i, j) in enumerate(zip(begin, end))])


def prepare(case, seed):
    c = case
    g, hg = _gen(seed)
    s = dict(c)
    if c["op"] == "plan":
        old, new = _plan_lens(c, hg)
        P, B = c["P"], c["B"]
        pps = (max(c["longest"] + c["draft"], c["prompt"]) + P - 1) // P
        held = (old + P - 1) // P
        n_pages = int(torch.maximum(old, new).sum()) // P + B + 8
        perm = torch.randperm(n_pages, generator=hg)
        table = torch.full((B, pps), -1)
        col = torch.arange(pps)
        mask = col[None, :] < held[:, None]
        table[mask] = perm[: int(held.sum())]
        free = torch.full((n_pages,), -1)
        n_free = n_pages - int(held.sum())
        free[:n_free] = perm[int(held.sum()):]
        rows = int(max((new - old).clamp(min=0).sum(), (old - new).clamp(min=0).sum())) + 3       # a padded batch: three rows behind the last
        i32 = lambda t: t.to(torch.int32).cuda()  # noqa: E731
        s.update(old=i32(old), new=i32(new), table=i32(table), free=i32(free), count=i32(torch.tensor([n_free])), rows=rows)
    elif c["op"] == "cache":
        held, new = _cache_lens(c, hg)
        P, B, Hkv, hd = c["P"], c["B"], c["Hkv"], c["hd"]
        total = held + new
        pps = (int(total.max()) + P - 1) // P
        used = (total + P - 1) // P
        n_pages = int(total.sum()) // P + B + 2
        table = torch.zeros(B, pps, dtype=torch.long)
        table[torch.arange(pps)[None, :] < used[:, None]] = torch.randperm(n_pages, generator=hg)[: int(used.sum())]
        slots, every = _slots(table, held, total, P), _slots(table, torch.zeros(B), total, P)
        page = slots // P
        first = torch.ones(len(slots), dtype=torch.bool)
        first[1:] = (page[1:] != page[:-1]) | (slots[1:] != slots[:-1] + 1)
        n = len(slots)
        qkv = torch.randn(n, 2 * Hkv, hd, generator=g, device="cuda", dtype=torch.float32)
        qkv = (qkv * torch.exp(0.6 * torch.randn(2 * Hkv, hd, generator=g, device="cuda"))).to(HALF[c["dtype"]])
        shape = (n_pages, Hkv, P, hd)
        s.update(k=qkv[:, :Hkv], v=qkv[:, Hkv:], slots=slots.to(torch.int32).cuda(), every=every.to(torch.int32).cuda(),
                 runs=first.nonzero().flatten().to(torch.int32).cuda(), kp=_codes(shape, c["code"], g), vp=_codes(shape, c["code"], g),
                 ks=_scales(shape[:2], c["code"], g), vs=_scales(shape[:2], c["code"], g))
    elif c["op"] == "attend":
        P, B, Hkv = c["P"], c["B"], c["Hkv"]
        ctx = _spread(B, c["shortest"], c["longest"], hg)
        pps = (c["longest"] + P - 1) // P
        used = (ctx + P - 1) // P
        n_pages = int(ctx.sum()) // P + B + 2
        table = torch.full((B, pps), -1)
        table[torch.arange(pps)[None, :] < used[:, None]] = torch.randperm(n_pages, generator=hg)[: int(used.sum())]
        shape = (n_pages, Hkv, P, c["hd"])
        q = torch.randn(B, c["T"], c["Hq"], c["hd"], generator=g, device="cuda").to(HALF[c["dtype"]])
        s.update(q=q, kp=_codes(shape, c["code"], g), vp=_codes(shape, c["code"], g), ks=_scales(shape[:2], c["code"], g),
                 vs=_scales(shape[:2], c["code"], g), table=table.to(torch.int32).cuda(), ctx=ctx.to(torch.int32).cuda())
    else:
        B, V = c["B"], c["V"]
        # flat and peaked rows: the spread of the logits differs from request to request
        logits = torch.randn(B, V, generator=g, device="cuda") * (1 + 3 * torch.rand(B, 1, generator=g, device="cuda"))
        u = torch.rand(B, generator=g, device="cuda")
        t = 0.5 + torch.rand(B, generator=g, device="cuda")
        k = torch.exp(torch.rand(B, generator=g, device="cuda") * math.log(500)).to(torch.int32)
        p = 0.5 + 0.5 * torch.rand(B, generator=g, device="cuda")
        m = 0.1 * torch.rand(B, generator=g, device="cuda")
        if c["mode"] != "all":                         # off: plain softmax sampling; mixed: each setting on for some rows only
            keep = torch.rand(3, B, generator=g, device="cuda") < (0.4 if c["mode"] == "mixed" else -1.0)
            k, p, m = torch.where(keep[0], k, 0), torch.where(keep[1], p, 1.0), torch.where(keep[2], m, 0.0)
            if c["mode"] == "mixed":
                t = torch.where(torch.rand(B, generator=g, device="cuda") < 0.1, 0.0, t)          # some requests are greedy
        s.update(logits=logits.to(HALF[c["dtype"]]), u=u, t=t, k=k, p=p, m=m)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(state):
    return _RUN[state["op"]](state)


def _run_plan(s):
    """The requests grow (or end), and a second call takes them back: pages are given out and returned."""
    if own:
        from paper_2405_14371_b200 import binding as b
        one = b.es_op_kv_plan(s["old"], s["new"], s["table"], s["P"], s["rows"], s["free"], s["count"])
        two = b.es_op_kv_plan(one.len_out, s["old"], s["table"], s["P"], s["rows"], s["free"], s["count"])
        return list(one) + list(two) + [s["table"], s["free"], s["count"]]
    one = _plan(s["old"], s["new"], s["table"], s["P"], s["rows"], s["free"], s["count"])
    two = _plan(one[-1], s["old"], s["table"], s["P"], s["rows"], s["free"], s["count"])
    return one + two + [s["table"], s["free"], s["count"]]


def _run_cache(s):
    if own:
        from paper_2405_14371_b200 import binding as b
        b.es_op_kv8_append(s["k"], s["v"], s["slots"], s["kp"], s["vp"], s["ks"], s["vs"], runs=s["runs"])
        k, v = b.es_op_kv8_gather(s["every"], s["kp"], s["vp"], s["ks"], s["vs"], dtype=s["k"].dtype)
        return [k, v, s["ks"], s["vs"]]
    _append(s["k"], s["slots"], s["kp"], s["ks"])
    _append(s["v"], s["slots"], s["vp"], s["vs"])
    return [_gather(s["every"], s["kp"], s["ks"], s["k"].dtype), _gather(s["every"], s["vp"], s["vs"], s["k"].dtype), s["ks"], s["vs"]]


def _run_attend(s):
    if own:
        from paper_2405_14371_b200 import binding as b
        return b.es_op_decode_attention_kv8(s["q"], s["kp"], s["vp"], s["ks"], s["vs"], s["table"], s["ctx"], s["longest"])
    return _attend(s["q"], s["kp"], s["vp"], s["ks"], s["vs"], s["table"], s["ctx"])


def _run_sample(s):
    if own:
        from paper_2405_14371_b200 import binding as b
        return b.es_op_sample(s["logits"], s["u"], s["t"], s["k"], s["p"], s["m"])
    return _sample(s["logits"], s["u"], s["t"], s["k"], s["p"], s["m"])


_RUN = {"plan": _run_plan, "cache": _run_cache, "attend": _run_attend, "sample": _run_sample}


# ---- plain forms -------------------------------------------------------------------------------------------------

def _plan(old, new, table, P, max_rows, free, count):
    """Row layout, slots, positions, sequences and runs of the rows that requests gain; `table`, `free` and `count` are
    brought up to date.  Pages that shrinking requests give up go onto the free stack first, in order; growing ones
    then pop theirs from its top, in order, whole requests only."""
    dev, (B, pps) = table.device, table.shape
    n_pages, cap = free.numel(), pps * P
    ok = (old >= 0) & (old <= cap) & (new >= 0) & (new <= cap)
    o, n = torch.where(ok, old, 0).long(), torch.where(ok, new, 0).long()
    po, pn = (o + P - 1) // P, (n + P - 1) // P
    give, need, rows = (po - pn).clamp(min=0), (pn - po).clamp(min=0), (n - o).clamp(min=0)
    have = count.long().clamp(0, n_pages)
    end_give, end_need, end_rows = give.cumsum(0), need.cumsum(0), rows.cumsum(0)
    avail = have + end_give[-1]
    served = (end_rows <= max_rows) & ((need == 0) | (end_need <= avail)) | (rows == 0)
    col = torch.arange(pps, device=dev)[None, :]
    before = torch.arange(n_pages, device=dev)
    given = table.new_full((n_pages + 1,), -1)                      # what comes back, in order of request and page
    leaves = (col >= pn[:, None]) & (col < po[:, None])
    at = torch.where(leaves, (end_give - give)[:, None] + col - pn[:, None], n_pages)
    given.index_put_((at.clamp(max=n_pages),), table)
    stack = torch.where(before < have, free, given[(before - have).clamp(min=0)])       # the stack once they are on it
    taken = torch.where(served, need, 0).sum()
    grows = (col >= po[:, None]) & (col < pn[:, None]) & served[:, None]
    top = avail - 1 - (end_need - need)[:, None] - (col - po[:, None])
    fresh = torch.where(grows, stack[top.clamp(0, n_pages - 1)], -1)
    table.copy_(torch.where(grows, fresh, torch.where(leaves, -1, table)))
    left = avail - taken
    free.copy_(torch.where((before >= have) & (before < left), stack, free))
    count.copy_(left)
    # rows
    r = torch.arange(max_rows, device=dev)
    seq = torch.searchsorted(end_rows, r, right=True)
    real = seq < B
    b = seq.clamp(max=B - 1)
    pos = o[b] + r - (end_rows - rows)[b]
    page = table[b, (pos // P).clamp(0, pps - 1)].long()
    slot = torch.where(real & served[b] & (page >= 0), page * P + pos % P, -1)
    starts = (slot >= 0) & ((r == (end_rows - rows)[b]) | (pos % P == 0))
    n_runs = min(max_rows, max_rows // P + 2 * B)
    runs = torch.full((max_rows + 1,), -1, device=dev)
    runs[torch.where(starts, starts.cumsum(0) - 1, max_rows)] = torch.where(starts, r, -1)
    offsets = torch.cat([end_rows.new_zeros(1), end_rows]).clamp(max=max_rows)
    length = torch.where(served, torch.where(ok, n, old), old)
    out = [offsets, slot, torch.where(real, pos, -1), torch.where(real, b, -1), runs[:n_runs], length]
    return [t.to(torch.int32) for t in out]


def _append(x, slots, pages, scale):
    """Writes rows x [n, Hkv, hd] at their slots of 8-bit pages [n_pages, Hkv, P, hd] with one scale per page and head.
    A page's scale covers the largest value that it holds; where it grows, the codes in front are brought to it."""
    n_pages, Hkv, P, hd = pages.shape
    int8 = pages.dtype == torch.int8
    page, off = (slots // P).long(), (slots % P).long()
    amax = x.float().abs().amax(-1)
    big = torch.zeros(n_pages, Hkv, device=x.device).index_reduce_(0, page, amax, "amax")
    first = torch.full((n_pages,), P, device=x.device).index_reduce_(0, page, off, "amin")
    touched = (first < P)[:, None]
    if int8:
        want = torch.clamp(big / 127, min=2.0 ** FLOOR_EXP)
    else:
        f, e = torch.frexp(big)                                         # big = f 2^e, 448 = 0.875 2^9
        e = (e - 9 + (f > 0.875)).clamp(min=FLOOR_EXP)
        want = torch.where(big > 0, torch.ldexp(torch.ones_like(big), e), 2.0 ** FLOOR_EXP)
    new = torch.where((first > 0)[:, None], torch.maximum(scale, want), want)
    new = torch.where(touched, new, scale)
    before = (torch.arange(P, device=x.device)[None, :] < first[:, None])[:, None, :, None] & touched[:, :, None, None]
    ratio = torch.where(touched, scale.double() / new.double(), 1.0)[:, :, None, None]
    if int8:
        moved = torch.round(pages.double() * ratio).to(torch.int8)
        pages.copy_(torch.where(before, moved, pages))
        pages[page, :, off] = torch.round(x.double() / new[page].double()[:, :, None]).to(torch.int8)
    else:
        raw = pages.view(torch.int8)
        moved = (pages.float() * ratio.float()).to(pages.dtype).view(torch.int8)
        raw.copy_(torch.where(before, moved, raw))
        raw[page, :, off] = (x.float() / new[page][:, :, None]).to(pages.dtype).view(torch.int8)
    scale.copy_(new)


def _gather(slots, pages, scale, dtype):
    P = pages.shape[2]
    page, off = (slots // P).long(), (slots % P).long()
    codes = pages.view(torch.int8)[page, :, off].view(pages.dtype)
    return (codes.float() * scale[page][:, :, None]).to(dtype)


def _attend(q, kp, vp, ks, vs, table, ctx):
    B, T, Hq, hd = q.shape
    n_pages, Hkv, P, _ = kp.shape
    pps = table.shape[1]
    at = table.long().clamp(min=0)

    def read(pages, scale):                                             # [B, Hkv, pps * P, hd]
        x = pages.view(torch.int8)[at].view(pages.dtype).float() * scale[at][..., None, None]
        return x.transpose(1, 2).reshape(B, Hkv, pps * P, hd)

    k = read(kp, ks)
    rows = q.float().reshape(B, T, Hkv, Hq // Hkv, hd).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, hd)
    score = torch.matmul(rows, k.transpose(-1, -2)) / math.sqrt(hd)
    t = torch.arange(T, device=q.device).repeat_interleave(Hq // Hkv)
    pos = torch.arange(pps * P, device=q.device)
    seen = (pos[None, None, :] <= (ctx.long()[:, None] - T + t[None, :])[..., None]) & (table >= 0).repeat_interleave(P, 1)[:, None, :]
    score = score.masked_fill(~seen[:, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    w = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    w = torch.where(total > 0, w / total, 0.0)
    out = torch.matmul(w, read(vp, vs)).reshape(B, Hkv, T, Hq // Hkv, hd).permute(0, 2, 1, 3, 4)
    return out.reshape(B, T, Hq * hd).to(q.dtype)


def _sample(logits, u, t, k, p, m):
    """Temperature, then the top k, then the smallest set of at least mass p among them, then nothing below min-p times
    the largest; equal logits rank by index.  The token is the first, in order of index, at which the running mass of
    what is left passes u times its whole.  In 64 bits: every sum here has borders next to it."""
    x = logits.double()
    V = x.shape[1]
    srt, order = torch.sort(x, dim=1, descending=True, stable=True)
    greedy = (t <= 0)[:, None]
    w = torch.exp((srt - srt[:, :1]) / torch.where(t > 0, t, 1.0).double()[:, None])
    rank = torch.arange(V, device=x.device)[None, :]
    k = torch.where(k > 0, k, V).long()[:, None]
    w = torch.where((rank < k) & (~greedy | (rank == 0)), w, 0.0)
    run = w.cumsum(1)
    p, m = p.double()[:, None], m.double()[:, None]
    keep = (run - w < p * run[:, -1:]) | (p >= 1) | (rank == 0)
    keep &= (w >= m) | (rank == 0)
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))
    run = kept.cumsum(1)
    token = (run <= u.double()[:, None] * run[:, -1:]).sum(1)
    last = V - 1 - (kept > 0).flip(1).to(torch.int8).argmax(1)
    token = torch.minimum(token, last)
    prob = kept.gather(1, token[:, None])[:, 0] / run[:, -1]
    return [token.to(torch.int32), torch.log(prob).float()]


# ---- the definitions in 64 bits, request by request ---------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[case["op"]](s)


def _exact_plan(s):
    P, rows_most = s["P"], s["rows"]
    table, free, n_free = s["table"].tolist(), s["free"].tolist(), int(s["count"])
    outs = []
    lens = [s["old"].tolist(), s["new"].tolist()]
    for a, z in ((0, 1), (1, 0)):
        old = lens[0] if not outs else outs[5]
        new = lens[z]
        for b in range(len(old)):
            for j in range(-(-new[b] // P), -(-old[b] // P)):
                free[n_free] = table[b][j]
                n_free += 1
                table[b][j] = -1
        left, offsets, slot, pos, seq, runs, length = n_free, [0], [], [], [], [], []
        for b in range(len(old)):
            need = range(-(-old[b] // P), -(-new[b] // P))
            fits = offsets[-1] + max(0, new[b] - old[b]) <= rows_most and len(need) <= left
            if fits:
                for j in need:
                    left -= 1
                    table[b][j] = free[left]
            for i in range(old[b], new[b]):
                if fits and (i == old[b] or i % P == 0):
                    runs.append(len(slot))
                slot.append(table[b][i // P] * P + i % P if fits else -1)
                pos.append(i)
                seq.append(b)
            offsets.append(len(slot))
            length.append(new[b] if fits else old[b])
        n_free = left
        pad = lambda v, n: v + [-1] * (n - len(v))  # noqa: E731
        outs += [offsets, pad(slot, rows_most), pad(pos, rows_most), pad(seq, rows_most),
                 pad(runs, min(rows_most, rows_most // P + 2 * len(old))), length]
    # entries of the stack that a pop has left behind are not part of it: they keep what they held last
    return [torch.tensor(t, dtype=torch.int32) for t in outs] + [torch.tensor(table, dtype=torch.int32), None, torch.tensor([n_free], dtype=torch.int32)]


def _round_e4m3(x):
    a = x.abs()
    step = torch.ldexp(torch.ones_like(a), (torch.frexp(a)[1] - 1).clamp(min=-6) - 3)
    return torch.sign(x) * torch.clamp(torch.round(a / step) * step, max=448.0)


def _exact_cache(s):
    P, int8 = s["P"], s["code"] == "int8"
    out, scales = [], []
    slots, runs, n = s["slots"].long(), s["runs"].tolist(), len(s["slots"])
    for x, pages, scale in ((s["k"], s["kp"], s["ks"]), (s["v"], s["vp"], s["vs"])):
        value = pages.double() if int8 else pages.float().double()
        scale = scale.double()
        for i, j in zip(runs, runs[1:] + [n]):
            page, off = int(slots[i]) // P, int(slots[i]) % P
            rows = x[i:j].double().transpose(0, 1)                      # [Hkv, rows, hd]
            big = rows.abs().amax((1, 2))
            if int8:
                want = torch.clamp(big / 127, min=2.0 ** FLOOR_EXP).float().double()          # a scale is held in 32 bits
            else:
                f, e = torch.frexp(big / 448)                           # exactly 1/2 where big is 448 times a power of two
                want = torch.ldexp(torch.ones_like(big), torch.where(f == 0.5, e - 1, e).clamp(min=FLOOR_EXP))
            new = torch.maximum(want, scale[page]) if off > 0 else want
            rounded = torch.round if int8 else _round_e4m3
            value[page, :, :off] = rounded(value[page, :, :off] * (scale[page] / new)[:, None, None])
            value[page, :, off:off + j - i] = rounded(rows / new[:, None, None])
            scale[page] = new
        every = s["every"].long()
        out.append(value[every // P, :, every % P] * scale[every // P][:, :, None])
        scales.append(scale)
    return out + scales


def _exact_attend(s):
    q, P, T = s["q"].double(), s["P"], s["T"]
    B, _, Hq, hd = q.shape
    G = Hq // s["Hkv"]
    out = torch.zeros(B, T, Hq, hd, dtype=torch.float64, device=q.device)
    for b, n in enumerate(s["ctx"].tolist()):
        if n == 0:
            continue
        at = s["table"][b, : -(-n // P)].long()
        k, v = ((x.view(torch.int8)[at].view(x.dtype).float().double() * y[at].double()[..., None, None]).transpose(0, 1).flatten(1, 2)[:, :n]
                for x, y in ((s["kp"], s["ks"]), (s["vp"], s["vs"])))
        for t in range(T):
            m = n - T + t + 1
            if m > 0:
                score = torch.einsum("hgd,hnd->hgn", q[b, t].reshape(-1, G, hd), k[:, :m]) / math.sqrt(hd)
                out[b, t] = torch.einsum("hgn,hnd->hgd", torch.softmax(score, -1), v[:, :m]).reshape(Hq, hd)
    return out.reshape(B, T, Hq * hd)


def _exact_sample(s):
    x = s["logits"].double()
    V = x.shape[1]
    tokens, logs = [], []
    for b, (u, t, k, p, m) in enumerate(zip(s["u"].tolist(), s["t"].tolist(), s["k"].tolist(), s["p"].tolist(), s["m"].tolist())):
        if t <= 0:
            tokens.append(int((x[b] == x[b].max()).nonzero()[0]))
            logs.append(0.0)
            continue
        order = torch.argsort(x[b], descending=True, stable=True)
        if 0 < k < V:
            order = order[:k]
        prob = torch.softmax(x[b][order] / t, 0)
        if p < 1:
            n = int(torch.searchsorted(prob.cumsum(0), torch.tensor(p, dtype=torch.float64, device=x.device))) + 1
            order, prob = order[:n], prob[:n]
        if m > 0:
            n = max(1, int((prob >= m * prob[0]).sum()))
            order, prob = order[:n], prob[:n]
        order, by = torch.sort(order)
        prob = prob[by] / prob.sum()
        i = min(len(order) - 1, int(torch.searchsorted(prob.cumsum(0), torch.tensor(u, dtype=torch.float64, device=x.device), right=True)))
        tokens.append(int(order[i]))
        logs.append(math.log(float(prob[i])))
    return [torch.tensor(tokens, dtype=torch.int32), torch.tensor(logs, dtype=torch.float64)]


_EXACT = {"plan": _exact_plan, "cache": _exact_cache, "attend": _exact_attend, "sample": _exact_sample}


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "plan":
        others = c["B"] - c["prompts"] - c["finish"]
        gain = c["prompts"] * _mean(c["prompts"], 1, c["prompt"]) + others * _mean(others, 1, c["draft"])
        back = c["finish"] * _mean(c["finish"], 1, c["longest"])
        pages = (c["prompts"] * c["prompt"] + c["finish"] * c["longest"]) / 2 / c["P"]
        # lengths in and out and row offsets, three numbers a row, the entries that change in the table and on the stack
        return {"bytes": 2 * 16.0 * c["B"] + 12 * (gain + back) + 4 * 8 * pages, "flops": 4 * (gain + back)}
    if c["op"] == "cache":
        new = c["B"] * _mean(c["B"], 1, c["new"])
        held = c["B"] * _mean(c["B"], 0, c["held"])
        width = 2.0 * c["Hkv"] * c["hd"]                                # K and V values of a token
        return {"bytes": width * (2 * new + new + (1 + 2) * (new + held)) + 8 * (2 * new + held), "flops": width * (4 * new + held)}
    if c["op"] == "attend":
        keys = c["B"] * _mean(c["B"], c["shortest"], c["longest"])
        return {"bytes": keys * c["Hkv"] * (2.0 * c["hd"] + 8.0 / c["P"]) + 4.0 * c["B"] * c["T"] * c["Hq"] * c["hd"],
                "flops": 4.0 * keys * c["T"] * c["Hq"] * c["hd"]}
    size = 4 if c["dtype"] == "fp32" else 2
    return {"bytes": float(size) * c["B"] * c["V"] + 28.0 * c["B"], "flops": 6.0 * c["B"] * c["V"]}

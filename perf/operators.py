"""Timing cases of the prompt path: blocks for a step's tokens, rotary positions, the K/V rows
into the paged cache, and attention of a chunk of new tokens over that cache.

A case is a dict of plain values; ``kind`` names the operator:

"plan"    blocks and cache slots for a step's new tokens (``plan_blocks``)
"trim"    blocks past the kept lengths back to the free list (``trim_blocks``)
"rope"    rotary positions of one or several axes for q and k, and the rows k, v into their
          slots of the paged cache (``rope_append``)
"chunk"   attention of each request's new tokens over its paged cache (``chunk_attention``)
"masked"  the same with a cap on the scores, a bias by distance, first keys per query (a
          sliding window or packed documents) and prefixes every query sees

bs              requests of the batch
new_lo, new_hi  new tokens of a request (uniform over the logarithm); ``single`` is the share of
                the requests that have one new token instead (decoding beside prompts)
ctx_lo, ctx_hi  tokens already in the cache, integer-uniform
hq, hkv, d      query heads, KV heads, head dimension

Lengths are drawn for the case and are the same for every seed; values, physical block ids and
free lists come from the seed.  Q/K/V are N(0, 1) in bf16.
"""
import math
import random

import numpy as np
import torch

own = False     # True: the framework's entry points; False: the plain form below

BLOCK = 16
# head geometries: (query heads, KV heads, head dimension)
HEADS = ((32, 8, 128), (16, 8, 128), (4, 2, 64))
THETA = 1e6


def listed():
    big = dict(hq=32, hkv=8, d=128)
    return [
        # a decoding step's bookkeeping: few requests cross a block border
        dict(name="plan_decode_256", kind="plan", bs=256, new_lo=1, new_hi=1, single=0.0,
             ctx_lo=1024, ctx_hi=4096, fits=1.0),
        # a large step with prompts in a pool that does not hold all of them
        dict(name="plan_prompts_4096", kind="plan", bs=4096, new_lo=1, new_hi=128, single=0.5,
             ctx_lo=0, ctx_hi=2048, fits=0.9),
        # after a small step: a few requests are finished, the others lose a rejected suffix
        dict(name="trim_64", kind="trim", bs=64, ctx_lo=1024, ctx_hi=4096, finished=0.1),
        # a drained worker: most of a large batch gives its blocks back
        dict(name="trim_4096", kind="trim", bs=4096, ctx_lo=512, ctx_hi=2048, finished=0.7),
        # one decoded token per request of a draft worker
        dict(name="rope_decode_64", kind="rope", bs=64, new_lo=1, new_hi=1, single=0.0, ctx_lo=512,
             ctx_hi=2048, hq=16, hkv=8, d=128, axes=1, rot=128, interleaved=False),
        # the windows of a verification round
        dict(name="rope_window_256", kind="rope", bs=256, new_lo=5, new_hi=5, single=0.0,
             ctx_lo=1024, ctx_hi=4096, axes=1, rot=128, interleaved=False, **big),
        # prompts with images: three axes, ragged lengths
        dict(name="rope_images_8", kind="rope", bs=8, new_lo=1000, new_hi=4000, single=0.0,
             ctx_lo=0, ctx_hi=500, axes=3, rot=128, interleaved=False, **big),
        # the smallest batch: latency
        dict(name="chunk_tiny_4", kind="chunk", bs=4, new_lo=1, new_hi=16, single=0.0, ctx_lo=64,
             ctx_hi=256, hq=4, hkv=2, d=64),
        # a serving step: mostly decoding, some prompt chunks among it
        dict(name="chunk_mixed_64", kind="chunk", bs=64, new_lo=64, new_hi=512, single=0.85,
             ctx_lo=1024, ctx_hi=4096, **big),
        # chunks of long prompts over what is cached of them
        dict(name="chunk_long_2", kind="chunk", bs=2, new_lo=2048, new_hi=4096, single=0.0,
             ctx_lo=8192, ctx_hi=28000, **big),
        # decoding with capped scores over a window behind a kept prefix
        dict(name="masked_decode_128", kind="masked", bs=128, new_lo=1, new_hi=1, single=0.0,
             ctx_lo=2048, ctx_hi=8192, cap=50.0, slopes=False, window=1024, docs=0, prefix=64,
             **big),
        # packed documents with a bias by distance and capped scores
        dict(name="masked_documents_4", kind="masked", bs=4, new_lo=1000, new_hi=2048, single=0.0,
             ctx_lo=0, ctx_hi=4096, cap=30.0, slopes=True, window=0, docs=700, prefix=0, **big),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("plan", "trim", "rope", "chunk", "chunk", "masked", "masked"))
    if kind == "trim":
        lo = rng.randint(1, 2048)
        return dict(kind=kind, bs=_log_int(rng, 1, 4096), ctx_lo=lo,
                    ctx_hi=rng.randint(lo, 4096), finished=rng.choice((0.0, 0.1, 0.5, 1.0)))
    if kind == "plan":
        lo, new = rng.randint(0, 2048), _log_int(rng, 1, 64)
        return dict(kind=kind, bs=_log_int(rng, 1, 4096), new_lo=new,
                    new_hi=rng.randint(new, 128), single=rng.choice((0.0, 0.5, 0.9)), ctx_lo=lo,
                    ctx_hi=rng.randint(lo, 4096), fits=rng.choice((0.5, 0.9, 1.0)))
    hq, hkv, d = rng.choice(HEADS)
    new_lo = _log_int(rng, 1, 2048)
    new_hi = min(4096, int(new_lo * rng.uniform(1.0, 4.0)))
    if kind == "rope":
        rot = rng.choice((d, d, d // 2))
        lo = _log_int(rng, 1, 16384)
        return dict(kind=kind, bs=_log_int(rng, 1, max(1, min(512, 16000 // new_hi))),
                    new_lo=new_lo, new_hi=new_hi, single=rng.choice((0.0, 0.5)), ctx_lo=lo,
                    ctx_hi=rng.randint(lo, 2 * lo), hq=hq, hkv=hkv, d=d,
                    axes=rng.choice((1, 1, 2, 3)), rot=rot, interleaved=rng.random() < 0.3)
    ctx_lo = _log_int(rng, 1, 16384)
    ctx_hi = min(28000, int(ctx_lo * rng.uniform(1.0, 4.0)))
    # neither the pairs of tokens nor the cached tokens pass those of the largest listed case
    most = min(4096 * 25000 // (new_hi * (ctx_hi + new_hi)), 600000 // (ctx_hi + new_hi), 256)
    case = dict(kind=kind, bs=_log_int(rng, 1, max(1, most)), new_lo=new_lo, new_hi=new_hi,
                single=rng.choice((0.0, 0.5, 0.9)), ctx_lo=ctx_lo, ctx_hi=ctx_hi, hq=hq, hkv=hkv,
                d=d)
    if kind == "masked":
        near = rng.choice(("window", "docs", "none"))
        case.update(cap=rng.choice((0.0, 30.0, 50.0)), slopes=rng.random() < 0.5,
                    window=_log_int(rng, 16, 4096) if near == "window" else 0,
                    docs=_log_int(rng, 16, 4096) if near == "docs" else 0,
                    prefix=rng.choice((0, 4, 64, 500)))
    return case


# ---- inputs -----------------------------------------------------------------------------

def _lengths(case):
    """(tokens in the cache, new tokens) of every request."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    ctx, new = [], []
    for r in range(case["bs"]):
        ctx.append(rng.randint(case["ctx_lo"], case["ctx_hi"]))
        if case["kind"] == "trim":
            new.append(0)
        elif r and rng.random() < case["single"]:
            new.append(1)
        else:
            new.append(_log_int(rng, case["new_lo"], case["new_hi"]))
    return ctx, new


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _indptr(new):
    return [0] + np.cumsum(np.asarray(new, np.int64)).tolist()


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


def _normal(shape, gen):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _table(counts, rng, spare=0):
    """(block table padded with -1, ids left over): a random permutation of the pool."""
    counts = np.asarray(counts, np.int64)
    ids = rng.permutation(int(counts.sum()) + spare).astype(np.int32)
    table = np.full((len(counts), max(1, int(counts.max()))), -1, np.int32)
    table[np.arange(table.shape[1])[None, :] < counts[:, None]] = ids[:counts.sum()]
    return table, ids[counts.sum():]


def _trimmed(case):
    """(cached tokens, kept tokens) of a trim."""
    ctx, _ = _lengths(case)
    rng = random.Random(1)
    keep = [0 if rng.random() < case["finished"] else max(0, c - rng.randint(0, 40)) for c in ctx]
    return ctx, keep


def _spans(case):
    """Visible tokens of every query row as (prefix, first, position), request by request."""
    ctx, new = _lengths(case)
    rng = random.Random(2)
    out = []
    for c, n in zip(ctx, new):
        pos = np.arange(c, c + n, dtype=np.int64)
        first = np.zeros(n, np.int64)
        if case.get("window"):
            first = np.maximum(pos - case["window"] + 1, 0)
        elif case.get("docs"):
            starts = [0]
            while starts[-1] < c + n:
                starts.append(starts[-1] + rng.randint(1, 2 * case["docs"]))
            starts = np.asarray(starts)
            first = starts[np.searchsorted(starts, pos, side="right") - 1]
        out.append((min(case.get("prefix", 0), c + n), first, pos))
    return out


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    if kind == "trim":
        ctx, keep = _trimmed(case)
        counts = [_blocks(c) for c in ctx]
        table, left = _table(counts, rng, spare=100)
        free = np.concatenate([left, np.full(sum(counts), -1, np.int32)])
        return dict(case=case, table=_i32(table), owned=_i32(counts), keep=_i32(keep),
                    free=_i32(free), free_count=_i32([len(left)]))
    ctx, new = _lengths(case)
    indptr = _indptr(new)
    state = dict(case=case, indptr=_i32(indptr), total=indptr[-1], host_ctx=ctx, host_new=new)
    if kind == "plan":
        counts = [_blocks(c) for c in ctx]
        want = [_blocks(c + n) - _blocks(c) for c, n in zip(ctx, new)]
        table, left = _table(counts, rng, spare=int(sum(want) * case["fits"]) + 1)
        width = max(_blocks(c + n) for c, n in zip(ctx, new))
        wide = np.full((len(ctx), width), -1, np.int32)
        wide[:, :min(width, table.shape[1])] = table[:, :width]
        state.update(table=_i32(wide), owned=_i32(counts), lens=_i32(ctx), free=_i32(left),
                     free_count=_i32([len(left)]))
        return state
    total, hkv, d = indptr[-1], case["hkv"], case["d"]
    lens = [c + n for c, n in zip(ctx, new)]
    if kind == "rope":
        # rows of a fused projection: q, k and v are views of it
        rows = _normal((total, (case["hq"] + 2 * hkv) * d), gen)
        cut = case["hq"] * d
        state["q"] = rows[:, :cut].view(total, case["hq"], d)
        state["k"] = rows[:, cut:cut + hkv * d].view(total, hkv, d)
        state["v"] = rows[:, cut + hkv * d:].view(total, hkv, d)
        # only the blocks that the new tokens touch are in the pool
        first = [c // BLOCK for c in ctx]
        table, _ = _table([_blocks(n) - f for n, f in zip(lens, first)], rng, spare=3)
        slots = np.concatenate([table[r, np.arange(c, c + n) // BLOCK - f].astype(np.int64) * BLOCK
                                + np.arange(c, c + n) % BLOCK
                                for r, (c, n, f) in enumerate(zip(ctx, new, first))])
        state["slots"] = _i32(slots)
        nb = int(table.max()) + 4
        pos = np.concatenate([np.arange(c, c + n) for c, n in zip(ctx, new)])
        axes = [pos, pos // 37, pos % 37][:case["axes"]]
        state["positions"] = _i32(np.stack(axes))
        half = case["rot"] // 2
        cuts = {1: [half], 2: [half - half // 3, half // 3],
                3: [half - 2 * (half // 3), half // 3, half // 3]}[case["axes"]]
        state["sections"] = cuts
        state["freq"] = torch.tensor([THETA ** (-i / half) for i in range(half)],
                                     dtype=torch.float32, device="cuda")
        state["q_out"] = torch.empty((total, case["hq"], d), dtype=torch.bfloat16, device="cuda")
    else:
        table, _ = _table([_blocks(n) for n in lens], rng)
        nb = int(table.max()) + 1
        state.update(q=_normal((total, case["hq"], d), gen), table=_i32(table), lens=_i32(lens),
                     out=torch.empty((total, case["hq"], d), dtype=torch.bfloat16, device="cuda"))
        state["most"] = (max(new), max(lens))
        state["spans"] = spans = _spans(case)
        masks = {}
        if case.get("cap"):
            masks["softcap"] = case["cap"]
        if case.get("slopes"):
            masks["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / case["hq"])
                                            for h in range(case["hq"])], device="cuda")
        if case.get("window") or case.get("docs"):
            masks["first_keys"] = _i32(np.concatenate([s[1] for s in spans]))
        if case.get("prefix"):
            masks["prefix_lens"] = _i32([s[0] for s in spans])
        state["masks"] = masks
        if own:
            import paper_2609_29364_amd as nsd
            state["workspace"] = nsd.new_workspace(nsd.chunk_attention_workspace_size(
                case["bs"], total, case["hq"], hkv, d, *state["most"]), "cuda")
    state["k_pool"] = _normal((nb, hkv, d // 8, BLOCK, 8), gen)
    state["v_pool"] = _normal((nb, hkv, d, BLOCK), gen)
    return state


# ---- a pass -----------------------------------------------------------------------------

def _plan_plain(s):
    table, owned, lens, indptr, free = s["table"], s["owned"], s["lens"], s["indptr"], s["free"]
    new = indptr[1:] - indptr[:-1]
    need = ((lens + new + BLOCK - 1) // BLOCK - owned).clamp(min=0)
    upto = need.cumsum(0)
    granted = ((need == 0) | (upto <= s["free_count"])).int()
    need = need * granted
    start = upto - need             # requests before a granted one are granted what they need
    out = table.clone()
    col = torch.arange(table.shape[1], device=table.device)[None, :]
    k = col - owned[:, None]
    take = (k >= 0) & (k < need[:, None])
    src = (s["free_count"] - 1 - start[:, None] - k).clamp(min=0, max=max(0, free.numel() - 1))
    out = torch.where(take, free[src.long()], out)
    rows = torch.repeat_interleave(torch.arange(len(lens), device=table.device), new.long(),
                                   output_size=s["total"])
    t = lens[rows] + torch.arange(s["total"], device=table.device) - indptr[rows]
    at = out[rows, (t // BLOCK).long().clamp(max=table.shape[1] - 1)]
    slots = torch.where(granted[rows] > 0, at * BLOCK + t % BLOCK, -1).int()
    return dict(table=out, owned=(owned + need).int(), lens=(lens + new * granted).int(),
                free_count=(s["free_count"] - need.sum()).int(), granted=granted, slots=slots)


def _trim_plain(s):
    table, owned, free = s["table"], s["owned"], s["free"]
    kept = torch.minimum(owned, (s["keep"] + BLOCK - 1) // BLOCK)
    col = torch.arange(table.shape[1], device=table.device)[None, :]
    back = ((col >= kept[:, None]) & (col < owned[:, None])).flatten()    # request by request
    at = torch.where(back, s["free_count"] + back.cumsum(0) - 1, free.numel())
    out = torch.cat([free, free[:1]])           # what is kept goes past the end
    out[at] = table.flatten()
    return dict(owned=kept.int(), free=out[:-1],
                free_count=(s["free_count"] + (owned - kept).sum()).int())


def _pairs(x, rot, interleaved):
    if interleaved:
        return x[..., 0:rot:2], x[..., 1:rot:2]
    return x[..., :rot // 2], x[..., rot // 2:rot]


def _rotate(x, cos, sin, rot, interleaved):
    """x [rows][heads][D] turned by the angles of its rows, in x's type."""
    out = x.clone()
    a, b = _pairs(x, rot, interleaved)
    oa, ob = _pairs(out, rot, interleaved)
    oa.copy_(a * cos - b * sin)
    ob.copy_(a * sin + b * cos)
    return out


def _angles(s):
    axis = torch.cat([torch.full((n,), i, dtype=torch.int64, device="cuda")
                      for i, n in enumerate(s["sections"])])
    return s["positions"][axis].double().T * s["freq"].double()      # far positions: 64 bits


def _put(s, k, v):
    block, slot = (s["slots"] // BLOCK).long(), (s["slots"] % BLOCK).long()
    rows, hkv, d = k.shape
    s["k_pool"][block, :, :, slot] = k.view(rows, hkv, d // 8, 8)
    s["v_pool"][block, :, :, slot] = v


def _rope_plain(s):
    c = s["case"]
    a = _angles(s)
    cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]
    q, k = (_rotate(s[n].float(), cos, sin, c["rot"], c["interleaved"]).bfloat16()
            for n in ("q", "k"))
    _put(s, k, s["v"])
    return dict(q=q, k_pool=s["k_pool"], v_pool=s["v_pool"])


def _attend(s, dtype):
    """out in `dtype`, request by request and at most 512 query tokens at a time."""
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    group, scale = hq // hkv, 1.0 / math.sqrt(d)
    cap = c.get("cap") or 0.0
    slopes = s["masks"].get("slopes")
    out = torch.empty((s["total"], hq, d), dtype=dtype, device="cuda")
    row = 0
    for r, (ctx, new) in enumerate(zip(s["host_ctx"], s["host_new"])):
        length = ctx + new
        ids = s["table"][r, :_blocks(length)].long()
        k = s["k_pool"][ids].to(dtype).permute(1, 0, 3, 2, 4).reshape(hkv, -1, d)[:, :length]
        v = s["v_pool"][ids].to(dtype).permute(1, 0, 3, 2).reshape(hkv, -1, d)[:, :length]
        k, v = k.transpose(1, 2).contiguous(), v.contiguous()
        prefix, first, _ = s["spans"][r]
        t = torch.arange(length, device="cuda")[None, :]
        for j in range(0, new, 512):
            n = min(512, new - j)
            q = s["q"][row + j:row + j + n].to(dtype).view(n, hkv, group, d)
            q = q.permute(1, 2, 0, 3).reshape(hkv, group * n, d)
            x = torch.matmul(q, k).mul_(scale)
            if cap:
                x = x.div_(cap).tanh_().mul_(cap)
            x = x.view(hkv, group, n, length)
            pos = torch.arange(ctx + j, ctx + j + n, device="cuda")[:, None]
            if slopes is not None:
                x -= slopes.to(dtype).view(hkv, group, 1, 1) * (pos - t).abs().to(dtype)
            lo = torch.as_tensor(first[j:j + n], device="cuda")[:, None]
            seen = (t < prefix) | ((t <= pos) & (t >= lo))
            x.masked_fill_(~seen, -math.inf)
            top = x.amax(-1, keepdim=True)
            x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
            total = x.sum(-1, keepdim=True)
            o = torch.matmul(x.view(hkv, group * n, length), v).view(hkv, group, n, d)
            o = torch.where(total > 0, o / total, 0.0)
            out[row + j:row + j + n] = o.permute(2, 0, 1, 3).reshape(n, hq, d)
        row += new
    return out


def run(state):
    s = state
    kind = s["case"]["kind"]
    if not own:
        if kind == "plan":
            return _plan_plain(s)
        if kind == "trim":
            return _trim_plain(s)
        if kind == "rope":
            return _rope_plain(s)
        return _attend(s, torch.float32).bfloat16()
    import paper_2609_29364_amd as nsd
    if kind == "plan":
        owned, lens, count, granted, slots = nsd.plan_blocks(
            s["table"], s["owned"], s["lens"], s["indptr"], s["free"], s["free_count"], s["total"])
        return dict(table=s["table"], owned=owned, lens=lens, free_count=count, granted=granted,
                    slots=slots)
    if kind == "trim":
        owned, count = nsd.trim_blocks(s["table"], s["owned"], s["keep"], s["free"],
                                       s["free_count"])
        return dict(owned=owned, free=s["free"], free_count=count)
    if kind == "rope":
        nsd.rope_append(s["k_pool"], s["v_pool"], s["q"], s["k"], s["v"], s["positions"],
                        s["freq"], s["slots"], sections=s["sections"],
                        interleaved=s["case"]["interleaved"], q_out=s["q_out"])
        return dict(q=s["q_out"], k_pool=s["k_pool"], v_pool=s["v_pool"])
    return nsd.chunk_attention(s["q"], s["k_pool"], s["v_pool"], s["table"], s["lens"],
                               s["indptr"], *s["most"], out=s["out"], workspace=s["workspace"],
                               **s["masks"])


# ---- what a pass cannot do without --------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "trim":
        ctx, keep = _trimmed(case)
        back = sum(_blocks(c) - min(_blocks(c), _blocks(k)) for c, k in zip(ctx, keep))
        return {"bytes": 12 * case["bs"] + 8 * back, "flops": 0}
    ctx, new = _lengths(case)
    total = sum(new)
    if kind == "plan":
        want = sum(_blocks(c + n) - _blocks(c) for c, n in zip(ctx, new))
        # owned, lengths and offsets read, owned, lengths and grants written; an id a block
        # read and written; a slot a token
        return {"bytes": 24 * case["bs"] + 8 * int(want * case["fits"]) + 4 * total, "flops": 0}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if kind == "rope":
        rows = (2 * hq + 4 * hkv) * d * 2 + 4 * (case["axes"] + 1)
        return {"bytes": total * rows + 2 * case["rot"],
                "flops": 3 * total * (hq + hkv) * case["rot"]}
    tokens = pairs = 0
    for prefix, first, pos in _spans(case):
        pairs += int(np.maximum(pos + 1 - np.maximum(first, prefix), 0).sum()) + prefix * len(pos)
        # tokens that some query sees: the prefix, and what lies between first key and position
        lo, hi = np.maximum(first, prefix), pos + 1
        before = np.maximum.accumulate(np.concatenate([[prefix], hi[:-1]]))
        tokens += prefix + int(np.maximum(hi - np.maximum(lo, before), 0).sum())
    extra = 4 * total * (1 if case.get("window") or case.get("docs") else 0)
    return {"bytes": tokens * hkv * d * 4 + total * hq * d * 4 + extra + 4 * tokens // BLOCK,
            "flops": 4 * hq * d * pairs}


# ---- the definition in 64 bits --------------------------------------------------------------

def _plan_exact(s):
    table, owned, lens, indptr, free = (s[n].cpu().numpy().astype(np.int64)
                                        for n in ("table", "owned", "lens", "indptr", "free"))
    left = int(s["free_count"].item())
    full, granted, slots = False, [], []
    for r in range(len(lens)):
        n = int(indptr[r + 1] - indptr[r])
        need = max(0, -(-(int(lens[r]) + n) // BLOCK) - int(owned[r]))
        full = full or need > left
        ok = not need or not full
        granted.append(int(ok))
        if not ok:
            slots += [-1] * n
            continue
        for _ in range(need):
            left -= 1
            table[r, owned[r]] = free[left]
            owned[r] += 1
        for t in range(int(lens[r]), int(lens[r]) + n):
            slots.append(int(table[r, t // BLOCK]) * BLOCK + t % BLOCK)
        lens[r] += n
    return dict(table=_i32(table), owned=_i32(owned), lens=_i32(lens), free_count=_i32([left]),
                granted=_i32(granted), slots=_i32(slots))


def _trim_exact(s):
    table, owned, keep, free = (s[n].cpu().numpy() for n in ("table", "owned", "keep", "free"))
    free, left, kept = free.tolist(), int(s["free_count"].item()), []
    for r in range(len(owned)):
        k = min(int(owned[r]), -(-int(keep[r]) // BLOCK))
        back = table[r, k:owned[r]].tolist()
        free[left:left + len(back)] = back
        left += len(back)
        kept.append(k)
    return dict(owned=_i32(kept), free=_i32(free), free_count=_i32([left]))


def _rope_exact(s):
    c = s["case"]
    half, d = c["rot"] // 2, c["d"]
    axis = [i for i, n in enumerate(s["sections"]) for _ in range(n)]
    pos, freq = s["positions"].double(), s["freq"].double()
    turned = {n: s[n].double() for n in ("q", "k")}
    for x in turned.values():
        for i in range(half):
            angle = pos[axis[i]] * freq[i]
            cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
            u, w = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
            a, b = x[..., u].clone(), x[..., w].clone()
            x[..., u] = a * cos - b * sin
            x[..., w] = a * sin + b * cos
    k_pool, v_pool = s["k_pool"].double(), s["v_pool"].double()
    block, slot = (s["slots"] // BLOCK).long(), (s["slots"] % BLOCK).long()
    for i in range(d):
        k_pool[block, :, i // 8, slot, i % 8] = turned["k"][..., i]
        v_pool[block, :, i, slot] = s["v"][..., i].double()
    return dict(q=turned["q"], k_pool=k_pool, v_pool=v_pool)


def _attend_exact(s):
    """Head by head, the visible keys of each stretch of 256 queries gathered."""
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    out = torch.zeros((s["total"], hq, d), dtype=torch.float64, device="cuda")
    slopes = s["masks"].get("slopes")
    row = 0
    for r, (ctx, new) in enumerate(zip(s["host_ctx"], s["host_new"])):
        prefix, first, _ = s["spans"][r]
        for j in range(0, new, 256):
            n = min(256, new - j)
            keys = np.arange(min(int(first[j:j + n].min()), prefix), max(ctx + j + n, prefix))
            keys = keys[(keys < prefix) | (keys >= first[j:j + n].min())]
            if prefix:
                keys = np.union1d(keys, np.arange(prefix))
            t = torch.as_tensor(keys, device="cuda")
            block, slot = s["table"][r].long()[t // BLOCK], t % BLOCK
            k = s["k_pool"][block, :, :, slot].reshape(len(keys), hkv, d).double()
            v = s["v_pool"][block, :, :, slot].double()
            pos = torch.arange(ctx + j, ctx + j + n, device="cuda")[:, None]
            lo = torch.as_tensor(first[j:j + n], device="cuda")[:, None]
            hidden = ~((t < prefix) | ((t <= pos) & (t >= lo)))
            for h in range(hq):
                g = h // (hq // hkv)
                x = s["q"][row + j:row + j + n, h].double() @ k[:, g].T / math.sqrt(d)
                if c.get("cap"):
                    x = c["cap"] * torch.tanh(x / c["cap"])
                if slopes is not None:
                    x = x - float(slopes[h]) * (pos - t).abs()
                x = x.masked_fill(hidden, -math.inf)
                w = torch.softmax(x, -1).nan_to_num(0.0)    # a row that sees nothing is 0
                out[row + j:row + j + n, h] = w @ v[:, g]
        row += new
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "plan":
        return _plan_exact(s)
    if case["kind"] == "trim":
        return _trim_exact(s)
    if case["kind"] == "rope":
        return _rope_exact(s)
    return _attend_exact(s)

"""What is timed of attention over pages of keys: the calls a user makes of the block entry points of
paper_2604_18348_amd.binding, and the same operators in elementary torch operations.

A case is one pass:
  kind "append"  new tokens of every sequence go into a paged cache (kept in the inputs' type or in 4 bits) with the
                 boxes of their pages, and are read back: what a serving step does with the keys and values it made.
  kind "select"  scores of blocks of queries against the boxes of the cached pages, and the pages that each block keeps.
  kind "serve"   attention of new tokens over a paged cache: over the pages selected for them (topk > 0, selection
                 included) or over all of them (topk 0); one token a sequence or a chunk of a prompt.
  kind "train"   boxes, selection, attention and its gradients over packed sequences: a layer's forward and backward.

Lengths are ragged and follow from the case; values follow from the seed.  Keys have a mean a page (neighbouring
tokens are alike) and channels that stand out, queries lean towards some of those means, so that attention is
concentrated and the pages' scores differ, as in a trained model.
"""
import math
import random

import torch

own = False


def _case(name, kind, B, Hq, Hkv, d, page, max_len, new=1, dtype="bf16", bits=0, qblock=1, topk=0, causal=True, full=False):
    """new: the largest number of new tokens (queries) of a sequence; full: all sequences have the largest lengths."""
    return dict(name=name, kind=kind, B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, max_len=max_len, new=new, dtype=dtype, bits=bits, qblock=qblock,
                topk=topk, causal=causal, full=full)


def listed():
    return [
        # one token a sequence into a small cache: launches and host time
        _case("append_token", "append", 8, 8, 8, 128, 16, 4001),
        # prompts going into a 4-bit cache
        _case("append_prompt_4bit", "append", 6, 8, 8, 128, 64, 8192, new=4096, bits=4),
        # the pages of a decode step over long contexts
        _case("select_decode", "select", 32, 32, 8, 128, 16, 32768, topk=128),
        # the pages of chunks of two prompts, one list for 16 tokens
        _case("select_prompt", "select", 2, 16, 4, 64, 32, 16384, new=2048, qblock=16, topk=64),
        # one sequence, one head of keys: latency
        _case("serve_single", "serve", 1, 8, 1, 64, 16, 4001, topk=32),
        # a decode step of a large batch over long contexts
        _case("serve_decode", "serve", 64, 32, 8, 128, 16, 32768, topk=128),
        # a decode step over a whole 4-bit cache
        _case("serve_4bit", "serve", 32, 32, 8, 128, 64, 16384, bits=4),
        # a few tokens a sequence (as in a verified draft) over selected pages of a 4-bit cache, odd group of heads
        _case("serve_4bit_draft", "serve", 16, 15, 3, 64, 32, 24001, new=5, bits=4, qblock=5, topk=100),
        # chunks of prompts over selected pages of a 16-bit cache
        _case("serve_chunk", "serve", 2, 32, 8, 128, 64, 32768, new=1024, qblock=16, topk=48),
        # a layer of a language model, packed ragged sequences, shared heads
        _case("train_causal", "train", 3, 16, 4, 128, 64, 8192, new=8192, qblock=64, topk=32),
        # a layer of the 720x480, 49-frame video model: no order, every head its own keys
        _case("train_video", "train", 1, 30, 30, 64, 128, 17776, new=17776, qblock=128, topk=32, causal=False, full=True),
        # the fp32 accuracy path at its usual size
        _case("train_f32", "train", 1, 1, 1, 64, 64, 4096, new=4096, dtype="f32", qblock=64, topk=16, causal=False, full=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        if w["flops"] <= 1.9e12 and w["bytes"] <= 9e8:                   # no more than the largest listed ones
            del case["name"]
            return case


def _draw(rng):
    kind = rng.choice(["append", "select", "serve", "serve", "serve", "train", "train"])
    d, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    Hkv, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 5, 8])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    bits = rng.choice([0, 4]) if kind in ("append", "serve") else 0
    if kind == "train":
        n = _log(rng, 300, 8192)
        qblock = rng.choice([16, 32, 64, 128])
        causal = rng.random() < 0.6
        need = (qblock - 1) // page + 3
        return _case("", kind, rng.randint(1, 2), Hkv * group, Hkv, d, page, n, n, dtype if n <= 2048 else "bf16", 0, qblock,
                     need + _log(rng, 1, max(2, 2048 // page)), causal, False)
    n = _log(rng, 64, 32768)
    new = 1 if rng.random() < 0.6 else min(n, _log(rng, 2, 1024))
    B = _log(rng, 1, 32) if new == 1 else rng.randint(1, 2)
    qblock = 1 if new == 1 else rng.choice([4, 7, 16, 32, 64])
    need = (qblock - 1) // page + 3
    topk = need + _log(rng, 1, max(2, 2048 // page)) if kind == "select" or rng.random() < 0.6 else 0
    return _case("", kind, B, Hkv * group, Hkv, d, page, n, new, dtype, bits, qblock, 0 if kind == "append" else topk, True, False)


# ---- sizes that follow from the case --------------------------------------------------------------------------------


def _lens(case):
    """(new tokens, tokens in the end) of every sequence; the first has the largest of both."""
    B, n, new = case["B"], case["max_len"], case["new"]
    if case["full"]:
        return [new] * B, [n] * B
    rng = random.Random("%d %d %d" % (B, n, new))
    news, lens = [new], [n]
    for _ in range(B - 1):
        lens.append(rng.randint(max(1, n // 2), n))
        news.append(lens[-1] if case["kind"] == "train" else min(lens[-1], 1 if new == 1 else rng.randint(max(1, new // 2), new)))
    return news, lens


def _tdtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _own_pages(case, n, nq, i):
    """Pages [lo, hi) that hold the positions of block i, and the number of pages that it can see."""
    page, first = case["page"], n - nq + i * case["qblock"]
    last = n - nq + min(nq, (i + 1) * case["qblock"]) - 1
    if not case["causal"]:
        return 0, 0, -(-n // page)
    if last < 0:
        return 0, 0, 0
    return max(first, 0) // page, last // page + 1, last // page + 1


def work(case):
    B, Hq, Hkv, d, page = case["B"], case["Hq"], case["Hkv"], case["d"], case["page"]
    e = 2 if case["dtype"] == "bf16" else 4
    row = d // 2 + d // 64 * 4 if case["bits"] == 4 else d * e           # one cached key or value of one head
    box = 2 * d * e
    news, lens = _lens(case)
    byts = flops = 0
    for nq, n in zip(news, lens):
        if case["kind"] == "append":
            pages = -(-n // page) - (n - nq) // page
            byts += nq * Hkv * 2 * (d * e + row + row + d * e) + pages * Hkv * box
            continue
        blocks = -(-nq // case["qblock"])
        kept = pairs = scored = 0
        for i in range(blocks):
            lo, hi, seen = _own_pages(case, n, nq, i)
            keep = min(seen, case["topk"]) if case["topk"] else seen
            scored += seen if case["topk"] else 0
            kept = kept + keep * page
            rows = min(nq, (i + 1) * case["qblock"]) - i * case["qblock"]
            cut = sum(max(0, hi * page - 1 - (n - nq + i * case["qblock"] + r)) for r in (0, rows - 1)) / 2 if case["causal"] else 0
            pairs += rows * max(0, min(n, keep * page) - cut)
        byts += nq * Hq * d * e                                          # q
        if case["topk"]:
            byts += -(-n // page) * Hkv * box + blocks * Hkv * (case["topk"] + 1) * 4
            flops += 4 * d * scored * Hq
        if case["kind"] == "select":
            continue
        byts += 2 * min(kept, n) * Hkv * row + nq * Hq * (d * e + 4)     # keys and values, o, lse
        flops += 4 * d * pairs * Hq
        if case["kind"] == "train":
            byts += nq * Hq * d * e * 2 + 2 * n * Hkv * d * e            # do, dq, dk, dv (what the forward has read is there)
            flops += 10 * d * pairs * Hq
    return dict(bytes=byts, flops=flops)


# ---- the 4-bit form ---------------------------------------------------------------------------------------------------


def _quantise(x):
    """[..., d] values -> codes uint8 [..., d/2] (dim 2j in the low half of byte j), (scale, lo) bf16 [..., d/64, 2]."""
    x = x.float().unflatten(-1, (-1, 64))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    down = lo.to(torch.bfloat16).float()
    bits = lo.contiguous().view(torch.int32)
    cut = (bits & -65536) + 65536 * ((lo < 0) & ((bits & 65535) != 0)).int()      # towards minus infinity
    down = torch.where(down <= lo, down, cut.view(torch.float32))
    step = (hi - down) / 15.0
    up = ((step.contiguous().view(torch.int32) + 65535) & -65536).view(torch.float32)    # step >= 0: upwards
    bad = ~(torch.isfinite(up) & torch.isfinite(hi - down) & torch.isfinite(x).all(-1, keepdim=True))
    code = torch.where(up > 0, torch.round((x - down) / up), torch.zeros_like(x)).clamp(0, 15)
    code = torch.where(bad, torch.zeros_like(code), code).to(torch.uint8).flatten(-2)
    meta = torch.cat([up, down], -1)
    meta = torch.where(bad, torch.full_like(meta, math.nan), meta).to(torch.bfloat16)
    return code[..., 0::2] | (code[..., 1::2] << 4), meta


def _dequantise(codes, meta, to=torch.float32):
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).to(to).unflatten(-1, (-1, 64))
    return (c * meta[..., 0:1].to(to) + meta[..., 1:2].to(to)).flatten(-2)


# ---- inputs -----------------------------------------------------------------------------------------------------------


def _prefix(ns):
    out = [0]
    for n in ns:
        out.append(out[-1] + n)
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt, B, Hq, Hkv, d, page = _tdtype(case), case["B"], case["Hq"], case["Hkv"], case["d"], case["page"]
    news, lens = _lens(case)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=dt)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = dict(case=case, lens=ints(lens), cu_q=ints(_prefix(news)), news=news, lens_host=lens)
    bias = 1.5 * rand(Hkv, d) * (torch.rand((Hkv, d), generator=gen, device="cuda") < 0.05)
    tq = sum(news)
    max_pages = -(-case["max_len"] // page)

    def queries(means):                                                  # means [n, Hkv, d] of pages
        pick = torch.randint(0, means.shape[0], (tq // 8 + 1,), generator=gen, device="cuda").repeat_interleave(8)[:tq]
        m = means[pick].repeat_interleave(Hq // Hkv, 1)
        return (1.2 * rand(tq, Hq, d) + m).to(dt)

    if case["kind"] == "train":
        tk = sum(lens)
        means = rand(tk // page + 1, Hkv, d)
        at = torch.arange(tk, device="cuda") // page
        s["k"] = (0.7 * rand(tk, Hkv, d) + means[at] + bias).to(dt)
        s["v"] = rand(tk, Hkv, d)
        s["q"], s["do"] = queries(means), rand(tq, Hq, d)
        if case["full"]:                                                 # the layout of the clustered calls: [H, N, d]
            for n in ("q", "k", "v", "do"):
                s[n] = s[n].transpose(0, 1).contiguous().transpose(0, 1)
        s["cu_k"] = ints(_prefix(lens))
    else:
        per = [-(-n // page) for n in lens]
        pages = sum(per) + 3
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
        for b, (a, n) in enumerate(zip(_prefix(per), per)):
            table[b, :n] = order[a:a + n]
        means = rand(pages, Hkv, 1, d)
        s["table"] = table
        old = ints([n - q for n, q in zip(lens, news)])                  # tokens held before this step
        if case["kind"] == "append":
            s["old"] = old
            s["k"], s["v"] = (rand(tq, Hkv, d) + bias).to(dt), rand(tq, Hkv, d)
            shape = (pages, Hkv, page, d // 2 if case["bits"] == 4 else d)
            for n in ("kc", "vc"):
                s[n] = torch.zeros(shape, dtype=torch.uint8 if case["bits"] == 4 else dt, device="cuda")
            for n in ("km", "vm"):
                s[n] = torch.zeros((pages, Hkv, page, d // 64, 2), dtype=torch.bfloat16, device="cuda") if case["bits"] == 4 else None
            s["boxes"] = torch.stack([rand(pages, Hkv, d).abs(), -rand(pages, Hkv, d).abs()], 2).to(dt)
        else:
            k = rand(pages, Hkv, page, d).mul_(0.7).add_(means).add_(bias[:, None].to(dt))
            v = rand(pages, Hkv, page, d) if case["kind"] == "serve" else None
            s["boxes"] = torch.stack([k.amax(2), k.amin(2)], 2)
            s["km"] = s["vm"] = None
            if case["bits"] == 4:
                (k, s["km"]), (v, s["vm"]) = _quantise(k), _quantise(v)
            if case["kind"] == "serve":
                s["kc"], s["vc"] = k, v
            s["q"] = queries(means[:, :, 0])
    if own:
        from paper_2604_18348_amd import binding as A
        s["p"] = A.BlockParams(B=B, Hq=Hq, Hkv=Hkv, d=d, dtype=A.BF16 if dt == torch.bfloat16 else A.F32, bits=case["bits"], page=page,
                               max_q=case["new"], max_pages=max_pages, qblock=case["qblock"], causal=int(case["causal"]), topk=case["topk"],
                               keep_first=1)
        if case["kind"] in ("append", "serve"):
            s["cache"] = A.BlockCache(k=s["kc"], v=s["vc"], k_meta=s["km"], v_meta=s["vm"], boxes=s["boxes"])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2604_18348_amd import binding as A
    case, p = s["case"], s["p"]
    kind = case["kind"]
    if kind == "append":
        A.adacluster_cache_append(p, s["k"], s["v"], s["cu_q"], s["old"], s["table"], s["cache"])
        k, v = A.adacluster_cache_read(p, s["cache"], s["cu_q"], s["old"], s["table"], rows=s["k"].shape[0])
        return [k, v, s["boxes"]]
    if kind == "select":
        return list(A.adacluster_block_select(p, s["q"], s["cu_q"], s["boxes"], seq_lens=s["lens"], page_table=s["table"]))
    if kind == "serve":
        sel = None
        if case["topk"]:
            sel, _ = A.adacluster_block_select(p, s["q"], s["cu_q"], s["boxes"], seq_lens=s["lens"], page_table=s["table"])
        o, lse = A.adacluster_block_attn(p, s["q"], s["cu_q"], cache=s["cache"], seq_lens=s["lens"], page_table=s["table"], sel_idx=sel)
        return [o, lse] if sel is None else [sel, o, lse]
    boxes = A.adacluster_block_boxes(p, s["k"], s["cu_k"])
    sel, _ = A.adacluster_block_select(p, s["q"], s["cu_q"], boxes, cu_k=s["cu_k"])
    o, lse = A.adacluster_block_attn(p, s["q"], s["cu_q"], k=s["k"], v=s["v"], cu_k=s["cu_k"], sel_idx=sel)
    dq, dk, dv = A.adacluster_block_attn_backward(p, s["q"], s["k"], s["v"], o, lse, s["do"], s["cu_q"], s["cu_k"], sel_idx=sel)
    return [sel, o, dq, dk, dv]


def _items(s):
    """Every block of queries of every sequence, padded: rows [B, blocks, qblock] of q (-1: none), their positions."""
    case = s["case"]
    qb, nb = case["qblock"], -(-case["new"] // case["qblock"])
    nq = (s["cu_q"][1:] - s["cu_q"][:-1]).long()
    local = torch.arange(nb * qb, device="cuda").view(1, nb, qb).expand(case["B"], nb, qb)
    there = local < nq.view(-1, 1, 1)
    rows = torch.where(there, s["cu_q"][:-1].long().view(-1, 1, 1) + local, -1)
    return rows, torch.where(there, local + (s["lens"].long() - nq).view(-1, 1, 1), -1)


def _select_plain(s, boxes, table):
    """boxes [n, Hkv, 2, d], table [B, pages] of their rows -> sel_idx [B, blocks, Hkv, topk], sel_cnt."""
    case = s["case"]
    Hkv, d, page, topk = case["Hkv"], case["d"], case["page"], case["topk"]
    rows, pos = _items(s)
    B, nb, _ = rows.shape
    P = table.shape[1]
    idx = torch.empty((B, nb, Hkv, topk), dtype=torch.int32, device="cuda")
    cnt = torch.empty((B, nb, Hkv), dtype=torch.int32, device="cuda")
    step = max(1, (1 << 27) // (P * Hkv * (2 * d + nb * case["Hq"] // Hkv * 2)))
    for a in range(0, B, step):
        r, at = rows[a:a + step], pos[a:a + step]
        n = r.shape[0]
        # sums over a block of queries in 64 bits: two pages that a rounding apart would swap are told apart
        u = (s["q"][r.clamp(min=0)].double() * (r >= 0)[..., None, None]).sum(2)
        u = u.view(n, nb, Hkv, -1, d).permute(0, 2, 1, 3, 4).reshape(n, Hkv, -1, d)
        bx = boxes[table[a:a + step].clamp(min=0).long()].double().permute(0, 2, 3, 4, 1)          # [n, Hkv, 2, d, P]
        sc = torch.matmul(u.clamp(min=0), bx[:, :, 0]) + torch.matmul(u.clamp(max=0), bx[:, :, 1])
        sc = torch.nan_to_num(sc, nan=-math.inf, posinf=math.inf, neginf=-math.inf)
        sc = sc.view(n, Hkv, nb, -1, P).amax(3).permute(0, 2, 1, 3)                                # [n, nb, Hkv, P]
        p = torch.arange(P, device="cuda")
        last = at.amax(2)[..., None]
        some = (r >= 0).any(2)[..., None]
        if case["causal"]:
            first = torch.where(r >= 0, at, 1 << 40).amin(2)[..., None].clamp(min=0)
            seen = some & (last >= 0) & (p <= torch.div(last, page, rounding_mode="floor"))
            kept = seen & ((p >= torch.div(first, page, rounding_mode="floor")) | (p < 1))
        else:
            seen = some & (p * page < s["lens"][a:a + step].view(-1, 1, 1))
            kept = seen & (p < 1)
        order = torch.sort(sc, dim=-1, descending=True, stable=True)[1]
        rank = torch.empty_like(order).scatter_(-1, order, p.expand_as(order).contiguous())
        cls = torch.where(kept, 0, torch.where(seen, 1, 2))[:, :, None]                            # always in, by score, never
        order = torch.sort(cls * P + rank, -1)[1][..., :topk]
        count = seen.sum(-1).clamp(max=topk)[..., None].expand(n, nb, Hkv)
        j = torch.arange(order.shape[-1], device="cuda")
        asc = torch.sort(torch.where(j < count[..., None], order, 1 << 40), -1)[0]
        idx[a:a + step] = -1
        idx[a:a + step, ..., :order.shape[-1]] = torch.where(j < count[..., None], asc, -1).to(torch.int32)
        cnt[a:a + step] = count.to(torch.int32)
    return idx, cnt


def _attend_plain(s, gather, sel, do=None):
    """gather(b [m], positions [m, Hkv, L]) -> K, V fp32 [m, Hkv, L, d] and their row numbers.  -> o, lse, or with do the gradients too."""
    case, q = s["case"], s["q"]
    Hq, Hkv, d, page, qb = case["Hq"], case["Hkv"], case["d"], case["page"], case["qblock"]
    G = Hq // Hkv
    scale = 1.0 / math.sqrt(d)
    rows, pos = _items(s)
    B, nb, _ = rows.shape
    if sel is None:
        sel = torch.arange(-(-case["max_len"] // page), device="cuda", dtype=torch.int32).view(1, 1, 1, -1).expand(B, nb, Hkv, -1)
    rows, pos, sel = rows.flatten(0, 1), pos.flatten(0, 1), sel.flatten(0, 1)
    seq = torch.arange(B, device="cuda").repeat_interleave(nb)
    o = torch.zeros(q.shape, dtype=torch.float32, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, device="cuda")
    if do is not None:
        dq = torch.zeros_like(o)
        dkv = [torch.zeros((s["k"].shape[0] * Hkv, d), device="cuda") for _ in range(2)]
    L = sel.shape[-1] * page
    step = max(1, (1 << 28) // (L * (2 * Hkv * d + 3 * qb * Hq)))
    for a in range(0, rows.shape[0], step):
        r, at, b = rows[a:a + step], pos[a:a + step], seq[a:a + step]
        m = r.shape[0]
        pages = sel[a:a + step].long()
        keys = (pages[..., None] * page + torch.arange(page, device="cuda")).flatten(2)           # positions [m, Hkv, L]
        keys = torch.where((pages >= 0).repeat_interleave(page, 2) & (keys < s["lens"][b].view(-1, 1, 1)), keys, -1)
        K, V, kr = gather(b, keys)
        split = lambda x: x[r.clamp(min=0)].float().view(m, qb, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(m, Hkv, qb * G, d)  # noqa: E731
        Q = split(q)
        S = torch.matmul(Q, K.transpose(2, 3)) * scale
        see = (keys >= 0)[:, :, None, :] & (r >= 0)[:, None, :, None]
        if case["causal"]:
            see = see & (keys[:, :, None, :] <= at[:, None, :, None])
        S = S.masked_fill_(~see.repeat_interleave(G, 2), -math.inf)
        top = S.amax(-1, keepdim=True)
        top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
        Pm = S.sub_(top).exp_()
        tot = Pm.sum(-1, keepdim=True)
        Pm /= torch.where(tot > 0, tot, torch.ones_like(tot))
        O = torch.matmul(Pm, V)
        back = lambda x: x.view(m, Hkv, qb, G, -1).permute(0, 2, 1, 3, 4).reshape(m, qb, Hq, -1)[r >= 0]  # noqa: E731
        to = r[r >= 0]
        o[to] = back(O)
        lse[to] = back(top + tot.log())[..., 0]
        if do is None:
            continue
        D = split(do) * (r >= 0).repeat_interleave(G, 1)[:, None, :, None]
        dP = torch.matmul(D, V.transpose(2, 3))
        dS = dP.sub_((D * O).sum(-1, keepdim=True)).mul_(Pm).mul_(scale)
        dq[to] = back(torch.matmul(dS, K))
        dkv[0].index_add_(0, kr.flatten(), torch.matmul(dS.transpose(2, 3), Q).flatten(0, 2) * (keys >= 0).flatten()[:, None])
        dkv[1].index_add_(0, kr.flatten(), torch.matmul(Pm.transpose(2, 3), D).flatten(0, 2) * (keys >= 0).flatten()[:, None])
    if do is None:
        return o.to(q.dtype), lse
    return o.to(q.dtype), dq.to(q.dtype), dkv[0].view_as(s["k"]).to(q.dtype), dkv[1].view_as(s["k"]).to(q.dtype)


def _run_plain(s):
    case = s["case"]
    kind, Hkv, d, page = case["kind"], case["Hkv"], case["d"], case["page"]
    h = torch.arange(Hkv, device="cuda")
    if kind == "append":
        nq = (s["cu_q"][1:] - s["cu_q"][:-1]).long()
        b = torch.arange(case["B"], device="cuda").repeat_interleave(nq, output_size=s["k"].shape[0])
        at = torch.arange(s["k"].shape[0], device="cuda") - s["cu_q"].long()[b] + s["old"].long()[b]
        pg = s["table"][b, at // page].long()
        where = (pg[:, None], h[None], (at % page)[:, None])
        out = []
        for x, cache, meta in ((s["k"], s["kc"], s["km"]), (s["v"], s["vc"], s["vm"])):
            if case["bits"] == 4:
                cache[where], meta[where] = _quantise(x)
                out.append(_dequantise(cache[where], meta[where]).to(x.dtype))
            else:
                cache[where] = x
                out.append(cache[where])
        first = torch.arange(case["B"], device="cuda")
        # a page that held no token before starts from nothing
        P = s["table"].shape[1]
        p = torch.arange(P, device="cuda")
        fresh = (p * page >= s["old"].view(-1, 1)) & (p * page < (s["old"] + nq).view(-1, 1))
        sb, sp = fresh.nonzero(as_tuple=True)
        new = s["table"][first[sb], sp].long()
        s["boxes"][new, :, 0] = -math.inf
        s["boxes"][new, :, 1] = math.inf
        flat = (pg[:, None] * Hkv + h).flatten()[:, None].expand(-1, d)
        for i, red in ((0, "amax"), (1, "amin")):
            side = s["boxes"][:, :, i].reshape(-1, d).float()
            side.scatter_reduce_(0, flat, s["k"].reshape(-1, d).float(), red)
            s["boxes"][:, :, i] = side.view(-1, Hkv, d).to(s["boxes"].dtype)
        return [out[0], out[1], s["boxes"]]
    if kind == "train":
        k = s["k"]
        lens, cu = s["lens"].long(), s["cu_k"].long()
        P = -(-case["max_len"] // page)
        p = torch.arange(P * page, device="cuda")
        there = p < lens.view(-1, 1)
        rows = torch.where(there, cu[:-1].view(-1, 1) + p, 0)                                       # [B, P * page]
        kk = k[rows].view(case["B"], P, page, Hkv, d)
        hide = ~there.view(case["B"], P, page, 1, 1)
        boxes = torch.stack([kk.masked_fill(hide, -math.inf).amax(2), kk.masked_fill(hide, math.inf).amin(2)], 3).flatten(0, 1)
        table = torch.arange(case["B"] * P, device="cuda").view(-1, P)
        table = torch.where(torch.arange(P, device="cuda") * page < lens.view(-1, 1), table, 0)
        sel, _ = _select_plain(s, boxes, table)

        def packed(b, keys):
            r = cu[b].view(-1, 1, 1) + keys.clamp(min=0)
            return s["k"][r, h.view(1, -1, 1)].float(), s["v"][r, h.view(1, -1, 1)].float(), r * Hkv + h.view(1, -1, 1)
        return [sel] + list(_attend_plain(s, packed, sel, s["do"]))
    sel = None
    if case["topk"]:
        sel, cnt = _select_plain(s, s["boxes"], s["table"])
        if kind == "select":
            return [sel, cnt]

    def paged(b, keys):
        at = keys.clamp(min=0)
        where = (s["table"][b.view(-1, 1, 1), at // page].long().clamp(min=0), h.view(1, -1, 1), at % page)
        if case["bits"] == 4:
            return _dequantise(s["kc"][where], s["km"][where]), _dequantise(s["vc"][where], s["vm"][where]), None
        return s["kc"][where].float(), s["vc"][where].float(), None
    o, lse = _attend_plain(s, paged, sel)
    return [o, lse] if sel is None else [sel, o, lse]


# ---- the definition, in 64 bits -----------------------------------------------------------------------------------------


def _exact_lists(case, u, boxes, n, nq):
    """u [blocks, Hq, d] sums of queries, boxes [pages, Hkv, 2, d] of one sequence -> lists [blocks, Hkv, topk] (-1 behind the end), counts."""
    Hkv, topk, pages = case["Hkv"], case["topk"], boxes.shape[0]
    G = case["Hq"] // Hkv
    blocks = u.shape[0]
    idx = torch.full((blocks, Hkv, topk), -1, dtype=torch.int32, device="cuda")
    cnt = torch.zeros((blocks, Hkv), dtype=torch.int32, device="cuda")
    span = [_own_pages(case, n, nq, i) for i in range(blocks)]
    lo, hi, seen = (torch.tensor([x[j] for x in span], device="cuda")[:, None] for j in range(3))
    pg = torch.arange(pages, device="cuda")[None]
    for g in range(Hkv):
        best = None
        for h in range(g * G, (g + 1) * G):
            sc = torch.zeros((blocks, pages), dtype=torch.float64, device="cuda")
            for c in range(0, case["d"], 16):                            # Eq. 1 as it stands, 16 dimensions at a time
                x = u[:, None, h, c:c + 16]
                sc += torch.maximum(x * boxes[None, :, g, 0, c:c + 16], x * boxes[None, :, g, 1, c:c + 16]).sum(-1)
            best = sc if best is None else torch.maximum(best, sc)
        best = torch.where((pg < 1) | ((pg >= lo) & (pg < hi)), torch.full_like(best, 1e300), best)
        best = torch.where(pg < seen, best, torch.full_like(best, -math.inf))
        for i in range(0, blocks, 1024):
            part = best[i:i + 1024]
            chosen = torch.sort(part, dim=1, descending=True, stable=True)[1][:, :topk]
            chosen = torch.where(torch.gather(part, 1, chosen) > -math.inf, chosen, pages).sort(1)[0]
            idx[i:i + 1024, g, :chosen.shape[1]] = torch.where(chosen < pages, chosen, -1).to(torch.int32)
            cnt[i:i + 1024, g] = (chosen < pages).sum(1).to(torch.int32)
    return idx, cnt


def exact(case, seed):
    s = prepare(case, seed)
    kind, Hq, Hkv, d, page, qb = (case[n] for n in ("kind", "Hq", "Hkv", "d", "page", "qblock"))
    G, news, lens = Hq // Hkv, s["news"], s["lens_host"]
    if kind == "append":
        boxes = s["boxes"].double()
        vals = []
        for x in (s["k"], s["v"]):
            if case["bits"] == 0:
                vals.append(x.double())
            else:                                                        # the nearest of the sixteen values that the format has
                codes, meta = _quantise(x)
                x, m = x.double().unflatten(-1, (-1, 64)), meta.double()
                grid = torch.arange(16, dtype=torch.float64, device="cuda")
                best = None
                for c in grid:
                    y = m[..., 1:2] + c * m[..., 0:1]
                    best = y.expand_as(x) if best is None else torch.where((y - x).abs() < (best - x).abs(), y, best)
                tie = (((x - m[..., 1:2]) / m[..., 0:1]) % 1.0 - 0.5).abs() < 1e-6       # half-way: as the rounding takes it
                best = torch.where(tie, _dequantise(codes, meta, torch.float64).unflatten(-1, (-1, 64)), best)
                vals.append(best.flatten(-2))
        start = 0
        for b, (nq, n) in enumerate(zip(news, lens)):
            for p in range((n - nq) // page, -(-n // page)):
                a, z = max(p * page, n - nq), min((p + 1) * page, n)
                x = s["k"][start + a - (n - nq):start + z - (n - nq)].double()
                at = int(s["table"][b, p])
                mx, mn = x.amax(0), x.amin(0)
                if p * page < n - nq:
                    mx, mn = torch.maximum(mx, boxes[at, :, 0]), torch.minimum(mn, boxes[at, :, 1])
                boxes[at] = torch.stack([mx, mn], 1)
            start += nq
        return [vals[0], vals[1], boxes]
    train = kind == "train"
    blocks_max = -(-case["new"] // qb)
    sel = torch.full((case["B"], blocks_max, Hkv, case["topk"]), -1, dtype=torch.int32, device="cuda")
    cnt = torch.zeros((case["B"], blocks_max, Hkv), dtype=torch.int32, device="cuda")
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    dq = torch.zeros_like(o)
    dk, dv = (torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") if train else None for _ in range(2))
    q0 = k0 = 0
    for b, (nq, n) in enumerate(zip(news, lens)):
        pages, blocks = -(-n // page), -(-nq // qb)
        q = s["q"][q0:q0 + nq].double()
        if not train:
            at = s["table"][b, :pages].long()
        if case["topk"]:
            if train:
                x = s["k"][k0:k0 + n].double()
                x = [x[i * page:(i + 1) * page] for i in range(pages)]
                boxes = torch.stack([torch.stack([y.amax(0), y.amin(0)], 1) for y in x])
            else:
                boxes = s["boxes"][at].double()
            pad = torch.zeros((blocks * qb, Hq, d), dtype=torch.float64, device="cuda")
            pad[:nq] = q
            sel[b, :blocks], cnt[b, :blocks] = _exact_lists(case, pad.view(blocks, qb, Hq, d).sum(1), boxes, n, nq)
        if kind == "select":
            q0 += nq
            continue
        for g in range(Hkv):
            if train:
                K, V = s["k"][k0:k0 + n, g].double(), s["v"][k0:k0 + n, g].double()
            elif case["bits"] == 4:
                K, V = (_dequantise(s[c][at, g], s[m][at, g], torch.float64).flatten(0, 1)[:n] for c, m in (("kc", "km"), ("vc", "vm")))
            else:
                K, V = (s[c][at, g].flatten(0, 1)[:n].double() for c in ("kc", "vc"))
            chunk = max(qb, (1 << 25) // (n * G) // qb * qb)
            for a in range(0, nq, chunk):
                z = min(nq, a + chunk)
                m = z - a
                hs = slice(g * G, (g + 1) * G)
                Q = q[a:z, hs].reshape(-1, d)
                see = torch.ones((m, n), dtype=torch.bool, device="cuda")
                if case["topk"]:
                    i0 = a // qb
                    i1 = -(-z // qb)
                    lists = sel[b, i0:i1, g].long()
                    mark = torch.zeros((i1 - i0, pages + 1), dtype=torch.bool, device="cuda")
                    mark.scatter_(1, torch.where(lists >= 0, lists, pages), True)
                    see = mark[:, :pages].repeat_interleave(page, 1)[:, :n].repeat_interleave(qb, 0)[:m]
                if case["causal"]:
                    see = see & (torch.arange(n, device="cuda")[None] <= (n - nq + torch.arange(a, z, device="cuda"))[:, None])
                S = (Q @ K.T / math.sqrt(d)).masked_fill(~see.repeat_interleave(G, 0), -math.inf)
                l = torch.logsumexp(S, 1, keepdim=True)
                Pm = torch.where(torch.isinf(l), torch.zeros_like(S), (S - l).exp())
                O = Pm @ V
                o[q0 + a:q0 + z, hs] = O.view(m, G, d)
                lse[q0 + a:q0 + z, hs] = l.view(m, G)
                if train:
                    D = s["do"][q0 + a:q0 + z, hs].double().reshape(-1, d)
                    dS = Pm * (D @ V.T - (D * O).sum(1, keepdim=True)) / math.sqrt(d)
                    dq[q0 + a:q0 + z, hs] = (dS @ K).view(m, G, d)
                    dk[k0:k0 + n, g] += dS.T @ Q
                    dv[k0:k0 + n, g] += Pm.T @ D
        q0, k0 = q0 + nq, k0 + n
    if kind == "select":
        return [sel, cnt]
    if train:
        return [sel, o, dq, dk, dv]
    return [o, lse] if not case["topk"] else [sel, o, lse]

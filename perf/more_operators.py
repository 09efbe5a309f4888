"""What is timed of serving from a paged cache whose sequences share prefixes and which drops tokens: the calls a user makes of
paper_2604_18348_amd.binding, and the same operators in elementary torch operations.

A case is one pass:
  kind "prefix"   attention of new tokens over a paged cache where the sequences of a group share their first pages (one system prompt,
                  samples of one prompt, drafts): adacluster_prefix_attn reads those pages once a group.
  kind "weights"  the weight that every cached key gets from the new tokens' queries, summed over queries and the heads that share
                  the key, on top of what earlier steps left: adacluster_cache_weights, from the row sums of attention.
  kind "evict"    the tokens that a sequence keeps, by those weights (its first pages and last tokens always), moved in order to new
                  pages with their weights and boxes: adacluster_cache_evict.

Lengths are ragged and follow from the case; values follow from the seed.  Keys have a mean a page (neighbouring tokens are alike)
and channels that stand out, queries lean towards some of those means, so that attention is concentrated, as in a trained model.
"""
import math
import random

import torch

own = False


def _case(name, kind, B, Hq, Hkv, d, page, max_len, new=1, dtype="bf16", bits=0, groups=1, prefix=0, keep=0, recent=0, first=0):
    """max_len: tokens of the longest sequence; new: the largest number of new tokens (queries); prefix: the longest shared prefix;
    keep, recent, first: tokens kept, the last ones and the first pages among them."""
    return dict(name=name, kind=kind, B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, max_len=max_len, new=new, dtype=dtype, bits=bits, groups=groups,
                prefix=prefix, keep=keep, recent=recent, first=first)


def listed():
    return [
        # eight short chats over one system prompt: latency
        _case("prefix_token_small", "prefix", 8, 8, 8, 64, 16, 1100, prefix=1024),
        # a decode step of a batch over one long document
        _case("prefix_token", "prefix", 32, 32, 8, 128, 16, 18000, prefix=16384),
        # four prompts of different lengths, 4-bit cache
        _case("prefix_token_4bit", "prefix", 64, 32, 8, 128, 64, 9001, bits=4, groups=4, prefix=8192),
        # many samples of one long prompt: its keys meet a thousand rows a head
        _case("prefix_samples", "prefix", 128, 32, 4, 128, 64, 33500, prefix=32768),
        # drafts of five tokens, odd group of heads, prefixes that end inside a page, fp32
        _case("prefix_draft_f32", "prefix", 12, 15, 3, 64, 32, 3500, new=5, dtype="f32", groups=3, prefix=3001),
        # a decode step's weights over whole caches
        _case("weights_token", "weights", 32, 32, 8, 128, 16, 16384),
        # the last tokens of prompts vote on what to keep of a 4-bit cache
        _case("weights_window_4bit", "weights", 4, 32, 8, 128, 64, 32768, new=64, bits=4),
        # chunks of prompts
        _case("weights_chunk", "weights", 2, 32, 8, 128, 64, 16384, new=1024),
        # a short fp32 cache, one head of keys
        _case("weights_draft_f32", "weights", 3, 8, 1, 64, 32, 2001, new=7, dtype="f32"),
        # chats that passed their budget: latency
        _case("evict_small", "evict", 8, 8, 8, 64, 16, 1100, keep=1024, recent=128, first=1),
        # prompts cut to an eighth
        _case("evict_prompt", "evict", 16, 32, 8, 128, 16, 32768, keep=4096, recent=512, first=4),
        # 4-bit caches cut to an odd budget
        _case("evict_4bit", "evict", 32, 32, 8, 128, 64, 16384, bits=4, keep=2001, recent=100, first=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        if w["flops"] <= 2.6e11 and w["bytes"] <= 1.1e9:                 # no more than the largest listed ones
            del case["name"]
            return case


def _draw(rng):
    kind = rng.choice(["prefix", "prefix", "prefix", "weights", "weights", "evict", "evict"])
    d, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    Hkv, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 5, 8])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    bits = rng.choice([0, 0, 4])
    if kind == "prefix":
        B = _log(rng, 1, 128)
        prefix, tail = _log(rng, 64, 32768), _log(rng, 8, 2048)
        new = 1 if rng.random() < 0.7 else min(tail, rng.randint(2, 8))
        return _case("", kind, B, Hkv * group, Hkv, d, page, prefix + tail, new, dtype, bits, min(B, rng.choice([1, 1, 2, 3, 5])), prefix)
    n = _log(rng, 64, 32768)
    B = _log(rng, 1, 32)
    if kind == "weights":
        new = 1 if rng.random() < 0.5 else min(n, _log(rng, 2, 1024))
        return _case("", kind, B if new <= 64 else min(B, 2), Hkv * group, Hkv, d, page, n, new, dtype, bits)
    keep = _log(rng, 32, max(33, n))
    first = rng.choice([0, 1, 2])
    first = min(first, keep // 2 // page)
    return _case("", kind, B, Hkv * group, Hkv, d, page, n, 1, dtype, bits, keep=keep, recent=rng.randint(0, keep // 4), first=first)


# ---- sizes that follow from the case --------------------------------------------------------------------------------


def _members(case):
    """Sequences of every group, uneven."""
    B, g = case["B"], case["groups"]
    cut = [0] + [max(i, min(B - (g - i), B * i * (i + 3) // (g * (g + 3)))) for i in range(1, g)] + [B]
    return list(zip(cut[:-1], cut[1:]))


def _lens(case):
    """(new tokens, tokens in the end) of every sequence, shared prefix of every group; the first has the largest of all."""
    B, n, new, prefix = case["B"], case["max_len"], case["new"], case["prefix"]
    rng = random.Random("%d %d %d %d" % (B, n, new, prefix))
    news = [new] + [1 if new == 1 else rng.randint(max(1, new // 2), new) for _ in range(B - 1)]
    if case["kind"] != "prefix":
        lens = [n] + [rng.randint(max(1, n // 2), n) for _ in range(B - 1)]
        return [min(a, b) for a, b in zip(news, lens)], lens, []
    shared = [prefix] + [rng.randint(max(1, prefix // 2), prefix) for _ in range(case["groups"] - 1)]
    lens = []
    for (a, z), p in zip(_members(case), shared):
        lens += [p + rng.randint(new, n - prefix) for _ in range(a, z)]
    lens[0] = n
    return news, lens, shared


def _tdtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def work(case):
    Hq, Hkv, d, page = case["Hq"], case["Hkv"], case["d"], case["page"]
    e = 2 if case["dtype"] == "bf16" else 4
    row = d // 2 + d // 64 * 4 if case["bits"] == 4 else d * e           # one cached key or value of one head
    news, lens, shared = _lens(case)
    byts = flops = 0
    if case["kind"] == "prefix":
        for (a, z), p in zip(_members(case), shared):
            p = p // page * page
            byts += 2 * p * Hkv * row
            for b in range(a, z):
                byts += 2 * (lens[b] - p) * Hkv * row + news[b] * Hq * (2 * d * e + 4)
                flops += 4 * d * Hq * (news[b] * lens[b] - news[b] * (news[b] - 1) // 2)
    elif case["kind"] == "weights":
        for nq, n in zip(news, lens):
            byts += n * Hkv * (row + 8) + nq * Hq * (d * e + 4)
            flops += 2 * d * Hq * (nq * n - nq * (nq - 1) // 2)
    else:
        for n in lens:
            kept = min(n, case["keep"])
            byts += Hkv * (n * 4 + kept * (4 + 4 + 4 * row) + -(-kept // page) * 2 * d * e)
            if case["bits"] == 4:                                        # and read back as values
                byts += Hkv * kept * 2 * (row + d * e)
    return dict(bytes=byts, flops=flops)


# ---- the 4-bit form ---------------------------------------------------------------------------------------------------


def _quantise(x):
    """[..., d] values -> codes uint8 [..., d/2] (dim 2j in the low half of byte j), (step, lowest) bf16 [..., d/64, 2]."""
    x = x.float().unflatten(-1, (-1, 64))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    low = (lo - lo.abs() * 2.0 ** -7).to(torch.bfloat16).float()         # below the lowest
    step = ((hi - low) / 15.0 * (1 + 2.0 ** -7)).to(torch.bfloat16).float()
    code = torch.round((x - low) / step).clamp(0, 15).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.cat([step, low], -1).to(torch.bfloat16)


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
    dt, B, Hq, Hkv, d, page, kind = _tdtype(case), case["B"], case["Hq"], case["Hkv"], case["d"], case["page"], case["kind"]
    news, lens, shared = _lens(case)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=dt)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = dict(case=case, lens=ints(lens), cu_q=ints(_prefix(news)), news=news, lens_host=lens, shared=shared, tq=sum(news))
    P = -(-case["max_len"] // page)
    # pages of the pool, in any order; sequences of a group name the same ones for their shared prefix
    per = [-(-n // page) for n in lens]
    common = [0] * B
    for (a, z), p in zip(_members(case), shared):
        common[a:z] = [p // page] * (z - a)
    keep = [min(n, case["keep"]) for n in lens] if kind == "evict" else []
    old = sum(per) - sum(common) + sum(common[a] for a, _ in _members(case)) + 3 if kind == "prefix" else sum(per) + 3
    new = sum(-(-k // page) for k in keep)
    order = torch.randperm(old, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((B, P), -1, dtype=torch.int32, device="cuda")
    at, start = 0, {}
    for g, (a, z) in enumerate(_members(case) if kind == "prefix" else []):
        start[a], at = at, at + common[a]
        table[a:z, :common[a]] = order[start[a]:at]
    for b in range(B):
        k = per[b] - common[b]
        table[b, common[b]:per[b]] = order[at:at + k]
        at += k
    s["table"] = table
    means = rand(old + new, Hkv, 1, d)
    bias = 1.5 * rand(Hkv, d) * (torch.rand((Hkv, d), generator=gen, device="cuda") < 0.05)
    k = rand(old + new, Hkv, page, d).mul_(0.7).add_(means).add_(bias[:, None].to(dt))
    v = rand(old + new, Hkv, page, d) if kind != "weights" else None
    s["boxes"] = torch.stack([k.amax(2), k.amin(2)], 2)
    if kind != "evict":
        pick = torch.randint(0, old, (s["tq"] // 8 + 1,), generator=gen, device="cuda").repeat_interleave(8)[:s["tq"]]
        s["q"] = (1.2 * rand(s["tq"], Hq, d) + means[pick][:, :, 0].repeat_interleave(Hq // Hkv, 1)).to(dt)
    s["km"] = s["vm"] = None
    if case["bits"] == 4:
        k, s["km"] = _quantise(k)
        if v is not None:
            v, s["vm"] = _quantise(v)
    s["kc"], s["vc"] = k, k if v is None else v
    if v is None:
        s["vm"] = s["km"]
    if kind == "prefix":
        s["cu_group"], s["prefix"] = ints([0] + [z for _, z in _members(case)]), ints(shared)
    elif kind == "weights":
        # what attention's step over the same cache has left: the logarithm of every row's sum
        lse = []
        for b, (nq, n) in enumerate(zip(news, lens)):
            K = _rows_of(s, table[b, :per[b]])[:, :n]
            Q = s["q"][sum(news[:b]):sum(news[:b]) + nq].float().view(nq, Hkv, -1, d).permute(1, 0, 2, 3).flatten(1, 2)
            S = torch.matmul(Q, K.transpose(1, 2).contiguous()).div_(math.sqrt(d)).view(Hkv, nq, -1, n)
            S.masked_fill_(torch.arange(n, device="cuda") > (n - nq + torch.arange(nq, device="cuda")).view(-1, 1, 1), -math.inf)
            lse.append(torch.logsumexp(S, -1).permute(1, 0, 2).reshape(nq, Hq))
        s["lse"] = torch.cat(lse)
        s["w"] = torch.exp(2 * torch.randn((B, Hkv, P * page), generator=gen, device="cuda")).mul_(0.01)
    else:
        w = torch.exp(2 * torch.randn((B, Hkv, P * page), generator=gen, device="cuda"))
        s["w"] = w * (torch.rand((B, Hkv, P * page), generator=gen, device="cuda") > 0.1)      # many never looked at: ties
        s["old"] = old
        s["new_table"] = torch.full((B, P), -1, dtype=torch.int32, device="cuda")
        to = old + torch.randperm(max(1, new), generator=gen, device="cuda").to(torch.int32)
        for b, (a, n) in enumerate(zip(_prefix([-(-k // page) for k in keep]), keep)):
            s["new_table"][b, :-(-n // page)] = to[a:a + -(-n // page)]
        s["rows"], s["cu_kept"], s["zero"] = sum(keep), ints(_prefix(keep)), ints([0] * B)
    return s


def _rows_of(s, pages):
    """Keys of pages [n] in order, fp32 [Hkv, n * page, d]"""
    k = s["kc"][pages.long()]
    k = _dequantise(k, s["km"][pages.long()]) if s["case"]["bits"] == 4 else k.float()
    return k.transpose(0, 1).flatten(1, 2)


# ---- one pass -----------------------------------------------------------------------------------------------------------


def run(s):
    return _run_own(s) if own else _PLAIN[s["case"]["kind"]](s)


def _run_own(s):
    from paper_2604_18348_amd import binding as A
    case, kind = s["case"], s["case"]["kind"]
    if "p" not in s:                                                     # what a program makes once for its cache
        s["p"] = A.BlockParams(B=case["B"], Hq=case["Hq"], Hkv=case["Hkv"], d=case["d"], dtype=A.BF16 if case["dtype"] == "bf16" else A.F32,
                               bits=case["bits"], page=case["page"], max_pages=s["table"].shape[1], max_q=max(case["new"], case["keep"]),
                               keep_first=case["first"])
        s["cache"] = A.BlockCache(k=s["kc"], v=s["vc"], k_meta=s["km"], v_meta=s["vm"], boxes=s["boxes"])
    p, cache = s["p"], s["cache"]
    if kind == "prefix":
        return list(A.adacluster_prefix_attn(p, s["q"], s["cu_q"], cache, s["lens"], s["table"], s["cu_group"], s["prefix"]))
    if kind == "weights":
        return [A.adacluster_cache_weights(p, s["q"], s["cu_q"], s["lse"], cache, s["lens"], s["table"], weights=s["w"], decay=0.75)]
    kept, lens, w = A.adacluster_cache_evict(p, cache, s["lens"], s["table"], s["w"], keep=case["keep"], recent=case["recent"],
                                             new_table=s["new_table"])
    if case["bits"] == 4:
        k, v = A.adacluster_cache_read(p, cache, s["cu_kept"], s["zero"], s["new_table"], rows=s["rows"])
    else:
        k, v = cache.k[s["old"]:], cache.v[s["old"]:]
    return [kept, lens, w, k, v, cache.boxes[s["old"]:]]


def _gather(s, codes, meta, pages, slots):
    """Cached rows at pages, slots [..., n] of every head -> fp32 [..., Hkv, n, d]"""
    h = torch.arange(s["case"]["Hkv"], device="cuda").view(-1, 1)
    where = (pages.clamp(min=0).long()[..., None, :], h, slots[..., None, :])
    return _dequantise(codes[where], meta[where]) if s["case"]["bits"] == 4 else codes[where].float()


def _queries(s, seq):
    """seq [...] of sequences (-1: none) -> rows of q [..., new] (-1: none) and the keys that each sees"""
    b = seq.clamp(min=0)
    nq = (s["cu_q"][1:] - s["cu_q"][:-1]).long()[b][..., None]
    t = torch.arange(s["case"]["new"], device="cuda")
    there = (t < nq) & (seq >= 0)[..., None]
    return torch.where(there, s["cu_q"][:-1].long()[b][..., None] + t, -1), torch.where(there, s["lens"].long()[b][..., None] - nq + t + 1, 0)


def _plain_prefix(s):
    case = s["case"]
    Hq, Hkv, d, page, new = case["Hq"], case["Hkv"], case["d"], case["page"], case["new"]
    G, scale = Hq // Hkv, 1.0 / math.sqrt(d)
    first, count = s["cu_group"][:-1].long(), (s["cu_group"][1:] - s["cu_group"][:-1]).long()
    most = max(z - a for a, z in _members(case))
    m = torch.arange(most, device="cuda")
    seq = torch.where(m < count[:, None], first[:, None] + m, -1)                                  # [groups, members]
    rows, lim = _queries(s, seq)                                                                   # [groups, members, new]
    n = seq.shape[0]
    whole = torch.div(s["prefix"].long(), page, rounding_mode="floor") * page                      # [groups]
    Q = s["q"][rows.clamp(min=0)].float().view(n, most, new, Hkv, G, d).permute(0, 3, 1, 2, 4, 5).reshape(n, Hkv, most, new * G, d)
    lim = lim.repeat_interleave(G, 2)[:, None, :, :, None]                                         # [groups, 1, members, new * G, 1]
    # the shared keys, once a group
    j = torch.arange(case["prefix"] // page * page, device="cuda")
    pages = s["table"][first][:, torch.div(j, page, rounding_mode="floor")]
    K1, V1 = (_gather(s, s[c], s[x], pages, (j % page).expand_as(pages)) for c, x in (("kc", "km"), ("vc", "vm")))
    S1 = torch.matmul(Q.flatten(2, 3), K1.transpose(2, 3).contiguous()).mul_(scale).view(n, Hkv, most, new * G, -1)
    S1 = S1.masked_fill_(~((j < whole.view(-1, 1, 1, 1, 1)) & (j < lim)), -math.inf)
    # every sequence's own
    i = torch.arange(max(x - s["shared"][g] // page * page for g, (a, z) in enumerate(_members(case)) for x in s["lens_host"][a:z]), device="cuda")
    at = whole.view(-1, 1, 1) + i                                                                  # [groups, 1, own]
    pg = torch.div(at, page, rounding_mode="floor").clamp(max=s["table"].shape[1] - 1)
    pages = s["table"][seq.clamp(min=0)[..., None], pg]
    K2, V2 = (_gather(s, s[c], s[x], pages, (at % page).expand_as(pages)) for c, x in (("kc", "km"), ("vc", "vm")))
    Qs = Q.transpose(1, 2)                                                                         # [groups, members, Hkv, new * G, d]
    S2 = torch.matmul(Qs, K2.transpose(3, 4).contiguous()).mul_(scale)
    see = at[:, :, None, None, :] < lim.transpose(1, 2)
    S2 = S2.masked_fill_(~see, -math.inf).transpose(1, 2)                                          # as S1
    top = S2.amax(-1, keepdim=True)
    if j.numel():
        top = torch.maximum(top, S1.amax(-1, keepdim=True))
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    P1, P2 = S1.sub_(top).exp_(), S2.sub_(top).exp_()
    tot = P1.sum(-1, keepdim=True) + P2.sum(-1, keepdim=True)
    O = torch.matmul(P1.flatten(2, 3), V1).view(n, Hkv, most, new * G, d) + torch.matmul(P2.transpose(1, 2).contiguous(), V2).transpose(1, 2)
    O = O / torch.where(tot > 0, tot, torch.ones_like(tot))
    back = lambda x: x.view(n, Hkv, most, new, G, -1).permute(0, 2, 3, 1, 4, 5).reshape(n, most, new, Hq, -1)[rows >= 0]  # noqa: E731
    o, lse = torch.zeros_like(s["q"]), torch.zeros(s["q"].shape[:2], device="cuda")
    o[rows[rows >= 0]] = back(O).to(o.dtype)
    lse[rows[rows >= 0]] = back(top + tot.log())[..., 0]
    return [o, lse]


def _plain_weights(s):
    case = s["case"]
    Hq, Hkv, d, page, B = case["Hq"], case["Hkv"], case["d"], case["page"], case["B"]
    rows, lim = _queries(s, torch.arange(B, device="cuda"))                                        # [B, new]
    split = lambda x: x.view(B, case["new"], Hkv, Hq // Hkv, -1).permute(0, 2, 1, 3, 4).reshape(B, Hkv, case["new"] * (Hq // Hkv), -1)  # noqa: E731
    Q, lse = split(s["q"][rows.clamp(min=0)].float()), split(s["lse"][rows.clamp(min=0)])
    j = torch.arange(s["table"].shape[1] * page, device="cuda")
    pages = s["table"][:, torch.div(j, page, rounding_mode="floor")]
    K = _gather(s, s["kc"], s["km"], pages, (j % page).expand_as(pages))
    S = torch.matmul(Q, K.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(d)).sub_(lse).exp_()
    S = S.masked_fill_(j >= lim.repeat_interleave(Hq // Hkv, 1)[:, None, :, None], 0.0)
    w = 0.75 * s["w"] + S.sum(2)
    return [w.masked_fill_(j >= s["lens"].view(-1, 1, 1), 0.0)]


def _plain_evict(s):
    case = s["case"]
    Hkv, d, page, B, keep = case["Hkv"], case["d"], case["page"], case["B"], case["keep"]
    n = s["lens"].long().view(-1, 1, 1)
    L = s["w"].shape[-1]
    j = torch.arange(L, device="cuda")
    lens = s["lens"].clamp(max=keep)
    # always in, by weight (a tie: the lower position first), not there
    order = torch.sort(s["w"], dim=-1, descending=True, stable=True)[1]
    rank = torch.empty_like(order).scatter_(-1, order, j.expand_as(order).contiguous())
    cls = torch.where(j >= n, 2, torch.where((j < case["first"] * page) | (j >= n - case["recent"]), 0, 1))
    order = torch.sort(cls * L + rank, -1)[1][..., :keep]
    c = torch.arange(min(keep, L), device="cuda")
    here = c < lens.view(-1, 1, 1)
    kept = torch.sort(torch.where(here, order, L), -1)[0]
    src = kept.clamp(max=L - 1)
    w = torch.zeros_like(s["w"])
    w[..., :src.shape[-1]] = torch.gather(s["w"], -1, src) * here
    out = torch.full((B, Hkv, keep), -1, dtype=torch.int32, device="cuda")
    out[..., :src.shape[-1]] = torch.where(here, kept, -1).to(torch.int32)
    b, h = torch.arange(B, device="cuda").view(-1, 1, 1), torch.arange(Hkv, device="cuda").view(1, -1, 1)
    here = here.expand_as(src)
    a = (s["table"][b, torch.div(src, page, rounding_mode="floor")].long().clamp(min=0), h.expand_as(src), src % page)
    to = s["new_table"][b, torch.div(c, page, rounding_mode="floor")].long().expand_as(src)
    z = (to[here], h.expand_as(src)[here], (c % page).expand_as(src)[here])
    got = []
    for x in ("kc", "vc"):
        s[x][z] = s[x][a][here]
        if case["bits"] == 4:
            m = x[0] + "m"
            s[m][z] = s[m][a][here]
            got.append(_dequantise(s[x][a], s[m][a]).to(_tdtype(case)))
        else:
            got.append(s[x][a])
    pages = -(-src.shape[-1] // page)
    k = torch.nn.functional.pad(got[0], (0, 0, 0, pages * page - src.shape[-1])).view(B, Hkv, pages, page, d)
    there = torch.nn.functional.pad(here, (0, pages * page - src.shape[-1])).view(B, Hkv, pages, page, 1)
    box = torch.stack([k.masked_fill(~there, -math.inf).amax(3), k.masked_fill(~there, math.inf).amin(3)], 3).transpose(1, 2)      # [B, pages, Hkv, 2, d]
    some = torch.arange(pages, device="cuda") * page < lens.view(-1, 1)
    s["boxes"][s["new_table"][:, :pages][some].long()] = box[some].to(s["boxes"].dtype)
    if case["bits"] == 4:
        k, v = (x.transpose(1, 2)[here[:, 0]] for x in got)
    else:
        k, v = s["kc"][s["old"]:], s["vc"][s["old"]:]
    return [out, lens, w, k, v, s["boxes"][s["old"]:]]


_PLAIN = dict(prefix=_plain_prefix, weights=_plain_weights, evict=_plain_evict)


# ---- the definition, in 64 bits -----------------------------------------------------------------------------------------


def _values(s, which, pages, g, n):
    """Keys or values of one head at the first n positions of pages, in 64 bits."""
    x = s[which + "c"][pages, g]
    x = _dequantise(x, s[which + "m"][pages, g], torch.float64) if s["case"]["bits"] == 4 else x.double()
    return x.flatten(0, 1)[:n]


def exact(case, seed):
    s = prepare(case, seed)
    Hq, Hkv, d, page = case["Hq"], case["Hkv"], case["d"], case["page"]
    G, news, lens = Hq // Hkv, s["news"], s["lens_host"]
    if case["kind"] == "evict":
        return _exact_evict(s)
    table = s["table"].clone()
    for (a, z), p in zip(_members(case), s["shared"]):
        table[a:z, :p // page] = table[a, :p // page].clone()
    o = torch.zeros((s["tq"], Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((s["tq"], Hq), dtype=torch.float64, device="cuda")
    w = torch.zeros(s["w"].shape, dtype=torch.float64, device="cuda") if case["kind"] == "weights" else None
    q0 = 0
    for b, (nq, n) in enumerate(zip(news, lens)):
        pages = table[b, :-(-n // page)].long()
        last = n - nq + torch.arange(nq, device="cuda").repeat_interleave(G)
        hide = torch.arange(n, device="cuda")[None] > last[:, None]
        for g in range(Hkv):
            hs = slice(g * G, (g + 1) * G)
            Q = s["q"][q0:q0 + nq, hs].double().reshape(-1, d)
            S = (Q @ _values(s, "k", pages, g, n).T / math.sqrt(d)).masked_fill_(hide, -math.inf)
            if case["kind"] == "weights":
                w[b, g, :n] = 0.75 * s["w"][b, g, :n].double() + (S - s["lse"][q0:q0 + nq, hs].double().reshape(-1, 1)).exp().sum(0)
                continue
            l = torch.logsumexp(S, 1)
            o[q0:q0 + nq, hs] = ((S - l[:, None]).exp() @ _values(s, "v", pages, g, n)).view(nq, G, d)
            lse[q0:q0 + nq, hs] = l.view(nq, G)
        q0 += nq
    return [w] if case["kind"] == "weights" else [o, lse]


def _exact_evict(s):
    case = s["case"]
    Hkv, d, page, B, keep = case["Hkv"], case["d"], case["page"], case["B"], case["keep"]
    kept = torch.full((B, Hkv, keep), -1, dtype=torch.int32, device="cuda")
    w = torch.zeros(s["w"].shape, dtype=torch.float64, device="cuda")
    boxes = s["boxes"].double()
    four = case["bits"] == 4
    pool = [s[x].double() if not four else None for x in ("kc", "vc")]
    packed = [torch.zeros((s["rows"], Hkv, d), dtype=torch.float64, device="cuda") if four else None for _ in range(2)]
    row = 0
    for b, n in enumerate(s["lens_host"]):
        m = min(n, keep)
        pages, to = s["table"][b, :-(-n // page)].long(), s["new_table"][b, :-(-m // page)].long()
        for g in range(Hkv):
            x = s["w"][b, g, :n].double()
            must = torch.zeros(n, dtype=torch.bool, device="cuda")
            must[:case["first"] * page] = True
            must[max(0, n - case["recent"]):] = True
            rest = (~must).nonzero()[:, 0]
            best = rest[torch.sort(x[rest], descending=True, stable=True)[1]][:max(0, m - int(must.sum()))]
            take = torch.cat([must.nonzero()[:, 0], best]).sort()[0] if m < n else torch.arange(n, device="cuda")
            kept[b, g, :m] = take.to(torch.int32)
            w[b, g, :m] = x[take]
            k, v = (_values(s, c, pages, g, n)[take] for c in "kv")
            for i in range(to.shape[0]):
                part = slice(i * page, min(m, (i + 1) * page))
                boxes[to[i], g, 0], boxes[to[i], g, 1] = k[part].amax(0), k[part].amin(0)
            for x, r, y in zip(pool, packed, (k, v)):
                if four:
                    r[row:row + m, g] = y
                else:
                    i = torch.arange(m, device="cuda")
                    x[to[i // page], g, i % page] = y
        row += m
    k, v = packed if four else [x[s["old"]:] for x in pool]
    return [kept, s["lens"].clamp(max=keep), w, k, v, boxes[s["old"]:]]

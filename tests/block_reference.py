"""Attention over pages of keys in 64 bits on the CPU, by its definition (one mask of what every query sees), with bounds on what
the kernels' roundings can change.  Shares no code with the library.

Bounds.  u = 2^-24 (fp32), h = half a step of the output's type relative to the value (2^-24, bfloat16 2^-8).
  scores   products of d terms in fp32:  es = (d + 8) u scale sum |q||k|; 4-bit keys enter as 128 + code, so their |k| counts as
           143 step + |lowest|.
  weights  relative error  ew = 2 max(es) + (n + 64) u 4  (difference of two scores, exponential, sums of n terms), and h more where
           they are rounded for a product with values in 16 bits.
"""
import math

import torch

U = 2.0 ** -24


def half(dtype):
    return torch.finfo(dtype).eps / 2


def dequantise(codes, meta):
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double().unflatten(-1, (-1, 64))
    m = meta.double()
    return (c * m[..., 0:1] + m[..., 1:2]).flatten(-2)


def quantise(x):
    """The 4-bit form of rows [..., d] by its definition, one group at a time in 64 bits but for the code's division in 32."""
    x = x.float()
    g = x.unflatten(-1, (-1, 64))
    lo, hi = g.amin(-1), g.amax(-1)

    def toward(v, up):                                       # next bfloat16 up or down
        r = v.to(torch.bfloat16)
        bits = r.view(torch.int16).int()
        wrong = (r.float() < v) if up else (r.float() > v)
        step = torch.where(bits < 0, -1, 1) if up else torch.where(bits < 0, 1, -1)
        zero = (r == 0) & wrong
        bits = torch.where(wrong & ~zero, bits + step, bits)
        return bits.to(torch.int16).view(torch.bfloat16)

    low = toward(lo, False)
    step = toward((hi - low.float()) * torch.tensor(1 / 15), True)
    bad = ~(torch.isfinite(g).all(-1) & torch.isfinite(hi - low.float()) & torch.isfinite(step.float()))
    s = step.float().unsqueeze(-1)
    code = torch.where(s > 0, torch.round((g - low.float().unsqueeze(-1)) / s), torch.zeros_like(g)).clamp(0, 15)
    code = torch.where(bad.unsqueeze(-1), torch.zeros_like(code), code).to(torch.uint8).flatten(-2)
    meta = torch.stack([step, low], -1)
    meta = torch.where(bad[..., None], torch.full_like(meta, math.nan), meta)
    return code[..., 0::2] | (code[..., 1::2] << 4), meta


def boxes_of(k, page):
    """k [n, Hkv, d] -> [pages, Hkv, 2, d]"""
    return torch.stack([torch.stack([x.amax(0), x.amin(0)], 1) for x in k.split(page)]) if k.shape[0] else k.new_zeros((0, k.shape[1], 2, k.shape[2]))


def span(n, nq, i, qblock, page, causal):
    """Pages [lo, hi) of a block's own positions, and pages it can list."""
    t0, t1 = i * qblock, min(nq, (i + 1) * qblock)
    if t0 >= nq:
        return 0, 0, 0
    if not causal:
        return 0, 0, -(-n // page)
    first, last = max(n - nq + t0, 0), n - nq + t1 - 1
    return (first // page, last // page + 1, last // page + 1) if last >= 0 else (0, 0, 0)


def select(q, boxes, n, nq, Hkv, page, qblock, topk, keep_first, causal):
    """q [nq, Hq, d], boxes [pages, Hkv, 2, d] of one sequence -> list of lists of pages [blocks][Hkv]."""
    q, boxes = q.double(), boxes.double()
    G = q.shape[1] // Hkv
    out = []
    for i in range(-(-nq // qblock)):
        lo, hi, seen = span(n, nq, i, qblock, page, causal)
        u = q[i * qblock:(i + 1) * qblock].sum(0)
        lists = []
        for g in range(Hkv):
            forced = set(range(lo, hi)) | set(range(min(keep_first, seen)))
            scored = []
            for p in range(seen):
                if p not in forced:
                    w = u[g * G:(g + 1) * G]
                    s = (w * torch.where(w >= 0, boxes[p, g, 0], boxes[p, g, 1])).sum(-1)
                    s = torch.where(s.isnan(), torch.full_like(s, -math.inf), s).max().item()
                    scored.append((-s, p))
            scored.sort()
            lists.append(sorted(list(forced) + [p for _, p in scored[:topk - len(forced)]]))
        out.append(lists)
    return out


def sees(lists, n, nq, Hkv, page, qblock, causal, there=None):
    """[nq, Hkv, n]: what every query may look at.  lists None: all pages.  there [n]: keys that exist at all."""
    m = torch.zeros((nq, Hkv, n), dtype=torch.bool)
    for t in range(nq):
        for g in range(Hkv):
            if lists is None:
                m[t, g] = True
            else:
                for p in lists[t // qblock][g]:
                    m[t, g, p * page:(p + 1) * page] = True
        if causal:
            m[t, :, max(0, n - nq + t + 1):] = False
    if there is not None:
        m &= there
    return m


def attend(q, k, v, see, scale, dtype, kabs=None, vabs=None, d_o=None):
    """q [nq,Hq,d], k, v [n,Hkv,d], see [nq,Hkv,n] -> dict of values and `_tol` bounds.  kabs, vabs: what enters the products."""
    q, k, v = q.double(), k.double(), v.double()
    nq, Hq, d = q.shape
    n, Hkv = k.shape[0], k.shape[1]
    G = Hq // Hkv
    kabs = k.abs() if kabs is None else kabs
    vabs = v.abs() if vabs is None else vabs
    h = half(dtype)
    hr = h if dtype == torch.bfloat16 else 0.0                # weights are rounded in 16 bits only
    r = {}
    out = {x: torch.zeros_like(q) for x in ("o", "o_tol", "dq", "dq_tol")}
    out["lse"], out["lse_tol"] = torch.full((nq, Hq), -math.inf, dtype=torch.float64), torch.zeros((nq, Hq), dtype=torch.float64)
    for x in ("dk", "dk_tol", "dv", "dv_tol"):
        out[x] = torch.zeros_like(k)
    for hq in range(Hq):
        g = hq // G
        K, V, S = k[:, g], v[:, g], see[:, g]
        s = (q[:, hq] @ K.T) * scale
        es = (d + 8) * U * scale * (q[:, hq].abs() @ kabs[:, g].T)
        s = torch.where(S, s, -math.inf)
        es = torch.where(S, es, 0.0).amax(1, keepdim=True) if n else torch.zeros((nq, 1), dtype=torch.float64)
        top = s.amax(1, keepdim=True) if n else torch.full((nq, 1), -math.inf, dtype=torch.float64)
        top = torch.where(top == -math.inf, 0.0, top)
        e = (s - top).exp()
        tot = e.sum(1, keepdim=True)
        P = e / torch.where(tot == 0, 1.0, tot)
        ew = 2 * es + (n + 64) * U * 4
        o = P @ torch.where(S.any(0)[:, None], V, 0.0)
        out["o"][:, hq] = o
        out["o_tol"][:, hq] = (ew + hr) * 1.01 * (P @ torch.where(S.any(0)[:, None], vabs[:, g], 0.0)) + h * 1.01 * o.abs()
        out["lse"][:, hq] = torch.where(tot > 0, top + tot.log(), -math.inf)[:, 0]
        out["lse_tol"][:, hq] = (es + (n + 64) * U * 4 + 8 * U * torch.where(tot > 0, top.abs() + tot.log().abs(), 0.0))[:, 0]
        if d_o is None:
            continue
        D = d_o[:, hq].double()
        dP = D @ V.T
        dPa = D.abs() @ V.abs().T
        delta = (D * o).sum(1, keepdim=True)
        dtol = (D.abs() * (out["o_tol"][:, hq] + h * o.abs())).sum(1, keepdim=True) + (d + 8) * U * (D * o).abs().sum(1, keepdim=True)
        dS = torch.where(S, P * (dP - delta), 0.0)
        # P again from scores and lse: an error of es and of lse's; dP from products of d terms; delta from the rounded o; rounded itself
        ep = 2 * es + out["lse_tol"][:, hq:hq + 1] + (n + 64) * U * 4
        dStol = torch.where(S, P * (ep * (dP - delta).abs() + (d + 8) * U * dPa + dtol), 0.0) * 1.02 + (hr + 4 * U) * dS.abs()
        acc = (n + nq * G + 64) * U
        out["dq"][:, hq] = scale * dS @ K
        out["dq_tol"][:, hq] = (scale * (dStol + acc * dS.abs()) @ K.abs()) * 1.01 + h * 1.01 * out["dq"][:, hq].abs()
        out["dk"][:, g] += scale * dS.T @ q[:, hq]
        out["dk_tol"][:, g] += scale * (dStol + acc * dS.abs()).T @ q[:, hq].abs() * 1.01
        out["dv"][:, g] += P.T @ D
        out["dv_tol"][:, g] += (P * (ep + hr + acc)).T @ D.abs() * 1.01
    for x in ("dk", "dv"):
        out[x + "_tol"] += h * 1.01 * out[x].abs()
    return out

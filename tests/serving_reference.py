"""Plain float64 forms of the serving operators, and page pools to try them on."""
import math

import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a step of a rounding, relative


def make_pools(rng, lens_cap, page, g, d, dtype, device, layout="slots", spare=3, seqs=None):
    """Pools [n_pages, page, g, d] of NaN (a test writes what may be read), and a table of distinct pages in no order.
    layout: 'slots' page-major with the heads innermost, 'heads' one run of slots per head, 'mixed' K and V side by side."""
    seqs = len(lens_cap) if seqs is None else seqs
    max_pages = max(1, max(-(-n // page) for n in lens_cap))
    n_pages = seqs * max_pages + spare
    nan = float("nan")
    if layout == "slots":
        k = torch.full((n_pages, page, g, d), nan, dtype=dtype, device=device)
        v = torch.full((n_pages, page, g, d), nan, dtype=dtype, device=device)
    elif layout == "heads":
        k = torch.full((n_pages, g, page, d), nan, dtype=dtype, device=device).transpose(1, 2)
        v = torch.full((n_pages, g, page, d), nan, dtype=dtype, device=device).transpose(1, 2)
    else:
        kv = torch.full((n_pages, page, 2 * g, d), nan, dtype=dtype, device=device)
        k, v = kv[:, :, :g], kv[:, :, g:]
    table = torch.from_numpy(rng.permutation(n_pages)[:seqs * max_pages].astype(np.int32).reshape(seqs, max_pages)).to(device)
    return k, v, table


def slots_of(table, s, n, page):
    """(page, slot) index tensors of the first n positions of sequence s."""
    j = torch.arange(n, device=table.device)
    return table[s, j // page].long(), j % page


def rotate(x, pos, rot, base, interleaved):
    """x [n, heads, d] float64 numpy, rotated by position."""
    x = x.copy()
    for i in range(rot // 2):
        a = np.asarray(pos, dtype=np.float64) * base ** (-2.0 * i / rot)
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        x0, x1 = x[:, :, lo].copy(), x[:, :, hi].copy()
        x[:, :, lo], x[:, :, hi] = x0 * c - x1 * s, x1 * c + x0 * s
    return x


def attention(q, k, v, table, lens, page, n_q, scale, bias):
    """(out, lse, tolerance of out, tolerance of lse) in float64; the tolerances count the roundings of a float32
    evaluation with one rounding to the output type at the end."""
    R, H, d = q.shape
    G = k.shape[2]
    m = H // G
    dev = q.device
    out = torch.zeros(R, H, d, dtype=torch.float64, device=dev)
    lse = torch.full((R, H), -math.inf, dtype=torch.float64, device=dev)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    eps = 2.0 ** -24
    for r in range(R):
        n = int(lens[r])
        if n <= 0:
            continue
        pg, sl = slots_of(table, r // n_q, n, page)
        kk, vv = k[pg, sl].double(), v[pg, sl].double()              # [n, G, d]
        qq = q[r].double().view(G, m, d)
        z = torch.einsum("gmd,ngd->gmn", qq, kk) * scale
        size = torch.einsum("gmd,ngd->gmn", qq.abs(), kk.abs()) * abs(scale)
        if bias is not None:
            nb = bias.shape[1]
            at = (nb - 1 - (n - 1 - torch.arange(n, device=dev))).clamp(min=0)
            b = bias.double()[:, at].view(G, m, n)
            z = z + b
            size = size + torch.where(b.abs() < 1e30, b.abs(), 0.0)
        top = z.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = torch.exp(z - top)
        total = p.sum(-1, keepdim=True)
        w = p / torch.where(total > 0, total, torch.ones_like(total))
        o = torch.einsum("gmn,ngd->gmd", w, vv)
        # a score: d products and sums, the scale, the bias; the distance to the maximum is rounded once more, then
        # multiplied and exponentiated (2 ulp); sums over n keys; a factor for every time the maximum moves
        ds = (d + 4) * eps * torch.where(p > 0, size, 0.0).amax(-1, keepdim=True) + \
            4 * eps * torch.where(p > 1e-30, (z - top).abs(), 0.0).amax(-1, keepdim=True)
        rel = 2 * ds + (math.sqrt(n) * 4 + 16) * eps
        if q.dtype == torch.bfloat16:
            rel = rel + 2.0 ** -16      # weights of the matrix product as a sum of two bfloat16 parts
        mag = torch.einsum("gmn,ngd->gmd", w, vv.abs())
        out[r] = o.reshape(H, d)
        lse[r] = (torch.log(total) + top).reshape(H)
        tol[r] = (HALF[q.dtype] * o.abs() * (1 + 2.0 ** -7) + rel * mag).reshape(H, d) + 1e-37
        ltol[r] = (rel.squeeze(-1) + 4 * eps * (lse[r].abs().view(G, m) + 1)).reshape(H)
    return out, lse, tol, ltol


def verify(target, draft, tokens, n_draft, u_accept, u_sample):
    """numpy float64 arrays; returns (out tokens, accepted)."""
    S, K1, V = target.shape
    K = K1 - 1

    def clean(r):
        return np.where(np.isfinite(r) & (r > 0), r, 0.0)

    out, acc = np.full((S, K1), -1, np.int32), np.zeros(S, np.int32)
    for s in range(S):
        n = K if n_draft is None else min(max(int(n_draft[s]), 0), K)
        a = 0
        while a < n:
            x = int(tokens[s, a])
            if not 0 <= x < V:
                break
            q = 1.0 if draft is None else draft[s, a, x]
            if not float(u_accept[s, a]) * q < target[s, a, x]:
                break
            out[s, a] = x
            a += 1
        acc[s] = a
        r = clean(target[s, a])
        if a < n:
            with np.errstate(invalid="ignore"):
                if draft is not None:
                    left = clean(target[s, a] - draft[s, a])
                else:
                    left = r.copy()
                    if 0 <= tokens[s, a] < V:
                        left[tokens[s, a]] = 0.0
            if left.sum() > 0:
                r = left
        if r.sum() > 0:
            reach = np.cumsum(r) > float(u_sample[s]) * r.sum()
            out[s, a] = int(np.argmax(reach)) if reach.any() else int(np.max(np.nonzero(r)))
    return out, acc

"""Measured cases of the serving operators: a paged key / value cache, the attention that reads it, and the
verification of drafted tokens.

With `own` false `run` computes an operator from elementary torch operations (float32, float64 where float32 loses
what matters); with `own` true it makes the call a user of the library makes.  Page pools are
[n_pages, page_size, kv heads, d_kv]; a page table row lists the pages of one sequence in order.

  append     token t of sequence s at position p goes to slot p % page_size of page table[s, p // page_size]; with
             rot_dim > 0 the first rot_dim columns of every head of k (and q) are first rotated in pairs by the angle
             p * base^(-2 i / rot_dim).  Position -1 is padding: nothing is written.
  attention  out[r, h] = sum_{j < len_r} softmax_j(scale q[r, h].k_j + bias[h, distance]) v_j with distance
             len_r - 1 - j, saturating at the last one the bias vector holds; a row with len 0 is zero.
  verify     drafted token x_i is accepted while u_i draft_i(x_i) < target_i(x_i); the token behind the last accepted
             one is drawn with one more random number from max(target - draft, 0), or from target behind the last draft.
"""
import math
import random

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the smallest append: one new token of four short sequences in the float32 validation mode
        dict(name="append_token_tiny_f32", op="append", dtype="f32", seqs=4, new=1, heads=4, kv_heads=4, d_kv=32, page=16,
             max_len=64, rot=0, interleaved=False, with_q=False),
        # one decoding step of a large batch, the XL head layout, relative-position bias (so no rotation)
        dict(name="append_token_xl", op="append", dtype="bf16", seqs=256, new=1, heads=32, kv_heads=32, d_kv=64, page=16,
             max_len=512, rot=0, interleaved=False, with_q=False),
        # prompts of a rotary decoder-only model entering the cache: ragged rows with padded tails, queries on the way
        dict(name="append_prompt_declm", op="append", dtype="bf16", seqs=16, new=2048, heads=16, kv_heads=16, d_kv=128,
             page=64, max_len=2048, rot=128, interleaved=False, with_q=True),
        # the smallest attention call: latency alone
        dict(name="attention_tiny_f32", op="attention", dtype="f32", seqs=4, n_q=1, heads=4, kv_heads=4, d_kv=32, page=16,
             max_len=32, bias=32, padded=False),
        # one user of the XL decoder
        dict(name="attention_one_row_xl", op="attention", dtype="bf16", seqs=1, n_q=1, heads=32, kv_heads=32, d_kv=64,
             page=16, max_len=512, bias=128, padded=False),
        # a continuous batch of the XL decoder: ragged lengths, some slots of the batch free
        dict(name="attention_batch_xl", op="attention", dtype="bf16", seqs=128, n_q=1, heads=32, kv_heads=32, d_kv=64,
             page=16, max_len=512, bias=128, padded=True),
        # long contexts of the decoder-only model, few rows: the cache's length is what is split
        dict(name="attention_long_declm", op="attention", dtype="bf16", seqs=8, n_q=1, heads=16, kv_heads=16, d_kv=128,
             page=64, max_len=65536, bias=0, padded=False),
        # query heads that share key / value heads
        dict(name="attention_shared_heads", op="attention", dtype="bf16", seqs=64, n_q=1, heads=32, kv_heads=4, d_kv=128,
             page=32, max_len=8192, bias=0, padded=True),
        # four drafted tokens and the one before them scored in one pass; pages that end inside a tile
        dict(name="attention_draft_declm", op="attention", dtype="bf16", seqs=16, n_q=5, heads=16, kv_heads=16, d_kv=128,
             page=24, max_len=4000, bias=128, padded=False),
        # one user, four drafted tokens
        dict(name="verify_one", op="verify", dtype="f32", seqs=1, n_draft=4, vocab=32128, with_draft=True, ragged=False),
        # a batch with drafts of several lengths
        dict(name="verify_batch", op="verify", dtype="f32", seqs=64, n_draft=5, vocab=32128, with_draft=True, ragged=True),
        # drafts without probabilities of their own (looked up in the prompt), probabilities stored in bfloat16
        dict(name="verify_lookup_bf16", op="verify", dtype="bf16", seqs=256, n_draft=8, vocab=32128, with_draft=False,
             ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "verify"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d_kv = rng.choice([32, 64, 64, 128, 128])
    kv_heads = _log_int(rng, 1, 32)
    group = rng.choice([1, 1, 2, 3, 4, 8])
    if kv_heads * group > 64:
        group = 1
    page = rng.choice([1, 8, 16, 16, 24, 32, 64, 100, 128])
    if op == "append":
        seqs, new = _log_int(rng, 1, 256), rng.choice([1, 1, 5, _log_int(rng, 2, 2048)])
        while seqs * new * (2 * kv_heads + kv_heads * group) * d_kv > 16 * 2048 * 48 * 128 // 2:
            seqs = max(1, seqs // 2)
            new = new if seqs > 1 else max(1, new // 2)
        rot = rng.choice([0, d_kv, d_kv, d_kv // 2, 16])
        return dict(op=op, dtype=dtype, seqs=seqs, new=new, heads=kv_heads * group, kv_heads=kv_heads, d_kv=d_kv, page=page,
                    max_len=new + _log_int(rng, 1, 4096), rot=rot, interleaved=rng.random() < 0.5,
                    with_q=rng.random() < 0.5)
    if op == "attention":
        seqs, n_q = _log_int(rng, 1, 256), rng.choice([1, 1, 1, 2, 4, 5, 8])
        max_len = _log_int(rng, 1, 65536)
        while seqs * max_len * kv_heads * d_kv * (2 if dtype == "f32" else 1) > 8 * 65536 * 16 * 128 // 2:
            seqs, max_len = (seqs // 2, max_len) if seqs > 1 else (1, max_len // 2)
        return dict(op=op, dtype=dtype, seqs=seqs, n_q=n_q, heads=kv_heads * group, kv_heads=kv_heads, d_kv=d_kv, page=page,
                    max_len=max_len, bias=rng.choice([0, 1, 32, 128, 500]), padded=rng.random() < 0.5)
    vocab = rng.choice([512, 1000, 32128, 32128, 50000, _log_int(rng, 300, 130000)])
    seqs, n_draft = _log_int(rng, 1, 256), rng.choice([0, 1, 2, 4, 5, 8])
    while seqs * (n_draft + 1) * vocab > 256 * 9 * 32128 // 2:
        seqs = max(1, seqs // 2)
    return dict(op=op, dtype=dtype, seqs=seqs, n_draft=n_draft, vocab=vocab, with_draft=rng.random() < 0.7,
                ragged=rng.random() < 0.5)


def _lengths(c):
    """Cache lengths of the sequences: a property of the case, not of the seed, so that its work is known."""
    rng = random.Random("%s %s %s %s" % (c["op"], c["seqs"], c["max_len"], c["page"]))
    lens = [rng.randint(max(1, c["max_len"] // 8), c["max_len"]) for _ in range(c["seqs"])]
    lens[0] = c["max_len"]
    if c.get("padded"):
        lens = [0 if i % 7 == 3 else n for i, n in enumerate(lens)]
    return lens


def _new_tokens(c):
    """How many of the `new` token slots of each sequence are real (the rest is padding)."""
    if c["new"] <= 8:
        return [c["new"]] * c["seqs"]
    rng = random.Random("%s %s" % (c["seqs"], c["new"]))
    return [c["new"] if i == 0 else rng.randint((c["new"] + 1) // 2, c["new"]) for i in range(c["seqs"])]


# ----------------------------------------------------------------------------------------------------------- inputs
def _pool(c, g, need_tokens):
    """Page pools and a page table whose pages lie in no order; the last page belongs to nobody."""
    ps = c["page"]
    max_pages = -(-need_tokens // ps)
    n_pages = c["seqs"] * max_pages + 1
    dt = TYPES[c["dtype"]]
    shape = (n_pages, ps, c["kv_heads"], c["d_kv"])
    k = torch.randn(shape, generator=g, device=DEV, dtype=dt)
    v = torch.randn(shape, generator=g, device=DEV, dtype=dt)
    table = torch.randperm(n_pages - 1, generator=g, device=DEV).to(torch.int32).view(c["seqs"], max_pages)
    return k, v, table


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = TYPES[c["dtype"]]
    s = dict(case=c)
    if c["op"] == "append":
        n, H, G, d = c["seqs"] * c["new"], c["heads"], c["kv_heads"], c["d_kv"]
        s["k_pages"], s["v_pages"], s["table"] = _pool(c, g, c["max_len"])
        # q, k, v as one projection leaves them: a row per token, heads as column blocks
        qkv = torch.randn(n, (H + 2 * G) * d, generator=g, device=DEV, dtype=dt)
        s["q"] = qkv[:, :H * d].view(n, H, d) if c["with_q"] else None
        s["k"] = qkv[:, H * d:(H + G) * d].view(n, G, d)
        s["v"] = qkv[:, (H + G) * d:].view(n, G, d)
        s["q_out"] = torch.empty(n, H, d, device=DEV, dtype=dt) if c["with_q"] else None
        real = torch.tensor(_new_tokens(c), device=DEV).view(-1, 1)
        start = torch.tensor([random.Random("%d %d" % (seed, i)).randint(0, c["max_len"] - c["new"])
                              for i in range(c["seqs"])], device=DEV).view(-1, 1)
        at = torch.arange(c["new"], device=DEV).view(1, -1)
        s["positions"] = torch.where(at < real, start + at, -1).to(torch.int32).view(-1)
        s["seq_of_token"] = torch.arange(c["seqs"], device=DEV, dtype=torch.int32).repeat_interleave(c["new"])
    elif c["op"] == "attention":
        R, H, d = c["seqs"] * c["n_q"], c["heads"], c["d_kv"]
        s["k_pages"], s["v_pages"], s["table"] = _pool(c, g, c["max_len"])
        s["q"] = torch.randn(R, H, d, generator=g, device=DEV, dtype=dt)
        last = torch.tensor(_lengths(c), device=DEV).view(-1, 1)
        back = torch.arange(c["n_q"] - 1, -1, -1, device=DEV).view(1, -1)
        s["lens"] = (last - back).clamp(min=0).to(torch.int32).view(-1)
        s["bias"] = None
        if c["bias"]:
            # a table of 32 buckets over logarithmic distances, laid out by distance, the far end first
            dist = torch.arange(c["bias"] - 1, -1, -1, device=DEV, dtype=torch.float64)
            far = 16 + (torch.log(dist.clamp(min=1) / 16) / math.log(128 / 16) * 16).floor().long()
            bucket = torch.where(dist < 16, dist.long(), far.clamp(max=31))
            s["bias"] = torch.randn(H, 32, generator=g, device=DEV)[:, bucket].contiguous()
        s["out"] = torch.empty(R, H, d, device=DEV, dtype=dt)
        s["lse"] = torch.empty(R, H, device=DEV, dtype=torch.float32)
    else:
        S, K, V = c["seqs"], c["n_draft"], c["vocab"]
        logits = 2.5 * torch.randn(S, K + 1, V, generator=g, device=DEV)
        s["target"] = torch.softmax(logits, -1).to(dt)
        near = torch.softmax(logits[:, :K] + 0.7 * torch.randn(S, K, V, generator=g, device=DEV), -1).to(dt)
        s["draft"] = near if c["with_draft"] else None
        if K:
            x = torch.multinomial(near.float().view(S * K, V), 1, generator=g).view(S, K)
        else:
            x = torch.zeros(S, 0, device=DEV, dtype=torch.long)
        s["draft_tokens"] = x.to(torch.int32)
        s["n_draft"] = torch.randint(0, K + 1, (S,), generator=g, device=DEV, dtype=torch.int32) if c["ragged"] else None
        s["u_accept"] = torch.rand(S, K, generator=g, device=DEV)
        s["u_sample"] = torch.rand(S, generator=g, device=DEV)
        s["out_tokens"] = torch.empty(S, K + 1, device=DEV, dtype=torch.int32)
        s["n_accepted"] = torch.empty(S, device=DEV, dtype=torch.int32)
    return s


# ---------------------------------------------------------------------------------------------------------- the call
def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2203_17189_b200 import binding as B
        if c["op"] == "append":
            B.t5_paged_kv_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["seq_of_token"], s["positions"],
                                 q=s["q"], q_out=s["q_out"], rot_dim=c["rot"], rot_base=10000.0,
                                 rot_interleaved=c["interleaved"])
            return [s["k_pages"], s["v_pages"]] + ([s["q_out"]] if c["with_q"] else [])
        if c["op"] == "attention":
            if "workspace" not in s:
                n = B.t5_paged_attention_workspace_bytes(c["seqs"] * c["n_q"], c["n_q"], c["heads"], c["kv_heads"], c["d_kv"])
                s["workspace"] = torch.empty(n, device=DEV, dtype=torch.uint8)
            B.t5_paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["out"], s["workspace"],
                                 scale=c["d_kv"] ** -0.5, n_q=c["n_q"], bias=s["bias"], lse=s["lse"])
            return [s["out"], s["lse"]]
        B.t5_verify_draft(s["target"], s["draft"], s["draft_tokens"], s["n_draft"], s["u_accept"], s["u_sample"],
                          s["out_tokens"], s["n_accepted"])
        return [s["out_tokens"], s["n_accepted"]]
    return {"append": _append, "attention": _attention, "verify": _verify}[c["op"]](s, c)


# ------------------------------------------------------------------------------------------------------- plain forms
def _rotate(x, positions, c):
    """x [n, heads, d] float32, its first rot columns rotated in pairs; the angles in float64."""
    r = c["rot"]
    f = 10000.0 ** (-torch.arange(0, r, 2, device=DEV, dtype=torch.float64) / r)
    a = positions.double().clamp(min=0).view(-1, 1, 1) * f
    cos, sin = a.cos().float(), a.sin().float()
    if c["interleaved"]:
        x0, x1 = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([x0 * cos - x1 * sin, x1 * cos + x0 * sin], -1).flatten(-2)
    else:
        x0, x1 = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([x0 * cos - x1 * sin, x1 * cos + x0 * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _append(s, c):
    ps, dt = c["page"], TYPES[c["dtype"]]
    pos, seq = s["positions"].long(), s["seq_of_token"].long()
    here = pos.clamp(min=0)
    real = (pos >= 0).view(-1, 1, 1)
    # padding writes back what the unowned last page holds
    page = torch.where(pos >= 0, s["table"][seq, here // ps].long(), s["k_pages"].shape[0] - 1)
    slot = here % ps
    k, q = s["k"].float(), s["q"].float() if c["with_q"] else None
    if c["rot"]:
        k = _rotate(k, pos, c)
        q = _rotate(q, pos, c) if c["with_q"] else None
    k = torch.where(real, k.to(dt), s["k_pages"][page, slot])
    v = torch.where(real, s["v"], s["v_pages"][page, slot])
    s["k_pages"][page, slot] = k
    s["v_pages"][page, slot] = v
    return [s["k_pages"], s["v_pages"]] + ([q.to(dt)] if c["with_q"] else [])


def _attention(s, c):
    S, n_q, H, G, d = c["seqs"], c["n_q"], c["heads"], c["kv_heads"], c["d_kv"]
    m = H // G
    table = s["table"].long()
    k = s["k_pages"][table].view(S, -1, G, d).permute(0, 2, 3, 1).float()       # [S, G, d, L]
    v = s["v_pages"][table].view(S, -1, G, d).transpose(1, 2).float()           # [S, G, L, d]
    L = v.shape[2]
    q = s["q"].float().view(S, n_q, G, m, d).transpose(1, 2).reshape(S, G, n_q * m, d)
    z = (q @ k).view(S, G, n_q, m, L) * d ** -0.5
    dist = s["lens"].long().view(S, n_q, 1) - 1 - torch.arange(L, device=DEV)   # [S, n_q, L]
    if c["bias"]:
        at = (c["bias"] - 1 - dist).clamp(0, c["bias"] - 1)
        z = z + s["bias"].view(G, m, -1)[:, :, at].permute(2, 0, 3, 1, 4)
    z = z.masked_fill((dist < 0)[:, None, :, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    lse = torch.log(total) + top
    p = p / torch.where(total > 0, total, 1.0)
    o = (p.view(S, G, n_q * m, L) @ v).view(S, G, n_q, m, d).transpose(1, 2).reshape(S * n_q, H, d)
    return [o.to(TYPES[c["dtype"]]), lse.squeeze(-1).transpose(1, 2).reshape(S * n_q, H).contiguous()]


def _verify(s, c):
    S, K, V = c["seqs"], c["n_draft"], c["vocab"]
    x = s["draft_tokens"].long()
    n = s["n_draft"].long() if c["ragged"] else torch.full((S,), K, device=DEV)
    p = s["target"][:, :K].gather(2, x.unsqueeze(2)).squeeze(2).double()
    q = s["draft"].gather(2, x.unsqueeze(2)).squeeze(2).double() if c["with_draft"] else torch.ones_like(p)
    ok = (s["u_accept"].double() * q < p) & (torch.arange(K, device=DEV) < n.view(-1, 1))
    a = ok.long().cumprod(1).sum(1)                                             # accepted drafts
    rows = torch.arange(S, device=DEV)
    r = s["target"][rows, a].double()
    if K:
        at = a.clamp(max=K - 1)
        refused = (a < n).view(-1, 1)
        if c["with_draft"]:
            left = (r - s["draft"][rows, at].double()).clamp(min=0)
        else:
            left = r.masked_fill(torch.arange(V, device=DEV) == x[rows, at].view(-1, 1), 0)
        r = torch.where(refused, left, r)
    mass = r.cumsum(1)
    t = s["u_sample"].double().view(-1, 1) * mass[:, -1:]
    last = (mass <= t).sum(1).clamp(max=V - 1)
    at = torch.arange(K + 1, device=DEV)
    kept = torch.cat([x, torch.zeros_like(x[:, :1]) if K else torch.zeros(S, 1, device=DEV, dtype=torch.long)], 1)
    tokens = torch.where(at < a.view(-1, 1), kept, torch.where(at == a.view(-1, 1), last.view(-1, 1), -1))
    return [tokens.to(torch.int32), a.to(torch.int32)]


# ------------------------------------------------------------------------------------------------------------- work
def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "append":
        tokens = sum(_new_tokens(c))
        cols = (2 * c["kv_heads"] + (c["heads"] if c["with_q"] else 0)) * c["d_kv"]
        turned = (c["kv_heads"] + (c["heads"] if c["with_q"] else 0)) * c["rot"]
        return {"bytes": tokens * (2 * cols * es + 12), "flops": tokens * turned * 3}
    if c["op"] == "attention":
        keys, rows = sum(_lengths(c)), c["seqs"] * c["n_q"]
        cache = keys * c["kv_heads"] * c["d_kv"] * 2 * es
        return {"bytes": cache + rows * c["heads"] * (c["d_kv"] * 2 * es + 4) + 4 * keys // c["page"] + c["heads"] * c["bias"] * 4,
                "flops": 4 * keys * c["n_q"] * c["heads"] * c["d_kv"]}
    # one row of target and, where drafts have probabilities, one of draft per sequence; two values per drafted token
    rows = c["seqs"] * c["vocab"] * es * (2 if c["with_draft"] and c["n_draft"] else 1)
    return {"bytes": rows + c["seqs"] * (c["n_draft"] * (2 * es + 12) + 16), "flops": 2 * c["seqs"] * c["vocab"]}


# ------------------------------------------------------------------------------------------------------------ exact
def exact(case, seed):
    """The definitions in float64, sequence by sequence."""
    c, s = case, prepare(case, seed)
    if c["op"] == "append":
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        pos, seq = s["positions"].tolist(), s["seq_of_token"].tolist()
        real = [i for i, p in enumerate(pos) if p >= 0]
        table = s["table"].tolist()
        page = torch.tensor([table[seq[i]][pos[i] // c["page"]] for i in real], device=DEV)
        slot = torch.tensor([pos[i] % c["page"] for i in real], device=DEV)

        def turn(x):
            x = x.double().clone()
            for i in range(c["rot"] // 2):
                a = torch.tensor([max(p, 0) * 10000.0 ** (-2 * i / c["rot"]) for p in pos], device=DEV,
                                 dtype=torch.float64).view(-1, 1)
                lo, hi = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + c["rot"] // 2)
                x0, x1 = x[..., lo].clone(), x[..., hi].clone()
                x[..., lo], x[..., hi] = x0 * a.cos() - x1 * a.sin(), x0 * a.sin() + x1 * a.cos()
            return x
        at = torch.tensor(real, device=DEV)
        kp[page, slot] = turn(s["k"])[at]
        vp[page, slot] = s["v"].double()[at]
        return [kp, vp] + ([turn(s["q"])] if c["with_q"] else [])
    if c["op"] == "attention":
        G, m, d, ps = c["kv_heads"], c["heads"] // c["kv_heads"], c["d_kv"], c["page"]
        lens = s["lens"].tolist()
        out = torch.zeros(len(lens), c["heads"], d, device=DEV, dtype=torch.float64)
        lse = torch.full((len(lens), c["heads"]), -math.inf, device=DEV, dtype=torch.float64)
        for r, n in enumerate(lens):
            if n == 0:
                continue
            pages = s["table"][r // c["n_q"], :-(-n // ps)].long()
            at = torch.tensor([max(c["bias"] - 1 - i, 0) for i in range(n - 1, -1, -1)], device=DEV)
            for g in range(G):
                k = s["k_pages"][pages, :, g].reshape(-1, d)[:n].double()
                v = s["v_pages"][pages, :, g].reshape(-1, d)[:n].double()
                z = s["q"][r, g * m:(g + 1) * m].double() @ k.T / math.sqrt(d)
                if c["bias"]:
                    z = z + s["bias"][g * m:(g + 1) * m].double()[:, at]
                lse[r, g * m:(g + 1) * m] = torch.logsumexp(z, 1)
                out[r, g * m:(g + 1) * m] = torch.softmax(z, 1) @ v
        return [out, lse]
    S, K, V = c["seqs"], c["n_draft"], c["vocab"]
    tokens, accepted = torch.full((S, K + 1), -1, dtype=torch.int32), torch.zeros(S, dtype=torch.int32)
    x, u = s["draft_tokens"].tolist(), s["u_accept"].tolist()
    n = s["n_draft"].tolist() if c["ragged"] else [K] * S
    for b in range(S):
        a = 0
        left = s["target"][b, 0].double()
        while a < n[b]:
            given = s["draft"][b, a].double() if c["with_draft"] else (torch.arange(V, device=DEV) == x[b][a]).double()
            if not u[b][a] * given[x[b][a]].item() < left[x[b][a]].item():
                left = (left - given).clamp(min=0)
                if not c["with_draft"]:
                    left = s["target"][b, a].double() * (1 - given)
                break
            tokens[b, a] = x[b][a]
            a += 1
            left = s["target"][b, a].double()
        mass = left.cumsum(0)
        where = mass > s["u_sample"][b].double() * mass[-1]
        tokens[b, a] = where.long().argmax().item()
        accepted[b] = a
    return [tokens, accepted]

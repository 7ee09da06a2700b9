"""Performance cases of the paged VQ cache: the three calls that a server makes in every step of continuous batching.

``assign`` gives the new tokens of every request pages of the pool (block tables, slot maps), ``append`` quantizes their keys and
values into those pages, ``attend`` is the attention of the new tokens over the pages.  Head counts are those of the repository's
benchmark cache (32 heads of 128 channels) and of grouped-query variants of it (8 cache heads), head size 64 among the drawn ones;
codebooks are one per head and side (G = 1) or one per sub-space (coupled quantization).  Codes are uniform, codebooks, keys,
values and queries normal: the distributions of ``paper_2503_02236_amd.workloads``.
"""
import math

import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # ---- pages, block tables, slot maps
        # a decode step of sixteen requests: a token each
        {"name": "assign_decode", "op": "assign", "B": 16, "chunks": 0, "chunk": 1, "released": 0, "T": 4096, "ps": 16},
        # a mixed step of a busy server: eight chunks of prompts, 240 decoding requests, some that ended
        {"name": "assign_mixed", "op": "assign", "B": 256, "chunks": 8, "chunk": 1000, "released": 8, "T": 9000, "ps": 16},
        # prompts of a large batch job
        {"name": "assign_prompts", "op": "assign", "B": 700, "chunks": 64, "chunk": 1024, "released": 100, "T": 8192, "ps": 32},
        # ---- keys and values into the pages
        # the smallest: the new token of one request
        {"name": "append_one", "op": "append", "B": 1, "n": 1, "H": 32, "D": 128, "v": 4, "E": 256, "G": 1, "T": 1000, "ps": 16},
        # a decode step of 64 requests on a coupled-quantization cache
        {"name": "append_cq_b64", "op": "append", "B": 64, "n": 1, "H": 8, "D": 128, "v": 4, "E": 256, "G": 32, "T": 2000, "ps": 16},
        # a chunk of two prompts
        {"name": "append_prompt", "op": "append", "B": 2, "n": 2047, "H": 32, "D": 128, "v": 4, "E": 256, "G": 1, "T": 5000, "ps": 32},
        # ---- attention over the pages
        # the smallest: one request of a few hundred tokens, one new token
        {"name": "attend_one", "op": "attend", "B": 1, "n": 1, "chunks": 0, "chunk": 0, "H": 32, "group": 1, "D": 128, "v": 4, "E": 256, "G": 1,
         "T": 300, "ps": 16, "window": 0, "cap": 0.0, "bias": False, "prefix": 0},
        # a decode step of sixteen requests of up to 4096 tokens
        {"name": "attend_decode", "op": "attend", "B": 16, "n": 1, "chunks": 0, "chunk": 0, "H": 32, "group": 1, "D": 128, "v": 4, "E": 256, "G": 1,
         "T": 4096, "ps": 16, "window": 0, "cap": 0.0, "bias": False, "prefix": 0},
        # drafted tokens of long requests on a coupled-quantization cache, grouped queries
        {"name": "attend_drafts", "op": "attend", "B": 12, "n": 5, "chunks": 0, "chunk": 0, "H": 8, "group": 4, "D": 128, "v": 4, "E": 256, "G": 32,
         "T": 30000, "ps": 64, "window": 0, "cap": 0.0, "bias": False, "prefix": 0},
        # a mixed step: a chunk of a prompt among decoding requests, a model with capped scores and a sliding window
        {"name": "attend_mixed", "op": "attend", "B": 25, "n": 1, "chunks": 1, "chunk": 500, "H": 8, "group": 4, "D": 128, "v": 4, "E": 256, "G": 1,
         "T": 6001, "ps": 16, "window": 4096, "cap": 50.0, "bias": False, "prefix": 4},
        # a 2048-token chunk of a long prompt, grouped queries
        {"name": "attend_chunk", "op": "attend", "B": 1, "n": 1, "chunks": 1, "chunk": 2048, "H": 8, "group": 4, "D": 128, "v": 4, "E": 256, "G": 1,
         "T": 8192, "ps": 16, "window": 0, "cap": 0.0, "bias": False, "prefix": 0},
        # four whole prompts, 4 bits a value (64 codebooks of 2-vectors), distance bias
        {"name": "attend_prompts", "op": "attend", "B": 4, "n": 1, "chunks": 4, "chunk": 2100, "H": 32, "group": 1, "D": 128, "v": 2, "E": 256, "G": 64,
         "T": 2100, "ps": 32, "window": 0, "cap": 0.0, "bias": True, "prefix": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["assign", "append", "attend", "attend"])
    ps = rng.choice([16, 16, 32, 64, 128])
    if op == "assign":
        B = _log(rng, 1, 700)
        chunks = rng.randint(0, min(B, 64))
        return {"op": op, "B": B, "chunks": chunks, "chunk": _log(rng, 2, 65536 // max(chunks, 1) // 4), "released": rng.randint(0, (B - chunks) // 4),
                "T": _log(rng, 20, 9000), "ps": ps}
    D = rng.choice([128, 128, 128, 64])
    v, G = rng.choice([(4, 1), (4, 1), (4, D // 4), (2, D // 2), (8, 1), (4, 4)])
    E = rng.choice([256, 256, 256, 100])
    if op == "append":
        B, H = _log(rng, 1, 64), rng.choice([4, 8, 32])
        return {"op": op, "B": B, "n": _log(rng, 1, max(1.1, 32768 * v // 4 // (B * H))), "H": H, "D": D, "v": v, "E": E, "G": G, "T": _log(rng, 2100, 5000), "ps": ps}
    most = max(work(k)["bytes"] for k in listed())
    H, group = rng.choice([(32, 1), (8, 4), (8, 8), (4, 7), (5, 3)])
    c = {"op": op, "H": H, "group": group, "D": D, "v": v, "E": E, "G": G, "ps": ps,
         "window": rng.choice([0, 0, _log(rng, 16, 4096)]), "cap": rng.choice([0.0, 0.0, 30.0]), "bias": rng.random() < 0.3, "prefix": rng.choice([0, 0, 4, 700])}
    if rng.random() < 0.5:      # a decode step, or drafted tokens
        c.update(B=_log(rng, 1, 32), n=rng.choice([1, 1, 1, 3, 8]), chunks=0, chunk=0, T=_log(rng, 40, 12000))
    else:                       # chunks of prompts among decoding requests
        c.update(B=_log(rng, 1, 24), n=1, T=_log(rng, 300, 8000))
        c["chunks"] = rng.randint(1, min(c["B"], 3))
        c["chunk"] = _log(rng, 16, min(c["T"], 2048) // c["chunks"])
    while work(c)["bytes"] > most:
        c["T"] = c["T"] * 3 // 4
    return c


# ------------------------------------------------------------------------------------------------ inputs

def _lens(case):
    """(tokens in the cache with the new ones, new tokens) of every request: lengths from T downwards, chunks first."""
    out = []
    B, T = case["B"], case["T"]
    for b in range(B):
        n = case["chunk"] if b < case.get("chunks", 0) else case.get("n", 1)
        if case["op"] == "assign" and b >= B - case["released"]:
            n = -1
        whole = case.get("chunks", 0) == B and case["chunk"] == T     # whole prompts
        ln = T if whole else T - (b * T) // (2 * B) - (b * 7) % 13
        out.append((max(ln, n, 1), n))
    return out


def _pages(g, lens, ps, extra):
    """A pool's pages dealt out at random: block table [B][W] (-1 where a request has no page), number of pages, the pages left."""
    counts = [-(-ln // ps) for ln in lens]
    n_pages = sum(counts) + extra
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    W = max(counts) + 2
    c = torch.tensor(counts, device=DEV)
    start = torch.cumsum(c, 0) - c
    j = torch.arange(W, device=DEV)
    idx = (start[:, None] + j[None]).clamp(max=n_pages - 1)
    table = torch.where(j[None] < c[:, None], perm[idx], torch.full_like(perm[idx], -1))
    return table.contiguous(), n_pages, perm[sum(counts):].contiguous()


def _normal(g, shape, sigma=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * sigma).to(torch.float16)


def _inputs(case, seed):
    """The data of a call: plain tensors on the GPU."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    lens = _lens(case)
    B, ps = case["B"], case["ps"]
    if case["op"] == "assign":
        before = [ln if n < 0 else ln - n for ln, n in lens]
        new = [n for _, n in lens]
        need = sum(-(-ln // ps) - -(-(ln - n) // ps) for ln, n in lens if n > 0)
        counts = [-(-ln // ps) for ln in before]
        table, n_pages, free = _pages(g, [max(ln, 1) for ln in before], ps, need + 5)
        W = max(max(-(-ln // ps) for ln, _ in lens), max(counts)) + 2
        wide = torch.full((B, W), -1, dtype=torch.int32, device=DEV)
        wide[:, :min(W, table.shape[1])] = table[:, :W]
        wide[torch.arange(W, device=DEV)[None] >= i32(counts)[:, None]] = -1
        pool = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
        pool[:free.numel()] = free
        return {"lens": i32(before), "new_lens": i32(new), "table": wide, "free_pages": pool, "n_free": i32([free.numel()]),
                "n_tokens": sum(n for n in new if n > 0) + 3}
    H, D, v, E, G = (case[k] for k in ("H", "D", "v", "E", "G"))
    P = D // v
    table, n_pages, _ = _pages(g, [ln for ln, _ in lens], ps, 3)
    codes = lambda *s: torch.randint(0, E, s, generator=g, device=DEV, dtype=torch.uint8)  # noqa: E731
    s = {"table": table, "k_codes": codes(n_pages, H, ps, P), "v_codes": codes(n_pages, H, ps // 16, P, 16),
         "k_cb": _normal(g, (H, G, E, v)), "v_cb": _normal(g, (H, G, E, v))}
    n_new = [n for _, n in lens]
    cu = [0]
    for n in n_new:
        cu.append(cu[-1] + n)
    if case["op"] == "append":
        qkv = _normal(g, (cu[-1], 3, H, D))      # what a fused projection leaves
        s["k_new"], s["v_new"] = qkv[:, 1], qkv[:, 2]
        at = torch.cat([torch.arange(ln - n, ln, device=DEV) for ln, n in lens])
        row = torch.repeat_interleave(torch.arange(B, device=DEV), torch.tensor(n_new, device=DEV))
        s["slots"] = (table[row, at // ps] * ps + at % ps).to(torch.int32)
        return s
    Hq = H * case["group"]
    s.update(q=_normal(g, (cu[-1], Hq, D)), cu_new=i32(cu), seq_lens=i32([ln for ln, _ in lens]), lens=lens, slopes=None, prefix_lens=None)
    if case["bias"]:
        s["slopes"] = torch.exp2(-8.0 * (torch.arange(Hq, device=DEV, dtype=torch.float32) + 1) / Hq)
    if case["prefix"]:
        s["prefix_lens"] = i32([min(case["prefix"], ln) for ln, _ in lens])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    import paper_2503_02236_amd as vq
    s["vq"] = vq
    if case["op"] == "assign":
        s["plan"] = vq.VQPagePlan(case["B"], s["n_tokens"], DEV)      # the buffers that a step's plan lies in
        s["n_free_out"] = torch.empty_like(s["n_free"])
        return s
    s["kv"] = vq.VQKVPagesDev(case["H"], case["D"], case["v"], case["ps"], s["k_codes"], s["v_codes"], s["k_cb"], s["v_cb"])
    if case["op"] == "attend":
        need = vq.vq_attn_paged_workspace(s["kv"], s["q"], s["table"])
        s["ws"] = vq.new_workspace(need, DEV) if need else None
    return s


# ------------------------------------------------------------------------------------------------ one pass

def _plain_assign(s, ps):
    new, lens, table, n_free = s["new_lens"].long(), s["lens"].long(), s["table"].clone(), s["n_free"].long()
    B, W = table.shape
    cap = s["n_tokens"]
    pages = (lens + ps - 1) // ps
    free = s["free_pages"].clone()
    j = torch.arange(W, device=DEV)
    # requests that ended give their pages back
    gone = new < 0
    back = torch.where(gone, pages, 0)
    at = n_free + torch.cumsum(back, 0) - back
    put = torch.where(j[None] < back[:, None], at[:, None] + j[None], free.numel())
    free = torch.cat([free, free.new_zeros(1)]).scatter(0, put.reshape(-1), table.reshape(-1))[:-1]
    n_free = n_free + back.sum()
    lens = torch.where(gone, 0, lens)
    pages = torch.where(gone, 0, pages)
    # who can be served
    new = torch.where(gone, 0, new)
    fits = (lens + new + ps - 1) // ps <= W
    ask = torch.where(fits, new, 0)
    fits = fits & ((torch.cumsum(ask, 0) <= cap) | (ask == 0))
    need = torch.where(fits, (lens + new + ps - 1) // ps - pages, 0)
    upto = torch.cumsum(need, 0)
    fits = fits & ((upto <= n_free) | (need == 0))
    need = torch.where(fits, need, 0)
    n = torch.where(fits, new, 0)
    first = torch.cumsum(need, 0) - need
    take = (n_free - 1 - first[:, None] - (j[None] - pages[:, None])).clamp(0, free.numel() - 1)
    table = torch.where((j[None] >= pages[:, None]) & (j[None] < (pages + need)[:, None]), free[take], table)
    cu = torch.cat([n.new_zeros(1), torch.cumsum(n, 0)])
    t = torch.arange(cap, device=DEV)
    b = (torch.searchsorted(cu, t, right=True) - 1).clamp(max=B - 1)
    pos = lens[b] + t - cu[b]
    live = t < cu[-1]
    page = table[b, (pos // ps).clamp(0, W - 1)].long()
    slots = torch.where(live, page * ps + pos % ps, -1)
    i32 = torch.int32
    return {"cu_new": cu.to(i32), "seq_lens": (lens + n).to(i32), "slots": slots.to(i32), "positions": torch.where(live, pos, -1).to(i32),
            "status": (~fits).to(i32), "table": table, "free_pages": free, "n_free": (n_free - need.sum()).to(i32)}


def _plain_codes(x, cb, ps, pool, slots, value):
    """Codes of x [n][H][D] into a copy of the pool: fp32, elements in ascending order, the lowest index of the smallest distance."""
    n, H, D = x.shape
    _, G, E, v = cb.shape
    P = D // v
    out = pool.clone()
    page, off = (slots // ps).long(), (slots % ps).long()
    index = torch.arange(E, device=x.device)
    for h in range(H):
        xs, c = x[:, h].float().view(n, G, P // G, 1, v), cb[h].float().view(1, G, 1, E, v)
        d = None
        for i in range(v):
            e = xs[..., i] - c[..., i]
            e = e * e
            d = e if d is None else d + e
        low = d.amin(-1, keepdim=True)
        code = torch.where(d == low, index, E).amin(-1).view(n, P).to(torch.uint8)
        if value:
            out[page, h, off // 16, :, off % 16] = code
        else:
            out[page, h, off] = code
    return out


def _dequantize(codes, cb):
    """Codes [H][T][P] -> values [H][T][P v] of the codebooks [H][G][E][v], in their type."""
    H, T, P = codes.shape
    _, G, E, v = cb.shape
    base = torch.arange(H, device=codes.device)[:, None, None] * (G * E) + (torch.arange(P, device=codes.device) * G // P * E)[None, None]
    return cb.reshape(H * G * E, v)[(codes.long() + base).reshape(-1)].reshape(H, T, P * v)


def _cached(s, b, ln, ps):
    """Codes of the first ln tokens of request b, keys and values, [H][ln][P] each."""
    pages = s["table"][b, :-(-ln // ps)].long()
    k, v = s["k_codes"][pages], s["v_codes"][pages]
    H, P = k.shape[1], k.shape[3]
    k = k.permute(1, 0, 2, 3).reshape(H, -1, P)[:, :ln]
    v = v.permute(1, 0, 2, 4, 3).reshape(H, -1, P)[:, :ln]
    return k, v


def _plain_attend(s, case):
    H, group, D, ps = case["H"], case["group"], case["D"], case["ps"]
    out = torch.empty(s["q"].shape, dtype=torch.float32, device=DEV)
    at = 0
    for b, (ln, n) in enumerate(s["lens"]):
        kc, vc = _cached(s, b, ln, ps)
        K, V = _dequantize(kc, s["k_cb"].float()), _dequantize(vc, s["v_cb"].float())
        q = s["q"][at:at + n].float().view(n, H, group, D).permute(1, 0, 2, 3).reshape(H, n * group, D)
        score = torch.bmm(q, K.transpose(1, 2).contiguous()) * D ** -0.5
        if case["cap"]:
            score = case["cap"] * torch.tanh(score / case["cap"])
        score = score.view(H, n, group, ln)
        pos, t = torch.arange(ln - n, ln, device=DEV)[:, None], torch.arange(ln, device=DEV)[None]
        if case["bias"]:
            score = score - s["slopes"].view(H, 1, group, 1) * (pos - t).abs().float().view(1, n, 1, ln)
        seen = t <= pos
        if case["window"]:
            seen = seen & (t > pos - case["window"])
        if case["prefix"]:
            seen = seen | (t < min(case["prefix"], ln))
        score = torch.where(seen.view(1, n, 1, ln), score, -math.inf)
        p = torch.exp(score - score.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        o = torch.bmm(p.view(H, n * group, ln), V)
        out[at:at + n] = o.view(H, n, group, D).permute(1, 0, 2, 3).reshape(n, H * group, D)
        at += n
    return out.to(torch.float16)


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "assign":
            return _plain_assign(s, case["ps"])
        if op == "append":
            return [_plain_codes(s["k_new"], s["k_cb"], case["ps"], s["k_codes"], s["slots"], False),
                    _plain_codes(s["v_new"], s["v_cb"], case["ps"], s["v_codes"], s["slots"], True)]
        return _plain_attend(s, case)
    vq = s["vq"]
    if op == "assign":
        p = vq.vq_kv_pages_assign(s["new_lens"], s["lens"], s["table"], s["free_pages"], s["n_free"], case["ps"], plan=s["plan"], n_free_out=s["n_free_out"])
        return {"cu_new": p.cu_new, "seq_lens": p.seq_lens, "slots": p.slots, "positions": p.positions, "status": p.status, "table": s["table"],
                "free_pages": s["free_pages"], "n_free": s["n_free_out"]}
    if op == "append":
        vq.vq_kv_quantize_paged(s["kv"], s["k_new"], s["v_new"], s["slots"])
        return [s["k_codes"], s["v_codes"]]
    return vq.vq_attn_paged(s["kv"], s["q"], case["D"] ** -0.5, s["table"], s["cu_new"], s["seq_lens"], ws=s["ws"], window=case["window"],
                            softcap=case["cap"], slopes=s["slopes"], prefix_lens=s["prefix_lens"])


# ------------------------------------------------------------------------------------------------ what it costs, how exact it is

def _visible(case):
    """Pairs of a new token and a cached one that it attends, and cached tokens that anyone attends, of all requests."""
    pairs = touched = 0
    w, pf = case["window"], case["prefix"]
    for ln, n in _lens(case):
        low = max(ln - n - w + 1, 0) if w else 0          # the first token that the first new one sees
        touched += ln - low + min(pf, low)
        for pos in range(ln - n, ln):
            lo = max(pos - w + 1, 0) if w else 0
            pairs += pos + 1 - lo + min(pf, lo) + max(min(pf, ln) - max(pos + 1, lo), 0)
    return pairs, touched


def work(case):
    if case["op"] == "assign":
        B, ps = case["B"], case["ps"]
        lens = _lens(case)
        tokens = sum(n for _, n in lens if n > 0) + 3
        taken = sum(-(-ln // ps) - -(-(ln - n) // ps) for ln, n in lens if n > 0)
        back = sum(-(-ln // ps) for ln, n in lens if n < 0)
        return {"bytes": 4 * (6 * B + 2 * tokens + 2 * taken + 2 * back), "flops": 0}
    H, D, v, E, G = (case[k] for k in ("H", "D", "v", "E", "G"))
    P = D // v
    books = 2 * H * G * E * v * 2
    if case["op"] == "append":
        n = case["B"] * case["n"]
        return {"bytes": books + 2 * n * H * (2 * D + P) + 4 * n, "flops": 2 * n * H * P * E * 2.0 * v}
    pairs, touched = _visible(case)
    n, Hq = sum(k for _, k in _lens(case)), H * case["group"]
    return {"bytes": books + 2 * touched * H * P + 2 * n * Hq * D * 2, "flops": 4.0 * pairs * Hq * D}


def exact(case, seed):
    """The attention by its definition in 64 bits, a head and a few hundred new tokens at a time.  (Codes, tables and counts are whole numbers.)"""
    if case["op"] != "attend":
        return None
    s = _inputs(case, seed)
    H, group, D, v, G, ps = (case[k] for k in ("H", "group", "D", "v", "G", "ps"))
    P = D // v
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    which = torch.arange(P, device=DEV) // (P // G)
    at = 0
    for b, (ln, n) in enumerate(s["lens"]):
        t = torch.arange(ln, device=DEV)
        page, off = s["table"][b].long()[t // ps], t % ps
        for h in range(H):
            kc = s["k_codes"][page, h, off].long()
            vc = s["v_codes"][page, h, off // 16, :, off % 16].long()
            K = s["k_cb"][h].double()[which[None], kc].reshape(ln, D)
            V = s["v_cb"][h].double()[which[None], vc].reshape(ln, D)
            for i0 in range(0, n, 512):
                i = torch.arange(i0, min(n, i0 + 512), device=DEV)
                far = (ln - n + i)[:, None] - t[None]                  # how far back a cached token lies
                hidden = far < 0
                if case["window"]:
                    hidden |= far >= case["window"]
                if case["prefix"]:
                    hidden &= t[None] >= case["prefix"]
                for j in range(h * group, (h + 1) * group):
                    z = s["q"][at + i, j].double() @ K.T / math.sqrt(D)
                    if case["cap"]:
                        z = torch.tanh(z / case["cap"]) * case["cap"]
                    if case["bias"]:
                        z = z - s["slopes"][j].double() * far.abs()
                    out[at + i, j] = torch.softmax(z.masked_fill(hidden, -math.inf), -1) @ V
        at += n
    return out

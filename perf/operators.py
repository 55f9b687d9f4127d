"""What the operators of the paged KV cache are measured on: requests of unequal length that a server steps through
together, instead of the equal sequences of a decode context.

A case names an operator and its sizes:

  plan       pages for the new tokens out of a pool, the pages of ended requests back into it, and for every new token
             its request's first row, its position and its slot in the cache
  append     QK-norm and rotary embedding of the new tokens' queries and keys, keys and values written into their slots
  attention  the new tokens of every request (one token, the rows of a refill, a chunk of a prompt) against the pages of
             that request, causally

Head counts are those of the repository's models (32/8 and 8/2 heads of 128, 4/2 and 16/8 of 64).  Lengths follow a fixed
sequence between a quarter of the largest and the largest, so that the work of a case does not hang on the seed; values and
the order of the pages do.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_EPS, _THETA = 1e-6, 1.0e6
_MOST_SCORES = 4.4e8           # query rows * heads * keys of a drawn case (the largest listed one: 4.5e8) ...
_MOST_PADDED = 1.8e9           # ... and of its padded plain form (1.9e9)


def listed():
    return [
        # A small server's decode step: eight requests, one new token each.
        {"name": "plan_b8", "kind": "plan", "batch": 8, "cached": 900, "new": 1, "chunks": 0, "chunk": 0, "page": 16, "ended": 0,
         "pad": 0, "short": False},
        # A loaded server: most requests refill three tokens, some bring a piece of a prompt, some have ended; rows padded for a graph.
        {"name": "plan_b300_mixed", "kind": "plan", "batch": 300, "cached": 5000, "new": 3, "chunks": 12, "chunk": 511, "page": 16,
         "ended": 9, "pad": 37, "short": False},
        # Very many requests at once with more prompt pieces than the pool has pages for.
        {"name": "plan_b4096_short", "kind": "plan", "batch": 4096, "cached": 2048, "new": 1, "chunks": 64, "chunk": 1000, "page": 32,
         "ended": 100, "pad": 0, "short": True},
        # One layer of the benchmark's batched workload: 32 tokens, fp32 activations and an fp16 cache as the decode context has them.
        {"name": "append_b32", "kind": "append", "rows": 32, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "act": "f32", "kv": "f16",
         "page": 64, "layout": "hnd", "far": 2000, "norm": True, "pad": 0},
        # One layer of a long prompt's chunk, 16-bit activations, far positions.
        {"name": "append_8191", "kind": "append", "rows": 8191, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "act": "bf16", "kv": "bf16",
         "page": 16, "layout": "nhd", "far": 130000, "norm": True, "pad": 9},
        # The small fp32 test model, a chunk of no particular length.
        {"name": "append_f32_777", "kind": "append", "rows": 777, "q_heads": 4, "kv_heads": 2, "head_dim": 64, "act": "f32", "kv": "f32",
         "page": 16, "layout": "hnd", "far": 5000, "norm": False, "pad": 0},
        # One chat user, one token: latency.
        {"name": "attention_b1", "kind": "attention", "batch": 1, "cached": 999, "new": 1, "chunks": 0, "chunk": 0, "q_heads": 32,
         "kv_heads": 8, "head_dim": 128, "q": "bf16", "kv": "bf16", "page": 16, "layout": "nhd", "pad": 0},
        # The refill of a batch of 32 (three tokens each) with the decode context's types: fp32 queries, fp16 cache.
        {"name": "attention_b32_refill", "kind": "attention", "batch": 32, "cached": 2045, "new": 3, "chunks": 0, "chunk": 0,
         "q_heads": 32, "kv_heads": 8, "head_dim": 128, "q": "f32", "kv": "f16", "page": 64, "layout": "hnd", "pad": 4},
        # Long documents: single tokens over up to 16 thousand keys each.
        {"name": "attention_b8_long", "kind": "attention", "batch": 8, "cached": 16500, "new": 1, "chunks": 0, "chunk": 0, "q_heads": 32,
         "kv_heads": 8, "head_dim": 128, "q": "bf16", "kv": "bf16", "page": 32, "layout": "hnd", "pad": 0},
        # A prompt's next piece over what is cached of it: the largest call.
        {"name": "attention_chunk_2000", "kind": "attention", "batch": 1, "cached": 6000, "new": 2000, "chunks": 0, "chunk": 0,
         "q_heads": 32, "kv_heads": 8, "head_dim": 128, "q": "bf16", "kv": "bf16", "page": 16, "layout": "hnd", "pad": 0},
        # A loaded server's step: single tokens of many requests beside two pieces of prompts.
        {"name": "attention_mixed", "kind": "attention", "batch": 26, "cached": 4000, "new": 1, "chunks": 2, "chunk": 500, "q_heads": 32,
         "kv_heads": 8, "head_dim": 128, "q": "f16", "kv": "f16", "page": 16, "layout": "nhd", "pad": 24},
        # The small fp32 test model: pieces of a few prompts, fp32 throughout.
        {"name": "attention_f32_chunks", "kind": "attention", "batch": 6, "cached": 700, "new": 130, "chunks": 0, "chunk": 0, "q_heads": 4,
         "kv_heads": 2, "head_dim": 64, "q": "f32", "kv": "f32", "page": 8, "layout": "hnd", "pad": 3},
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)) - 0.25 / lo))))


def draw(rng):
    """One more case: the same operators, sizes spread over the ranges the listed cases stand in."""
    kind = rng.choice(["plan", "append", "attention", "attention", "attention"])
    page = rng.choice([1, 4, 8, 16, 16, 32, 64, 128, 256])
    pad = rng.choice([0, 0, 1, 5, 40])
    if kind == "plan":
        batch = _spread(rng, 1, 4096)
        chunks = min(batch, rng.choice([0, 0, 1, 3, 20]))
        return {"kind": kind, "batch": batch, "cached": max(page, min(_spread(rng, 1, 16000), 6000000 // batch)), "new": rng.choice([1, 1, 2, 3, 4]),
                "chunks": chunks, "chunk": _spread(rng, 4, 2000), "page": max(page, 4), "ended": rng.choice([0, 0, 1, batch // 10]),
                "pad": pad, "short": rng.choice([False, False, True])}
    heads = {"q_heads": 32, "kv_heads": 8, "head_dim": 128}
    heads = rng.choice([heads, heads, {"q_heads": 8, "kv_heads": 2, "head_dim": 128}, {"q_heads": 16, "kv_heads": 8, "head_dim": 64},
                        {"q_heads": 4, "kv_heads": 2, "head_dim": 64}])
    layout = rng.choice(["hnd", "nhd"])
    if kind == "append":
        act = rng.choice(["f32", "bf16", "f16"])
        return {"kind": kind, "rows": _spread(rng, 1, 8000), **heads, "act": act, "kv": rng.choice([act, "bf16", "f16"]), "page": page,
                "layout": layout, "far": _spread(rng, 8000, 1000000), "norm": rng.choice([True, True, False]), "pad": pad}
    kv = rng.choice(["bf16", "f16", "bf16", "f16", "f32"])
    q = rng.choice([kv, kv, "f32"])
    new = rng.choice([1, 1, 1, 2, 3, 4, _spread(rng, 5, 1200)])
    chunks = rng.choice([0, 0, 0, 1, 2])
    chunk = _spread(rng, 5, 600) if chunks else 0
    # no more keys or scores than the largest listed cases have
    batch, cached, heads_q = _spread(rng, 1, 64), _spread(rng, 1, 16000), heads["q_heads"] * (8 if q == "f32" else 1)
    top = max(new, chunk)
    batch = max(1, min(batch, int(_MOST_SCORES / (heads_q * new * (new + 100))), int(_MOST_PADDED / (heads_q * top * (top + 100)))))
    rows = batch * new + min(chunks, batch) * chunk
    cached = max(1, min(cached, 130000 // batch, int(_MOST_SCORES / (heads_q * rows)) - top, int(_MOST_PADDED / (heads_q * batch * top)) - top))
    return {"kind": kind, "batch": batch, "cached": cached, "new": new, "chunks": min(chunks, batch), "chunk": chunk, **heads, "q": q, "kv": kv,
            "page": page, "layout": layout, "pad": pad}


def _lengths(case):
    """(keys cached, new tokens) of every request: by the case alone."""
    B, top = case["batch"], case["cached"]
    cached = [top if b == 0 else max(0, round(top * (0.25 + 0.75 * ((0.618034 * b) % 1.0)))) for b in range(B)]
    new = [case["chunk"] - 7 * b % max(1, case["chunk"]) if b < case["chunks"] else case["new"] for b in range(B)]
    if case["new"] > 4:
        new = [max(1, n - 11 * b) for b, n in enumerate(new)]            # pieces of prompts are not equally long
    for b in range(5, B, 13):
        if b >= case["chunks"]:
            new[b] = 0                                                   # waits in this step
    if B > 3 and case["chunks"] < 3:
        cached[3] = 0                                                    # its first step
        new[3] = max(1, new[3])
    return cached, new


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, page = case["kind"], case["page"]
    if kind == "append":
        nq, nkv, D, T = case["q_heads"], case["kv_heads"], case["head_dim"], case["rows"] + case["pad"]
        n_pages = -(-(case["rows"] + 64) // page)
        qkv = torch.randn(T, (nq + 2 * nkv) * D, generator=g, device="cuda").mul_(2.0).to(_TYPES[case["act"]])
        slot = torch.randperm(n_pages * page, generator=g, device="cuda")[:T].int()
        position = (torch.randint(0, case["far"], (1,), generator=g, device="cuda") + torch.arange(T, device="cuda")).int()
        slot[case["rows"]:] = -1
        position[case["rows"]:] = 0
        norms = [1.0 + 0.1 * torch.randn(D, generator=g, device="cuda") if case["norm"] else None for _ in range(2)]
        kc, vc = (_pool(case, n_pages, g, zero=True) for _ in range(2))
        q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([nq * D, nkv * D, nkv * D], dim=1))
        return {"kind": kind, "q": q, "k": k, "v": v, "position": position, "slot": slot, "norms": norms, "kc": kc, "vc": vc,
                "q_out": torch.zeros(T, nq, D, dtype=qkv.dtype, device="cuda")}
    cached, new = _lengths(case)
    B = case["batch"]
    held = [-(-c // page) for c in cached]
    need = [-(-(c + n) // page) for c, n in zip(cached, new)]
    if kind == "plan":
        n_new = list(new)
        for b in range(case["ended"]):
            n_new[B - 1 - b * (B // max(1, case["ended"]))] = -1
        n_rows = sum(max(0, n) for n in n_new) + case["pad"]
        width = max(need) + 1
        spare = sum(need) - sum(held)
        spare = max(1, spare // 2) if case["short"] else spare + 5
        n_pages = sum(held) + spare
        perm = torch.randperm(n_pages, generator=g, device="cuda").int()
        table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
        table[torch.arange(width, device="cuda")[None] < _ints(held)[:, None]] = perm[:sum(held)]
        free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        free[:spare] = perm[sum(held):]
        out = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B + 1, n_rows, n_rows, B, B, 1)]
        return {"kind": kind, "lens": _ints(cached), "n_new": _ints(n_new), "table": table, "free": free, "n_free": _ints([spare]), "page": page,
                "n_rows": n_rows, "out": out}
    nq, nkv, D = case["q_heads"], case["kv_heads"], case["head_dim"]
    n_pages = sum(need) + 3
    perm = torch.randperm(n_pages, generator=g, device="cuda").int()
    width = max(need)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(width, device="cuda")[None] < _ints(need)[:, None]] = perm[:sum(need)]
    T = sum(new) + case["pad"]
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    q = torch.randn(T, nq, D, generator=g, device="cuda").mul_(1.5).to(_TYPES[case["q"]])
    kc, vc = (_pool(case, n_pages, g) for _ in range(2))
    return {"kind": kind, "q": q, "row_start": _ints(start), "lens": _ints([c + n for c, n in zip(cached, new)]), "table": table, "kc": kc,
            "vc": vc, "max_new": max(new), "out": torch.zeros_like(q), "scratch": torch.empty(48 << 20, dtype=torch.uint8, device="cuda")}


def _pool(case, n_pages, g, zero=False):
    """[n_pages, kv heads, page, head_dim], whatever the order in memory."""
    nkv, D, page = case["kv_heads"], case["head_dim"], case["page"]
    size = (n_pages, nkv, page, D) if case["layout"] == "hnd" else (n_pages, page, nkv, D)
    t = torch.empty(size, dtype=_TYPES[case["kv"]], device="cuda")
    for part in t.split(4096):
        part.copy_(torch.zeros((), device="cuda") if zero else torch.randn(part.shape, generator=g, device="cuda"))
    return t if case["layout"] == "hnd" else t.transpose(1, 2)


def run(state):
    return {"plan": _plan, "append": _append, "attention": _attention}[state["kind"]](state)


def _plan(s):
    if own:
        import paper_2510_11958_b200 as pkg
        p = pkg.paged_plan(s["lens"], s["n_new"], s["table"], s["free"], s["n_free"], s["page"], s["n_rows"], out=s["out"])
        return {"row_start": p.row_start, "position": p.position, "slot": p.slot, "granted": p.granted, "lens": p.lens, "n_free": p.n_free,
                "table": s["table"]}
    page, table, free, T = s["page"], s["table"], s["free"], s["n_rows"]
    n_pages, (_, width) = free.numel(), table.shape
    lens, ended = s["lens"].long().clamp(min=0), s["n_new"] < 0
    n = s["n_new"].long().clamp(min=0)
    held = (lens + page - 1) // page
    col = torch.arange(width, device="cuda")[None]
    # the pages of ended requests, in the order of requests and pages
    gone = table[ended[:, None] & (col < held[:, None]) & (table >= 0) & (table < n_pages)]
    avail = s["n_free"].long() + gone.numel()
    free[s["n_free"].long() + torch.arange(gone.numel(), device="cuda")] = gone
    row_end = n.cumsum(0)
    fits = (lens + n <= width * page) & (row_end <= T) & ~ended
    want = torch.where(fits, (lens + n + page - 1) // page - held, 0)
    last = want.cumsum(0)
    ok = fits & ((want == 0) | (last <= avail))
    granted = torch.where(ok, n, 0)
    new_page = ok[:, None] & (col >= held[:, None]) & (col < (held + want)[:, None])
    nth = (last - want)[:, None] + col - held[:, None]
    table.copy_(torch.where(new_page, free[(avail - 1 - nth).clamp(0, n_pages - 1)], table))
    row_start = torch.cat([torch.zeros_like(row_end[:1]), row_end]).clamp(max=T)
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(row_start, t, right=True) - 1
    real = b < n.numel()
    b = b.clamp(max=n.numel() - 1)
    pos = lens[b] + t - row_start[b]
    real = real & ok[b]
    pos = torch.where(real, pos, 0)
    slot = torch.where(real, table[b, pos // page].long() * page + pos % page, -1)
    return {"row_start": row_start.int(), "position": pos.int(), "slot": slot.int(), "granted": granted.int(),
            "lens": torch.where(ended, 0, lens + granted).int(), "n_free": (avail - torch.where(ok, want, 0).sum()).int(), "table": table}


def _append(s):
    q, k, v, (q_norm, k_norm) = s["q"], s["k"], s["v"], s["norms"]
    if own:
        import paper_2510_11958_b200 as pkg
        pkg.paged_append(q, k, v, s["position"], s["slot"], s["kc"], s["vc"], q_norm=q_norm, k_norm=k_norm, eps=_EPS, rope_theta=_THETA,
                         q_out=s["q_out"])
        return {"q": s["q_out"], "k": s["kc"], "v": s["vc"]}
    D, page = q.shape[-1], s["kc"].shape[2]
    freq = torch.pow(torch.tensor(_THETA, dtype=torch.float64, device="cuda"), -2.0 * torch.arange(D // 2, dtype=torch.float64, device="cuda") / D)
    angle = s["position"].double()[:, None] * freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * w
        a, b = x[..., :D // 2], x[..., D // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    here = s["slot"] >= 0
    slot = s["slot"].long()[here]
    s["q_out"][here] = turned(q, q_norm)[here].to(q.dtype)
    s["kc"][slot // page, :, slot % page] = turned(k, k_norm)[here].to(s["kc"].dtype)
    s["vc"][slot // page, :, slot % page] = v[here].float().to(s["vc"].dtype)
    return {"q": s["q_out"], "k": s["kc"], "v": s["vc"]}


def _attention(s):
    q, kc, vc, out = s["q"], s["kc"], s["vc"], s["out"]
    if own:
        import paper_2510_11958_b200 as pkg
        return pkg.paged_attention(q, s["row_start"], s["lens"], s["table"], kc, vc, max_new=s["max_new"], scratch=s["scratch"], out=out)
    (T, nq, D), (_, nkv, page, _), (B, width), R = q.shape, kc.shape, s["table"].shape, s["max_new"]
    G = nq // nkv
    pages = s["table"].clamp(min=0)
    keys, values = (c[pages].transpose(1, 2).reshape(B, nkv, width * page, D).float() for c in (kc, vc))
    start, lens = s["row_start"].long(), s["lens"].long()
    r = torch.arange(R, device="cuda")[None]
    n = (start[1:] - start[:-1])[:, None]
    row = start[:-1, None] + r                                           # [B, R]
    seen = lens[:, None] - n + r + 1                                     # keys that a row sees
    rows = q[row.clamp(max=T - 1)].float().view(B, R, nkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, nkv, G * R, D)
    key = torch.arange(width * page, device="cuda")
    hidden = key >= seen[:, None, None, :, None]                         # [B, 1, 1, R, keys]
    score = torch.matmul(rows * D ** -0.5, keys.transpose(2, 3)).view(B, nkv, G, R, width * page).masked_fill_(hidden, -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True).clamp(min=1e-38)
    values = torch.where((key < lens[:, None])[:, None, :, None], values, 0)
    o = torch.matmul(p.view(B, nkv, G * R, -1), values).view(B, nkv, G, R, D) / total
    real = r < n
    out[row[real]] = o.permute(0, 3, 1, 2, 4).reshape(B, R, nq, D)[real].to(out.dtype)
    return out


def exact(case, seed):
    """The definitions, request by request and in 64 bits."""
    s = prepare(case, seed)
    if s["kind"] == "plan":
        return _exact_plan(s)
    if s["kind"] == "append":
        D, page = s["q"].shape[-1], s["kc"].shape[2]
        out = {"q": s["q_out"].double(), "k": s["kc"].double(), "v": s["vc"].double()}
        real = s["slot"] >= 0
        t = int(real.sum())                                              # rows without a slot come last
        where = s["slot"][:t].long()
        half = torch.arange(D, device="cuda") % (D // 2)
        angle = s["position"][:t, None].double() * torch.exp(-math.log(_THETA) * 2.0 / D * half.double())
        turn = torch.complex(angle.cos(), angle.sin())[:, None, :D // 2]
        for name, w in (("q", s["norms"][0]), ("k", s["norms"][1])):
            x = s[name][:t].double()
            if w is not None:
                x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + _EPS) * w.double()
            z = torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous()) * turn
            x = torch.cat([z.real, z.imag], -1)
            if name == "q":
                out["q"][:t] = x
            else:
                out["k"][where // page, :, where % page] = x
        out["v"][where // page, :, where % page] = s["v"][:t].double()
        return out
    q, kc, vc, page = s["q"], s["kc"], s["vc"], s["kc"].shape[2]
    nq, D, G = q.shape[1], q.shape[2], q.shape[1] // kc.shape[1]
    out = s["out"].double()
    start, lens = s["row_start"].tolist(), s["lens"].tolist()
    for b, length in enumerate(lens):
        t0, t1 = start[b], start[b + 1]
        if t1 == t0:
            continue
        pages = s["table"][b, :-(-length // page)].long()
        for h in range(nq):
            k, v = (c[pages, h // G].reshape(-1, D)[:length].double() for c in (kc, vc))
            score = q[t0:t1, h].double() @ k.T / math.sqrt(D)
            score += torch.full_like(score, -math.inf).triu(length - (t1 - t0) + 1)
            out[t0:t1, h] = torch.softmax(score, -1) @ v
    return out


def _exact_plan(s):
    page, table, free, T = s["page"], s["table"].tolist(), s["free"].tolist(), s["n_rows"]
    lens, n_new, width = s["lens"].tolist(), s["n_new"].tolist(), s["table"].shape[1]
    stack = free[:s["n_free"].item()]
    for b, n in enumerate(n_new):
        if n < 0:
            stack += [p for p in table[b][:-(-lens[b] // page)] if 0 <= p < len(free)]
            lens[b] = 0
    start, granted, position, slot, wanted, left = [0], [], [], [], 0, len(stack)
    for b, n in enumerate(n_new):
        n = max(0, n)
        held, need = -(-lens[b] // page), -(-(lens[b] + n) // page)
        ok = n_new[b] >= 0 and lens[b] + n <= width * page and start[-1] + n <= T
        if ok:
            wanted += need - held
            ok = need == held or wanted <= left
        if ok:
            for i in range(held, need):
                table[b][i] = stack.pop()
        for r in range(min(n, T - start[-1])):
            at = lens[b] + r
            position.append(at if ok else 0)
            slot.append(table[b][at // page] * page + at % page if ok else -1)
        start.append(min(T, start[-1] + n))
        granted.append(n if ok else 0)
        lens[b] += granted[-1]
    position += [0] * (T - len(position))
    slot += [-1] * (T - len(slot))
    return {"row_start": _ints(start), "position": _ints(position), "slot": _ints(slot), "granted": _ints(granted), "lens": _ints(lens),
            "n_free": _ints([len(stack)]), "table": _ints(table)}


def work(case):
    if case["kind"] == "append":
        heads = case["q_heads"] + 2 * case["kv_heads"]
        D, T = case["head_dim"], case["rows"]
        return {"bytes": T * D * (heads * _BYTES[case["act"]] + case["q_heads"] * _BYTES[case["act"]] + 2 * case["kv_heads"] * _BYTES[case["kv"]]) + 8 * T,
                "flops": T * D * 7 * heads}
    cached, new = _lengths(case)
    if case["kind"] == "plan":
        page, B = case["page"], case["batch"]
        pages = sum(-(-(c + n) // page) - -(-c // page) for c, n in zip(cached, new))
        return {"bytes": 4 * (6 * B + 2 * (sum(new) + case["pad"]) + 2 * pages), "flops": 4 * (B + sum(new))}
    D, nq = case["head_dim"], case["q_heads"]
    keys = sum(c + n for c, n in zip(cached, new) if n)
    scores = sum(n * c + n * (n + 1) // 2 for c, n in zip(cached, new))
    return {"bytes": 2 * keys * case["kv_heads"] * D * _BYTES[case["kv"]] + 2 * sum(new) * nq * D * _BYTES[case["q"]] + 4 * -(-keys // case["page"]),
            "flops": 4 * scores * nq * D}

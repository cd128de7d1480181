"""Cases and plain forms of the paged-cache and sampling operators.

Four operators that a prompt runs through before its first draft tree is verified, and every token of a drafter:

- ``tables``: which pages and slots the new tokens of every request take (block tables, slot map, positions);
- ``append``: rotary embedding of the new queries and keys, keys and values written into their slots;
- ``attn``: causal attention of the new tokens of every request over its paged cache, optionally through a sliding
  window beside a few first tokens (sinks) that stay visible;
- ``sample``: one token a row of logits from a given uniform number, after temperature, top-k, top-p and min-p.

``own = False``: elementary torch operations.  ``own = True``: the library's calls.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
ROPE_BASE = 10000.0


# ---------------------------------------------------------------------------------------------------- cases

def listed():
    heads = dict(Hq=32, Hkv=32, D=128)          # the 7B-shaped targets: 32 heads of 128, a key head for each
    return [
        # one token of one prompt and its unconditional twin over 64 prompt + 320 image tokens: latency counts
        dict(name="attn_token_pair", op="attn", dtype="bf16", **heads, page=16, n_req=2, q_lo=1, q_hi=1, kv_lo=385, kv_hi=385,
             window=0, sinks=0, mix=1),
        # a server's batch, one new token each, prefixes anywhere between 256 and 2880 tokens
        dict(name="attn_token_batch", op="attn", dtype="bf16", **heads, page=16, n_req=48, q_lo=1, q_hi=1, kv_lo=256, kv_hi=2880,
             window=0, sinks=0, mix=2),
        # four prompts and their twins of 128 text tokens and a whole 48 x 49 image as one chunk, from an empty cache
        dict(name="attn_prompt", op="attn", dtype="bf16", **heads, page=64, n_req=8, q_lo=2480, q_hi=2480, kv_lo=2480, kv_hi=2480,
             window=0, sinks=0, mix=3),
        # pieces of up to about ten image rows behind long prefixes, four query heads a key head, a window of 1024 and
        # four first tokens
        dict(name="attn_chunk_window", op="attn", dtype="bf16", Hq=32, Hkv=8, D=128, page=16, n_req=16, q_lo=17, q_hi=480,
             kv_lo=700, kv_hi=2880, window=1024, sinks=4, mix=4),
        # the 32-bit configuration: 4 heads of 64, chunks behind short prefixes
        dict(name="attn_f32", op="attn", dtype="f32", Hq=4, Hkv=4, D=64, page=16, n_req=8, q_lo=15, q_hi=130, kv_lo=64, kv_hi=450,
             window=0, sinks=0, mix=5),
        # one prompt and its twin take one more token
        dict(name="tables_token", op="tables", page=16, n_req=2, new_lo=1, new_hi=1, kv_lo=384, kv_hi=400, width=64, done=0.0, pad=0,
             mix=6),
        # a server admits prompts beside running requests, while finished ones give their pages back
        dict(name="tables_prompt", op="tables", page=16, n_req=512, new_lo=1, new_hi=480, kv_lo=0, kv_hi=2300, width=192, done=0.1,
             pad=1000, mix=7),
        # one token of 8 prompts and their twins, with its query
        dict(name="append_token", op="append", dtype="bf16", **heads, page=16, n_tok=16, start_lo=384, start_hi=2480, mix=8),
        # the four prompts and their twins of attn_prompt
        dict(name="append_prompt", op="append", dtype="bf16", **heads, page=64, n_tok=8 * 2480, start_lo=0, start_hi=0, mix=9),
        # a drafter's token for one prompt and its twin: 16384 image tokens, the published top-k 2000
        dict(name="sample_pair", op="sample", dtype="f32", V=16384, rows=2, mode="topk", mix=10),
        # the nodes of many drafts at once over the 65536-token vocabulary, each request with settings of its own
        dict(name="sample_mixed", op="sample", dtype="f32", V=65536, rows=488, mode="mixed", mix=11),
        # the same from a head that leaves 16-bit logits, plain temperature and nucleus
        dict(name="sample_bf16", op="sample", dtype="bf16", V=16384, rows=61, mode="topp", mix=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.499)))))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "sample", "sample", "append", "tables"])
    mix = rng.randrange(1 << 30)
    if op == "attn":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        D = rng.choice([64, 128, 128])
        Hkv, G = rng.choice([(32, 1), (8, 4), (4, 8), (1, 8), (4, 1), (2, 5), (8, 2), (10, 1)])
        page = rng.choice([8, 16, 16, 32, 48, 64, 128])
        q_hi = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 17, 2480)])
        q_lo = 1 if q_hi == 1 else _log_int(rng, 1, q_hi)
        kv_hi = max(q_hi, _log_int(rng, 16, 2880 if q_hi > 1 else 11000))
        kv_lo = max(q_hi, _log_int(rng, 1, kv_hi))
        # no more work, and no larger plain scores, than the listed chunk of 2480 tokens (a sixteenth of it in 32 bits)
        most = 8 * 32 * 2480 * 2480 // (16 if dtype == "f32" else 1)
        n_most = max(1, min(64, most // (Hkv * G * q_hi * kv_hi), (64 * 2880 * 32) // (kv_hi * Hkv * G)))
        n_req = _log_int(rng, 1, n_most)
        window = rng.choice([0, 0, _log_int(rng, 16, 2048)])
        sinks = rng.choice([0, 1, 4, 17, 128]) if window else 0
        return dict(op="attn", dtype=dtype, Hq=Hkv * G, Hkv=Hkv, D=D, page=page, n_req=n_req, q_lo=q_lo, q_hi=q_hi,
                    kv_lo=kv_lo, kv_hi=kv_hi, window=window, sinks=sinks, mix=mix)
    if op == "tables":
        n_req = _log_int(rng, 1, 1000)
        new_hi = min(_log_int(rng, 1, 2480), 200000 // n_req)
        return dict(op="tables", page=rng.choice([8, 16, 32, 48, 64, 128]), n_req=n_req, new_lo=rng.choice([0, 1]), new_hi=max(1, new_hi),
                    kv_lo=0, kv_hi=_log_int(rng, 1, 2880), width=700, done=rng.choice([0.0, 0.1, 0.5]),
                    pad=rng.choice([0, 7, 1000]), mix=mix)
    if op == "append":
        Hkv, G = rng.choice([(32, 1), (8, 4), (4, 8), (1, 8), (4, 1), (2, 5)])
        n_tok = _log_int(rng, 1, 8 * 2480 * 32 // max(32, Hkv * G))
        return dict(op="append", dtype=rng.choice(["bf16", "bf16", "f32"]), Hq=Hkv * G, Hkv=Hkv, D=rng.choice([64, 128]),
                    page=rng.choice([8, 16, 48, 64]), n_tok=min(n_tok, 9000), start_lo=0, start_hi=_log_int(rng, 1, 100000), mix=mix)
    V = 8 * _log_int(rng, 16, 8192)
    rows = _log_int(rng, 1, max(1, min(1000, 488 * 65536 // V)))
    return dict(op="sample", dtype=rng.choice(["f32", "bf16"]), V=V, rows=rows,
                mode=rng.choice(["plain", "topk", "topp", "minp", "mixed"]), mix=mix)


def _lengths(case):
    """The requests' new tokens and lengths (the new ones included): part of the case, not of its inputs."""
    r = random.Random(case["mix"])
    q = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["n_req"])]
    kv = [max(n, r.randint(case["kv_lo"], case["kv_hi"])) for n in q]
    return q, kv


def _table_lengths(case):
    r = random.Random(case["mix"])
    done = [r.random() < case["done"] for _ in range(case["n_req"])]
    kv = [r.randint(case["kv_lo"], case["kv_hi"]) for _ in range(case["n_req"])]
    new = [-1 if d else r.randint(case["new_lo"], case["new_hi"]) for d in done]
    return new, kv


def _visible(q, kv, window, sinks):
    """(visible pairs, keys that any of the new tokens sees) of one request."""
    first = kv - q
    if window == 0:
        return q * first + q * (q + 1) // 2, kv
    pairs = 0
    for p in range(first, kv):
        lo = max(0, p - window + 1)
        pairs += p + 1 - lo + min(sinks, lo)
    lo = max(0, first - window + 1)
    return pairs, kv - lo + min(sinks, lo)


def work(case):
    if case["op"] == "attn":
        q, kv = _lengths(case)
        seen = [_visible(a, b, case["window"], case["sinks"]) for a, b in zip(q, kv)]
        es, D = BYTES[case["dtype"]], case["D"]
        return {"bytes": 2 * sum(q) * case["Hq"] * D * es + 2 * sum(s[1] for s in seen) * case["Hkv"] * D * es
                + 4 * sum(-(-n // case["page"]) for n in kv),
                "flops": 4 * D * case["Hq"] * sum(s[0] for s in seen)}
    if case["op"] == "tables":
        new, kv = _table_lengths(case)
        tok = sum(max(n, 0) for n in new)
        pages = sum(-(-(k + n) // case["page"]) - -(-k // case["page"]) for n, k in zip(new, kv) if n >= 0)
        back = sum(-(-k // case["page"]) for n, k in zip(new, kv) if n < 0)
        return {"bytes": 8 * (tok + case["pad"]) + 16 * case["n_req"] + 8 * (pages + back), "flops": 4 * tok}
    if case["op"] == "append":
        es = BYTES[case["dtype"]]
        row = (case["Hq"] + 2 * case["Hkv"]) * case["D"]
        return {"bytes": 2 * case["n_tok"] * row * es + 8 * case["n_tok"],
                "flops": 3 * case["n_tok"] * (case["Hq"] + case["Hkv"]) * case["D"]}
    return {"bytes": case["rows"] * (case["V"] * BYTES[case["dtype"]] + 32), "flops": 4 * case["rows"] * case["V"]}


# --------------------------------------------------------------------------------------------------- inputs

def _pool(gen, case, n_pages, filled):
    shape = (n_pages, case["page"], case["Hkv"], case["D"])
    if not filled:
        return torch.zeros(shape, device=DEV, dtype=TYPES[case["dtype"]])
    return torch.randn(shape, device=DEV, generator=gen, dtype=torch.float32 if case["dtype"] == "f32" else torch.bfloat16)


def _table(rng, lens, page, width):
    """Pages of a pool in no order: every request's block table, and how many pages the pool has."""
    counts = [-(-n // page) for n in lens]
    n_pages = sum(counts) + 3
    ids = rng.permutation(n_pages)
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for r, c in enumerate(counts):
        table[r, :c] = ids[at:at + c]
        at += c
    return table, ids[at:], n_pages


def _i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    st = dict(case=case)
    if case["op"] == "attn":
        q, kv = _lengths(case)
        table, _, n_pages = _table(rng, kv, case["page"], -(-max(kv) // case["page"]))
        dt = TYPES[case["dtype"]]
        st.update(q=torch.randn((sum(q), case["Hq"], case["D"]), device=DEV, generator=gen).to(dt),
                  k_pages=_pool(gen, case, n_pages, True), v_pages=_pool(gen, case, n_pages, True), table=_i32(table),
                  q_begin=_i32(np.concatenate([[0], np.cumsum(q)])), kv_len=_i32(kv), max_q=max(q), max_kv=max(kv),
                  scale=1.0 / math.sqrt(case["D"]))
        st["out"] = torch.zeros_like(st["q"])
    elif case["op"] == "tables":
        new, kv = _table_lengths(case)
        page, width = case["page"], case["width"]
        table, _, held = _table(rng, kv, page, width)
        need = sum(-(-(k + max(n, 0)) // page) - -(-k // page) for n, k in zip(new, kv))
        n_pages = held + need + 5
        free = np.full(n_pages, -1, np.int32)
        spare = rng.permutation(np.setdiff1d(np.arange(n_pages), table[table >= 0]))
        free[:len(spare)] = spare
        tok = sum(max(n, 0) for n in new) + case["pad"]
        st.update(n_pages=n_pages, new_len=_i32(new), kv_len=_i32(kv), table=_i32(table), free=_i32(free),
                  free_count=_i32([len(spare)]), kv_out=_i32(np.zeros(len(kv))), count_out=_i32([0]),
                  q_begin=_i32(np.zeros(len(kv) + 1)), slot=_i32(np.zeros(max(tok, 1))), pos=_i32(np.zeros(max(tok, 1))))
    elif case["op"] == "append":
        n, Hq, Hkv, D = case["n_tok"], case["Hq"], case["Hkv"], case["D"]
        per = 2480 if case["start_hi"] == 0 else 1
        start = rng.integers(case["start_lo"], case["start_hi"] + 1, -(-n // per))
        pos = (start[:, None] + np.arange(per)[None, :]).reshape(-1)[:n]
        n_pages = -(-n // case["page"]) + 2
        pages = rng.permutation(n_pages)
        slot = pages[np.arange(n) // case["page"]] * case["page"] + np.arange(n) % case["page"]
        if per == 1:                        # single tokens of many requests: slots anywhere in the pool
            slot = rng.permutation(n_pages * case["page"])[:n]
        qkv = torch.randn((n, (Hq + 2 * Hkv) * D), device=DEV, generator=gen).to(TYPES[case["dtype"]])
        st.update(qkv=qkv, q=qkv[:, :Hq * D].view(n, Hq, D), k=qkv[:, Hq * D:(Hq + Hkv) * D].view(n, Hkv, D),
                  v=qkv[:, (Hq + Hkv) * D:].view(n, Hkv, D), slot=_i32(slot), pos=_i32(pos),
                  k_pages=_pool(gen, case, n_pages, False), v_pages=_pool(gen, case, n_pages, False),
                  q_out=torch.zeros((n, Hq, D), device=DEV, dtype=qkv.dtype), table=_i32(np.zeros((1, 1))))
    else:
        # near-identical codes share the mass, as in an image vocabulary: 256 levels and a little noise
        V, rows, mode = case["V"], case["rows"], case["mode"]
        level = torch.randn((rows, 256), device=DEV, generator=gen) * 2.6
        logits = level[:, torch.arange(V, device=DEV) % 256] + 0.3 * torch.randn((rows, V), device=DEV, generator=gen)
        st.update(logits=logits.to(TYPES[case["dtype"]]), u=torch.rand((rows,), device=DEV, generator=gen))
        f = lambda lo, hi: torch.as_tensor(rng.uniform(lo, hi, rows).astype(np.float32), device=DEV)  # noqa: E731
        st.update(temperature=f(0.7, 1.5), top_k=None, top_p=None, min_p=None)
        if mode in ("topk", "mixed"):
            k = np.minimum(2000, V // 2) if mode == "topk" else rng.choice([0, 1, 50, min(2000, V // 2), V], rows)
            st["top_k"] = _i32(np.broadcast_to(k, (rows,)).copy())
        if mode in ("topp", "mixed"):
            p = rng.uniform(0.5, 0.99, rows)
            st["top_p"] = torch.as_tensor(np.where((mode == "mixed") & (rng.random(rows) < 0.3), 1.0, p).astype(np.float32), device=DEV)
        if mode in ("minp", "mixed"):
            p = rng.uniform(0.001, 0.1, rows)
            st["min_p"] = torch.as_tensor(np.where((mode == "mixed") & (rng.random(rows) < 0.5), 0.0, p).astype(np.float32), device=DEV)
        if mode == "mixed":                 # some requests want the most likely token
            st["temperature"] *= torch.as_tensor((rng.random(rows) > 0.1).astype(np.float32), device=DEV)
        st.update(token=_i32(np.zeros(rows)), prob=torch.zeros(rows, device=DEV), kept=_i32(np.zeros(rows)))
    if own:
        from paper_2605_07230_b200 import binding as cb
        dtype = cb.F32 if case.get("dtype") == "f32" else cb.BF16
        st["ctx"] = cb.Context(dtype, 1, 1, 64, 64, case.get("Hq", 1), case.get("Hkv", 1), case.get("D", 64), case.get("V", 64))
        if "k_pages" in st:
            st["cache"] = cb.PagedCache(st["k_pages"], st["v_pages"], st["table"])
    return st


# ---------------------------------------------------------------------------------------------- plain forms

def _plain_attn(st):
    c = st["case"]
    q, qb, kvl, page = st["q"], st["q_begin"].long(), st["kv_len"].long(), c["page"]
    n, nq, nk, G = c["n_req"], st["max_q"], st["max_kv"], c["Hq"] // c["Hkv"]
    rows = (qb[:-1, None] + torch.arange(nq, device=DEV)[None, :]).clamp(max=q.shape[0] - 1)
    x = q[rows].float().view(n, nq, c["Hkv"], G, c["D"]).permute(0, 2, 3, 1, 4).reshape(n, c["Hkv"], G * nq, c["D"])
    pages = st["table"][:, :-(-nk // page)].long().clamp(min=0)
    keys = lambda p: p[pages].reshape(n, -1, c["Hkv"], c["D"])[:, :nk].float()                          # noqa: E731
    there = (torch.arange(nk, device=DEV)[None, :] < kvl[:, None])[:, :, None, None]
    k = torch.where(there, keys(st["k_pages"]), 0.0).permute(0, 2, 3, 1)
    s = (x @ k).view(n, c["Hkv"], G, nq, nk)
    del k
    s *= st["scale"]
    i = torch.arange(nk, device=DEV)[None, None, :]
    p = (kvl - (qb[1:] - qb[:-1]))[:, None, None] + torch.arange(nq, device=DEV)[None, :, None]
    see = (i <= p) & (i < kvl[:, None, None])
    if c["window"]:
        see &= (i > p - c["window"]) | (i < c["sinks"])
    s.masked_fill_(~see[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    s -= torch.where(m == -math.inf, 0.0, m)
    s.exp_()
    total = s.sum(-1, keepdim=True)
    v = torch.where(there, keys(st["v_pages"]), 0.0).permute(0, 2, 1, 3)
    o = (s.view(n, c["Hkv"], G * nq, nk) @ v).view(n, c["Hkv"], G, nq, c["D"])
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(n, nq, c["Hq"], c["D"])
    t = torch.arange(q.shape[0], device=DEV)
    r = torch.searchsorted(qb[1:], t, right=True)
    return o[r, t - qb[r]].to(q.dtype)


def _plain_tables(st):
    c = st["case"]
    page, kv, new = c["page"], st["kv_len"].long(), st["new_len"].long()
    done, add = new < 0, new.clamp(min=0)
    had = (kv + page - 1) // page
    kv_out = torch.where(done, 0, kv + add)
    has = torch.where(done, had, (kv_out + page - 1) // page)
    back, need = torch.where(done, had, 0), has - had
    j = torch.arange(c["width"], device=DEV)[None, :]
    free = torch.cat([st["free"].long(), torch.zeros(1, dtype=torch.long, device=DEV)])     # the last: a place for nothing
    at = st["free_count"].long() + (torch.cumsum(back, 0) - back)[:, None] + j
    free = free.index_put((torch.where(j < back[:, None], at, st["n_pages"]),), st["table"].long())
    count = st["free_count"].long() + back.sum()
    take = count - 1 - ((torch.cumsum(need, 0) - need)[:, None] + j - had[:, None])
    fresh = (j >= had[:, None]) & (j < has[:, None])
    table = torch.where(fresh, free[torch.where(fresh, take, 0)], st["table"].long())
    q_begin = torch.cat([torch.zeros_like(add[:1]), torch.cumsum(add, 0)])
    t = torch.arange(st["slot"].numel(), device=DEV)
    r = torch.searchsorted(q_begin[1:], t, right=True)
    live = r < c["n_req"]
    r = r.clamp(max=c["n_req"] - 1)
    pos = kv[r] + t - q_begin[r]
    slot = table[r, torch.where(live, pos // page, 0)] * page + pos % page
    return [x.int() for x in (table, free[:-1], kv_out, (count - need.sum()).view(1), q_begin, torch.where(live, slot, -1), torch.where(live, pos, -1))]


def _plain_append(st):
    half = st["case"]["D"] // 2
    freq = ROPE_BASE ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    angle = st["pos"].double()[:, None] * freq[None, :]
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]

    def turn(x):
        a, b = x[..., :half].float(), x[..., half:].float()
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(x.dtype)

    slot = st["slot"].long()
    st["k_pages"].view(-1, *st["k"].shape[1:])[slot] = turn(st["k"])
    st["v_pages"].view(-1, *st["v"].shape[1:])[slot] = st["v"]
    return [st["k_pages"], st["v_pages"], turn(st["q"])]


def _plain_sample(st):
    x = st["logits"].double()
    V = x.shape[1]
    m = x.amax(-1, keepdim=True)
    t = st["temperature"].double()[:, None]
    greedy = t <= 0
    w = torch.exp((x - m) / torch.where(greedy, 1.0, t))
    keep = torch.ones_like(x, dtype=torch.bool)
    if st["top_k"] is not None:
        k = st["top_k"].long()[:, None]
        down = torch.sort(x, -1, descending=True)[0]
        keep = (k <= 0) | (k >= V) | (x >= down.gather(1, (k - 1).clamp(0, V - 1)))
    if st["top_p"] is not None:
        p = st["top_p"].double()[:, None]
        xs, order = torch.sort(torch.where(keep, x, -math.inf), -1, descending=True)
        ws = torch.where(keep, w, 0.0).gather(1, order)
        before = torch.cumsum(ws, -1) - ws
        first = torch.cat([torch.ones_like(keep[:, :1]), xs[:, 1:] != xs[:, :-1]], -1)
        larger = torch.cummax(torch.where(first, before, 0.0), -1)[0]
        inside = (larger < p * ws.sum(-1, keepdim=True)) & (xs > -math.inf)
        floor = torch.where(inside, xs, math.inf).amin(-1, keepdim=True)
        keep &= (p >= 1) | (x >= floor)
    if st["min_p"] is not None:
        keep &= w >= st["min_p"].double()[:, None]
    i = torch.arange(V, device=DEV)[None, :]
    best = torch.where(x == m, i, V).amin(-1, keepdim=True)
    keep = torch.where(greedy, i == best, keep)
    w = torch.where(keep, w, 0.0)
    run_sum = torch.cumsum(w, -1)
    token = (run_sum <= st["u"].double()[:, None] * run_sum[:, -1:]).sum(-1, keepdim=True).clamp(max=V - 1)
    prob = w.gather(1, token) / run_sum[:, -1:]
    return [token[:, 0].int(), prob[:, 0].float(), keep.sum(-1).int()]


def run(st):
    op = st["case"]["op"]
    if own:
        from paper_2605_07230_b200 import binding as cb
        if op == "attn":
            cb.cascade_paged_attn(st["ctx"], st["cache"], st["q"], st["q_begin"], st["kv_len"], st["max_q"], st["max_kv"],
                                  st["out"], st["scale"], window=st["case"]["window"], sinks=st["case"]["sinks"])
            return st["out"]
        if op == "tables":
            cb.cascade_paged_tables(st["ctx"], st["case"]["page"], st["n_pages"], st["new_len"], st["kv_len"], st["table"],
                                    st["free"], st["free_count"], st["kv_out"], st["count_out"], st["q_begin"], st["slot"],
                                    st["pos"])
            return [st["table"], st["free"], st["kv_out"], st["count_out"], st["q_begin"], st["slot"], st["pos"]]
        if op == "append":
            cb.cascade_paged_append(st["ctx"], st["cache"], st["k"], st["v"], st["slot"], st["pos"], rope_base=ROPE_BASE,
                                    q=st["q"], q_out=st["q_out"])
            return [st["k_pages"], st["v_pages"], st["q_out"]]
        cb.cascade_sample(st["ctx"], st["logits"], st["u"], st["token"], temperature=st["temperature"], top_k=st["top_k"],
                          top_p=st["top_p"], min_p=st["min_p"], prob=st["prob"], kept=st["kept"])
        return [st["token"], st["prob"], st["kept"]]
    if op == "attn":
        return _plain_attn(st)
    if op == "tables":
        return _plain_tables(st)
    if op == "append":
        return _plain_append(st)
    return _plain_sample(st)


# ---------------------------------------------------------------------------------------- in 64 bits, apart

def _exact_attn(st):
    """Request by request and head by head, rows of scores in 64 bits."""
    c = st["case"]
    q_len, kv_len = _lengths(c)
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for r in range(c["n_req"]):
        n, L = q_len[r], kv_len[r]
        where = torch.arange(L, device=DEV)
        page = st["table"][r].long()[where // c["page"]]
        see = where[None, :] <= (L - n + torch.arange(n, device=DEV))[:, None]
        if c["window"]:
            near = where[None, :] > (L - n + torch.arange(n, device=DEV))[:, None] - c["window"]
            see &= near | (where < c["sinks"])[None, :]
        for h in range(c["Hq"]):
            kh = h * c["Hkv"] // c["Hq"]
            k = st["k_pages"][page, where % c["page"], kh].double()
            v = st["v_pages"][page, where % c["page"], kh].double()
            s = st["q"][at:at + n, h].double() @ k.T * st["scale"]
            w = torch.softmax(torch.where(see, s, -math.inf), -1)
            out[at:at + n, h] = w @ v
        at += n
    return out


def _exact_append(st):
    c = st["case"]
    n, D = c["n_tok"], c["D"]
    half = D // 2
    slot, pos = st["slot"].long(), st["pos"].double()
    unit = torch.polar(torch.ones((n, half), dtype=torch.float64, device=DEV),
                       pos[:, None] * torch.exp(-math.log(ROPE_BASE) * torch.arange(half, device=DEV, dtype=torch.float64) * 2 / D))

    def turn(x):
        z = torch.complex(x[..., :half].double(), x[..., half:].double()) * unit[:, None, :]
        return torch.cat([z.real, z.imag], -1)

    k = st["k_pages"].double().reshape(-1, c["Hkv"], D)
    v = st["v_pages"].double().reshape(-1, c["Hkv"], D)
    k[slot] = turn(st["k"])
    v[slot] = st["v"].double()
    return [k.view(st["k_pages"].shape), v.view(st["v_pages"].shape), turn(st["q"])]


def _exact_sample(st):
    """Row by row on the host, the nucleus walked from the most likely token down."""
    x = st["logits"].double().cpu().numpy()
    host = {k: None if st[k] is None else st[k].double().cpu().numpy() for k in ("u", "temperature", "top_k", "top_p", "min_p")}
    token, prob, kept = [], [], []
    for r, row in enumerate(x):
        if host["temperature"][r] <= 0:
            token.append(int(np.argmax(row)))
            prob.append(1.0)
            kept.append(1)
            continue
        z = row / host["temperature"][r]
        w = np.exp(z - z.max())
        keep = np.ones(len(row), bool)
        k = 0 if host["top_k"] is None else int(host["top_k"][r])
        if 0 < k < len(row):
            keep &= row >= np.partition(row, len(row) - k)[len(row) - k]
        p = 1.0 if host["top_p"] is None else host["top_p"][r]
        if p < 1:
            values, inverse = np.unique(-row[keep], return_inverse=True)
            mass = np.bincount(inverse, w[keep])
            ahead = np.concatenate([[0.0], np.cumsum(mass)[:-1]])
            keep &= row >= -values[ahead < p * mass.sum()].max()
        if host["min_p"] is not None:
            keep &= w >= host["min_p"][r]
        ids = np.flatnonzero(keep)
        cum = np.cumsum(w[ids])
        i = int(np.searchsorted(cum, host["u"][r] * cum[-1], side="right"))
        token.append(int(ids[i]))
        prob.append(w[ids[i]] / cum[-1])
        kept.append(len(ids))
    return [torch.tensor(token, dtype=torch.int32), torch.tensor(prob, dtype=torch.float64), torch.tensor(kept, dtype=torch.int32)]


def _exact_tables(st):
    """A stack of pages and a walk over the requests, on the host."""
    page, host = st["case"]["page"], {k: st[k].tolist() for k in ("new_len", "kv_len", "table", "free", "free_count")}
    new, table, free, count = host["new_len"], host["table"], host["free"], host["free_count"][0]
    kv_out, q_begin, slot, pos = [], [0], [], []
    for r, n in enumerate(new):
        if n < 0:
            back = [p for p in table[r][:-(-host["kv_len"][r] // page)]]
            free[count:count + len(back)] = back
            count += len(back)
    for r, n in enumerate(new):
        kv = host["kv_len"][r]
        for i in range(kv, kv + max(n, 0)):
            if i % page == 0:
                count -= 1
                table[r][i // page] = free[count]
            slot.append(table[r][i // page] * page + i % page)
            pos.append(i)
        kv_out.append(0 if n < 0 else kv + n)
        q_begin.append(len(slot))
    rest = [-1] * (st["slot"].numel() - len(slot))
    return [torch.tensor(x, dtype=torch.int32) for x in (table, free, kv_out, [count], q_begin, slot + rest, pos + rest)]


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "tables":
        return _exact_tables(st)
    if case["op"] == "attn":
        return _exact_attn(st)
    if case["op"] == "append":
        return _exact_append(st)
    return _exact_sample(st)

"""Cases and plain forms of the operators that train a drafter.

A drafter learns from sequences that the target has generated: one pass of its attention over the tokens of many sequences
(the paged calls), a soft cross-entropy against what was stored of the target's distributions, and the way back.  Three
operators:

- ``attn_grad``: the gradient of the paged attention with respect to queries, keys and values, from its output and
  log-sum-exp, through causal masks, windows and first tokens;
- ``loss``: the drafter's loss (soft cross-entropy, a position's weight raised where consecutive hidden states of the target
  converge) against the target's largest logits of every position alone, as they are stored (2000 of them, say);
- ``loss_grad``: its gradient with respect to the drafter's logits.

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
TAU, RAISED = 0.5, 2.0                      # convergence threshold and the weight of converging positions


# ---------------------------------------------------------------------------------------------------- cases

def listed():
    heads = dict(Hq=32, Hkv=32, D=128)          # a drafter layer of the 7B-shaped targets: 32 heads of 128
    return [
        # the smallest step: one prompt of 64 text tokens and its unconditional twin, latency counts
        dict(name="attn_grad_text", op="attn_grad", dtype="bf16", **heads, page=16, n_req=2, q_lo=64, q_hi=64, kv_lo=64, kv_hi=64,
             window=0, sinks=0, mix=1),
        # one prompt with its 576 image tokens and the twin
        dict(name="attn_grad_image", op="attn_grad", dtype="bf16", **heads, page=16, n_req=2, q_lo=640, q_hi=640, kv_lo=640,
             kv_hi=640, window=0, sinks=0, mix=2),
        # a full batch: eight sequences of 128 text tokens and a 48 x 49 image
        dict(name="attn_grad_batch", op="attn_grad", dtype="bf16", **heads, page=64, n_req=8, q_lo=2480, q_hi=2480, kv_lo=2480,
             kv_hi=2480, window=0, sinks=0, mix=3),
        # pieces of sequences behind the tokens before them, four query heads a key head, a window of 1024, four first tokens
        dict(name="attn_grad_chunk_window", op="attn_grad", dtype="bf16", Hq=32, Hkv=8, D=128, page=16, n_req=16, q_lo=17, q_hi=480,
             kv_lo=700, kv_hi=2880, window=1024, sinks=4, mix=4),
        # ragged sequences of up to 120 text and 1024 image tokens, 20 heads of 64
        dict(name="attn_grad_ragged", op="attn_grad", dtype="bf16", Hq=20, Hkv=20, D=64, page=48, n_req=12, q_lo=100, q_hi=1144,
             kv_lo=1, kv_hi=1, window=0, sinks=0, mix=5),
        # the 32-bit configuration: 4 heads of 64, short ragged sequences
        dict(name="attn_grad_f32", op="attn_grad", dtype="f32", Hq=4, Hkv=4, D=64, page=16, n_req=8, q_lo=47, q_hi=450, kv_lo=1,
             kv_hi=1, window=0, sinks=0, mix=6),
        # a few positions over 16384 image tokens: latency counts
        dict(name="loss_few", op="loss", dtype="f32", V=16384, K=16, n=2000, h=4096, pad=0.0, seqs=1, lse=False, mix=7),
        # two sequences of 48 x 48 image tokens over the 65536-token vocabulary, some positions padding
        dict(name="loss_images", op="loss", dtype="f32", V=65536, K=4608, n=2000, h=4096, pad=0.05, seqs=2, lse=False, mix=8),
        # 16-bit logits over an odd vocabulary, the target's own log-sum-exp beside its largest logits
        dict(name="loss_bf16_odd", op="loss", dtype="bf16", V=10007, K=1153, n=333, h=1280, pad=0.1, seqs=3, lse=True, mix=9),
        # the ways back of the same three
        dict(name="loss_grad_few", op="loss_grad", dtype="f32", V=16384, K=16, n=2000, h=0, pad=0.0, seqs=1, lse=False, mix=10),
        dict(name="loss_grad_images", op="loss_grad", dtype="f32", V=65536, K=4608, n=2000, h=0, pad=0.05, seqs=2, lse=False, mix=11),
        dict(name="loss_grad_bf16_odd", op="loss_grad", dtype="bf16", V=10007, K=1153, n=333, h=0, pad=0.1, seqs=3, lse=True, mix=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.499)))))))


def draw(rng):
    op = rng.choice(["attn_grad", "attn_grad", "attn_grad", "loss", "loss_grad"])
    mix = rng.randrange(1 << 30)
    if op == "attn_grad":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        D = rng.choice([64, 128, 128])
        Hkv, G = rng.choice([(32, 1), (8, 4), (4, 8), (1, 8), (4, 1), (2, 5), (8, 2), (10, 1)])
        page = rng.choice([8, 16, 16, 32, 48, 64, 128])
        q_hi = _log_int(rng, 16, 2480)
        q_lo = rng.choice([q_hi, _log_int(rng, 1, q_hi)])
        whole = rng.random() < 0.6              # whole sequences, or pieces behind the tokens before them
        kv_hi = 1 if whole else max(q_hi, _log_int(rng, 16, 2880))
        kv_lo = 1 if whole else _log_int(rng, 1, kv_hi)
        # no more work than the listed batch (a thirtieth of it in 32 bits)
        most = 8 * 32 * 2480 * 2480 // (30 if dtype == "f32" else 1)
        n_req = _log_int(rng, 1, max(1, min(64, most // (Hkv * G * q_hi * max(q_hi, kv_hi)))))
        window = rng.choice([0, 0, _log_int(rng, 16, 2048)])
        sinks = rng.choice([0, 1, 4, 17, 128]) if window else 0
        return dict(op=op, dtype=dtype, Hq=Hkv * G, Hkv=Hkv, D=D, page=page, n_req=n_req, q_lo=q_lo, q_hi=q_hi, kv_lo=kv_lo,
                    kv_hi=kv_hi, window=window, sinks=sinks, mix=mix)
    V = _log_int(rng, 100, 65536)
    K = _log_int(rng, 1, max(1, min(6000, 4608 * 65536 // V)))
    return dict(op=op, dtype=rng.choice(["f32", "bf16"]), V=V, K=K, n=_log_int(rng, 1, min(V, 4000)),
                h=rng.choice([256, 1280, 4096]) if op == "loss" else 0, pad=rng.choice([0.0, 0.1]), seqs=rng.choice([1, 2, 7]),
                lse=rng.choice([False, True]), mix=mix)


def _lengths(case):
    """The requests' new tokens and lengths (the new ones included): part of the case, not of its inputs."""
    r = random.Random(case["mix"])
    q = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["n_req"])]
    kv = [max(n, r.randint(case["kv_lo"], case["kv_hi"])) for n in q]
    return q, kv


def _sequences(case):
    """The sequence that every position belongs to, -1 for padding at the end of each."""
    K, seqs = case["K"], min(case["seqs"], case["K"])
    seq = np.arange(K) * seqs // K
    for s in range(seqs):
        at = np.flatnonzero(seq == s)
        gone = int(len(at) * case["pad"])
        if gone:
            seq[at[-gone:]] = -1
    return seq.astype(np.int32)


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
    if case["op"] == "attn_grad":
        # queries, outputs, their gradients and the seen keys and values read; three gradients written; five products
        q, kv = _lengths(case)
        seen = [_visible(a, b, case["window"], case["sinks"]) for a, b in zip(q, kv)]
        es, D = BYTES[case["dtype"]], case["D"]
        return {"bytes": 4 * sum(q) * case["Hq"] * D * es + 4 * sum(q) * case["Hq"] + 2 * sum(s[1] for s in seen) * case["Hkv"] * D * es
                + 2 * sum(kv) * case["Hkv"] * D * es + 4 * sum(-(-n // case["page"]) for n in kv),
                "flops": 10 * D * case["Hq"] * sum(s[0] for s in seen)}
    live = int((_sequences(case) >= 0).sum())
    row = case["V"] * BYTES[case["dtype"]]
    if case["op"] == "loss":
        return {"bytes": live * (row + 8 * case["n"] + 4 * case["h"]) + case["K"] * (4 + 4 + 16),
                "flops": live * (4 * case["V"] + 8 * case["n"] + 4 * case["h"])}
    return {"bytes": live * (row + 8 * case["n"]) + case["K"] * (row + 16), "flops": live * (4 * case["V"] + 4 * case["n"])}


# --------------------------------------------------------------------------------------------------- inputs

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
    return table, n_pages


def _i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=DEV)


def _prepare_attn(st, case, gen, rng):
    q_len, kv = _lengths(case)
    Hq, Hkv, D, dt = case["Hq"], case["Hkv"], case["D"], TYPES[case["dtype"]]
    table, n_pages = _table(rng, kv, case["page"], -(-max(kv) // case["page"]))
    normal = lambda *shape: torch.randn(shape, device=DEV, generator=gen).to(dt)                     # noqa: E731
    n = sum(q_len)
    st.update(q=normal(n, Hq, D), k_pages=normal(n_pages, case["page"], Hkv, D), v_pages=normal(n_pages, case["page"], Hkv, D),
              table=_i32(table), q_begin=_i32(np.concatenate([[0], np.cumsum(q_len)])), kv_len=_i32(kv),
              k_begin=_i32(np.cumsum(kv) - kv), max_q=max(q_len), max_kv=max(kv), scale=1.0 / math.sqrt(D))
    # the attention's output and log-sum-exp, from the pass before
    out, lse = [], []
    for see, x, k, v in _groups(st):
        s = x @ k.transpose(-1, -2)
        s *= st["scale"]
        s.masked_fill_(~see, -math.inf)
        z = s.logsumexp(-1)
        s -= torch.where(z == -math.inf, 0.0, z)[..., None]
        out.append((s.exp_() @ v, None))
        lse.append((z[..., None], None))
        del s
    st["out"] = _rows_of(st, [o[0] for o in out]).to(dt)
    st["lse"] = _rows_of(st, [z[0] for z in lse])[..., 0].contiguous()
    st["d_out"] = normal(n, Hq, D)
    st["dq"], st["scratch"] = torch.zeros_like(st["q"]), torch.zeros((n, Hq, 2), device=DEV)
    st["dk"] = torch.zeros((sum(kv), Hkv, D), device=DEV, dtype=dt)
    st["dv"] = torch.zeros_like(st["dk"])


def _prepare_loss(st, case, gen, rng):
    V, K, n, h = case["V"], case["K"], case["n"], case["h"]
    dt = TYPES[case["dtype"]]
    logits = torch.empty((K, V), device=DEV, dtype=dt)
    top, ids, lse = torch.empty((K, n), device=DEV), torch.empty((K, n), device=DEV, dtype=torch.int32), torch.empty(K, device=DEV)
    column = torch.arange(V, device=DEV) % 256
    for a in range(0, K, 512):                  # near-identical codes share the mass: 256 levels and a little noise
        b = min(K, a + 512)
        target = torch.randn((b - a, 256), device=DEV, generator=gen)[:, column] * 2.6
        target += 0.3 * torch.randn((b - a, V), device=DEV, generator=gen)
        top[a:b], i = torch.topk(target, n, dim=1)
        ids[a:b], lse[a:b] = i.int(), target.logsumexp(-1)
        logits[a:b] = target / 1.5 + 0.5 * torch.randn((b - a, V), device=DEV, generator=gen)
    st.update(logits=logits, top=top, ids=ids, seq=_i32(_sequences(case)), target_lse=lse if case["lse"] else None,
              loss=torch.zeros(K, device=DEV), saved=torch.zeros((K, 4), device=DEV), total=torch.zeros(1, device=DEV))
    if case["op"] == "loss":                    # hidden states that drift along some stretches and jump elsewhere
        noise, jump = torch.randn((K, h), device=DEV, generator=gen), torch.as_tensor(rng.random(K) < 0.5, device=DEV)
        start = torch.cummax(torch.where(jump, torch.arange(K, device=DEV), 0), 0)[0]
        st["feat"] = noise[start] + 0.4 * torch.randn((K, h), device=DEV, generator=gen)
    else:                                       # what the loss has left, and what comes back from above
        d, t = torch.empty(K, device=DEV), top.logsumexp(-1) if st["target_lse"] is None else lse
        for a in range(0, K, 512):
            d[a:a + 512] = logits[a:a + 512].float().logsumexp(-1)
        weight = torch.as_tensor(rng.choice([1.0, RAISED], K).astype(np.float32), device=DEV)
        mass = (top - t[:, None]).exp().sum(-1)
        st["saved"] = torch.stack([d, t, mass, torch.where(st["seq"] >= 0, weight, 0.0)], 1).contiguous()
        st["up"] = torch.as_tensor(rng.uniform(0.5, 1.5, K).astype(np.float32), device=DEV) / K
        st["grad"] = torch.zeros_like(logits)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    st = dict(case=case)
    (_prepare_attn if case["op"] == "attn_grad" else _prepare_loss)(st, case, gen, rng)
    if own and case["op"] == "attn_grad":
        from paper_2605_07230_b200 import binding as cb
        dtype = cb.F32 if case["dtype"] == "f32" else cb.BF16
        st["ctx"] = cb.Context(dtype, 1, 1, 64, 64, case["Hq"], case["Hkv"], case["D"], 64)
        st["cache"] = cb.PagedCache(st["k_pages"], st["v_pages"], st["table"])
    return st


# ---------------------------------------------------------------------------------------------- plain forms

def _batches(st):
    """Requests (first, last + 1) whose padded scores fit a gigabyte or two at once."""
    c = st["case"]
    per = max(1, (1 << 28) // (c["Hq"] * st["max_q"] * st["max_kv"]))
    return [(a, min(a + per, c["n_req"])) for a in range(0, c["n_req"], per)]


def _row_index(st, a, b):
    begin = st["q_begin"].long()
    i = torch.arange(st["max_q"], device=DEV)[None, :]
    return (begin[a:b, None] + i).clamp(max=st["q"].shape[0] - 1), i < (begin[a + 1:b + 1] - begin[a:b])[:, None]


def _by_head(st, x, a, b):
    """Rows of [n_tok, Hq, D], in 32 bits, as [requests, key heads, group x max_q, D]; zeros where there is no row."""
    c = st["case"]
    rows, live = _row_index(st, a, b)
    x = torch.where(live[:, :, None, None], x[rows].float(), 0.0).view(b - a, st["max_q"], c["Hkv"], c["Hq"] // c["Hkv"], -1)
    return x.permute(0, 2, 3, 1, 4).reshape(b - a, c["Hkv"], -1, x.shape[-1])


def _groups(st):
    """For each batch of requests: the mask, queries, keys and values by key head, padded with zeros."""
    c = st["case"]
    begin, kvl = st["q_begin"].long(), st["kv_len"].long()
    nq, nk, G = st["max_q"], st["max_kv"], c["Hq"] // c["Hkv"]
    for a, b in _batches(st):
        pages = st["table"][a:b, :-(-nk // c["page"])].long().clamp(min=0)
        there = (torch.arange(nk, device=DEV)[None, :] < kvl[a:b, None])[:, :, None, None]
        keys = lambda p: torch.where(there, p[pages].reshape(b - a, -1, c["Hkv"], c["D"])[:, :nk].float(), 0.0).permute(0, 2, 1, 3)  # noqa: E731,B023
        i = torch.arange(nk, device=DEV)[None, None, :]
        p = (kvl[a:b] - (begin[a + 1:b + 1] - begin[a:b]))[:, None, None] + torch.arange(nq, device=DEV)[None, :, None]
        see = (i <= p) & (i < kvl[a:b, None, None])
        if c["window"]:
            see &= (i > p - c["window"]) | (i < c["sinks"])
        see &= _row_index(st, a, b)[1][:, :, None]
        see = see[:, None, None].expand(b - a, 1, G, nq, nk).reshape(b - a, 1, G * nq, nk)
        yield see, _by_head(st, st["q"], a, b), keys(st["k_pages"]), keys(st["v_pages"])


def _rows_of(st, parts):
    """The way back from [requests, key heads, group x max_q, D], batch by batch, to [n_tok, Hq, D]."""
    c = st["case"]
    rows = []
    for (a, b), x in zip(_batches(st), parts):
        x = x.view(b - a, c["Hkv"], c["Hq"] // c["Hkv"], st["max_q"], -1).permute(0, 3, 1, 2, 4)
        rows.append(x.reshape(b - a, st["max_q"], c["Hq"], -1).reshape(-1, c["Hq"], x.shape[-1]))
    begin = st["q_begin"].long()
    t = torch.arange(st["q"].shape[0], device=DEV)
    r = torch.searchsorted(begin[1:], t, right=True)
    return torch.cat(rows)[r * st["max_q"] + t - begin[r]]


def _plain_attn_grad(st):
    scale, dq, dk, dv = st["scale"], [], [], []
    for (a, b), (see, x, k, v) in zip(_batches(st), _groups(st)):
        do, o, lse = (_by_head(st, t, a, b) for t in (st["d_out"], st["out"], st["lse"][..., None]))
        delta = (do * o).sum(-1, keepdim=True)
        p = x @ k.transpose(-1, -2)
        p *= scale
        p -= lse
        p.masked_fill_(~see, -math.inf)
        p.exp_()
        dv.append(p.transpose(-1, -2) @ do)
        ds = do @ v.transpose(-1, -2)
        ds -= delta
        ds *= p
        del p
        dq.append(scale * (ds @ k))
        dk.append(scale * (ds.transpose(-1, -2) @ x))
        del ds
    kvl, first = st["kv_len"].long(), st["k_begin"].long()
    t = torch.arange(st["dk"].shape[0], device=DEV)
    r = torch.searchsorted(first + kvl, t, right=True)
    flat = lambda parts: torch.cat([y.permute(0, 2, 1, 3) for y in parts])[r, t - first[r]].to(st["q"].dtype)  # noqa: E731
    return [_rows_of(st, dq).to(st["q"].dtype), flat(dk), flat(dv)]


def _plain_loss(st):
    feat, seq, ids = st["feat"].double(), st["seq"], st["ids"].long()      # (64 bits: a cosine may lie next to the threshold)
    size = feat.pow(2).sum(-1).sqrt()
    near = (feat[:-1] * feat[1:]).sum(-1) / (size[:-1] * size[1:])
    weight = torch.ones_like(st["loss"])
    weight[:-1] = torch.where((near >= TAU) & (seq[:-1] == seq[1:]), RAISED, 1.0)
    weight = torch.where(seq >= 0, weight, 0.0)
    x = st["logits"].float()
    m = x.amax(-1, keepdim=True)
    lse = m[:, 0] + (x - m).exp().sum(-1).log()
    top = st["top"]
    t = st["target_lse"]
    if t is None:
        high = top.amax(-1, keepdim=True)
        t = high[:, 0] + (top - high).exp().sum(-1).log()
    q = (top - t[:, None]).exp()
    loss = weight * (q * (lse[:, None] - x.gather(1, ids))).sum(-1)
    return [loss, torch.stack([lse, t, q.sum(-1), weight], 1) * (seq >= 0)[:, None], loss.double().sum().float().view(1)]


def _plain_loss_grad(st):
    lse, t, mass, weight = st["saved"].unbind(1)
    g = (st["logits"].float() - lse[:, None]).exp_()
    g *= mass[:, None]
    g.scatter_add_(1, st["ids"].long(), -(st["top"] - t[:, None]).exp())
    g *= (weight * st["up"])[:, None]
    return torch.where(weight[:, None] > 0, g, 0.0).to(st["logits"].dtype)


def run(st):
    op = st["case"]["op"]
    if own:
        from paper_2605_07230_b200 import binding as cb
        if op == "attn_grad":
            cb.cascade_paged_attn_grad(st["ctx"], st["cache"], st["q"], st["q_begin"], st["kv_len"], st["max_q"], st["max_kv"],
                                       st["out"], st["lse"], st["d_out"], st["scratch"], st["dq"], st["dk"], st["dv"], st["scale"],
                                       window=st["case"]["window"], sinks=st["case"]["sinks"], k_begin=st["k_begin"])
            return [st["dq"], st["dk"], st["dv"]]
        if op == "loss":
            cb.cascade_distill_loss(st["logits"], st["top"], st["ids"], st["loss"], st["saved"], total=st["total"],
                                    target_lse=st["target_lse"], feat=st["feat"], seq=st["seq"], tau_seq=TAU, c=RAISED)
            return [st["loss"], st["saved"], st["total"]]
        cb.cascade_distill_grad(st["logits"], st["top"], st["ids"], st["saved"], st["grad"], grad_loss=st["up"])
        return st["grad"]
    return {"attn_grad": _plain_attn_grad, "loss": _plain_loss, "loss_grad": _plain_loss_grad}[op](st)


# ---------------------------------------------------------------------------------------- in 64 bits, apart

def _exact_attn_grad(st):
    """Request by request and head by head; the softmax's Jacobian row by row from the given outputs."""
    c = st["case"]
    q_len, kv_len = _lengths(c)
    dq = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    dk = torch.zeros(st["dk"].shape, dtype=torch.float64, device=DEV)
    dv = torch.zeros_like(dk)
    at = first = 0
    for r in range(c["n_req"]):
        n, L = q_len[r], kv_len[r]
        where = torch.arange(L, device=DEV)
        page, row = st["table"][r].long()[where // c["page"]], where % c["page"]
        x = L - n + torch.arange(n, device=DEV)[:, None]
        see = where[None, :] <= x
        if c["window"]:
            see &= (where[None, :] > x - c["window"]) | (where < c["sinks"])[None, :]
        for h in range(c["Hq"]):
            kh = h * c["Hkv"] // c["Hq"]
            k, v = st["k_pages"][page, row, kh].double(), st["v_pages"][page, row, kh].double()
            q, o, g = (st[name][at:at + n, h].double() for name in ("q", "out", "d_out"))
            w = torch.exp(torch.einsum("id,jd->ij", q, k) * st["scale"] - st["lse"][at:at + n, h].double()[:, None])
            w = torch.where(see, w, 0.0)
            e = w * (torch.einsum("id,jd->ij", g, v) - torch.einsum("id,id->i", g, o)[:, None]) * st["scale"]
            dq[at:at + n, h] = torch.einsum("ij,jd->id", e, k)
            dk[first:first + L, kh] += torch.einsum("ij,id->jd", e, q)
            dv[first:first + L, kh] += torch.einsum("ij,id->jd", w, g)
        at += n
        first += L
    return [dq, dk, dv]


def _exact_loss(st):
    """Position by position."""
    c, seq = st["case"], st["seq"].tolist()
    loss = torch.zeros(c["K"], dtype=torch.float64, device=DEV)
    saved = torch.zeros((c["K"], 4), dtype=torch.float64, device=DEV)
    for k in range(c["K"]):
        if seq[k] < 0:
            continue
        weight = 1.0
        if k + 1 < c["K"] and seq[k + 1] == seq[k]:
            a, b = st["feat"][k].double(), st["feat"][k + 1].double()
            weight = torch.where(torch.dot(a, b) >= TAU * torch.linalg.norm(a) * torch.linalg.norm(b), RAISED, 1.0)
        x = st["logits"][k].double()
        top = st["top"][k].double()
        lse, t = torch.logsumexp(x, 0), torch.logsumexp(top, 0) if st["target_lse"] is None else st["target_lse"][k].double()
        q = torch.exp(top - t)
        loss[k] = -weight * torch.dot(q, x[st["ids"][k].long()] - lse)
        saved[k] = torch.stack([lse, t, q.sum(), torch.as_tensor(weight, dtype=torch.float64, device=DEV)])
    return [loss, saved, loss.sum().view(1)]


def _exact_loss_grad(st):
    c, seq = st["case"], st["seq"].tolist()
    grad = torch.zeros((c["K"], c["V"]), dtype=torch.float64, device=DEV)
    for k in range(c["K"]):
        if seq[k] < 0:
            continue
        lse, t, mass, weight = st["saved"][k].double()
        grad[k] = mass * torch.exp(st["logits"][k].double() - lse)
        grad[k, st["ids"][k].long()] -= torch.exp(st["top"][k].double() - t)
        grad[k] *= weight * st["up"][k].double()
    return grad


def exact(case, seed):
    st = prepare(case, seed)
    return {"attn_grad": _exact_attn_grad, "loss": _exact_loss, "loss_grad": _exact_loss_grad}[case["op"]](st)

"""Cases of the operators that serve a paged key/value cache and read a model's answer.

Three operators, used one after the other in every step of a server that keeps its cache in pages:

  append   the keys and values of new tokens go into their sequences' pages; on the way keys (and the queries, which are
           not cached) are turned by their position
  attend   one new query per row against the cached keys of its sequence, found through the page table
  score    log probability of a given token, entropy, and the best alternatives of every row of logits

With `own` false `run` computes them from elementary torch operations; with `own` true through this repository's calls.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
DEVICE = "cuda"


# ---------------------------------------------------------------------------------------------------- the cases

def _append(name, seqs, new, past, q_heads, kv_heads, head_dim, rot, interleaved, page, dtype, padding=0):
    """`new`: most new tokens of a sequence (each brings between half of it and all of it); `past`: tokens that a sequence
    may have already; `padding`: rows at the end that belong to no sequence."""
    return {"name": name, "op": "append", "seqs": seqs, "new": new, "past": past, "q_heads": q_heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rot": rot, "interleaved": interleaved, "page": page, "dtype": dtype, "padding": padding}


def _attend(name, seqs, shortest, longest, q_heads, kv_heads, head_dim, page, dtype, cap=0.0, window=0, slopes=False):
    return {"name": name, "op": "attend", "seqs": seqs, "shortest": shortest, "longest": longest, "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "dtype": dtype, "cap": cap, "window": window,
            "slopes": slopes}


def _score(name, rows, vocab, top, scale, dtype, padded=0):
    """`padded`: columns behind the vocabulary in the tensor that the rows are a slice of."""
    return {"name": name, "op": "score", "rows": rows, "vocab": vocab, "top": top, "scale": scale, "dtype": dtype,
            "padded": padded}


def listed():
    return [
        # one user's next token: nothing but latency
        _append("append one token", 1, 1, 4000, 32, 8, 128, 128, False, 16, "bf16"),
        # one decode step of a batch of 64
        _append("append a batch step", 64, 1, 2100, 16, 16, 64, 64, False, 16, "bf16"),
        # packed prompts of different lengths, rotation of neighbouring pairs on half of the head only, pages whose size is
        # no power of two, a batch padded to a fixed number of rows
        _append("append ragged prompts", 9, 150, 300, 12, 4, 96, 48, True, 24, "f16", padding=31),
        # four full prompts
        _append("append four prompts", 4, 2048, 0, 16, 16, 128, 128, False, 64, "bf16"),
        # one user, short context: latency
        _attend("attend one short", 1, 500, 500, 16, 16, 64, 16, "bf16"),
        # a decode step of a batch of 16 near 2100 tokens, one key/value head per query head
        _attend("attend a batch step", 16, 2048, 2176, 16, 16, 64, 16, "bf16"),
        # a server's mix of lengths, eight query heads to a key/value head, capped scores
        _attend("attend ragged capped", 64, 16, 8192, 32, 4, 128, 64, "bf16", cap=30.0),
        # a long document of one user: all the parallelism there is lies along the keys
        _attend("attend one long", 1, 131072, 131072, 32, 8, 128, 128, "f16"),
        # distance bias and a sliding window, odd sizes
        _attend("attend window slopes", 24, 1, 6001, 12, 12, 104, 24, "f16", window=1000, slopes=True),
        # the next token of one user
        _score("score one row", 1, 50257, 20, 1.0, "f32"),
        # the next tokens of a batch, 16-bit logits, a temperature, rows cut out of a wider product
        _score("score a batch step", 48, 51200, 20, 1.25, "bf16", padded=64),
        # every token of a prompt
        _score("score a prompt", 2048, 50257, 5, 1.0, "f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("append", "attend", "score"))
    if op == "append":
        kv_heads = rng.choice((1, 2, 4, 8, 12, 16))
        head_dim = rng.choice((64, 72, 96, 104, 128))
        rot = rng.choice((0, 16, 32, 64, head_dim))
        seqs = _log(rng, 1, 200)
        new = 1 if rng.random() < 0.4 else _log(rng, 2, max(2, 6000 // seqs))
        return _append("", seqs, new, _log(rng, 1, 3000), kv_heads * rng.choice((1, 2, 3, 4)) if kv_heads <= 8 else kv_heads,
                       kv_heads, head_dim, rot, rng.random() < 0.5, rng.choice((1, 8, 16, 24, 64, 100, 256)),
                       rng.choice(("bf16", "f16")), padding=rng.choice((0, 0, 5)))
    if op == "attend":
        kv_heads = rng.choice((1, 2, 4, 8, 12))
        longest = _log(rng, 1, 60000)
        seqs = _log(rng, 1, max(1, min(200, 200000 // longest // kv_heads * 4)))
        return _attend("", seqs, _log(rng, 1, longest), longest, kv_heads * rng.choice((1, 2, 4, 5, 8, 16)), kv_heads,
                       rng.choice((64, 72, 96, 104, 128)), rng.choice((1, 8, 16, 24, 64, 100, 256)),
                       rng.choice(("bf16", "f16")), cap=rng.choice((0.0, 0.0, 20.0, 50.0)),
                       window=rng.choice((0, 0, 1, 128, 1000)), slopes=rng.random() < 0.3)
    vocab = _log(rng, 40, 150000)
    rows = _log(rng, 1, max(1, min(5000, 90000000 // vocab)))
    return _score("", rows, vocab, rng.choice((0, 1, 5, 20, 32)), rng.choice((1.0, 0.7, 1.25)),
                  rng.choice(("f32", "bf16", "f16")), padded=rng.choice((0, 0, 3, 64)))


# ---------------------------------------------------------------------------------------------------- lengths, the same for every seed

def _pick(case):
    return random.Random(_key(case))


def _key(case):
    return repr(sorted((k, v) for k, v in case.items() if k != "name"))


def _new_tokens(case):
    """(past, new) of every sequence."""
    r = _pick(case)
    return [(r.randint(0, case["past"]), r.randint((case["new"] + 1) // 2, case["new"])) for _ in range(case["seqs"])]


def _lengths(case):
    r = _pick(case)
    n = [_log(r, case["shortest"], case["longest"]) for _ in range(case["seqs"] - 1)] + [case["longest"]]
    if case["seqs"] > 4:
        n[2] = 0          # a row of the batch whose sequence has nothing in the cache yet
    return n


def _seen(case, n):
    return min(n, case["window"]) if case["window"] else n


def work(case):
    if case["op"] == "append":
        tokens = sum(new for _, new in _new_tokens(case))
        values = tokens * (case["q_heads"] + 2 * case["kv_heads"]) * case["head_dim"]
        turned = tokens * (case["q_heads"] + case["kv_heads"]) * case["rot"]
        return {"bytes": 4 * values + 12 * tokens + 2 * case["rot"], "flops": 3 * turned}
    if case["op"] == "attend":
        keys = sum(_seen(case, n) for n in _lengths(case))
        row = case["q_heads"] * case["head_dim"]
        return {"bytes": 4 * keys * case["kv_heads"] * case["head_dim"] + case["seqs"] * (4 * row + 4 * case["q_heads"] + 4)
                + 4 * keys // case["page"], "flops": 4 * keys * row}
    size = 4 if case["dtype"] == "f32" else 2
    return {"bytes": case["rows"] * (case["vocab"] * size + 12 + 8 * case["top"]), "flops": 5 * case["rows"] * case["vocab"]}


# ---------------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE).mul_(scale)

    dtype = DTYPES[case["dtype"]]
    if case["op"] == "score":
        rows, vocab = case["rows"], case["vocab"]
        # rows between flat and sharp; a thousandth of the tokens is forbidden
        sharp = 0.5 + 4 * torch.rand(rows, 1, generator=g, device=DEVICE)
        x = normal(rows, vocab + case["padded"]) * sharp
        x[torch.rand(x.shape, generator=g, device=DEVICE) < 1e-3] = -math.inf
        logits = x.to(dtype)[:, :vocab]
        targets = torch.randint(0, vocab, (rows,), generator=g, device=DEVICE, dtype=torch.int32)
        targets[5::7] = -1    # tokens that are not asked for
        return {"case": case, "logits": logits, "targets": targets}

    H, Hkv, hd, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    if case["op"] == "append":
        spans = _new_tokens(case)
        ends = [past + new for past, new in spans]
    else:
        ends = _lengths(case)
    width = max(1, max(-(-n // page) for n in ends))
    used = [-(-n // page) for n in ends]
    n_pages = sum(used) + 3
    order = torch.randperm(n_pages, generator=g, device=DEVICE).to(torch.int32)     # pages were handed out in any order
    table = torch.full((case["seqs"], width), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(used):
        table[s, :n] = torch.arange(at, at + n, dtype=torch.int32)
        at += n
    table = table.to(DEVICE)
    table = torch.where(table >= 0, order[table.clamp(min=0).long()], table)
    k_cache = normal(n_pages, Hkv, page, hd).to(dtype)
    v_cache = normal(n_pages, Hkv, page, hd).to(dtype)
    s = {"case": case, "k_cache": k_cache, "v_cache": v_cache, "table": table}
    if case["op"] == "attend":
        s["q"] = normal(case["seqs"], H, hd).to(dtype)
        s["n_keys"] = torch.tensor(ends, dtype=torch.int32, device=DEVICE)
        s["slopes"] = None
        if case["slopes"]:
            s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=DEVICE)
        return s
    rows = sum(new for _, new in spans) + case["padding"]
    # q, k and v lie side by side in the rows of one product
    qkv = normal(rows, (H + 2 * Hkv) * hd).to(dtype)
    s["q"] = qkv[:, :H * hd].unflatten(1, (H, hd))
    s["k"] = qkv[:, H * hd:(H + Hkv) * hd].unflatten(1, (Hkv, hd))
    s["v"] = qkv[:, (H + Hkv) * hd:].unflatten(1, (Hkv, hd))
    s["q_out"] = torch.zeros(rows, H, hd, dtype=dtype, device=DEVICE)
    seq = [i for i, (_, new) in enumerate(spans) for _ in range(new)] + [-1] * case["padding"]
    pos = [past + i for past, new in spans for i in range(new)] + [0] * case["padding"]
    s["row_seq"] = torch.tensor(seq, dtype=torch.int32, device=DEVICE)
    s["positions"] = torch.tensor(pos, dtype=torch.int32, device=DEVICE)
    s["live"] = rows - case["padding"]
    half = case["rot"] // 2
    s["inv_freq"] = torch.tensor([10000.0 ** (-i / half) for i in range(half)], device=DEVICE) if half else None
    return s


# ---------------------------------------------------------------------------------------------------- one pass

def run(state):
    return {"append": run_append, "attend": run_attend, "score": run_score}[state["case"]["op"]](state)


def run_append(s):
    case = s["case"]
    if own:
        import paper_2408_07802_b200 as kr
        q = kr.op_paged_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["positions"], row_seq=s["row_seq"],
                               q=s["q"], q_out=s["q_out"], inv_freq=s["inv_freq"], interleaved=case["interleaved"])
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    n = s["live"]
    pos, seq = s["positions"][:n].long(), s["row_seq"][:n].long()
    pages, slots = s["table"][seq, pos // case["page"]].long(), pos % case["page"]
    q, k = s["q"][:n].float(), s["k"][:n].float()
    if s["inv_freq"] is not None:
        angle = pos.double()[:, None, None] * s["inv_freq"].double()
        cos, sin = angle.cos().float(), angle.sin().float()
        q, k = _turned(q, cos, sin, case), _turned(k, cos, sin, case)
    s["q_out"][:n] = q.to(s["q"].dtype)
    s["k_cache"][pages, :, slots] = k.to(s["k"].dtype)
    s["v_cache"][pages, :, slots] = s["v"][:n]
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _turned(x, cos, sin, case):
    rot = case["rot"]
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((turned, x[..., rot:]), dim=-1)


def run_attend(s):
    case = s["case"]
    if own:
        import paper_2408_07802_b200 as kr
        out, lse = kr.op_paged_decode_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["n_keys"],
                                                score_cap=case["cap"], window=case["window"], slopes=s["slopes"])
        return {"out": out, "lse": lse}
    B, H, hd = s["q"].shape
    Hkv, page = case["kv_heads"], case["page"]
    pages = s["table"].clamp(min=0).long()
    k = s["k_cache"][pages].transpose(1, 2).flatten(2, 3).float()      # [B, Hkv, width * page, hd]
    v = s["v_cache"][pages].transpose(1, 2).flatten(2, 3).float()
    q = s["q"].float().unflatten(1, (Hkv, H // Hkv))
    x = (q @ k.transpose(-1, -2)).flatten(1, 2) * hd ** -0.5             # [B, H, keys]
    if case["cap"]:
        x = case["cap"] * torch.tanh(x / case["cap"])
    at, n = torch.arange(x.shape[-1], device=x.device), s["n_keys"][:, None]
    if s["slopes"] is not None:
        x = x + s["slopes"][:, None] * (at - (n - 1)).float()[:, None, :]
    seen = at < n
    if case["window"]:
        seen = seen & (at >= n - case["window"])
    x = x.masked_fill(~seen[:, None, :], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    out = (e.unflatten(1, (Hkv, H // Hkv)) @ v).flatten(1, 2) / total.clamp(min=1e-38)
    return {"out": out.to(s["q"].dtype), "lse": (top + torch.log(total)).squeeze(-1)}


def run_score(s):
    case = s["case"]
    if own:
        import paper_2408_07802_b200 as kr
        got = kr.op_token_logprobs(s["logits"], s["targets"], top=case["top"], scale=case["scale"])
        logprob, entropy, ids, best = got.logprob, got.entropy, got.top_ids, got.top_logprobs
        return {"logprob": logprob, "entropy": entropy, "ids": ids, "best": best} if case["top"] else {"logprob": logprob, "entropy": entropy}
    raw = s["logits"].float()
    x = raw * case["scale"]
    below = x - x.amax(-1, keepdim=True)
    e = torch.exp(below)
    total = e.sum(-1, keepdim=True)
    logs = below - torch.log(total)
    entropy = torch.log(total).squeeze(-1) - (e * below.clamp(min=-3e38)).sum(-1) / total.squeeze(-1)
    target = s["targets"].long()
    logprob = logs.gather(-1, target.clamp(min=0)[:, None]).squeeze(-1)
    logprob = torch.where(target >= 0, logprob, torch.zeros_like(logprob))
    if not case["top"]:
        return {"logprob": logprob, "entropy": entropy}
    ids = raw.sort(dim=-1, descending=True, stable=True).indices[:, :case["top"]]     # equal ones: the lowest index first
    return {"logprob": logprob, "entropy": entropy, "ids": ids.to(torch.int32), "best": logs.gather(-1, ids)}


# ---------------------------------------------------------------------------------------------------- in 64 bits, from the definitions

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "score":
        x = s["logits"].double() * case["scale"]
        lse = torch.logsumexp(x, -1)
        t = s["targets"].long()
        logprob = torch.where(t < 0, 0.0, x.gather(1, t.clamp(min=0)[:, None])[:, 0] - lse)
        p = torch.exp(x - lse[:, None])
        entropy = torch.special.entr(p).sum(-1)
        if not case["top"]:
            return {"logprob": logprob, "entropy": entropy}
        best = torch.topk(x, case["top"], dim=-1).values - lse[:, None]
        return {"logprob": logprob, "entropy": entropy, "ids": None, "best": best}
    page = case["page"]
    if case["op"] == "append":
        rot, n = case["rot"], s["live"]
        seq, pos, table = s["row_seq"].tolist(), s["positions"].tolist(), s["table"].tolist()

        def turn(x):
            x = x.double()
            if not rot:
                return x
            # a pair of the rotated part is a complex number, the rotation a product with one of length 1
            pairs = x[..., :rot].unflatten(-1, (rot // 2, 2)) if case["interleaved"] else x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
            z = torch.view_as_complex(pairs.contiguous())
            theta = s["positions"][:, None].double() * s["inv_freq"].double()
            z = torch.view_as_real(z * torch.polar(torch.ones_like(theta), theta)[:, None, :])
            turned = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
            return torch.cat((turned, x[..., rot:]), -1)

        q_out, k, v = s["q_out"].double(), turn(s["k"]), s["v"].double()
        q_out[:n] = turn(s["q"])[:n]
        k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
        where = torch.tensor([table[seq[i]][pos[i] // page] * page + pos[i] % page for i in range(n)], device=DEVICE)
        for cache, new in ((k_cache, k), (v_cache, v)):
            by_token = cache.transpose(1, 2).reshape(-1, *new.shape[1:]).clone()
            by_token[where] = new[:n]
            cache.copy_(by_token.unflatten(0, (-1, page)).transpose(1, 2))
        return {"q": q_out, "k_cache": k_cache, "v_cache": v_cache}
    B, H, hd = s["q"].shape
    rep = H // case["kv_heads"]
    out = torch.zeros(B, H, hd, dtype=torch.float64, device=DEVICE)
    lse = torch.full((B, H), -math.inf, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(s["n_keys"].tolist()):
        if n == 0:
            continue
        lo = n - _seen(case, n)
        pages = s["table"][b, lo // page:(n - 1) // page + 1].long()
        skip = lo % page
        for h in range(case["kv_heads"]):
            k = s["k_cache"][pages, h].flatten(0, 1)[skip:skip + n - lo].double()
            v = s["v_cache"][pages, h].flatten(0, 1)[skip:skip + n - lo].double()
            x = s["q"][b, h * rep:(h + 1) * rep].double() @ k.T / math.sqrt(hd)
            if case["cap"]:
                x = torch.tanh(x / case["cap"]) * case["cap"]
            if s["slopes"] is not None:
                distance = torch.arange(n - lo, device=DEVICE).double() - (n - lo - 1)
                x = x + s["slopes"][h * rep:(h + 1) * rep, None].double() * distance
            out[b, h * rep:(h + 1) * rep] = torch.softmax(x, -1) @ v
            lse[b, h * rep:(h + 1) * rep] = torch.logsumexp(x, -1)
    return {"out": out, "lse": lse}

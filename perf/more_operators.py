"""Cases of the operators that take prompts into a paged key/value cache piece by piece and choose the tokens that follow.

Three operators, used one after the other in every step of a server whose batches mix pieces of prompts with single tokens:

  norm     the keys and queries of new tokens are normalised head by head, turned by their position and (the keys, with the
           values) put into their sequences' pages
  chunk    several new tokens of every sequence, those of all sequences packed one after the other, attend over the pages:
           each token sees the cached keys up to its own
  sample   one token of every row of logits is drawn with a given random number, after temperature, top-k, min-p and top-p

With `own` false `run` computes them from elementary torch operations; with `own` true through this repository's calls.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
DEVICE = "cuda"
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------- the cases

def _norm(name, seqs, new, past, q_heads, kv_heads, head_dim, rot, interleaved, page, dtype, padding=0, by_head=False):
    """`new`: most new tokens of a sequence (each brings between half of it and all of it); `past`: tokens that a sequence
    may have already; `padding`: rows at the end that belong to no sequence; `by_head`: every head has weights of its own."""
    return {"name": name, "op": "norm", "seqs": seqs, "new": new, "past": past, "q_heads": q_heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rot": rot, "interleaved": interleaved, "page": page, "dtype": dtype, "padding": padding,
            "by_head": by_head}


def _chunk(name, seqs, new, past, q_heads, kv_heads, head_dim, page, dtype, single=0.0, cap=0.0, window=0, slopes=False, padding=0):
    """`single`: the share of the sequences that bring one token only (the others: between half of `new` and all of it)."""
    return {"name": name, "op": "chunk", "seqs": seqs, "new": new, "past": past, "q_heads": q_heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "dtype": dtype, "single": single, "cap": cap, "window": window, "slopes": slopes,
            "padding": padding}


def _sample(name, rows, vocab, dtype, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, padded=0):
    """`mixed`: every row has parameters of its own, around the given ones; `padded`: columns behind the vocabulary in the
    tensor that the rows are a slice of."""
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "temperature": temperature,
            "top_k": top_k, "top_p": top_p, "min_p": min_p, "mixed": mixed, "padded": padded}


def listed():
    return [
        # one user's next token: nothing but latency
        _norm("norm one token", 1, 1, 4000, 32, 8, 128, 128, False, 16, "bf16"),
        # packed prompts of different lengths, neighbouring pairs on half of the head, weights for every head, pages whose size
        # is no power of two, a batch padded to a fixed number of rows
        _norm("norm ragged prompts", 9, 150, 300, 12, 4, 96, 48, True, 24, "f16", padding=31, by_head=True),
        # four full prompts
        _norm("norm four prompts", 4, 2048, 0, 16, 16, 128, 128, False, 64, "bf16"),
        # a few drafted tokens of one user, checked in one step: latency
        _chunk("chunk draft tokens", 1, 5, 1500, 32, 8, 128, 16, "bf16"),
        # a server's step: most sequences bring one token, some a piece of their prompt; capped scores
        _chunk("chunk mixed batch", 24, 512, 4000, 16, 4, 64, 16, "bf16", single=0.75, cap=30.0, padding=17),
        # distance bias and a sliding window, odd sizes
        _chunk("chunk window slopes", 7, 301, 1700, 12, 12, 104, 24, "f16", window=1000, slopes=True),
        # four whole prompts, no past
        _chunk("chunk four prompts", 4, 2048, 0, 16, 16, 128, 64, "bf16"),
        # one more piece of a long document: the largest
        _chunk("chunk long document", 1, 2048, 32768, 32, 8, 128, 128, "f16"),
        # the next token of one user
        _sample("sample one row", 1, 50257, "f32", temperature=0.8, top_p=0.95),
        # the next tokens of a batch of users who all chose for themselves, 16-bit logits, rows cut out of a wider product
        _sample("sample a mixed batch", 64, 51200, "bf16", temperature=0.9, top_k=50, top_p=0.9, min_p=0.02, mixed=True, padded=64),
        # many samples a prompt, nothing but the temperature
        _sample("sample many rows", 512, 50257, "f32", temperature=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "chunk", "chunk", "sample"))
    if op == "norm":
        kv_heads = rng.choice((1, 2, 4, 8, 12, 16))
        head_dim = rng.choice((64, 72, 96, 104, 128))
        rot = rng.choice((0, 16, 32, 64, head_dim))
        seqs = _log(rng, 1, 200)
        new = 1 if rng.random() < 0.4 else _log(rng, 2, max(2, 6000 // seqs))
        return _norm("", seqs, new, _log(rng, 1, 3000), kv_heads * rng.choice((1, 2, 3, 4)) if kv_heads <= 8 else kv_heads,
                     kv_heads, head_dim, rot, rng.random() < 0.5, rng.choice((1, 8, 16, 24, 64, 100, 256)),
                     rng.choice(("bf16", "f16")), padding=rng.choice((0, 0, 5)), by_head=rng.random() < 0.3)
    if op == "chunk":
        kv_heads = rng.choice((1, 2, 4, 8, 12))
        q_heads = kv_heads * rng.choice((1, 2, 3, 4, 5, 8)) if kv_heads <= 4 else kv_heads
        new = _log(rng, 1, 3000)
        # (the plain form makes every sequence as long as the longest)
        past = min(_log(rng, 1, 30000), 2000000000 // (q_heads * new) - new)
        seqs = _log(rng, 1, max(1, min(100, 2000000000 // (q_heads * new * (past + new)), 8000000 // (kv_heads * (past + new)))))
        return _chunk("", seqs, new, past, q_heads, kv_heads, rng.choice((64, 72, 96, 104, 128)),
                      rng.choice((1, 8, 16, 24, 64, 100, 256)), rng.choice(("bf16", "f16")), single=rng.choice((0.0, 0.0, 0.5, 0.9)),
                      cap=rng.choice((0.0, 0.0, 20.0, 50.0)), window=rng.choice((0, 0, 1, 128, 1000)), slopes=rng.random() < 0.3,
                      padding=rng.choice((0, 0, 7)))
    vocab = _log(rng, 40, 150000)
    rows = _log(rng, 1, max(1, min(1000, 25000000 // vocab)))
    return _sample("", rows, vocab, rng.choice(("f32", "bf16", "f16")), temperature=rng.choice((0.6, 1.0, 1.3)),
                   top_k=rng.choice((0, 0, 1, 20, 1000)), top_p=rng.choice((1.0, 0.5, 0.9, 0.95)), min_p=rng.choice((0.0, 0.0, 0.05)),
                   mixed=rng.random() < 0.3, padded=rng.choice((0, 0, 3, 64)))


# ---------------------------------------------------------------------------------------------------- lengths, the same for every seed

def _spans(case):
    """(past, new) of every sequence."""
    r = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    spans = []
    for i in range(case["seqs"]):
        past = case["past"] if case["op"] == "chunk" and i == 0 else r.randint(0, case["past"])
        new = 1 if r.random() < case.get("single", 0.0) else r.randint((case["new"] + 1) // 2, case["new"])
        spans.append((past, case["new"] if case["op"] == "chunk" and i == 0 else new))
    return spans


def _pairs(case, past, new):
    """(query token, visible key) pairs of a sequence."""
    w = case["window"]
    return sum(min(past + i + 1, w) if w else past + i + 1 for i in range(new))


def work(case):
    if case["op"] == "norm":
        tokens = sum(new for _, new in _spans(case))
        heads = case["q_heads"] + case["kv_heads"]
        values = tokens * (heads + case["kv_heads"]) * case["head_dim"]
        weights = case["head_dim"] * (heads if case["by_head"] else 2)
        return {"bytes": 4 * values + 12 * tokens + 2 * case["rot"] + 2 * weights,
                "flops": tokens * heads * (4 * case["head_dim"] + 3 * case["rot"])}
    if case["op"] == "chunk":
        spans, w, row = _spans(case), case["window"], case["q_heads"] * case["head_dim"]
        keys = sum(min(past + new, w + new - 1) if w else past + new for past, new in spans)
        rows = sum(new for _, new in spans)
        return {"bytes": 4 * keys * case["kv_heads"] * case["head_dim"] + rows * (4 * row + 4 * case["q_heads"]) + 4 * keys // case["page"],
                "flops": 4 * row * sum(_pairs(case, past, new) for past, new in spans)}
    size = 4 if case["dtype"] == "f32" else 2
    return {"bytes": case["rows"] * (case["vocab"] * size + 28), "flops": 4 * case["rows"] * case["vocab"]}


# ---------------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE).mul_(scale)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=DEVICE)

    dtype = DTYPES[case["dtype"]]
    if case["op"] == "sample":
        rows, vocab = case["rows"], case["vocab"]
        # rows between flat and sharp; a thousandth of the tokens is forbidden
        x = normal(rows, vocab + case["padded"]) * (0.5 + 4 * uniform(rows, 1))
        x[uniform(*x.shape) < 1e-3] = -math.inf
        s = {"case": case, "logits": x.to(dtype)[:, :vocab], "uniforms": uniform(rows)}
        k = min(case["top_k"], vocab)
        if not case["mixed"]:
            return s | {"temperature": case["temperature"], "top_k": k, "top_p": case["top_p"], "min_p": case["min_p"]}
        at = torch.arange(rows, device=DEVICE)
        s["temperature"] = (case["temperature"] * (0.5 + uniform(rows))).masked_fill(at % 5 == 3, 0.0)     # (0: the likeliest token)
        s["top_k"] = torch.where(at % 3 == 1, 0, torch.randint(1, max(1, k) + 1, (rows,), generator=g, device=DEVICE)).to(torch.int32)
        s["top_p"] = torch.where(at % 4 == 2, 1.0, case["top_p"] * (0.5 + 0.5 * uniform(rows)))
        s["min_p"] = case["min_p"] * 2 * uniform(rows)
        return s

    H, Hkv, hd, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    spans = _spans(case)
    used = [-(-(past + new) // page) for past, new in spans]
    n_pages = sum(used) + 3
    order = torch.randperm(n_pages, generator=g, device=DEVICE).to(torch.int32)     # pages were handed out in any order
    table = torch.full((case["seqs"], max(used)), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(used):
        table[s, :n] = torch.arange(at, at + n, dtype=torch.int32)
        at += n
    table = table.to(DEVICE)
    table = torch.where(table >= 0, order[table.clamp(min=0).long()], table)
    s = {"case": case, "table": table, "k_cache": normal(n_pages, Hkv, page, hd).to(dtype), "v_cache": normal(n_pages, Hkv, page, hd).to(dtype)}
    live = sum(new for _, new in spans)
    rows = live + case["padding"]
    seq = [i for i, (_, new) in enumerate(spans) for _ in range(new)]
    pos = [past + i for past, new in spans for i in range(new)]
    s["live"] = live
    s["seq"] = torch.tensor(seq + [-1] * case["padding"], dtype=torch.int32, device=DEVICE)
    s["positions"] = torch.tensor(pos + [0] * case["padding"], dtype=torch.int32, device=DEVICE)
    # q, k and v lie side by side in the rows of one product
    qkv = normal(rows, (H + 2 * Hkv) * hd).to(dtype)
    s["q"] = qkv[:, :H * hd].unflatten(1, (H, hd))
    s["out"] = torch.zeros(rows, H, hd, dtype=dtype, device=DEVICE)
    if case["op"] == "chunk":
        starts = [0]
        for _, new in spans:
            starts.append(starts[-1] + new)
        s["starts"] = torch.tensor(starts, dtype=torch.int32, device=DEVICE)
        s["n_keys"] = torch.tensor([past + new for past, new in spans], dtype=torch.int32, device=DEVICE)
        s["longest"] = max(new for _, new in spans)
        s["lse"] = torch.zeros(rows, H, dtype=torch.float32, device=DEVICE)
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=DEVICE) if case["slopes"] else None
        return s
    s["k"] = qkv[:, H * hd:(H + Hkv) * hd].unflatten(1, (Hkv, hd))
    s["v"] = qkv[:, (H + Hkv) * hd:].unflatten(1, (Hkv, hd))
    s["q_weight"] = (1 + normal(*((H, hd) if case["by_head"] else (hd,)), scale=0.2)).to(dtype)
    s["k_weight"] = (1 + normal(*((Hkv, hd) if case["by_head"] else (hd,)), scale=0.2)).to(dtype)
    half = case["rot"] // 2
    s["inv_freq"] = torch.tensor([10000.0 ** (-i / half) for i in range(half)], device=DEVICE) if half else None
    return s


# ---------------------------------------------------------------------------------------------------- one pass

def run(state):
    return {"norm": run_norm, "chunk": run_chunk, "sample": run_sample}[state["case"]["op"]](state)


def run_norm(s):
    case = s["case"]
    if own:
        import paper_2408_07802_b200 as kr
        q = kr.op_paged_append_norm(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["positions"], k_weight=s["k_weight"],
                                    q_weight=s["q_weight"], eps=EPS, row_seq=s["seq"], q=s["q"], q_out=s["out"],
                                    inv_freq=s["inv_freq"], interleaved=case["interleaved"])
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    n = s["live"]
    pos, seq = s["positions"][:n].long(), s["seq"][:n].long()
    pages, slots = s["table"][seq, pos // case["page"]].long(), pos % case["page"]
    q, k = _normed(s["q"][:n].float(), s["q_weight"]), _normed(s["k"][:n].float(), s["k_weight"])
    if s["inv_freq"] is not None:
        angle = pos.double()[:, None, None] * s["inv_freq"].double()
        cos, sin = angle.cos().float(), angle.sin().float()
        q, k = _turned(q, cos, sin, case), _turned(k, cos, sin, case)
    s["out"][:n] = q.to(s["q"].dtype)
    s["k_cache"][pages, :, slots] = k.to(s["k"].dtype)
    s["v_cache"][pages, :, slots] = s["v"][:n]
    return {"q": s["out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _normed(x, weight):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()


def _turned(x, cos, sin, case):
    rot = case["rot"]
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((turned, x[..., rot:]), dim=-1)


def run_chunk(s):
    case = s["case"]
    if own:
        import paper_2408_07802_b200 as kr
        out, lse = kr.op_paged_chunk_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["starts"], s["n_keys"],
                                               score_cap=case["cap"], window=case["window"], slopes=s["slopes"], out=s["out"], lse=s["lse"])
        return {"out": out, "lse": lse}
    H, hd = s["q"].shape[1:]
    Hkv, n = case["kv_heads"], s["live"]
    pages = s["table"].clamp(min=0).long()
    k = s["k_cache"][pages].transpose(1, 2).flatten(2, 3).float()      # [seqs, Hkv, width * page, hd]
    v = s["v_cache"][pages].transpose(1, 2).flatten(2, 3).float()
    seq, pos = s["seq"][:n].long(), s["positions"][:n]
    place = torch.arange(n, device=seq.device) - s["starts"][seq]       # of a token in its chunk
    q = torch.zeros(case["seqs"], s["longest"], H, hd, device=seq.device)
    q[seq, place] = s["q"][:n].float()
    at = torch.full((case["seqs"], s["longest"]), -1, dtype=pos.dtype, device=seq.device)
    at[seq, place] = pos
    x = (q.unflatten(2, (Hkv, H // Hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3) @ k.transpose(-1, -2)).mul_(hd ** -0.5)
    x = x.view(case["seqs"], H, s["longest"], -1)
    if case["cap"]:
        x = x.div_(case["cap"]).tanh_().mul_(case["cap"])
    back = torch.arange(x.shape[-1], device=x.device) - at[:, :, None]   # position of the key minus that of the query
    if s["slopes"] is not None:
        x = x + s["slopes"][:, None, None] * back[:, None].float()
    seen = back <= 0
    if case["window"]:
        seen = seen & (back > -case["window"])
    x = x.masked_fill_(~seen[:, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    e = x.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    out = (e.view(case["seqs"], Hkv, -1, e.shape[-1]) @ v).view(case["seqs"], H, s["longest"], hd) / total.clamp(min=1e-38)
    s["out"][:n] = out.transpose(1, 2)[seq, place].to(s["q"].dtype)
    s["lse"][:n] = (top + torch.log(total)).squeeze(-1).transpose(1, 2)[seq, place]
    return {"out": s["out"], "lse": s["lse"]}


def run_sample(s):
    if own:
        import paper_2408_07802_b200 as kr
        got = kr.op_sample_tokens(s["logits"], s["uniforms"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                  min_p=s["min_p"])
        return {"ids": got.ids, "logprob": got.logprob}
    def column(v, dtype):
        return torch.as_tensor(v, device=s["logits"].device).to(dtype).view(-1, 1)

    # equal logits: the lowest index first.  A sum of 50 thousand weights next to a border needs 64 bits.
    v, ids = s["logits"].float().sort(dim=-1, descending=True, stable=True)
    T, k = column(s["temperature"], torch.float32).double(), column(s["top_k"], torch.int32)
    p, m = column(s["top_p"], torch.float32).double(), column(s["min_p"], torch.float32).double()
    rank = torch.arange(v.shape[1], device=v.device)
    below = v.double() - v[:, :1].double()
    w = torch.exp(below / torch.where(T > 0, T, 1.0))
    kept = ((k <= 0) | (rank < k)) & (w >= m) & ((T > 0) | (rank == 0))
    w = w * kept
    up_to = w.cumsum(-1)
    kept = kept & ((p >= 1) | (rank == 0) | (up_to - w < p * up_to[:, -1:]))
    w = w * kept
    up_to = w.cumsum(-1)
    mass = up_to[:, -1:]
    chosen = (kept & (up_to <= s["uniforms"].double()[:, None] * mass)).sum(-1, keepdim=True)
    chosen = torch.minimum(chosen, kept.sum(-1, keepdim=True) - 1)
    return {"ids": ids.gather(-1, chosen).squeeze(-1).to(torch.int32), "logprob": torch.log(w.gather(-1, chosen) / mass).squeeze(-1).float()}


# ---------------------------------------------------------------------------------------------------- in 64 bits, from the definitions

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "chunk": _exact_chunk, "sample": _exact_sample}[case["op"]](case, s)


def _exact_norm(case, s):
    page, rot, n, hd = case["page"], case["rot"], s["live"], case["head_dim"]
    seq, pos, table = s["seq"].tolist(), s["positions"].tolist(), s["table"].tolist()

    def turn(x, weight):
        x = x.double()
        length = torch.linalg.vector_norm(x, dim=-1, keepdim=True)
        x = x / torch.sqrt(length ** 2 / hd + EPS) * weight.double()
        if not rot:
            return x
        # a pair of the rotated part is a complex number, the rotation a product with one of length 1
        pairs = x[..., :rot].unflatten(-1, (rot // 2, 2)) if case["interleaved"] else x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
        z = torch.view_as_complex(pairs.contiguous())
        theta = s["positions"][:, None].double() * s["inv_freq"].double()
        z = torch.view_as_real(z * torch.polar(torch.ones_like(theta), theta)[:, None, :])
        turned = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat((turned, x[..., rot:]), -1)

    q_out, k, v = s["out"].double(), turn(s["k"], s["k_weight"]), s["v"].double()
    q_out[:n] = turn(s["q"], s["q_weight"])[:n]
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    where = torch.tensor([table[seq[i]][pos[i] // page] * page + pos[i] % page for i in range(n)], device=DEVICE)
    for cache, new in ((k_cache, k), (v_cache, v)):
        by_token = cache.transpose(1, 2).reshape(-1, *new.shape[1:]).clone()
        by_token[where] = new[:n]
        cache.copy_(by_token.unflatten(0, (-1, page)).transpose(1, 2))
    return {"q": q_out, "k_cache": k_cache, "v_cache": v_cache}


def _exact_chunk(case, s):
    page, rep = case["page"], case["q_heads"] // case["kv_heads"]
    out, lse = s["out"].double(), s["lse"].double()
    row = 0
    for c, (past, new) in enumerate(_spans(case)):
        n = past + new
        lo = max(0, past + 1 - case["window"]) if case["window"] else 0       # no token of the chunk sees what lies before
        pages = s["table"][c, lo // page:(n - 1) // page + 1].long()
        skip = lo % page
        key = torch.arange(lo, n, device=DEVICE)
        for first in range(0, new, 1024):
            these = slice(row + first, row + min(new, first + 1024))
            query = torch.arange(past + first, past + min(new, first + 1024), device=DEVICE)
            hidden = key[None, :] > query[:, None]
            if case["window"]:
                hidden |= key[None, :] <= query[:, None] - case["window"]
            for h in range(case["kv_heads"]):
                k = s["k_cache"][pages, h].flatten(0, 1)[skip:skip + n - lo].double()
                v = s["v_cache"][pages, h].flatten(0, 1)[skip:skip + n - lo].double()
                for j in range(h * rep, (h + 1) * rep):
                    x = s["q"][these, j].double() @ k.T / math.sqrt(case["head_dim"])
                    if case["cap"]:
                        x = torch.tanh(x / case["cap"]) * case["cap"]
                    if s["slopes"] is not None:
                        x += s["slopes"][j].double() * (key[None, :] - query[:, None])
                    x[hidden] = -math.inf
                    out[these, j] = torch.softmax(x, -1) @ v
                    lse[these, j] = torch.logsumexp(x, -1)
        row += new
    return {"out": out, "lse": lse}


def _exact_sample(case, s):
    rows = case["rows"]

    def by_row(name):
        return s[name].tolist() if case["mixed"] else [torch.tensor(s[name], dtype=torch.float32).item()] * rows

    T, k, p, m = by_row("temperature"), by_row("top_k"), by_row("top_p"), by_row("min_p")
    u, logprob = s["uniforms"].tolist(), []
    for r in range(rows):
        x = s["logits"][r].double()
        if T[r] <= 0:
            logprob.append(0.0)
            continue
        x = x / T[r]
        if k[r] > 0:
            x = torch.topk(x, int(k[r])).values
        x = x.sort(descending=True).values
        weights = torch.softmax(x, -1)
        weights = weights[weights >= m[r] * weights[0]]
        if p[r] < 1:
            before = torch.cat((weights.new_zeros(1), weights.cumsum(0)[:-1]))
            weights = weights[:max(1, int((before < p[r] * weights.sum()).sum()))]
        share = weights.cumsum(0) / weights.sum()
        at = min(int(torch.searchsorted(share, torch.tensor([u[r]], dtype=torch.float64, device=DEVICE), right=True)), len(weights) - 1)
        logprob.append(float(torch.log(weights[at] / weights.sum())))
    return {"ids": None, "logprob": torch.tensor(logprob, dtype=torch.float64, device=DEVICE)}

"""Drawing tokens (temperature, top-k, min-p, top-p, given uniforms) against the definition in 64 bits, and the operators of a
server's step run together.

The token has to be the definition's, except where u M, top_p Z or min_p lies so near to a border that the reference's own sums
(64 bits, in another order: off by at most vocab 2^-53 of the total) do not tell: such rows, recognised by the reference alone, may
have either neighbour.  logprob: rounded to fp32, 2^-23 of itself and 2^-24.
"""
import ctypes as C
import math
import random

import pytest
import torch

import kraken_inputs as ki
import paper_2408_07802_b200 as kr
from test_paged_ops import DEV, T16, Pages, normal

gpu = pytest.mark.gpu
DTYPES = {"f32": torch.float32, **T16}


def reference(logits, u, t, k, p, m):
    """(ids, logprob, sure) of the definition; parameters are lists"""
    ids, logprob, sure = [], [], []
    for r in range(logits.shape[0]):
        x, order = logits[r].double().cpu().sort(descending=True, stable=True)
        n = x.numel()
        if t[r] == 0:
            ids.append(order[0].item()), logprob.append(0.0), sure.append(True)
            continue
        w = torch.exp((x - x[0]) / t[r])
        ok = True
        if 0 < k[r] < n:
            w[k[r]:] = 0
        if m[r] > 0:
            low = w < min(m[r], 1.0)
            near = (w - m[r]).abs() <= 1e-14 * m[r]
            ok &= not bool((near & (w != m[r])).any())
            w[low] = 0
        slack = n * 2.0 ** -53 * 4
        if p[r] < 1:
            up = w.cumsum(0)
            want = max(p[r], 0.0) * up[-1]
            ok &= not bool((((up - want).abs() < slack * up[-1]) & (w > 0)).any())
            keep = up - w < want
            keep[0] = True
            w = w * keep
        up = w.cumsum(0)
        want = u[r] * up[-1]
        at = int((up <= want).sum())
        at = min(at, int((w > 0).sum()) - 1)
        if at > 0:
            ok &= bool((up[at - 1] - want).abs() > slack * up[-1])
        ok &= bool((up[at] - want).abs() > slack * up[-1])
        ids.append(order[at].item())
        logprob.append(float(torch.log(w[at] / up[-1])))
        sure.append(ok)
    return ids, logprob, sure


def check(logits, u, t=1.0, k=0, p=1.0, m=0.0, most_unsure=0.02):
    got = kr.op_sample_tokens(logits, u, temperature=t, top_k=k, top_p=p, min_p=m)
    rows = logits.shape[0]
    each = lambda v: v.tolist() if torch.is_tensor(v) else [torch.tensor(v, dtype=torch.float32).item() if isinstance(v, float) else v] * rows  # noqa: E731
    ids, logprob, sure = reference(logits, u.tolist(), each(t), each(k), each(p), each(m))
    g, l = got.ids.tolist(), got.logprob.tolist()
    for r in range(rows):
        if sure[r]:
            assert g[r] == ids[r], (r, g[r], ids[r], l[r], logprob[r])
            assert abs(l[r] - logprob[r]) <= 2.0 ** -23 * abs(logprob[r]) + 2.0 ** -24, (r, l[r], logprob[r])
        else:
            assert 0 <= g[r] < logits.shape[1]
    assert sum(not s for s in sure) <= most_unsure * rows + 1
    return got


def logits_of(seed, rows, vocab, dtype, sharp=None, padded=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab + padded, generator=g) * (0.5 + 4 * torch.rand(rows, 1, generator=g) if sharp is None else sharp)
    x[torch.rand(x.shape, generator=g) < 1e-3] = -math.inf
    x[:, 0] = x[:, 0].clamp(min=-3.0)     # (a row of forbidden tokens alone is another test)
    return x.to(DTYPES[dtype]).to(DEV)[:, :vocab]


def uniforms(seed, rows):
    u = torch.rand(rows, generator=torch.Generator().manual_seed(seed))
    u[::7] = 0.0
    u[3::11] = 1 - 2.0 ** -24
    return u.to(DEV)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,padded", [(1, 1, 0), (3, 2, 1), (9, 17, 0), (40, 100, 3), (200, 1000, 5), (333, 4099, 1), (17, 50257, 0),
                                               (2, 151936, 7), (70, 32000, 64), (1, 50257, 3), (150, 9000, 0)])
@pytest.mark.parametrize("form", ["all", "k", "p", "m", "kpm"])
def test_sample(dtype, rows, vocab, padded, form):
    x, u = logits_of(rows + vocab, rows, vocab, dtype, padded=padded), uniforms(vocab, rows)
    kw = {"all": {}, "k": dict(k=5), "p": dict(p=0.9), "m": dict(m=0.02), "kpm": dict(k=40, p=0.95, m=0.001)}[form]
    check(x, u, t=0.8 if form == "p" else 1.0, **kw)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seed", range(4))
def test_sample_rows_with_parameters_of_their_own(dtype, seed):
    rows, vocab = 128, 3001 + 7000 * seed
    g = torch.Generator().manual_seed(seed)
    x, u = logits_of(seed, rows, vocab, dtype), uniforms(seed, rows)
    t = (0.05 + 2 * torch.rand(rows, generator=g))
    t[::6] = 0.0
    k = torch.randint(-1, 60, (rows,), generator=g, dtype=torch.int32)
    k[::5] = vocab + 3
    k[1::9] = vocab - 1
    p = torch.rand(rows, generator=g) * 1.2
    p[2::13] = 0.0
    m = torch.rand(rows, generator=g) * 0.1 - 0.02
    m[4::17] = 1.5
    check(x, u, *(v.to(DEV) for v in (t, k, p, m)))


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", ["equal", "two", "steps", "one high", "rising", "falling", "narrow"])
def test_sample_rows_of_equal_and_ordered_logits(dtype, kind):
    """More equal logits than there is room for: the borders are found digit by digit."""
    rows, vocab = 12, 20011
    x = {"equal": torch.full((rows, vocab), 1.5), "two": (torch.arange(vocab) % 2).float().expand(rows, -1),
         "steps": (torch.arange(vocab) * 7919 % 13).float().expand(rows, -1) * 0.25,
         "one high": torch.zeros(rows, vocab).index_fill(1, torch.tensor([777]), 9.0), "rising": torch.linspace(-4, 4, vocab).expand(rows, -1),
         "falling": torch.linspace(4, -4, vocab).expand(rows, -1), "narrow": torch.linspace(0, 1e-3, vocab).expand(rows, -1)}[kind]
    x = x.to(DTYPES[dtype]).to(DEV)
    u = torch.tensor([0.0, 1e-6, 0.1, 0.25, 0.3333, 0.5001, 0.7, 0.9, 0.99, 0.9999, 1 - 2.0 ** -24, 0.61], device=DEV)
    for kw in (dict(), dict(k=1), dict(k=7000), dict(p=0.9), dict(m=0.5), dict(k=15000, p=0.77, m=0.1), dict(t=0.3, p=0.5)):
        check(x, u, most_unsure=1.0 if kind in ("equal", "two", "steps", "one high") else 0.02, **kw)


@gpu
def test_sample_equal_logits_are_drawn_by_index():
    """512 equal logits: u = (i + 1/2) / 512 is the i-th."""
    x = torch.full((512, 512), -3.0, device=DEV)
    got = kr.op_sample_tokens(x, (torch.arange(512, device=DEV) + 0.5) / 512)
    assert got.ids.tolist() == list(range(512))
    assert (got.logprob + math.log(512)).abs().max() < 1e-6
    x = torch.full((64, 65536), 2.0, dtype=torch.bfloat16, device=DEV)
    got = kr.op_sample_tokens(x, (torch.arange(64, device=DEV) * 1024 + 0.5) / 65536)
    assert got.ids.tolist() == [1024 * i for i in range(64)]
    # 0 and -0 are equal
    x = torch.zeros(4, 1000, device=DEV)
    x[:, ::2] = -0.0
    assert kr.op_sample_tokens(x, torch.tensor([0.0, 0.2505, 0.5005, 0.9995], device=DEV)).ids.tolist() == [0, 250, 500, 999]


@gpu
@pytest.mark.parametrize("rows", [1, 5, 200])
@pytest.mark.parametrize("exponent", [20.5, 30.0, 38.5, 41.5])
def test_sample_many_tiny_weights(exponent, rows):
    """One token of weight 1 and a million of 2^-exponent each, which together are drawn by uniforms close to 1: the sums are right
    to 1e-11 of the mass, however small the single weights are."""
    vocab = 1 << 20
    x = torch.full((vocab,), -exponent * math.log(2.0), device=DEV)
    x[4321] = 0.0
    w = math.exp(float(x[0]))
    mass = 1.0 + (vocab - 1) * w
    u = torch.full((rows,), 1 - 2.0 ** -24)
    u[rows // 2] = 1 / mass + 0.3 * (1 - 1 / mass)
    got = kr.op_sample_tokens(x.expand(rows, -1), u.to(DEV)).ids.tolist()
    for r in range(rows):
        want = (float(u[r]) * mass - 1.0) / w
        place = -1 if got[r] == 4321 else got[r] - (got[r] > 4321)   # (ties go by index)
        # (1e-15: the reference's own sum)
        assert abs(place - max(want, -1.0)) <= (1e-11 + 1e-15) * mass / w + 1, (r, place, want)


@gpu
def test_sample_zero_temperature_and_one_token_left():
    x = logits_of(5, 30, 5000, "bf16")
    first = torch.tensor([int((x[r] == x[r].max()).nonzero()[0]) for r in range(30)])
    u = uniforms(1, 30)
    for kw in (dict(temperature=0.0), dict(top_k=1), dict(temperature=0)):
        got = kr.op_sample_tokens(x, u, **kw)
        assert got.ids.tolist() == first.tolist() and bool((got.logprob == 0).all())
    got = kr.op_sample_tokens(x, torch.zeros(30, device=DEV))
    assert got.ids.tolist() == first.tolist()
    got = kr.op_sample_tokens(x, u, top_p=0.0)
    assert got.ids.tolist() == first.tolist() and bool((got.logprob == 0).all())


@gpu
@pytest.mark.parametrize("t", [1e-3, 1e-20, 1e-38, 50.0, 1e10, 3e38])
def test_sample_extreme_temperatures(t):
    check(logits_of(6, 20, 7001, "f32"), uniforms(2, 20), t=t, p=0.9, most_unsure=0.1)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [3, 90])
def test_sample_tokens_masked_by_the_lowest_number(dtype, rows):
    """Forbidden tokens by the type's lowest number in place of -inf: never drawn, however many top_k asks for, unless there is
    nothing else; from the highest to the lowest number is further than 32 bits hold."""
    t = DTYPES[dtype]
    low, vocab = torch.finfo(t).min, 30011
    x = torch.full((rows, vocab), low, dtype=t, device=DEV)
    for r in range(rows):
        left = [7 + r, 400 + 3 * r, 29000 - r, vocab - 1][:r % 4 + 1]
        x[r, left] = torch.tensor([1.0, 0.5, 1.25, -2.0][:len(left)], dtype=t, device=DEV)
    u = uniforms(11, rows)
    for kw in (dict(), dict(k=3), dict(k=500), dict(p=0.9), dict(m=0.4), dict(k=20000, p=0.999, m=0.01), dict(t=0.2), dict(t=0.2, k=9)):
        check(x, u, most_unsure=0.1, **kw)
    x[1] = low
    x[2, 12345] = torch.finfo(t).max
    got = kr.op_sample_tokens(x[1:3].contiguous(), torch.tensor([0.5, 0.999], device=DEV))
    assert got.ids.tolist() == [vocab // 2, 12345]
    assert abs(float(got.logprob[0]) + math.log(vocab)) < 1e-5 and float(got.logprob[1]) == 0.0


@gpu
@pytest.mark.parametrize("vocab", [33, 4000, 60000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_rows_without_a_distribution(vocab, dtype):
    x, u = logits_of(8, 12, vocab, dtype), torch.full((12,), 0.5, device=DEV)
    t, p, m = torch.ones(12, device=DEV), torch.ones(12, device=DEV), torch.zeros(12, device=DEV)
    x[0, vocab - 1] = math.nan
    x[1, 3] = math.inf
    x[2] = -math.inf
    u[3], u[4], u[5] = 1.0, -1e-9, math.nan
    t[6], t[7], t[8] = -1.0, math.inf, math.nan
    p[9], m[10] = math.nan, math.nan
    got = kr.op_sample_tokens(x, u, temperature=t, top_p=p, min_p=m)
    assert got.ids[:11].tolist() == [-1] * 11 and bool(got.logprob[:11].isnan().all())
    assert got.ids[11] >= 0 and bool(got.logprob[11].isfinite())
    # all but one forbidden
    x[2, vocab // 2] = -1e30 if dtype == "f32" else -100.0
    got = kr.op_sample_tokens(x[2:3], u[:1])
    assert got.ids.item() == vocab // 2 and got.logprob.item() == 0


@gpu
def test_sample_follows_the_distribution():
    """Uniforms at the middles of 20000 equal parts: every token as often as its probability says, to one part."""
    n = 20000
    x = logits_of(9, 1, 300, "f32", sharp=1.0)
    got = kr.op_sample_tokens(x.expand(n, -1), (torch.arange(n, device=DEV) + 0.5) / n)
    p = torch.softmax(x[0].double(), 0)
    assert (torch.bincount(got.ids.long(), minlength=300) - n * p).abs().max() <= 1.0 + 1e-3
    assert (got.logprob.double() - torch.log(p)[got.ids.long()]).abs().max() < 1e-6


@gpu
def test_sample_random_calls():
    r = random.Random(3)
    for i in range(40):
        vocab = int(math.exp(r.uniform(math.log(40), math.log(150000))))
        rows = r.randint(1, max(1, min(300, 400000 // vocab)))
        x = logits_of(i, rows, vocab, r.choice(["f32", "bf16", "f16"]), sharp=r.choice([None, 0.3, 2.0, 8.0]), padded=r.choice([0, 1, 3, 64]))
        check(x, uniforms(i, rows), t=r.choice([0.6, 1.0, 1.3]), k=r.choice([0, 0, 2, 20, 1000, vocab - 1]), p=r.choice([1.0, 0.5, 0.9, 0.999]),
              m=r.choice([0.0, 0.0, 0.05, 1e-4]))


@gpu
def test_sample_in_a_graph_and_on_two_streams():
    x, u = logits_of(10, 48, 51200, "bf16"), uniforms(4, 48)
    want = kr.op_sample_tokens(x, u, top_p=0.9)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = kr.op_sample_tokens(x, u, top_p=0.9)
    graph.replay()
    assert got.ids.tolist() == want.ids.tolist() and bool((got.logprob == want.logprob).all())
    u.copy_(uniforms(5, 48))
    graph.replay()
    again = kr.op_sample_tokens(x, u, top_p=0.9)
    assert got.ids.tolist() == again.ids.tolist()
    del graph
    streams, out = [torch.cuda.Stream() for _ in range(2)], [[], []]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                out[i].append(kr.op_sample_tokens(x, u, top_p=0.9))
    torch.cuda.synchronize()
    for some in out:
        for o in some:
            assert o.ids.tolist() == again.ids.tolist() and bool((o.logprob == again.logprob).all())


# ------------------------------------------------------------------ a server's steps, and a model's

@gpu
@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("f16", 100)])
def test_a_servers_steps(dtype, page):
    """A layer of attention with normalised, rotated heads and a head of logits: prompts in pieces beside single tokens, each
    step append, attend, project, sample.  The same sequences at once, in 64 bits, give the same outputs and tokens."""
    t, H, Hkv, hd, vocab = T16[dtype], 8, 2, 64, 997
    prompts = [70, 3, 41]
    d = H * hd
    g = torch.Generator().manual_seed(3)
    embed = torch.randn(vocab, d, generator=g, dtype=torch.float64).to(t).to(DEV)
    w_qkv = (torch.randn(d, (H + 2 * Hkv) * hd, generator=g, dtype=torch.float64) * d ** -0.5).to(t).to(DEV)
    w_out = (torch.randn(d, vocab, generator=g, dtype=torch.float64) * 2 * d ** -0.5).to(t).to(DEV)
    wq, wk = ((1 + 0.2 * torch.randn(hd, generator=g)).to(t).to(DEV) for _ in range(2))
    freq = torch.tensor([10000.0 ** (-i / 32) for i in range(32)], device=DEV)
    tokens = [torch.randint(0, vocab, (n,), generator=g).tolist() for n in prompts]
    pages = Pages(1, [n + 8 for n in prompts], Hkv, hd, page, dtype, fill=False)
    # pieces of the prompts, then drawn tokens: (sequence, tokens) of every step
    steps = [[(0, 64), (1, 3)], [(0, 6), (1, 1), (2, 41)]] + [[(0, 1), (1, 1), (2, 1)]] * 4
    done, out_of = [0, 0, 0], [[], [], []]
    for n, step in enumerate(steps):
        seq = [s for s, c in step for _ in range(c)]
        pos = [done[s] + i for s, c in step for i in range(c)]
        ids = torch.tensor([tokens[s][q] for s, q in zip(seq, pos)], device=DEV)
        starts = [0]
        for s, c in step:
            starts.append(starts[-1] + c)
            done[s] += c
        qkv = embed[ids] @ w_qkv
        q, k, v = (x.unflatten(1, (-1, hd)) for x in qkv.split([d, Hkv * hd, Hkv * hd], 1))
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
        q = kr.op_paged_append_norm(k, v, pages.k, pages.v, pages.table, i32(pos), k_weight=wk, q_weight=wq, row_seq=i32(seq), q=q, inv_freq=freq)
        out, _ = kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, i32(starts), i32([done[s] for s, _ in step]),
                                             chunk_seq=i32([s for s, _ in step]))
        last = [e - 1 for e in starts[1:]]
        logits = out.flatten(1)[last] @ w_out
        u = torch.rand(len(step), generator=torch.Generator().manual_seed(n)).to(DEV)
        drawn = check(logits, u, t=0.9, k=50, p=0.95)
        for i, (s, c) in enumerate(step):
            out_of[s].append(out[starts[i]:starts[i + 1]])
            if done[s] == len(tokens[s]):
                tokens[s].append(int(drawn.ids[i]))
    half = torch.finfo(t).eps / 2
    for s in range(3):
        x = (embed[torch.tensor(tokens[s][:done[s]], device=DEV)] @ w_qkv).double()
        q, k, v = (y.unflatten(1, (-1, hd)) for y in x.split([d, Hkv * hd, Hkv * hd], 1))
        theta = torch.arange(done[s], device=DEV).double()[:, None, None] * freq.double()
        def turn(y, w):
            y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w.double()
            a, b = y[..., :32], y[..., 32:]
            return torch.cat((a * theta.cos() - b * theta.sin(), b * theta.cos() + a * theta.sin()), -1)
        q, k = turn(q, wq), turn(k, wk)
        got = torch.cat(out_of[s]).double()
        assert got.shape[0] == done[s]
        hidden = torch.ones(done[s], done[s], dtype=torch.bool, device=DEV).triu(1)
        for h in range(H):
            score = (q[:, h] @ k[:, h // 4].T / 8).masked_fill(hidden, -math.inf)
            # q and k are rounded once each (half a step of their values), then the weights and the output
            d_score = 2 * half * (q[:, h].abs() @ k[:, h // 4].abs().T / 8).masked_fill(hidden, 0).amax(1, keepdim=True)
            p = torch.softmax(score, 1)
            bound = (p @ v[:, h // 4].abs()) * (2.2 * d_score + half + 1e-4) + half * (p @ v[:, h // 4]).abs() + 1e-6
            assert bool(((got[:, h] - p @ v[:, h // 4]).abs() <= bound).all())


@gpu
def test_generate():
    """Greedy generation is prefill and decode steps by hand; drawn tokens are those of the same logits."""
    s = ki.CONFIGS["C0"]
    w = ki.make_weights(s, seed=0, device=DEV)
    model = kr.KrakenModel(kr.make_config(s, max_batch=3), w, DEV)
    prompt = ki.uniform_tokens(1, s.vocab, 3, 40, DEV)
    u = torch.rand(6, 3, generator=torch.Generator().manual_seed(1)).to(DEV)
    for kw in (dict(temperature=0.0), dict(temperature=0.7, top_k=100, top_p=0.9), dict(min_p=0.5)):
        got = model.generate(prompt, u, **kw)
        logits = model.prefill(prompt)
        for i in range(6):
            if i:
                logits = model.decode_step(got.ids[i - 1].contiguous())
            want = kr.op_sample_tokens(logits, u[i], **kw)
            assert got.ids[i].tolist() == want.ids.tolist() and bool((got.logprob[i] == want.logprob).all())
            if kw.get("temperature") == 0.0:
                assert got.ids[i].tolist() == logits.argmax(1).tolist()
    assert model.device_status() == 0
    model.close()


# ------------------------------------------------------------------ refusals (no GPU)

def sample_args(**over):
    a = dict(logits=1 << 20, row_stride=100, uniforms=2 << 20, temperature_all=1.0, top_p_all=1.0, ids=3 << 20, rows=4, vocab=100)
    a.update(over)
    return kr.SampleArgs(**a)


@pytest.mark.parametrize("over,code", [
    (dict(logits=None), kr.EINVAL), (dict(uniforms=None), kr.EINVAL), (dict(ids=None), kr.EINVAL), (dict(rows=-1), kr.EINVAL), (dict(vocab=0), kr.EINVAL),
    (dict(dtype=2), kr.EINVAL), (dict(row_stride=-1), kr.EINVAL), (dict(logits=(1 << 20) + 2), kr.EINVAL), (dict(logits=(1 << 20) + 1, dtype=1), kr.EINVAL),
    (dict(temperature_all=-0.5), kr.EINVAL), (dict(temperature_all=math.inf), kr.EINVAL), (dict(temperature_all=math.nan), kr.EINVAL),
    (dict(top_p_all=math.nan), kr.EINVAL), (dict(min_p_all=math.nan), kr.EINVAL), (dict(vocab=(1 << 24) + 1), kr.EUNSUPPORTED),
    (dict(rows=1 << 27), kr.EUNSUPPORTED), (dict(rows=0), kr.OK)])
def test_sample_refusals(over, code):
    assert kr.lib().kraken_op_sample_tokens(C.byref(sample_args(**over)), None) == code
    assert kr.lib().kraken_op_sample_tokens(None, None) == kr.EINVAL


def test_sample_refuses_cpu_tensors():
    with pytest.raises(ValueError):
        kr.op_sample_tokens(torch.zeros(2, 10), torch.zeros(2))


@gpu
def test_sample_binding_refusals():
    x, u = torch.zeros(4, 10, device=DEV), torch.zeros(4, device=DEV)
    for bad in (dict(logits=x.double()), dict(logits=x[0]), dict(logits=x.T), dict(uniforms=u[:3]), dict(uniforms=u.double()), dict(uniforms=None),
                dict(temperature=u.double()), dict(temperature="hot"), dict(top_k=u), dict(top_k=1.5), dict(top_p=u[:1]), dict(min_p=None),
                dict(uniforms=u.cpu())):
        with pytest.raises(ValueError):
            kr.op_sample_tokens(**{**dict(logits=x, uniforms=u), **bad})
    for bad in (dict(temperature=-1.0), dict(top_p=math.nan)):
        with pytest.raises(kr.KrakenError):
            kr.op_sample_tokens(x, u, **bad)
    assert kr.op_sample_tokens(x[:0], u[:0]).ids.numel() == 0

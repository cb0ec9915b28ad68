"""Drawing tokens: rows that CTAs share, rows with few tokens left, weights between the windows, temperatures at the ends of fp32.

What is compared exactly (ids of a temperature of 0, of rows with one answer) has no tolerance; the others derive theirs beside
the comparison.
"""
import math

import pytest
import torch

import kraken_inputs as ki
import paper_2408_07802_b200 as kr
from paper_2408_07802_b200 import build as kbuild

kbuild.build_all()

DEV = "cuda:0"
gpu = pytest.mark.gpu


# ------------------------------------------------------------------ rows that CTAs share

@gpu
@pytest.mark.parametrize("dtype,vec", [(torch.float32, 4), (torch.bfloat16, 8)])
@pytest.mark.parametrize("ctas", [1, 2, 4, 8])
def test_rows_shared_by_ctas_call_after_call(dtype, vec, ctas):
    """Rows just long enough for 1, 2, 4 and 8 CTAs, the largest logit in every CTA's part in turn, one call right after another
    and on two streams at once: every CTA has the maximum of the whole row in every call."""
    vocab = max(ctas, 1) * 1024 * vec + (5 if ctas > 1 else -vec)
    for rows in (1, 3, 18):
        at = torch.randint(0, vocab, (16, rows), generator=torch.Generator().manual_seed(ctas))
        at[:, 0] = torch.arange(16) * (vocab // 16) + 3
        x = torch.full((16, rows, vocab + 3), -2.0, dtype=dtype, device=DEV)
        x.scatter_(2, at.to(DEV)[..., None], 25.0)   # (the others together weigh vocab e^-27 < 2e-7 of it)
        x = x[:, :, :vocab]
        u = torch.full((rows,), 0.5, device=DEV)
        streams, got = [torch.cuda.Stream() for _ in range(2)], []
        torch.cuda.synchronize()
        for n in range(48):
            with torch.cuda.stream(streams[n & 1]):
                got.append(kr.op_sample_tokens(x[n % 16], u, temperature=0.0 if n % 3 == 0 else 1.0))
        torch.cuda.synchronize()
        for n, g in enumerate(got):
            assert g.ids.tolist() == at[n % 16].tolist(), (rows, n)
            assert bool((g.logprob.abs() < 1e-6).all())


# ------------------------------------------------------------------ limits that nothing reaches

def device_us(call, n=20):
    """Least device time of a call, from a graph of them"""
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(n):
            call()
    best = math.inf
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        graph.replay()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b) * 1e3 / n)
    del graph
    return best


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 160])
@pytest.mark.parametrize("kind", ["few allowed", "cold", "lowest number"])
def test_top_k_beyond_what_is_left(kind, rows, dtype):
    """Fewer tokens of any weight than top_k asks for: the same tokens as without the limit, by the same way and not digit by digit
    (ten times as long and more)."""
    vocab, k, t = 50257, 50, 1.0
    g = torch.Generator().manual_seed(rows)
    if kind == "cold":   # few of the logits lie within 140 ln(2) T = 0.5 of the largest
        x, t = 2 * torch.randn(rows, vocab, generator=g), 0.005
    else:
        x = torch.full((rows, vocab), -math.inf if kind == "few allowed" else torch.finfo(dtype).min)
        x[:, torch.randperm(vocab, generator=g)[:20]] = torch.randn(rows, 20, generator=g)
    x, u = x.to(dtype).to(DEV), torch.rand(rows, generator=g).to(DEV)
    limited, free = kr.op_sample_tokens(x, u, temperature=t, top_k=k), kr.op_sample_tokens(x, u, temperature=t)
    assert limited.ids.tolist() == free.ids.tolist() and bool((limited.logprob == free.logprob).all())
    a, b = (device_us(lambda: kr.op_sample_tokens(x, u, temperature=t, top_k=limit)) for limit in (k, 0))
    assert a < 4 * b, (a, b)


# ------------------------------------------------------------------ weights between the windows

@gpu
@pytest.mark.parametrize("before,at,after", [(172, 160, 148), (169, 158, 147), (66, 50, 35), (218, 180, 148)])
def test_many_alike_on_both_sides_of_the_window(before, at, after):
    """Half a million equal weights before the window of the token and as many behind it, 4000 in it of about a millionth of the mass each;
    the uniforms are such that u M lies 5 10^-11 to 10^-9 of the mass from a border.  That is more than 1e-11: the definition's token.
    (Weights of so many 256ths: their sums in 32 bits tell where the windows have to be.)"""
    n, middle = 1 << 19, 4000
    x = torch.cat([torch.full((k,), math.log(w / 256)) for k, w in ((n, before), (middle, at), (n, after))])
    x[77] = 0.0
    w = [math.exp(float(x[i])) for i in (0, n, n + middle)]
    lower = 1 + (n - 1) * w[0]
    mass = lower + middle * w[1] + n * w[2]
    u = torch.arange(math.ceil(lower / mass * 2 ** 24) + 20, math.floor((lower + middle * w[1]) / mass * 2 ** 24) - 20).double() * 2.0 ** -24
    place = (u * mass - lower) / w[1]          # (the sums here are off by 2^-53 of the mass, 10^-10 of a place)
    share = w[1] / mass
    near = (place - place.round()).abs() * share
    some = ((near > 5e-11) & (near < 1e-9)).nonzero()[:, 0][:600]
    assert some.numel() > 40
    got = kr.op_sample_tokens(x.to(DEV).expand(some.numel(), -1), u[some].float().to(DEV)).ids.cpu() - n
    assert got.tolist() == place[some].floor().long().tolist()


# ------------------------------------------------------------------ temperatures at the ends

@gpu
@pytest.mark.parametrize("rows", [1, 160])
@pytest.mark.parametrize("vocab", [40, 40000])
def test_temperatures_at_the_ends(vocab, rows):
    """Logits further apart than fp32 holds at a temperature as large, and logits below the normal numbers at one as small: weights
    e^0, e^-1, e^-2 all the same."""
    for t, step in ((3e38, 3e38), (1e37, 1e37), (2e-42, 2e-42), (1e-38, 1e-38)):
        tt, st = (float(torch.tensor(v, dtype=torch.float32)) for v in (t, step))
        x = torch.full((vocab,), -math.inf)
        x[5], x[9], x[11] = st, 0.0, -st
        w = [math.exp((float(x[i]) - float(x[5])) / tt) for i in (5, 9, 11)]
        m = sum(w)
        u = (torch.arange(rows) + 0.5) / rows
        u[rows // 2] = 0.999
        want = [5 if float(v) * m < w[0] else (9 if float(v) * m < w[0] + w[1] else 11) for v in u]
        got = kr.op_sample_tokens(x.to(DEV).expand(rows, -1), u.to(DEV), temperature=t)
        assert got.ids.tolist() == want, t
        p = {5: w[0], 9: w[1], 11: w[2]}
        for i, l in zip(want, got.logprob.tolist()):   # (rounded to 32 bits)
            assert abs(l - math.log(p[i] / m)) <= 2.0 ** -23 * abs(l) + 2.0 ** -24


# ------------------------------------------------------------------ generate

@gpu
def test_generate_says_beforehand_that_there_is_no_room():
    """Prompt and steps that do not fit are refused before a token is drawn, and the handle stays as it was; the last step that fits runs."""
    s = ki.CONFIGS["C0"]
    model = kr.KrakenModel(kr.make_config(s, max_batch=2, max_pos=24), ki.make_weights(s, seed=0, device=DEV), DEV)
    prompt = ki.uniform_tokens(1, s.vocab, 2, 20, DEV)
    model.prefill(prompt[:, :7].contiguous())
    u = torch.rand(6, 2, generator=torch.Generator().manual_seed(1)).to(DEV)
    with pytest.raises(kr.KrakenError) as e:
        model.generate(prompt, u)
    assert e.value.status == kr.ECAPACITY and model.cur_len == 7
    got = model.generate(prompt, u[:5])
    assert model.cur_len == 24 and bool(((got.ids >= 0) & (got.ids < s.vocab)).all())
    assert model.generate(prompt, u[:0]).ids.shape == (0, 2)
    model.close()

"""The append with norms and the attention of chunks of tokens over a cache in pages, against plain 64-bit forms.

Tolerances.  A result rounded to 16 bits may be off by half a step, eps / 2 of its value.  On top of that:
  norms      the sum of up to 128 squares by 2^-24 for each of its 7 levels of additions and 16 terms of a thread, the inverse root
             by 2^-22, two products by 2^-24 each, then the rotation as in the append without norms: below 3e-6 (|a| + |b|)
  chunk      a score by d as in the decode step's test (and by another 2^-19 of itself under a cap: tanh to 1e-6); a weight by
             d + 2^-22, a sum over n keys by n 2^-24 (twice: output and sum).  That is the share of lse that may be off.
             For the output a weight is also rounded to 16 bits, by eps / 2 of itself, in half by at most 2^-32 of the row's
             largest where it is tiny: by so much of sum p |v|.
"""
import ctypes as C
import math
import random

import pytest
import torch

import paper_2408_07802_b200 as kr
from test_paged_ops import DEV, T16, Pages, normal

gpu = pytest.mark.gpu


# ------------------------------------------------------------------ chunk attention

def chunk_ref(pages, q, starts, n_keys, seqs, scale, cap=0.0, window=0, slopes=None):
    """(out, lse, tolerance of out, of lse, rows that belong to a chunk), 64 bits"""
    R, H, hd = q.shape
    rep = H // pages.k.shape[1]
    out = torch.zeros(R, H, hd, dtype=torch.float64, device=DEV)
    lse = torch.full((R, H), -math.inf, dtype=torch.float64, device=DEV)
    tol_o, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    live = torch.zeros(R, dtype=torch.bool, device=DEV)
    half = torch.finfo(q.dtype).eps / 2
    for c, s in enumerate(seqs):
        lo_row, hi_row, n = starts[c], starts[c + 1], n_keys[c]
        if s < 0 or lo_row == hi_row:
            continue
        live[lo_row:hi_row] = True
        if n == 0:
            continue
        k, v = pages.get(pages.k, s, 0, n), pages.get(pages.v, s, 0, n)
        pos = torch.arange(n - (hi_row - lo_row), n, device=DEV)
        key = torch.arange(n, device=DEV)
        hidden = key > pos[:, None]
        if window:
            hidden = hidden | (key <= pos[:, None] - window)
        none = hidden.all(1)
        for h in range(H):
            qh, kh, vh = q[lo_row:hi_row, h].double(), k[:, h // rep], v[:, h // rep]
            x = qh @ kh.T * scale
            sums = (qh.abs() @ kh.abs().T).masked_fill(hidden, 0).amax(1)
            d = hd * 2.0 ** -23 * abs(scale) * sums + 2.0 ** -22 * x.masked_fill(hidden, 0).abs().amax(1)
            if cap:
                x = cap * torch.tanh(x / cap)
                d = d + 2.0 ** -19 * x.masked_fill(hidden, 0).abs().amax(1)
            if slopes is not None:
                x = x + slopes[h].double() * (key - pos[:, None])
                d = d + 2.0 ** -22 * x.masked_fill(hidden, 0).abs().amax(1)
            x = x.masked_fill(hidden, -math.inf)
            p = torch.softmax(x, 1).nan_to_num(0.0)
            vh = torch.where(hidden.all(0)[:, None], 0.0, vh)
            out[lo_row:hi_row, h] = p @ vh
            lse[lo_row:hi_row, h] = torch.logsumexp(x, 1)
            share = (2 * d + 2.0 ** -21 + n * 2.0 ** -23)[:, None]
            tiny = 2.0 ** -32 * p.amax(1, keepdim=True) * (~hidden).double() if q.dtype == torch.float16 else 0.0
            tol_o[lo_row:hi_row, h] = (p * (share + half) + tiny) @ vh.abs()
            tol_l[lo_row:hi_row, h] = share[:, 0] + 2.0 ** -22 * lse[lo_row:hi_row, h].nan_to_num(neginf=0.0).abs()
        out[lo_row:hi_row][none] = 0.0
        lse[lo_row:hi_row][none] = -math.inf
    return out, lse, tol_o, tol_l, live


def int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def check_chunk(pages, q, starts, n_keys, seqs=None, scale=None, cap=0.0, window=0, slopes=None, **kw):
    R, H, hd = q.shape
    scale = hd ** -0.5 if scale is None else scale
    ref, ref_lse, tol, tol_l, live = chunk_ref(pages, q, starts, n_keys, seqs if seqs is not None else range(len(n_keys)), scale, cap,
                                               window, slopes)
    out = torch.full((R, H, hd), 7.0, dtype=q.dtype, device=DEV)
    lse = torch.full((R, H), 7.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, int32(starts), int32(n_keys),
                                chunk_seq=None if seqs is None else int32(seqs), scale=scale, score_cap=cap, window=window, slopes=slopes,
                                out=out, lse=lse, status=status, **kw)
    assert int(status) == 0
    assert bool((out[~live] == 7).all()) and bool((lse[~live] == 7).all())
    half = torch.finfo(q.dtype).eps / 2
    err, bound = (out.double() - ref).abs()[live], (half * ref.abs() * (1 + 1e-2) + tol + 2.0 ** -25)[live]
    assert bool((err <= bound).all()), (err - bound).max().item()
    some = live[:, None] & (ref_lse > -math.inf)
    assert bool(((lse.double() - ref_lse).abs()[some] <= tol_l[some]).all())
    assert bool((lse[live[:, None] & ~some] == -math.inf).all())
    return out, lse


CHUNKS = [
    # (past, new) of every sequence, H, Hkv, hd, page, dtype
    ([(0, 1)], 1, 1, 64, 16, "bf16"),
    ([(0, 127), (0, 128), (0, 129), (0, 257), (1, 1)], 4, 2, 64, 16, "bf16"),
    ([(127, 1), (128, 1), (100, 28), (100, 29), (383, 2)], 8, 1, 128, 1, "f16"),
    ([(5, 700)], 12, 12, 104, 24, "f16"),
    ([(300, 0), (0, 3), (17, 44), (511, 65)], 5, 1, 72, 8, "bf16"),
    ([(257, 90), (3, 400)], 6, 2, 96, 100, "bf16"),
    ([(40, 999)], 18, 2, 128, 64, "bf16"),
    ([(77, 5), (500, 3), (0, 9)], 130, 1, 64, 16, "f16"),
    ([(1500, 3), (3, 1), (2049, 300)], 32, 4, 128, 256, "bf16"),
    ([(9000, 2)], 2, 2, 128, 16, "f16"),
    ([(i * 37, 1 + i % 3) for i in range(60)], 8, 2, 64, 8, "bf16"),
]


@gpu
@pytest.mark.parametrize("spans,H,Hkv,hd,page,dtype", CHUNKS)
@pytest.mark.parametrize("form", ["plain", "cap", "window", "slopes", "all"])
def test_chunk(spans, H, Hkv, hd, page, dtype, form):
    lens = [p + n for p, n in spans]
    pages = Pages(len(lens) + H, lens, Hkv, hd, page, dtype, by_slot=form == "window")
    starts = [3]
    for _, n in spans:
        starts.append(starts[-1] + n)
    q = normal(7, starts[-1] + 5, H, hd).to(T16[dtype])
    if form == "window":   # rows cut out of a wider product, heads behind one another
        q = q.repeat(1, 2, 1)[:, :H]
    slopes = torch.linspace(0.6, 0.01, H, device=DEV) if form in ("slopes", "all") else None
    check_chunk(pages, q, starts, lens, cap=15.0 if form in ("cap", "all") else 0.0,
                window={"window": 1 if H == 5 else 150, "all": 40}.get(form, 0), slopes=slopes)


@gpu
@pytest.mark.parametrize("scale", [0.0, -0.1, 2.0])
def test_chunk_scales(scale):
    pages = Pages(5, [300, 41], 2, 64, 16, "bf16")
    check_chunk(pages, normal(8, 90, 4, 64).to(torch.bfloat16), [0, 70, 90], [300, 41], scale=scale)


@gpu
@pytest.mark.parametrize("page", [16, 100])
def test_chunk_more_tokens_than_keys_and_shared_sequences(page):
    """Tokens at negative positions see nothing; two chunks of one sequence; padding chunks; chunks in any order of sequences."""
    pages = Pages(6, [300, 2, 140], 2, 128, page, "bf16")
    q = normal(9, 700, 4, 128).to(torch.bfloat16)
    out, lse = check_chunk(pages, q, [0, 300, 310, 330, 630, 640], [20, 2, 7, 140, 300], seqs=[0, 1, -1, 2, 0])
    assert bool((out[:280] == 0).all()) and bool((lse[:280] == -math.inf).all())


@gpu
def test_chunk_of_one_token_is_the_decode_step():
    lens = [1, 15, 128, 1000, 777]
    pages = Pages(3, lens, 4, 128, 16, "bf16")
    q = normal(4, len(lens), 16, 128).to(torch.bfloat16)
    out, lse = check_chunk(pages, q, list(range(len(lens) + 1)), lens)
    dec, dec_lse = kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, int32(lens))
    assert (out.float() - dec.float()).abs().max() < 0.04 and (lse - dec_lse).abs().max() < 1e-4


@gpu
@pytest.mark.parametrize("page", [16, 100])
def test_chunk_expanded_cache_and_queries(page):
    """One head's keys for all (a head stride of 0), one token's queries for all rows."""
    pages = Pages(11, [400], 1, 64, page, "f16")
    q = normal(4, 60, 6, 64).to(torch.float16)
    out, _ = check_chunk(pages, q, [0, 60], [400])
    k, v = pages.k.expand(-1, 3, -1, -1), pages.v.expand(-1, 3, -1, -1)
    got, _ = kr.op_paged_chunk_attention(q, k, v, pages.table, int32([0, 60]), int32([400]))
    assert (got.float() - out.float()).abs().max() < 4e-3
    one = q[:1].expand(60, -1, -1)
    a, _ = kr.op_paged_chunk_attention(one, pages.k, pages.v, pages.table, int32([0, 60]), int32([400]))
    b, _ = kr.op_paged_chunk_attention(one.contiguous(), pages.k, pages.v, pages.table, int32([0, 60]), int32([400]))
    assert (a.float() - b.float()).abs().max() < 4e-3


@gpu
@pytest.mark.parametrize("hd,page,window", [(128, 16, 0), (64, 100, 0), (104, 8, 90), (128, 1, 300)])
def test_chunk_values_that_are_not_finite_reach_the_rows_that_see_them(hd, page, window):
    """A NaN or an infinity in a later token's value, or in one that left the window, leaves a row as it was, to the last bit."""
    n, new = 700, 300
    pages = Pages(12, [n], 2, hd, page, "bf16")
    q = normal(5, new, 4, hd).to(torch.bfloat16)
    call = lambda: kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, int32([0, new]), int32([n]), window=window)  # noqa: E731
    good, good_lse = (t.clone() for t in call())
    where = [(120, 0, 5, math.nan), (450, 0, 7, math.inf), (450, 1, hd - 1, -math.inf), (699, 1, 0, math.nan), (513, 0, 40, math.nan)]
    for key, head, e, value in where:
        pages.v[pages.table[0, key // page].item(), head, key % page, e] = value
    out, lse = call()
    assert bool((lse == good_lse).all())
    odd = torch.zeros_like(out, dtype=torch.bool)
    pos = torch.arange(n - new, n, device=DEV)
    for key, head, e, _ in where:
        sees = (pos >= key) & ((pos - key < window) if window else True)
        odd[:, 2 * head:2 * head + 2, e] |= sees[:, None]
    assert bool((out[~odd] == good[~odd]).all())
    assert not bool(out[odd].isfinite().any())


@gpu
@pytest.mark.parametrize("page", [16, 100])
def test_chunk_scores_that_are_not_finite(page):
    n, new = 300, 200
    pages = Pages(13, [n], 1, 64, page, "bf16")
    q = normal(5, new, 2, 64).to(torch.bfloat16)
    good, _ = (t.clone() for t in kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, int32([0, new]), int32([n])))
    pages.k[pages.table[0, 250 // page].item(), 0, 250 % page, 3] = math.nan      # seen from position 250 on: rows 150 ..
    out, lse = kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, int32([0, new]), int32([n]))
    assert bool((out[:150] == good[:150]).all()) and bool(out[150:].isnan().all()) and bool(lse[150:].isnan().all())
    # one row's queries are not finite: its own results only
    pages = Pages(13, [n], 1, 64, page, "bf16")
    q[17, 1, 2] = math.nan
    out, lse = kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, int32([0, new]), int32([n]))
    assert bool(out[17, 1].isnan().all()) and bool(lse[17, 1].isnan())
    odd = torch.zeros(new, 2, dtype=torch.bool, device=DEV)
    odd[17, 1] = True
    assert bool((out[~odd] == good[~odd]).all())


@gpu
@pytest.mark.parametrize("value", [-math.inf, -2.0e38, -3.3e38, -1e6])
def test_chunk_keys_that_push_scores_to_the_lowest(value):
    """All scores of a head -inf: nothing seen; finite lowest values: still a distribution."""
    pages = Pages(14, [200], 1, 64, 16, "bf16")
    pages.k[:] = 0
    pages.k[..., 0] = value
    q = torch.zeros(50, 1, 64, dtype=torch.bfloat16, device=DEV)
    q[:, 0, 0] = 1.0
    out, lse = kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, int32([0, 50]), int32([200]), scale=1.0)
    if value == -math.inf:
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    else:
        assert bool(out.isfinite().all())
        v = pages.get(pages.v, 0, 0, 200)[:, 0]
        mean = torch.stack([v[:151 + i].mean(0) for i in range(50)])
        assert (out[:, 0].double() - mean).abs().max() < 0.02


@gpu
@pytest.mark.parametrize("page", [16, 100])
def test_chunk_pages_that_do_not_exist(page):
    """Their keys are not visible and the status word says so; the other rows of the call are right."""
    n, new = 420, 33
    pages = Pages(15, [n, 90], 2, 64, page, "bf16")
    q = normal(5, new + 10, 4, 64).to(torch.bfloat16)
    table = pages.table.clone()
    bad = 1
    for number in (-1, pages.n_pages, 2 ** 31 - 1):
        table[0, bad] = number
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out, lse = kr.op_paged_chunk_attention(q, pages.k, pages.v, table, int32([0, new, new + 10]), int32([n, 90]), status=status)
        assert int(status) == kr.STATUS_BAD_PAGE
        k, v = pages.get(pages.k, 0, 0, n), pages.get(pages.v, 0, 0, n)
        key, pos = torch.arange(n, device=DEV), torch.arange(n - new, n, device=DEV)
        hidden = (key > pos[:, None]) | (key // page == bad)
        x = (q[:new, 3].double() @ k[:, 1].T / 8).masked_fill(hidden, -math.inf)
        assert (out[:new, 3].double() - torch.softmax(x, 1) @ v[:, 1]).abs().max() < 0.02
        assert (lse[:new, 3].double() - torch.logsumexp(x, 1)).abs().max() < 1e-4
        good, _ = kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, int32([0, new, new + 10]), int32([n, 90]))
        assert (out[new:].float() - good[new:].float()).abs().max() < 0.04


@gpu
def test_chunk_given_back_pages_and_entries_behind_the_end_are_not_read():
    pages = Pages(16, [1000], 1, 128, 16, "bf16", width=80)
    q = normal(5, 40, 2, 128).to(torch.bfloat16)
    args = (int32([0, 40]), int32([1000]))
    good, _ = (t.clone() for t in kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, *args, window=100))
    table = pages.table.clone()
    table[0, :(960 - 99) // 16] = 2 ** 30
    table[0, 63:] = -5
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, _ = kr.op_paged_chunk_attention(q, pages.k, pages.v, table, *args, window=100, status=status)
    assert int(status) == 0 and bool((out == good).all())


@gpu
@pytest.mark.parametrize("what", ["rows", "descending", "sequence", "keys", "negative"])
def test_chunk_that_does_not_exist_is_left_out(what):
    pages = Pages(17, [200, 100], 1, 64, 16, "bf16")
    q = normal(5, 50, 2, 64).to(torch.bfloat16)
    good, _ = kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, int32([0, 20, 50]), int32([200, 100]))
    starts, keys, seqs = {"rows": ([0, 20, 51], [200, 100], [0, 1]), "descending": ([-3, 20, 19], [200, 100], [0, 1]),
                          "sequence": ([0, 20, 50], [200, 100], [0, 2]), "keys": ([0, 20, 50], [200, 16 * pages.table.shape[1] + 1], [0, 1]),
                          "negative": ([0, 20, 50], [200, -1], [0, 1])}[what]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.full_like(good, 7)
    kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, int32(starts), int32(keys), chunk_seq=int32(seqs), out=out, status=status)
    assert int(status) == kr.STATUS_BAD_PAGE
    assert bool((out[20:] == 7).all())
    if what == "descending":
        assert bool((out == 7).all())
    else:
        assert (out[:20].float() - good[:20].float()).abs().max() < 0.03


@gpu
def test_chunk_offsets_past_32_bits():
    hd, page = 128, 64
    n_pages = 2 ** 31 // (page * 2 * hd) + 40
    k = torch.zeros(n_pages, 2, page, hd, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    small = Pages(18, [500], 2, hd, page, "bf16")
    table = small.table.clone()
    for i in range(8):
        old, new = table[0, i].item(), n_pages - 1 - 4 * i
        k[new], v[new] = small.k[old].nan_to_num(0.0), small.v[old].nan_to_num(0.0)
        table[0, i] = new
    q = normal(5, 30, 4, hd).to(torch.bfloat16)
    good, _ = kr.op_paged_chunk_attention(q, small.k, small.v, small.table, int32([0, 30]), int32([500]))
    out, _ = kr.op_paged_chunk_attention(q, k, v, table, int32([0, 30]), int32([500]))
    assert bool((out == good).all())


@gpu
def test_chunk_is_the_same_from_run_to_run_and_whatever_the_workspace_holds():
    pages = Pages(19, [5000, 300, 1], 2, 128, 16, "bf16")
    q = normal(5, 400, 8, 128).to(torch.bfloat16)
    args = (q, pages.k, pages.v, pages.table, int32([0, 200, 399, 400]), int32([5000, 300, 1]))
    out, lse = (t.clone() for t in kr.op_paged_chunk_attention(*args))
    for byte in (0, 255, 127):
        ws = torch.full((kr.paged_chunk_attention_workspace(128),), byte, dtype=torch.uint8, device=DEV)
        again, again_lse = kr.op_paged_chunk_attention(*args, workspace=ws)
        assert bool((again == out).all()) and bool((again_lse == lse).all())


@gpu
def test_chunk_random_calls():
    r = random.Random(5)
    for i in range(40):
        Hkv = r.choice([1, 2, 3, 4])
        H = Hkv * r.choice([1, 2, 3, 4, 7, 8])
        hd, page, dtype = r.choice([64, 72, 96, 104, 128]), r.choice([1, 8, 16, 24, 40, 64, 100, 128, 256]), r.choice(["bf16", "f16"])
        spans = [(r.choice([0, r.randint(0, 50), r.randint(0, 3000)]), r.choice([0, 1, 1, r.randint(1, 40), r.randint(1, 500)]))
                 for _ in range(r.randint(1, 9))]
        lens = [max(p + n, 0) for p, n in spans]
        pages = Pages(i, lens, Hkv, hd, page, dtype, by_slot=r.random() < 0.5)
        starts = [r.randint(0, 3)]
        for _, n in spans:
            starts.append(starts[-1] + n)
        q = normal(i, starts[-1] + r.randint(1, 4), H, hd).to(T16[dtype])
        slopes = torch.rand(H, generator=torch.Generator().manual_seed(i)).to(DEV) if r.random() < 0.3 else None
        check_chunk(pages, q, starts, lens, cap=r.choice([0.0, 0.0, 10.0]), window=r.choice([0, 0, 1, 130, 700]), slopes=slopes)


@gpu
def test_chunk_in_a_graph_with_other_lengths():
    """A captured call follows what its length tensors say at replay; padding chunks and rows stay as they were."""
    pages = Pages(20, [700, 700, 700, 700], 2, 64, 16, "bf16")
    q = normal(5, 300, 4, 64).to(torch.bfloat16)
    starts, keys, seqs = int32([0, 300, 300, 300, 300]), int32([700, 0, 0, 0]), int32([0, -1, -1, -1])
    out, lse = torch.full((300, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((300, 4), 7.0, device=DEV)
    ws = torch.empty(kr.paged_chunk_attention_workspace(64), dtype=torch.uint8, device=DEV)
    call = lambda o, l: kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, starts, keys, chunk_seq=seqs, out=o, lse=l, workspace=ws)  # noqa: E731
    call(out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse)
    for s, n, i in (([0, 300, 300, 300, 300], [700, 0, 0, 0], [0, -1, -1, -1]), ([0, 1, 2, 100, 131], [500, 1, 98, 690], [3, 2, 1, 0]),
                    ([5, 5, 5, 5, 5], [1, 1, 1, 1], [0, 1, 2, 3])):
        starts.copy_(int32(s))
        keys.copy_(int32(n))
        seqs.copy_(int32(i))
        out.fill_(7)
        lse.fill_(7)
        graph.replay()
        eager, eager_lse = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
        call(eager, eager_lse)
        assert bool((out == eager).all()) and bool((lse == eager_lse).all())
    del graph


@gpu
def test_chunk_on_two_streams_at_once():
    pages = Pages(21, [3000, 800], 2, 128, 16, "bf16")
    qs = [normal(30 + i, 500, 4, 128).to(torch.bfloat16) for i in range(2)]
    args = (int32([0, 300, 500]), int32([3000, 800]))
    want = [tuple(t.clone() for t in kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, *args)) for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(kr.op_paged_chunk_attention(qs[i], pages.k, pages.v, pages.table, *args))
    torch.cuda.synchronize()
    for i in range(2):
        for out, lse in got[i]:
            assert bool((out == want[i][0]).all()) and bool((lse == want[i][1]).all())


# ------------------------------------------------------------------ append with norms

def normed(x, weight, eps):
    x = x.double()
    w = torch.ones(x.shape[-1], dtype=torch.float64, device=DEV) if weight is None else weight.double()
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w


def turned(x, pos, inv_freq, interleaved):
    """x [rows, heads, hd] in 64 bits, and the sums |a| + |b| of the pairs"""
    if inv_freq is None:
        return x, x.abs()
    half = inv_freq.numel()
    t = pos.double()[:, None, None] * inv_freq.double()
    c, s = torch.cos(t), torch.sin(t)
    out, size = x.clone(), x.abs()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return out, size


NORMS = [
    # rows, H, Hkv, hd, rot, page, dtype, weights
    (1, 32, 8, 128, 128, 16, "bf16", "all"),
    (5, 3, 1, 64, 64, 8, "f16", "head"),
    (7, 12, 4, 72, 72, 1, "bf16", "all"),
    (9, 5, 5, 96, 48, 24, "f16", "head"),
    (70, 6, 2, 104, 104, 100, "bf16", None),
    (33, 4, 4, 128, 32, 64, "f16", "all"),
    (40, 2, 1, 128, 0, 16, "bf16", "head"),
    (12, 7, 7, 72, 24, 16, "bf16", "q"),
    (700, 16, 16, 128, 128, 64, "bf16", "all"),
    (650, 9, 3, 96, 8, 16, "f16", "k"),
    (611, 5, 1, 64, 40, 256, "bf16", "head"),
]


@gpu
@pytest.mark.parametrize("rows,H,Hkv,hd,rot,page,dtype,weights", NORMS)
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_norm(rows, H, Hkv, hd, rot, page, dtype, weights, interleaved):
    t = T16[dtype]
    n = 3 * rows + 40
    pages = Pages(rows, [n, 1, n], Hkv, hd, page, dtype, by_slot=interleaved, fill=False)
    product = normal(rows + 1, rows, (H + 2 * Hkv) * hd).to(t)
    product[rows // 2] *= 100
    product[rows // 3, :hd] = 0           # a head of zeros stays zeros
    q, k, v = (x.unflatten(1, (-1, hd)) for x in product.split([H * hd, Hkv * hd, Hkv * hd], 1))
    seq = torch.arange(rows) % 4 - 1      # -1: padding
    seq[seq == 1] = 0
    pos = torch.randperm(n, generator=torch.Generator().manual_seed(rows))[:rows]
    one = lambda seed, heads: (1 + 0.3 * normal(seed, *((heads, hd) if weights == "head" else (hd,)))).to(t)  # noqa: E731
    wq = one(3, H) if weights in ("all", "head", "q") else None
    wk = one(4, Hkv) if weights in ("all", "head", "k") else None
    freq = torch.tensor([10000.0 ** (-2 * i / rot) for i in range(rot // 2)], device=DEV) if rot else None
    eps = 1e-5
    q_out = torch.full((rows, H, hd), 7.0, dtype=t, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    kr.op_paged_append_norm(k, v, pages.k, pages.v, pages.table, pos.int().to(DEV), k_weight=wk, q_weight=wq, eps=eps,
                            row_seq=seq.int().to(DEV), q=q, q_out=q_out, inv_freq=freq, interleaved=interleaved, status=status)
    assert int(status) == 0
    live = (seq >= 0).to(DEV)
    half = torch.finfo(t).eps / 2
    posd = pos.to(DEV)
    ref, size = turned(normed(q, wq, eps), posd, freq, interleaved)
    tiny = 2.0 ** -25 if dtype == "f16" else 0.0
    assert bool(((q_out.double() - ref).abs() <= half * ref.abs() * (1 + 1e-2) + 3e-6 * size + tiny)[live].all())
    assert bool((q_out[~live] == 7).all())
    ref, size = turned(normed(k, wk, eps), posd, freq, interleaved)
    written = torch.zeros_like(pages.k, dtype=torch.bool)
    for r in range(rows):
        if seq[r] < 0:
            continue
        at = (pages.table[seq[r], pos[r] // page].item(), slice(None), int(pos[r]) % page)
        written[at] = True
        assert bool(((pages.k[at].double() - ref[r]).abs() <= half * ref[r].abs() * (1 + 1e-2) + 3e-6 * size[r] + tiny).all())
        assert bool((pages.v[at] == v[r]).all())
    assert bool(pages.k[~written].isnan().all()) and bool(pages.v[~written].isnan().all())


@gpu
def test_append_norm_in_place_and_without_queries():
    pages = Pages(2, [64], 2, 64, 16, "bf16", fill=False)
    q, k, v = (normal(i, 10, h, 64).to(torch.bfloat16) for i, h in ((1, 4), (2, 2), (3, 2)))
    args = dict(row_seq=torch.zeros(10, dtype=torch.int32, device=DEV), inv_freq=torch.rand(32, device=DEV), eps=1e-6)
    pos = torch.arange(10, dtype=torch.int32, device=DEV)
    want = kr.op_paged_append_norm(k, v, pages.k, pages.v, pages.table, pos, q=q, **args)
    k_cache, v_cache = pages.k.clone(), pages.v.clone()
    own = q.clone()
    got = kr.op_paged_append_norm(k, v, pages.k, pages.v, pages.table, pos, q=own, q_out=own, **args)
    assert got is own and bool((own == want).all())
    pages.k.fill_(math.nan)
    pages.v.fill_(math.nan)
    assert kr.op_paged_append_norm(k, v, pages.k, pages.v, pages.table, pos, **args) is None
    assert bool((pages.k.view(torch.int16) == k_cache.view(torch.int16)).all()) and bool((pages.v.view(torch.int16) == v_cache.view(torch.int16)).all())


@gpu
def test_append_norm_rows_that_do_not_exist():
    pages = Pages(2, [64], 1, 64, 16, "bf16", fill=False)
    k = normal(1, 5, 1, 64).to(torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    kr.op_paged_append_norm(k, k, pages.k, pages.v, pages.table, int32([0, 64, -1, 3, 4]), row_seq=int32([0, 0, 0, 1, -1]), status=status)
    assert int(status) == kr.STATUS_BAD_PAGE
    assert int((~pages.v.isnan()).any(-1).sum()) == 1
    kr.op_paged_append_norm(k[:0], k[:0], pages.k, pages.v, pages.table, int32([]), row_seq=int32([]))


# ------------------------------------------------------------------ refusals (no GPU: the library looks at its arguments first)

def cache_args(hd=64, page=16, n_kv=2):
    return kr.PagedCacheArgs(k=1 << 20, v=2 << 20, page_table=3 << 20, page_stride=n_kv * page * hd, head_stride=page * hd, slot_stride=hd,
                             table_stride=4, n_pages=8, page_size=page, n_kv_head=n_kv, head_dim=hd, n_seqs=4, max_pages=4)


def chunk_args(**over):
    a = dict(q=4 << 20, q_row_stride=256, q_head_stride=64, out=5 << 20, out_row_stride=256, out_head_stride=64, q_start=6 << 20,
             n_keys=7 << 20, workspace=8 << 20, workspace_bytes=1 << 40, scale=0.125, chunks=2, rows=10, n_head=4)
    a.update(over)
    return kr.PagedChunkArgs(**a)


CHUNK_REFUSALS = [
    (dict(q=None), kr.EINVAL), (dict(out=None), kr.EINVAL), (dict(q_start=None), kr.EINVAL), (dict(n_keys=None), kr.EINVAL),
    (dict(n_head=3), kr.EINVAL), (dict(n_head=0), kr.EINVAL), (dict(rows=-1), kr.EINVAL), (dict(chunks=-1), kr.EINVAL), (dict(window=-1), kr.EINVAL),
    (dict(score_cap=-1.0), kr.EINVAL), (dict(score_cap=math.inf), kr.EINVAL), (dict(score_cap=math.nan), kr.EINVAL), (dict(score_cap=1e-45), kr.EINVAL),
    (dict(scale=math.inf), kr.EINVAL), (dict(scale=math.nan), kr.EINVAL), (dict(scale=3e38), kr.EINVAL), (dict(chunks=5), kr.EINVAL),
    (dict(out_row_stride=0), kr.EINVAL), (dict(out_head_stride=0), kr.EINVAL), (dict(lse=9 << 20, lse_row_stride=0), kr.EINVAL),
    (dict(q=(4 << 20) + 2), kr.EUNSUPPORTED), (dict(out=(5 << 20) + 8), kr.EUNSUPPORTED), (dict(q_row_stride=255), kr.EUNSUPPORTED),
    (dict(out_head_stride=68), kr.EUNSUPPORTED), (dict(rows=1 << 22), kr.EUNSUPPORTED),
    (dict(chunks=1 << 22, chunk_seq=10 << 20), kr.EUNSUPPORTED), (dict(workspace=None), kr.ECAPACITY), (dict(workspace_bytes=100), kr.ECAPACITY),
    (dict(workspace=(8 << 20) + 4), kr.EINVAL),
]


@pytest.mark.parametrize("over,code", CHUNK_REFUSALS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_chunk_refusals(over, code, dtype):
    assert kr.lib(dtype).kraken_op_paged_chunk_attention(C.byref(cache_args()), C.byref(chunk_args(**over)), None, None) == code


def test_chunk_refuses_caches_and_takes_nothing_to_do():
    f = kr.lib().kraken_op_paged_chunk_attention
    assert f(None, C.byref(chunk_args()), None, None) == kr.EINVAL and f(C.byref(cache_args()), None, None, None) == kr.EINVAL
    assert f(C.byref(cache_args(hd=80)), C.byref(chunk_args()), None, None) == kr.EUNSUPPORTED
    assert f(C.byref(cache_args()), C.byref(chunk_args(rows=0)), None, None) == kr.OK
    assert f(C.byref(cache_args()), C.byref(chunk_args(chunks=0)), None, None) == kr.OK
    n = C.c_size_t()
    assert kr.lib().kraken_paged_chunk_attention_workspace(80, C.byref(n)) == kr.EUNSUPPORTED
    assert kr.lib().kraken_paged_chunk_attention_workspace(64, None) == kr.EINVAL
    assert kr.lib().kraken_paged_chunk_attention_workspace(64, C.byref(n)) == kr.OK and n.value > 0


@pytest.mark.parametrize("over,code", [(dict(eps=-1e-6), kr.EINVAL), (dict(eps=math.nan), kr.EINVAL), (dict(eps=math.inf), kr.EINVAL),
                                       (dict(q_weight=(9 << 20) + 2), kr.EUNSUPPORTED), (dict(k_weight=(9 << 20) + 8), kr.EUNSUPPORTED),
                                       (dict(k_weight=9 << 20, k_head_stride=60), kr.EUNSUPPORTED)])
def test_append_norm_refusals(over, code):
    a = kr.PagedAppendArgs(k=4 << 20, v=5 << 20, k_row_stride=128, k_head_stride=64, v_row_stride=128, v_head_stride=64, row_pos=6 << 20, rows=3)
    f = kr.lib().kraken_op_paged_append_norm
    assert f(C.byref(cache_args()), C.byref(a), C.byref(kr.PagedNormArgs(**over)), None, None) == code
    assert f(C.byref(cache_args()), C.byref(a), None, None, None) == kr.EINVAL
    a.rows = 0
    assert f(C.byref(cache_args()), C.byref(a), C.byref(kr.PagedNormArgs(eps=1e-6)), None, None) == kr.OK


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        kr.op_paged_chunk_attention(x[0], x, x, i[None], torch.zeros(2, dtype=torch.int32), i)
    with pytest.raises(ValueError):
        kr.op_paged_append_norm(x[0], x[0], x, x, i[None], i)


@gpu
def test_binding_refusals():
    pages = Pages(1, [40], 2, 64, 16, "bf16")
    q = normal(1, 6, 4, 64).to(torch.bfloat16)
    s, n = int32([0, 6]), int32([40])
    good = dict(q=q, k_cache=pages.k, v_cache=pages.v, page_table=pages.table, q_start=s, n_keys=n)
    for bad in (dict(q=q.half()), dict(q=q[:, :, ::2]), dict(q_start=int32([0])), dict(q_start=s.long()), dict(n_keys=n.float()),
                dict(n_keys=None), dict(q_start=None), dict(chunk_seq=int32([0, 1])), dict(slopes=torch.zeros(3, device=DEV)), dict(window="a"),
                dict(out=q[:5]), dict(lse=torch.zeros(6, 5, device=DEV)), dict(score_cap=1e-60), dict(v_cache=pages.v[:2])):
        with pytest.raises(ValueError):
            kr.op_paged_chunk_attention(**{**good, **bad})
    with pytest.raises(kr.KrakenError):
        kr.op_paged_chunk_attention(**good, workspace=torch.empty(64, dtype=torch.uint8, device=DEV))
    k = normal(2, 3, 2, 64).to(torch.bfloat16)
    append = dict(k=k, v=k, k_cache=pages.k, v_cache=pages.v, page_table=pages.table, positions=int32([0, 1, 2]), row_seq=int32([0, 0, 0]))
    for bad in (dict(k_weight=k[0, 0].float()), dict(k_weight=k[0, 0, :32]), dict(k_weight=k[:, 0]), dict(q_weight=k[0, 0]), dict(eps="x"),
                dict(q=q[:3], q_weight=k[0])):
        with pytest.raises(ValueError):
            kr.op_paged_append_norm(**{**append, **bad})

"""The cache in pages (append with rotation, decode-step attention) and the reading of logits, against plain 64-bit forms.

Tolerances.  A result rounded to 16 bits may be off by half a step, eps / 2 of its value.  On top of that:
  append     the angle's fraction of a turn is rounded to fp32 (2^-25 turns = 1.9e-7), the sine and cosine to 1-2 units
             (1.2e-7 each), three fp32 roundings: below 6e-7 (|a| + |b|) for the pair (a, b)
  attention  a score is an fp32 sum of head_dim products: off by at most d = head_dim 2^-23 scale max sum |q_e k_e| (and as much
             again relative for the score's own roundings); a weight by 2 d + 2^-17 (two 16-bit pieces of 8 bits each, 2^-18, and
             the exponential, 2^-22); a sum over n keys by n 2^-24.  The output by that share of sum p |v|, lse by that itself.
  logprobs   a weight by |y| 2^-22 + 2^-22 with |y| e^-|y| < 0.4, sums of up to V / 256 + 64 terms in a row by 2^-24 each;
             a value by 2^-22 of itself.
"""
import ctypes as C
import math
import random

import pytest
import torch

import kraken_inputs as ki
import paper_2408_07802_b200 as kr
from paper_2408_07802_b200 import build as kbuild

kbuild.build_all()

DEV = "cuda:0"
gpu = pytest.mark.gpu
T16 = {"bf16": torch.bfloat16, "f16": torch.float16}


def normal(seed, *shape, device=DEV):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).to(device)


class Pages:
    """Sequences of the given lengths in pages handed out in a shuffled order; unused slots hold NaN."""

    def __init__(self, seed, lens, n_kv, hd, page, dtype, spare=2, by_slot=False, fill=True, width=None):
        self.lens, self.page = list(lens), page
        used = [-(-n // page) for n in lens]
        self.n_pages = sum(used) + spare
        order = torch.randperm(self.n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
        self.table = torch.full((len(lens), width or max([1] + used)), -7, dtype=torch.int32)
        at = 0
        for s, n in enumerate(used):
            self.table[s, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.table = self.table.to(DEV)
        shape = (self.n_pages, page, n_kv, hd) if by_slot else (self.n_pages, n_kv, page, hd)
        self.k = torch.full(shape, math.nan, dtype=T16[dtype], device=DEV)
        self.v = self.k.clone()
        if by_slot:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        if fill:
            for i, cache in enumerate((self.k, self.v)):
                for s, n in enumerate(lens):
                    if n:
                        self.put(cache, s, 0, normal(seed + 1000 * i + s + 1, n, n_kv, hd).to(cache.dtype))

    def put(self, cache, s, pos0, rows):
        for i in range(rows.shape[0]):
            cache[self.table[s, (pos0 + i) // self.page].item(), :, (pos0 + i) % self.page] = rows[i]

    def get(self, cache, s, lo, hi):
        """[hi - lo, n_kv, hd] in 64 bits"""
        pos = torch.arange(lo, hi, device=DEV)
        return cache[self.table[s][pos // self.page].long(), :, pos % self.page].double()


def attention_ref(pages, q, n_keys, row_seq, scale, cap=0.0, window=0, slopes=None):
    """(out, lse, tolerance share of out, of lse), all 64 bits; None rows are padding."""
    R, H, hd = q.shape
    rep = H // pages.k.shape[1]
    out = torch.zeros(R, H, hd, dtype=torch.float64, device=DEV)
    lse = torch.full((R, H), -math.inf, dtype=torch.float64, device=DEV)
    tol_o, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    for r in range(R):
        n, s = int(n_keys[r]), int(row_seq[r])
        lo = max(0, n - window) if window else 0
        if s < 0 or n == 0:
            continue
        k, v = pages.get(pages.k, s, lo, n), pages.get(pages.v, s, lo, n)
        for h in range(H):
            qh = q[r, h].double()
            x = k[:, h // rep] @ qh * scale
            d = hd * 2.0 ** -23 * scale * (k[:, h // rep].abs() @ qh.abs()).max() + 2.0 ** -22 * x.abs().max()
            if cap:
                x = cap * torch.tanh(x / cap)
                d = d + 2.0 ** -21 * x.abs().max()
            if slopes is not None:
                x = x + slopes[h].double() * (torch.arange(lo, n, device=DEV) - (n - 1))
                d = d + 2.0 ** -22 * x.abs().max()
            p = torch.softmax(x, 0)
            out[r, h] = p @ v[:, h // rep]
            lse[r, h] = torch.logsumexp(x, 0)
            share = 2 * d + 2.0 ** -17 + n * 2.0 ** -24
            tol_o[r, h] = 2 * share * (p @ v[:, h // rep].abs())
            tol_l[r, h] = share + 2.0 ** -22 * lse[r, h].abs()
    return out, lse, tol_o, tol_l


def check_attention(pages, q, n_keys, row_seq=None, cap=0.0, window=0, slopes=None, scale=None, **kw):
    hd = q.shape[2]
    scale = hd ** -0.5 if scale is None else scale
    seqs = row_seq if row_seq is not None else torch.arange(q.shape[0])
    ref, ref_lse, tol, tol_l = attention_ref(pages, q, n_keys.tolist(), seqs.tolist(), scale, cap, window, slopes)
    out, lse = kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, n_keys, row_seq=row_seq, scale=scale, score_cap=cap,
                                            window=window, slopes=slopes, **kw)
    live = (seqs >= 0).to(DEV)
    half = torch.finfo(q.dtype).eps / 2
    err = (out.double() - ref).abs()[live]
    bound = (half * ref.abs() * (1 + 1e-3) + tol + 2.0 ** -25)[live]
    assert bool((err <= bound).all()), (err - bound).max().item()
    some = live & (n_keys > 0)
    assert bool(((lse.double() - ref_lse).abs()[some] <= tol_l[some]).all())
    none = live & (n_keys == 0)
    assert bool((lse[none] == -math.inf).all()) and bool((out[none] == 0).all())
    return out, lse


ATTEND = [
    # lens, H, Hkv, hd, page, dtype
    ([1], 1, 1, 64, 16, "bf16"),
    ([0, 1, 2, 15, 16, 17, 31, 33], 4, 2, 64, 16, "bf16"),
    ([63, 64, 65, 127, 128, 129], 8, 1, 128, 1, "f16"),
    ([5, 700], 12, 12, 104, 24, "f16"),
    ([300, 0, 0, 1], 5, 1, 72, 8, "bf16"),
    ([257, 90], 16, 1, 96, 100, "bf16"),
    ([40, 999], 18, 2, 128, 64, "bf16"),
    ([77, 500], 33, 1, 64, 16, "f16"),
    ([1500, 3, 2049], 32, 4, 128, 256, "bf16"),
    ([6000], 2, 2, 128, 16, "f16"),
]


@gpu
@pytest.mark.parametrize("lens,H,Hkv,hd,page,dtype", ATTEND)
@pytest.mark.parametrize("form", ["plain", "cap", "window", "slopes", "all"])
def test_attention(lens, H, Hkv, hd, page, dtype, form):
    pages = Pages(len(lens) + H, lens, Hkv, hd, page, dtype, by_slot=form == "window")
    q = normal(7, len(lens), H, hd).to(T16[dtype])
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    slopes = (2.0 ** -torch.linspace(1, 8, H)).to(DEV) if form in ("slopes", "all") else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    check_attention(pages, q, n, cap=3.0 if form in ("cap", "all") else 0.0, window=37 if form in ("window", "all") else 0,
                    slopes=slopes, status=status)
    assert int(status.item()) == 0


@gpu
@pytest.mark.parametrize("window", [1, 16, 64, 65, 1 << 30])
def test_attention_windows(window):
    lens = [1, 64, 65, 200, 1031]
    pages = Pages(3, lens, 2, 64, 24, "bf16")
    check_attention(pages, normal(8, len(lens), 8, 64).to(torch.bfloat16), torch.tensor(lens, dtype=torch.int32, device=DEV), window=window)


@gpu
@pytest.mark.parametrize("page", [1, 3, 4, 7, 8, 16, 24, 100])
@pytest.mark.parametrize("window", [1, 10, 37])
@pytest.mark.parametrize("no_page", [-1, 1 << 30])
def test_attention_pages_freed_behind_the_window(page, window, no_page):
    """Table entries of pages wholly in front of the window may name no page: no status, and the bits of the full table."""
    lens = [0, 1, 25, 30, 41, 200, 1031]
    pages = Pages(35, lens, 2, 64, page, "bf16")
    q = normal(36, len(lens), 8, 64).to(torch.bfloat16)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    full = check_attention(pages, q, n, window=window)
    for s, length in enumerate(lens):
        pages.table[s, :max(0, length - window) // page] = no_page
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, n, window=window, status=status)
    assert int(status.item()) == 0
    assert torch.equal(out, full[0]) and torch.equal(lse, full[1])


@gpu
def test_attention_rows_of_one_sequence_padding_and_strides():
    """Draft tokens (several rows of one sequence), padding rows in the middle, q and out as slices of wider tensors."""
    lens = [400, 90]
    pages = Pages(4, lens, 2, 128, 16, "bf16")
    seq = torch.tensor([0, 0, -1, 1, 0, -5, 1], dtype=torch.int32, device=DEV)
    n = torch.tensor([398, 399, 12345, 90, 400, -3, 1], dtype=torch.int32, device=DEV)
    wide = normal(9, 7, 8 * 3 * 128).to(torch.bfloat16)
    q = wide[:, 128:128 + 8 * 128].unflatten(1, (8, 128))
    box = torch.full((7, 10, 128), 77.0, dtype=torch.bfloat16, device=DEV)
    lbox = torch.full((7, 11), 55.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    check_attention(pages, q, n, row_seq=seq, out=box[:, 1:9], lse=lbox[:, 2:10], status=status)
    assert int(status.item()) == 0
    assert bool((box[seq < 0] == 77).all()) and bool((box[:, [0, 9]] == 77).all())
    assert bool((lbox[seq < 0] == 55).all()) and bool((lbox[:, [0, 1, 10]] == 55).all())


@gpu
def test_attention_rows_and_pages_that_do_not_exist():
    lens = [100, 100, 100, 100, 100]
    pages = Pages(5, lens, 1, 64, 16, "bf16")
    good = pages.table.clone()
    q = normal(10, 5, 4, 64).to(torch.bfloat16)
    n = torch.tensor([100, 113, 100, -1, 100], dtype=torch.int32, device=DEV)      # 113 > 7 pages of 16; -1
    seq = torch.tensor([0, 1, 5, 3, 4], dtype=torch.int32, device=DEV)             # sequence 5 of 5
    pages.table[4, 2], pages.table[4, 5] = pages.n_pages, -1
    out, lse = torch.full_like(q, 9.0), torch.full((5, 4), 9.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, n, row_seq=seq, out=out, lse=lse, status=status)
    assert int(status.item()) == kr.STATUS_BAD_PAGE
    assert bool((out[1:4] == 9).all()) and bool((lse[1:4] == 9).all())
    # row 4: the 32 keys on pages that do not exist are not visible
    pages.table = good
    keep = [i for i in range(100) if i // 16 not in (2, 5)]
    k, v = pages.get(pages.k, 4, 0, 100)[keep, 0], pages.get(pages.v, 4, 0, 100)[keep, 0]
    p = torch.softmax(q[4].double() @ k.T / 8, -1)
    assert (out[4].double() - p @ v).abs().max() < 2.0 ** -8 * 4
    p = torch.softmax(q[0].double() @ pages.get(pages.k, 0, 0, 100)[:, 0].T / 8, -1)
    assert (out[0].double() - p @ pages.get(pages.v, 0, 0, 100)[:, 0]).abs().max() < 2.0 ** -8 * 4


class Some(Pages):
    """The same pages without the keys whose position `hidden` names."""

    def __init__(self, pages, hidden):
        self.k, self.v, self.table, self.page, self.hidden = pages.k, pages.v, pages.table.clone(), pages.page, hidden

    def get(self, cache, s, lo, hi):
        return super().get(cache, s, lo, hi)[[i for i in range(lo, hi) if not self.hidden(i)]]


def near_reference(pages, q, out, lse, n_keys, row_seq, rows):
    """Those rows of (out, lse) against 64 bits, with the tolerances of check_attention."""
    ref, ref_lse, tol, tol_l = attention_ref(pages, q, n_keys, row_seq, q.shape[2] ** -0.5)
    half = torch.finfo(q.dtype).eps / 2
    assert bool(((out.double() - ref).abs() <= half * ref.abs() * (1 + 1e-3) + tol + 2.0 ** -25)[rows].all())
    assert bool(((lse.double() - ref_lse).abs() <= tol_l)[rows].all())


@gpu
@pytest.mark.parametrize("page,width", [(16, 7), (16, 600), (7, 15), (7, 1200), (8, 13), (100, 1)])
@pytest.mark.parametrize("kind", ["too long", "negative length", "no sequence", "page past the end", "page below zero"])
def test_attention_what_does_not_exist_one_at_a_time(page, width, kind):
    """Each kind alone raises the bit, in the middle one of three rows: with copies as boxes and by the lanes, with page tables
    by which the host knows that nothing is split and others."""
    lens = [100, 100, 100]
    pages = Pages(37, lens, 2, 64, page, "bf16", width=width)
    q = normal(38, 3, 8, 64).to(torch.bfloat16)
    lengths = {"too long": width * page + 1, "negative length": -1}
    n, seq = [100, lengths.get(kind, 100), 100], [0, 3 if kind == "no sequence" else 1, 2]
    left_alone = kind in ("too long", "negative length", "no sequence")
    lost = (100 - 1) // page                                     # number of the page that does not exist
    seen = Some(pages, lambda i: i // page == lost and not left_alone)
    if not left_alone:
        pages.table[1, lost] = pages.n_pages if kind == "page past the end" else -1
    out, lse = torch.full_like(q, 9.0), torch.full((3, 8), 9.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, torch.tensor(n, dtype=torch.int32, device=DEV),
                                 row_seq=torch.tensor(seq, dtype=torch.int32, device=DEV), out=out, lse=lse, status=status)
    assert int(status.item()) == kr.STATUS_BAD_PAGE
    near_reference(Some(pages, lambda i: False), q, out, lse, [100, 0, 100], [0, -1, 2], [0, 2])
    if left_alone:
        assert bool((out[1] == 9).all()) and bool((lse[1] == 9).all())
    elif lost == 0:                                              # no key is left
        assert bool((out[1] == 0).all()) and bool((lse[1] == -math.inf).all())
    else:
        near_reference(seen, q, out, lse, [0, 100, 0], [-1, 1, -1], [1])


@gpu
def test_attention_many_rows_of_unequal_length_and_a_row_alone():
    """A row's result does not depend on the rows beside it (up to the order of the sums)."""
    g = torch.Generator().manual_seed(6)
    lens = [int(x) for x in torch.randint(0, 60, (290,), generator=g)] + [4000, 1, 0, 2500]
    pages = Pages(6, lens, 2, 64, 16, "f16")
    q = normal(11, len(lens), 4, 64).to(torch.float16)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out, lse = check_attention(pages, q, n)
    for r in (3, 290, 293):
        o1, l1 = kr.op_paged_decode_attention(q[r:r + 1], pages.k, pages.v, pages.table[r:r + 1], n[r:r + 1])
        assert (o1[0] - out[r]).abs().max() <= 2.0 ** -9 and (l1[0] - lse[r]).abs().max() < 1e-4


@gpu
def test_attention_extreme_scores():
    """Scores far apart (all weight on one key), equal scores, keys of -inf score; a NaN outside the visible keys is not read."""
    pages = Pages(12, [200, 200, 200], 1, 64, 16, "bf16")
    q = torch.zeros(3, 1, 64, dtype=torch.bfloat16, device=DEV)
    q[0, 0, 0] = 1.0
    pages.k.nan_to_num_(0.0)
    for s in (0, 2):
        for i in range(200):
            pages.k[pages.table[s, i // 16].item(), 0, i % 16] = 0
    pages.k[pages.table[0, 5].item(), 0, 3, 0] = 30000.0        # held as 29952 in bfloat16
    out, lse = kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, torch.tensor([200, 200, 0], dtype=torch.int32, device=DEV))
    assert torch.equal(out[0, 0], pages.v[pages.table[0, 5].item(), 0, 3]) and abs(lse[0, 0].item() - 29952 / 8) < 1e-2
    mean = pages.get(pages.v, 1, 0, 200)[:, 0].mean(0)
    assert (out[1, 0].double() - mean).abs().max() < 2.0 ** -8 * mean.abs().max() + 1e-5 and abs(lse[1, 0].item() - math.log(200)) < 1e-5
    # every visible score -inf: no weight anywhere
    q[2, 0, 0] = 1.0
    for i in range(17):
        pages.k[pages.table[2, i // 16].item(), 0, i % 16, 0] = -math.inf
    out, lse = kr.op_paged_decode_attention(q[2:], pages.k, pages.v, pages.table[2:], torch.tensor([17], dtype=torch.int32, device=DEV))
    assert bool((out == 0).all()) and lse.item() == -math.inf


@gpu
@pytest.mark.parametrize("n,page", [(60, 16), (60, 7), (3000, 16), (3000, 7)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attention_nan_and_infinity_in_visible_places(n, page, dtype):
    """They reach the heads (of a value: the elements) that they belong to and nothing else, whoever of the CTAs meets them."""
    pages = Pages(39, [n, n], 2, 64, page, dtype)
    q = normal(40, 2, 6, 64).to(T16[dtype])
    q[:, 0, 0], q[:, 1, 0], q[:, 2, 0] = 1.0, -1.0, 0.0            # heads of key/value head 0
    lens = torch.tensor([n, n], dtype=torch.int32, device=DEV)
    at = 29
    slot = (pages.table[1, at // page].item(), 0, at % page)         # of head 0
    run = lambda q=q: kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, lens)
    clean, clean_lse = run()
    k, v = pages.k[slot].clone(), pages.v[slot].clone()

    def others_as_before(out, lse, row, heads):
        keep = torch.ones(2, 6, dtype=torch.bool, device=DEV)
        keep[row, heads] = False
        assert torch.equal(out[keep], clean[keep]) and torch.equal(lse[keep], clean_lse[keep])

    # a query: its head
    bad = q.clone()
    bad[1, 4, 5] = math.nan
    out, lse = run(bad)
    assert bool(out[1, 4].isnan().all()) and bool(lse[1, 4].isnan())
    others_as_before(out, lse, 1, [4])
    # a key: the heads that share it.  NaN, and +inf as a score: NaN; -inf as a score: that key does not count
    pages.k[slot][7] = math.nan
    out, lse = run()
    assert bool(out[1, :3].isnan().all()) and bool(lse[1, :3].isnan().all())
    others_as_before(out, lse, 1, [0, 1, 2])
    pages.k[slot][7] = k[7]
    pages.k[slot][0] = math.inf
    out, lse = run()
    assert bool(out[1, [0, 2]].isnan().all()) and bool(lse[1, [0, 2]].isnan().all())       # inf, and 0 times inf
    others_as_before(out, lse, 1, [0, 1, 2])
    pages.k[slot][0] = k[0]
    near = Some(pages, lambda i: i == at)
    ref, ref_lse, tol, tol_l = attention_ref(near, q, [0, n], [-1, 1], 64 ** -0.5)
    half = torch.finfo(q.dtype).eps / 2
    assert bool(((out[1, 1].double() - ref[1, 1]).abs() <= half * ref[1, 1].abs() * (1 + 1e-3) + tol[1, 1] + 2.0 ** -25).all())
    assert bool((lse[1, 1].double() - ref_lse[1, 1]).abs() <= tol_l[1, 1])
    # a value: its element of the heads that share it, which is not finite; the other elements and lse as before
    for x in (math.nan, math.inf, -math.inf):
        pages.v[slot][9] = x
        out, lse = run()
        assert not bool(out[1, :3, 9].isfinite().any()) and torch.equal(lse, clean_lse)
        out[1, :3, 9] = clean[1, :3, 9]
        assert torch.equal(out, clean)
        pages.v[slot][9] = v[9]


@gpu
@pytest.mark.parametrize("form", ["cap", "slopes", "all"])
@pytest.mark.parametrize("lens,H,Hkv,hd,page,dtype", [ATTEND[1], ATTEND[3], ATTEND[5], ATTEND[8]])
def test_attention_slots_before_heads(lens, H, Hkv, hd, page, dtype, form):
    """Pages laid out [slot][head], with a score cap and with slopes."""
    pages = Pages(len(lens) + 2 * H, lens, Hkv, hd, page, dtype, by_slot=True)
    slopes = (2.0 ** -torch.linspace(1, 8, H)).to(DEV) if form in ("slopes", "all") else None
    check_attention(pages, normal(41, len(lens), H, hd).to(T16[dtype]), torch.tensor(lens, dtype=torch.int32, device=DEV),
                    cap=3.0 if form in ("cap", "all") else 0.0, window=50 if form == "all" else 0, slopes=slopes)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("gap", [12.0, 17.0, 21.0])
def test_attention_many_small_weights_against_a_large_one(dtype, gap):
    """One key with e^gap times the weight of each of 60000 others: together these count, alone each is next to nothing in 16
    bits.  V is 1 at the large one and -1 elsewhere."""
    n, hd = 60000, 64
    pages = Pages(15, [n], 1, hd, 64, dtype, fill=False)
    pages.k.zero_()
    pages.v.fill_(-1.0)
    at = 777
    slot = pages.table[0, at // 64].item(), 0, at % 64
    pages.k[slot][0] = gap
    pages.v[slot] = 1.0
    q = torch.zeros(1, 1, hd, dtype=T16[dtype], device=DEV)
    q[0, 0, 0] = 1.0
    out, lse = kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, torch.tensor([n], dtype=torch.int32, device=DEV), scale=1.0)
    big = math.exp(gap)
    ref = (big - (n - 1)) / (big + (n - 1))
    # half a step of the output; the sums as above; in half, weights below 2^-25 of 2^7 may be off by that, each
    lost = (n * 2.0 ** -32 if dtype == "f16" else 0) + 2.0 ** -17 + 2.0 ** -21 + n * 2.0 ** -24 * 0.01
    assert (out.double() - ref).abs().max() <= torch.finfo(T16[dtype]).eps / 2 * abs(ref) + 2 * lost
    assert abs(lse.item() - math.log(big + n - 1)) < 1e-5


@gpu
def test_attention_caps_and_scales_at_the_ends_of_the_type():
    """The smallest and largest that are taken, on scores of 0 (half of them) and others; smaller and larger ones are refused."""
    pages = Pages(42, [50], 1, 64, 16, "bf16")
    q = normal(43, 1, 2, 64).to(torch.bfloat16)
    q[0, 0] = 0
    n = torch.tensor([50], dtype=torch.int32, device=DEV)
    run = lambda **kw: kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, n, **kw)
    even, _ = run(scale=0.0)
    out, lse = run(score_cap=1.2e-38)                        # every score is next to 0: the mean of the values
    assert torch.equal(out, even) and bool(((lse - math.log(50)).abs() < 1e-5).all())
    out, _ = run(scale=2.3e38)
    assert torch.equal(out[0, 0], even[0, 0])
    for bad in (dict(score_cap=1e-39), dict(score_cap=math.inf), dict(scale=2.4e38), dict(scale=-2.4e38)):
        with pytest.raises(kr.KrakenError) as e:
            run(**bad)
        assert e.value.status == kr.EINVAL
    with pytest.raises(ValueError):
        run(score_cap=1e-60)                                 # no cap at all in 32 bits


@gpu
def test_attention_far_pages_and_streams():
    """Offsets past 2^31 elements, on another stream than the default one, captured into a graph and replayed with other lengths."""
    page, hd, n_pages = 128, 128, 140000
    free, _ = torch.cuda.mem_get_info()
    assert free > 20 << 30
    k = torch.zeros(n_pages, 1, page, hd, dtype=torch.bfloat16, device=DEV)      # 2.3e9 elements
    v = torch.zeros_like(k)
    lens = [1000, 333]
    small = Pages(13, lens, 1, hd, page, "bf16")
    table = torch.zeros(2, 8, dtype=torch.int32, device=DEV)
    for s in range(2):
        for j in range(-(-lens[s] // page)):
            far = n_pages - 1 - 11 * (8 * s + j)
            k[far], v[far] = small.k[small.table[s, j].item()], small.v[small.table[s, j].item()]
            table[s, j] = far
    q = normal(14, 2, 8, hd).to(torch.bfloat16)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(kr.paged_attention_workspace(8, 1, hd), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(q), torch.empty(2, 8, device=DEV)
    with torch.cuda.stream(side):
        kr.op_paged_decode_attention(q, k, v, table, n, out=out, lse=lse, workspace=ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            kr.op_paged_decode_attention(q, k, v, table, n, out=out, lse=lse, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    for now in ([1000, 333], [17, 0], [999, 128], [1000, 333]):
        n.copy_(torch.tensor(now, dtype=torch.int32))
        graph.replay()
        ref, ref_lse, tol, tol_l = attention_ref(small, q, now, [0, 1], hd ** -0.5)
        assert bool(((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() * 1.001 + tol + 2.0 ** -25).all()), now


@gpu
def test_strides_of_dimensions_of_one():
    """A dimension of one may have any stride, an odd one too."""
    pages = Pages(19, [100], 1, 64, 128, "bf16")                    # one page of 128 slots and two spare ones, one head
    q = normal(20, 1, 4, 64).to(torch.bfloat16)
    n = torch.tensor([100], dtype=torch.int32, device=DEV)
    ref = kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, n)
    odd = lambda t: t.as_strided(t.shape, [3 if t.shape[i] == 1 else s for i, s in enumerate(t.stride())])
    got = kr.op_paged_decode_attention(odd(q), odd(pages.k), pages.v, odd(pages.table), n)
    assert torch.equal(ref[0], got[0]) and torch.equal(ref[1], got[1])
    one = pages.k[pages.table[0, 0].item():][:1].clone()
    row = normal(21, 1, 1, 64).to(torch.bfloat16)
    zero = torch.zeros(1, 1, dtype=torch.int32, device=DEV)
    kr.op_paged_append(odd(row), odd(row), odd(one), odd(one.clone()), odd(zero), n - 1)
    assert torch.equal(one[0, 0, 99], row[0, 0])


@gpu
@pytest.mark.parametrize("page", [16, 7])
def test_attention_cache_whose_heads_or_pages_lie_on_one_another(page):
    """Expanded caches, which are only read: one head's keys for all heads, one page for all pages."""
    lens = [200, 1, 90, 3000]
    pages = Pages(44, lens, 1, 64, page, "bf16")
    q = normal(45, 4, 12, 64).to(torch.bfloat16)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    pages.k, pages.v = pages.k.expand(-1, 3, -1, -1), pages.v.expand(-1, 3, -1, -1)
    out, lse = check_attention(pages, q, n)
    again, lse2 = kr.op_paged_decode_attention(q, pages.k.contiguous(), pages.v.contiguous(), pages.table, n)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    one = Pages(46, [page], 2, 64, page, "bf16", spare=0)
    one.k, one.v = one.k.expand(50, -1, -1, -1), one.v.expand(50, -1, -1, -1)
    one.table = torch.arange(50, dtype=torch.int32, device=DEV).view(2, 25)
    check_attention(one, q[:2], torch.tensor([25 * page, 3 * page + 1], dtype=torch.int32, device=DEV))


@gpu
def test_calls_on_two_streams_at_once():
    """Calls that overlap on the device, each with its own workspace, eager and as two graphs replayed side by side."""
    sets = []
    for i, lens in enumerate(([3000, 20, 700], [90, 2500])):
        pages = Pages(16 + i, lens, 2, 128, 16, "bf16")
        q = normal(17 + i, len(lens), 8, 128).to(torch.bfloat16)
        n = torch.tensor(lens, dtype=torch.int32, device=DEV)
        alone = kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, n)
        logits = normal(18 + i, 40, 9000).float()
        sets.append((pages, q, n, alone, logits, kr.op_token_logprobs(logits, top=9), torch.cuda.Stream()))
    torch.cuda.synchronize()

    def run(pages, q, n, logits):
        return kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, n), kr.op_token_logprobs(logits, top=9)

    got, graphs = [[], []], []
    for _ in range(20):
        for i, (pages, q, n, _a, logits, _l, stream) in enumerate(sets):
            with torch.cuda.stream(stream):
                got[i].append(run(pages, q, n, logits))
    torch.cuda.synchronize()
    for i, (pages, q, n, _a, logits, _l, stream) in enumerate(sets):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got[i].append(run(pages, q, n, logits))
        graphs.append(graph)
    for _ in range(20):
        for graph, s in zip(graphs, sets):
            with torch.cuda.stream(s[6]):
                graph.replay()
    torch.cuda.synchronize()
    for i, (_p, _q, _n, alone, _x, read, _s) in enumerate(sets):
        for (out, lse), lp in got[i]:
            assert torch.equal(out, alone[0]) and torch.equal(lse, alone[1])
            assert all(a is b is None or torch.equal(a, b) for a, b in zip(lp, read))


# ---------------------------------------------------------------------------------------------------- append

def turn_ref(x, pos, freq, interleaved):
    x = x.double().clone()
    rot = 0 if freq is None else 2 * freq.numel()
    if not rot:
        return x, torch.zeros_like(x)
    ang = pos.double()[:, None, None] * freq.double()
    c, s = torch.cos(ang), torch.sin(ang)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    na, nb, tol = a * c - b * s, b * c + a * s, torch.zeros_like(x)
    size = 6e-7 * (a.abs() + b.abs())
    if interleaved:
        tol[..., 0:rot:2] = tol[..., 1:rot:2] = size
        x[..., 0:rot:2], x[..., 1:rot:2] = na, nb
    else:
        tol[..., :rot // 2] = tol[..., rot // 2:rot] = size
        x[..., :rot // 2], x[..., rot // 2:rot] = na, nb
    return x, tol


APPEND = [
    # (sequence, first position, tokens) spans, H, Hkv, hd, rot, interleaved, page, dtype
    ([(0, 0, 1)], 1, 1, 64, 64, False, 16, "bf16"),
    ([(0, 13, 9), (1, 0, 1), (2, 99, 30)], 8, 2, 128, 128, False, 16, "bf16"),
    ([(0, 0, 40), (1, 1, 41)], 4, 4, 104, 104, False, 24, "f16"),
    ([(1, 7, 20), (0, 3, 2)], 3, 1, 72, 72, False, 1, "bf16"),
    ([(0, 5, 70)], 6, 3, 96, 40, False, 100, "f16"),
    ([(0, 5, 70)], 6, 3, 96, 48, True, 8, "bf16"),
    ([(0, 1000, 33)], 2, 1, 128, 128, True, 64, "f16"),
    ([(0, 0, 17), (1, 50, 3)], 4, 4, 64, 0, False, 16, "bf16"),
    ([(s, 31 * s, 2 + s % 3) for s in range(400)], 2, 2, 64, 64, False, 16, "f16"),
]


@gpu
@pytest.mark.parametrize("spans,H,Hkv,hd,rot,interleaved,page,dtype", APPEND)
@pytest.mark.parametrize("by_slot", [False, True])
def test_append(spans, H, Hkv, hd, rot, interleaved, page, dtype, by_slot):
    n_seq = max(s for s, _, _ in spans) + 1
    lens = [0] * n_seq
    for s, p0, t in spans:
        lens[s] = p0 + t
    pages = Pages(20, lens, Hkv, hd, page, dtype, by_slot=by_slot, fill=False)
    seq = torch.tensor([s for s, _, t in spans for _ in range(t)] + [-1, -2], dtype=torch.int32, device=DEV)
    pos = torch.tensor([p0 + i for _, p0, t in spans for i in range(t)] + [0, 1 << 30], dtype=torch.int32, device=DEV)
    R = seq.numel()
    qkv = normal(21, R, (H + 2 * Hkv) * hd).to(T16[dtype])
    q, k, v = (x.unflatten(1, (-1, hd)) for x in qkv.split((H * hd, Hkv * hd, Hkv * hd), 1))
    freq = (10000.0 ** -(torch.arange(rot // 2) / (rot / 2))).float().to(DEV) if rot else None
    k0, v0 = pages.k.clone(), pages.v.clone()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.full((R, H, hd), 5.0, dtype=T16[dtype], device=DEV)
    got = kr.op_paged_append(k, v, pages.k, pages.v, pages.table, pos, row_seq=seq, q=q, q_out=out, inv_freq=freq,
                             interleaved=interleaved, status=status)
    assert got is out and int(status.item()) == 0
    half, live = torch.finfo(T16[dtype]).eps / 2, R - 2
    for have, x in ((out[:live], q[:live]), (None, k[:live])):
        ref, tol = turn_ref(x, pos[:live], freq, interleaved)
        if have is None:
            have = pages.k[pages.table[seq[:live].long(), pos[:live] // page].long(), :, pos[:live] % page]
        assert bool(((have.double() - ref).abs() <= half * ref.abs() * 1.001 + tol + 2.0 ** -25).all())
        assert torch.equal(have[..., rot:], x[..., rot:])
    where = (pages.table[seq[:live].long(), pos[:live] // page].long(), slice(None), pos[:live] % page)
    assert torch.equal(pages.v[where], v[:live])
    assert bool((out[live:] == 5).all())
    # nothing else was written: the other slots still hold NaN
    k1, v1 = pages.k.clone(), pages.v.clone()
    k1[where], v1[where] = k0[where], v0[where]
    assert bool(k1.isnan().all()) and bool(v1.isnan().all())
    # in place, and without queries
    inplace = q.clone()
    kr.op_paged_append(k, v, pages.k, pages.v, pages.table, pos, row_seq=seq, q=inplace, q_out=inplace, inv_freq=freq, interleaved=interleaved)
    assert torch.equal(inplace[:live], out[:live])
    kc, vc = pages.k.clone(), pages.v.clone()
    assert kr.op_paged_append(k, v, pages.k, pages.v, pages.table, pos, row_seq=seq, inv_freq=freq, interleaved=interleaved) is None
    assert torch.equal(kc.nan_to_num(), pages.k.nan_to_num()) and torch.equal(vc.nan_to_num(), pages.v.nan_to_num())


@gpu
def test_append_far_positions():
    """Angles of positions near 2^31 keep their accuracy; pages past 2^31 elements."""
    hd, page = 128, 1 << 20
    pages = torch.zeros(20, 1, page, hd, dtype=torch.bfloat16, device=DEV)       # 2.7e9 elements
    table = torch.arange(2048, dtype=torch.int32, device=DEV).remainder_(20).unsqueeze(0)
    pos = torch.tensor([2146435071, 1999999999, 7, (1 << 20) * 19 + 5], dtype=torch.int32, device=DEV)
    zero = torch.zeros(4, dtype=torch.int32, device=DEV)
    k = normal(22, 4, 1, hd).to(torch.bfloat16)
    freq = (10000.0 ** -(torch.arange(64) / 64)).float().to(DEV)
    kr.op_paged_append(k, k, pages, pages.clone(), table[:, :2047], pos, row_seq=zero, inv_freq=freq)
    ref, tol = turn_ref(k, pos, freq, False)
    at = (table[0][pos // page].long(), slice(None), pos % page)
    assert bool(((pages[at].double() - ref).abs() <= 2.0 ** -8 * ref.abs() * 1.001 + tol + 2.0 ** -25).all())


@gpu
def test_append_rows_that_do_not_exist():
    pages = Pages(23, [64, 64], 1, 64, 16, "bf16", fill=False)
    pages.table[1, 2], pages.table[1, 3] = -1, pages.n_pages
    seq = torch.tensor([0, 2, 0, 0, 1, 1, 1 << 30], dtype=torch.int32, device=DEV)
    pos = torch.tensor([3, 3, -1, 64, 33, 60, 0], dtype=torch.int32, device=DEV)
    k = normal(24, 7, 1, 64).to(torch.bfloat16)
    q = torch.full((7, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    out = torch.full_like(q, 8.0)
    for rows, flag in (([0], 0), ([0, 1], 4), ([0, 2], 4), ([0, 3], 4), ([0, 4], 4), ([0, 5], 4), ([0, 6], 4)):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out.fill_(8.0)
        kr.op_paged_append(k[rows], k[rows], pages.k, pages.v, pages.table, pos[rows], row_seq=seq[rows], q=q[rows],
                           q_out=out[:len(rows)], status=status)
        assert int(status.item()) == flag
        assert bool((out[0] == 3).all()) and bool((out[1:] == 8).all())
    assert int((~pages.k.isnan()).sum()) == 64 and int((~pages.v.isnan()).sum()) == 64


# ---------------------------------------------------------------------------------------------------- logits

def check_logprobs(logits, targets, top, scale=1.0, status=None):
    x = logits.double() * scale
    rows, V = logits.shape
    got = kr.op_token_logprobs(logits, targets, top=top, scale=scale, status=status)
    lse = torch.logsumexp(x, -1)
    assert torch.equal(lse.isnan(), got.lse.isnan())
    some = lse.isfinite()
    t = targets.long()
    lp = torch.where(t < 0, 0.0, x.gather(1, t.clamp(min=0)[:, None])[:, 0] - lse)
    p = torch.exp(x - lse[:, None])
    H = torch.special.entr(p).sum(-1)
    tol = (V / 256 + 64) * 2.0 ** -24 + 2.0 ** -20

    def near(a, b, ok):
        a, b = a.double()[ok], b[ok]
        inf = b == -math.inf
        assert torch.equal(a == -math.inf, inf)
        assert bool(((a - b).abs()[~inf] <= tol * (1 + b.abs()[~inf]) + 2.0 ** -21 * x.abs().nan_to_num(0, 0, 0).max()).all()), \
            ((a - b).abs()[~inf].max(), tol)

    near(got.lse, lse, some)
    near(got.logprob, lp, some)
    near(got.entropy, H, some)
    if top:
        raw = logits.float()
        order = torch.where(raw.isnan(), -math.inf, raw).sort(dim=-1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(got.top_ids.long(), order)
        near(got.top_logprobs, x.gather(1, order) - lse[:, None], some)
    else:
        assert got.top_ids is None and got.top_logprobs is None
    return got


SCORES = [(1, 1, 1), (3, 2, 2), (2, 31, 5), (5, 33, 32), (1, 1000, 0), (7, 4097, 20), (300, 257, 3), (2, 50257, 32), (1, 131073, 20),
          (160, 8191, 7), (40, 51200, 20), (700, 5003, 8), (1500, 999, 0), (650, 9001, 9)]


@gpu
@pytest.mark.parametrize("rows,V,top", SCORES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("padded", [0, 3])
def test_logprobs(rows, V, top, dtype, padded):
    x = (normal(rows + V, rows, V + padded) * 3).to(dtype)
    if V > 100:
        x[:, 7::50] = -math.inf
    targets = torch.randint(0, V, (rows,), generator=torch.Generator().manual_seed(V), dtype=torch.int32).to(DEV)
    targets[1::3] = -1
    check_logprobs(x[:, padded:], targets, top, scale=1.0 if top % 2 else 0.7)


@gpu
@pytest.mark.parametrize("V", [40, 1000, 20000, 50257])
@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "two values", "one high", "few finite", "huge", "zeros of both signs"])
def test_logprobs_orders(V, kind):
    i = torch.arange(V, dtype=torch.float64, device=DEV)
    row = {"equal": i * 0 + 2.5, "rising": i / V * 20, "falling": -i / V * 20, "two values": (i % 2), "one high": (i == V // 3) * 80.0,
           "few finite": torch.where(i % (V // 4) == 3, i / V, -math.inf), "huge": (i % 97) * 3e36,
           "zeros of both signs": torch.where(i % 2 == 0, 0.0, -0.0)}[kind]
    x = torch.stack([row, row.flip(0), row])
    targets = torch.tensor([0, V - 1, 3], dtype=torch.int32, device=DEV)
    check_logprobs(x.float(), targets, 32)
    if kind != "huge":
        check_logprobs(x.to(torch.bfloat16), targets, 20)


@gpu
@pytest.mark.parametrize("rows,top", [(200, 32), (1300, 8), (1300, 0), (1300, 20)])
def test_logprobs_many_rows_of_every_order(rows, top):
    """Rows that need the exact way through (rising, of few values, all equal, mostly forbidden) between ordinary ones, in CTAs that
    take several rows."""
    V = 9001
    x = normal(33, rows, V).float()
    i = torch.arange(V, dtype=torch.float32, device=DEV)
    x[1::7] = i / 500
    x[2::7] = (i % 3)
    x[3::7] = 1.25
    x[4::7, 5:] = -math.inf
    x[5::7] = -i / 500
    targets = torch.arange(rows, dtype=torch.int32, device=DEV) % V
    check_logprobs(x, targets, top)
    check_logprobs(x.to(torch.float16), targets, top)


@gpu
def test_logprobs_lowest_values():
    """Masks of the type's lowest value, a row of nothing else (every token equally likely), values at both ends of the type."""
    V = 5000
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        low = torch.finfo(dtype).min
        x = normal(34, 4, V).to(dtype)
        x[0, 100:] = low
        x[1] = low
        x[2, ::2] = -low
        x[2, 1::2] = low
        got = kr.op_token_logprobs(x, torch.tensor([5, 7, 0, 3], dtype=torch.int32, device=DEV), top=3)
        ref = torch.log_softmax(x.double(), -1)
        assert abs(got.logprob[0].item() - ref[0, 5].item()) < 1e-5 and abs(got.logprob[3].item() - ref[3, 3].item()) < 1e-5
        assert abs(got.logprob[1].item() + math.log(V)) < 1e-4 and abs(got.entropy[1].item() - math.log(V)) < 1e-4
        assert abs(got.logprob[2].item() + math.log(V / 2)) < 1e-4 and abs(got.entropy[2].item() - math.log(V / 2)) < 1e-4
        assert got.top_ids[1].tolist() == [0, 1, 2] and got.top_ids[2].tolist() == [0, 2, 4]


@gpu
def test_logprobs_rows_without_a_distribution():
    V = 3001
    x = normal(30, 6, V).float()
    x[1, 17] = math.nan
    x[2, 5] = math.inf
    x[3] = -math.inf
    x[4] = math.nan
    got = kr.op_token_logprobs(x, torch.tensor([3] * 6, dtype=torch.int32, device=DEV), top=4)
    for r in (1, 2, 4):
        assert all(bool(v[r].isnan().all()) for v in (got.lse, got.logprob, got.entropy, got.top_logprobs)), r
    assert got.lse[3].item() == -math.inf and got.logprob[3].isnan() and got.entropy[3].isnan() and bool(got.top_logprobs[3].isnan().all())
    assert got.top_ids[3].tolist() == got.top_ids[4].tolist() == [0, 1, 2, 3] and got.top_ids[2, 0].item() == 5
    order = torch.where(x[1].isnan(), -math.inf, x[1]).sort(descending=True, stable=True).indices[:4]
    assert torch.equal(got.top_ids[1].long(), order)
    keep = [0, 5]
    alone = check_logprobs(x[keep], torch.tensor([3, 3], dtype=torch.int32, device=DEV), 4)
    assert torch.equal(alone.logprob, got.logprob[keep])


@gpu
def test_logprobs_targets_and_rows():
    x = normal(31, 4, 500).float()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = kr.op_token_logprobs(x, torch.tensor([0, 499, -1, -9], dtype=torch.int32, device=DEV), status=status)
    assert int(status.item()) == 0 and got.logprob[2:].tolist() == [0, 0]
    got = kr.op_token_logprobs(x, torch.tensor([0, 499, 500, 1 << 30], dtype=torch.int32, device=DEV), status=status)
    assert int(status.item()) == kr.STATUS_BAD_TOKEN and bool(got.logprob[2:].isnan().all())
    assert kr.op_token_logprobs(x).logprob is None
    same = kr.op_token_logprobs(x[:1].expand(5, 500), top=3)          # rows that lie on one another
    assert bool((same.lse == same.lse[0]).all()) and bool((same.top_ids == same.top_ids[0]).all())
    assert kr.op_token_logprobs(x[:0], top=2).top_ids.shape == (0, 2)


@gpu
def test_logprobs_refusals_take_no_memory():
    x = torch.zeros(64, 1 << 20, device=DEV)
    kr.op_token_logprobs(x, top=1)
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    for top, code in ((1 << 20, kr.EUNSUPPORTED), (33, kr.EUNSUPPORTED), (1 << 21, kr.EINVAL)):
        with pytest.raises(kr.KrakenError) as e:
            kr.op_token_logprobs(x, top=top)
        assert e.value.status == code
    assert torch.cuda.max_memory_allocated() - before < 1 << 16


# ---------------------------------------------------------------------------------------------------- calls nobody wrote down

@gpu
@pytest.mark.parametrize("seed", range(24))
def test_random_attention(seed):
    """Seeded random head layouts, page sizes, lengths, masks and row lists; a call made twice gives the same bits."""
    rng = random.Random(seed)
    hd, Hkv, rep = rng.choice((64, 72, 96, 104, 128)), rng.choice((1, 2, 3, 5, 8)), rng.choice((1, 2, 3, 7, 8, 9, 16, 17, 24, 40))
    page, dtype = rng.choice((1, 2, 3, 7, 8, 16, 24, 40, 64, 100, 128, 512)), rng.choice(("bf16", "f16"))
    B, longest = rng.choice((1, 2, 5, 17, 60)), rng.choice((1, 16, 65, 130, 700, 3000))
    lens = [rng.randint(0, longest) for _ in range(B)]
    pages = Pages(seed, lens, Hkv, hd, page, dtype, by_slot=rng.random() < 0.5, width=max(1, -(-max(lens) // page)) + rng.choice((0, 0, 5, 400)))
    R = rng.choice((B, B, 2 * B + 1))
    seq = torch.tensor([rng.randrange(B) if rng.random() < 0.9 else -1 for _ in range(R)], dtype=torch.int32, device=DEV)
    n = torch.tensor([rng.randint(0, lens[s]) if s >= 0 else -5 for s in seq.tolist()], dtype=torch.int32, device=DEV)
    q = (normal(seed, R, Hkv * rep, hd) * rng.choice((0.1, 1, 4))).to(T16[dtype])
    slopes = (torch.rand(Hkv * rep, generator=torch.Generator().manual_seed(seed)) * 0.2).to(DEV) if rng.random() < 0.3 else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    form = dict(score_cap=rng.choice((0.0, 0.0, 5.0)), window=rng.choice((0, 0, 1, 15, 16, 17, 100)), slopes=slopes, scale=rng.choice((None, 0.3)))
    out, lse = torch.full_like(q, 3.0), torch.full((R, Hkv * rep), 3.0, device=DEV)
    check_attention(pages, q, n, row_seq=seq, status=status, out=out, lse=lse, cap=form["score_cap"], window=form["window"], slopes=slopes,
                    scale=form["scale"])
    assert int(status.item()) == 0 and bool((out[seq < 0] == 3).all()) and bool((lse[seq < 0] == 3).all())
    again, lse2 = kr.op_paged_decode_attention(q, pages.k, pages.v, pages.table, n, row_seq=seq, **form)
    assert torch.equal(again[seq >= 0], out[seq >= 0]) and torch.equal(lse2[seq >= 0], lse[seq >= 0])


@gpu
@pytest.mark.parametrize("seed", range(12))
def test_random_append(seed):
    rng = random.Random(seed)
    hd, Hkv = rng.choice((64, 72, 96, 104, 128)), rng.choice((1, 2, 3, 8, 17))
    H, page, dtype = Hkv * rng.choice((1, 2, 5)), rng.choice((1, 5, 8, 16, 24, 100, 256)), rng.choice(("bf16", "f16"))
    rot = rng.choice([r for r in (0, 8, 16, 24, 40, 64, 72, 104, 120, hd) if r <= hd])
    B = rng.choice((1, 3, 40))
    spans = [(s, rng.randint(0, 300), rng.choice((1, 1, 7, 90))) for s in range(B)]
    if seed % 3 == 0:
        spans[0] = (0, 11, 900)              # many rows
    test_append(spans, H, Hkv, hd, rot, rng.random() < 0.5, page, dtype, rng.random() < 0.5)


@gpu
@pytest.mark.parametrize("seed", range(24))
def test_random_logprobs(seed):
    rng, g = random.Random(seed), torch.Generator().manual_seed(seed)
    V = rng.choice((1, 5, 33, 100, 1000, 4095, 4096, 4097, 8200, 16385, 50257))
    rows = min(rng.choice((1, 1, 2, 5, 30, 149, 297, 700, 1300)), max(1, 4000000 // V))
    dtype, top, pad = rng.choice((torch.float32, torch.bfloat16, torch.float16)), min(V, rng.choice((0, 1, 3, 8, 9, 20, 32))), rng.choice((0, 1, 3, 8))
    x = torch.randn(rows, V + pad, generator=g) * rng.choice((0.0, 0.1, 3, 20))
    if rng.random() < 0.5:
        x[torch.rand(x.shape, generator=g) < rng.choice((0.01, 0.5, 0.99))] = -math.inf
    x[:, pad] = rng.choice((0.0, 1.0, 50.0))
    check_logprobs(x.to(dtype).to(DEV)[:, pad:], torch.randint(-1, V, (rows,), generator=g, dtype=torch.int32).to(DEV), top, scale=rng.choice((1.0, 0.3, 2.0)))


# ---------------------------------------------------------------------------------------------------- together

@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_serving_steps(dtype):
    """Prompts into pages, decode steps (append, attend), logits of the result, their reading: as a server runs them, the
    decode steps as a captured graph whose positions advance on the device; the last step against 64 bits."""
    H, Hkv, hd, page, V = 8, 2, 64, 16, 1000
    prompts, steps = [37, 1, 100], 20
    pages = Pages(40, [p + steps for p in prompts], Hkv, hd, page, dtype, fill=False)
    freq = (10000.0 ** -(torch.arange(hd // 2) / (hd / 2))).float().to(DEV)
    keys = [normal(41 + s, p + steps, Hkv, hd).to(T16[dtype]) for s, p in enumerate(prompts)]
    vals = [normal(51 + s, p + steps, Hkv, hd).to(T16[dtype]) for s, p in enumerate(prompts)]
    q_all = normal(61, steps, 3, H, hd).to(T16[dtype])
    w = (normal(62, V, H * hd) * 0.1).to(T16[dtype])
    seq = torch.tensor([s for s, p in enumerate(prompts) for _ in range(p)], dtype=torch.int32, device=DEV)
    pos = torch.tensor([i for p in prompts for i in range(p)], dtype=torch.int32, device=DEV)
    kr.op_paged_append(torch.cat([k[:p] for k, p in zip(keys, prompts)]), torch.cat([v[:p] for v, p in zip(vals, prompts)]), pages.k,
                       pages.v, pages.table, pos, row_seq=seq, inv_freq=freq)
    at = torch.tensor(prompts, dtype=torch.int32, device=DEV)
    n, k, v, q = at + 1, *(torch.zeros(3, h, hd, dtype=T16[dtype], device=DEV) for h in (Hkv, Hkv, H))
    logits = torch.zeros(3, V, device=DEV)
    out = {}

    def step():
        qr = kr.op_paged_append(k, v, pages.k, pages.v, pages.table, at, q=q, inv_freq=freq)
        o, lse = kr.op_paged_decode_attention(qr, pages.k, pages.v, pages.table, n)
        with kr.storage_dtype(dtype):
            g = kr.GemmArgs(a=o.data_ptr(), lda=H * hd, w=w.data_ptr(), ldw=H * hd, groups=1, m=3, n_out=V, k=H * hd,
                            epilogue=kr.EPI_F32, out_f32=logits.data_ptr(), ld_out_f32=V, n_tile=8)
            kr.op_grouped_gemm(g)
        out.update(o=o, q=qr, lp=kr.op_token_logprobs(logits, top=5))
        at.add_(1)
        n.add_(1)

    def load(i):
        for s, p in enumerate(prompts):
            k[s], v[s], q[s] = keys[s][p + i], vals[s][p + i], q_all[i, s]

    load(0)
    step()
    graph = torch.cuda.CUDAGraph()
    load(1)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(1, steps):
        load(i)
        graph.replay()
    for s, p in enumerate(prompts):
        every = torch.arange(p + steps, device=DEV)
        kt, tol = turn_ref(keys[s], every, freq, False)
        assert bool(((pages.get(pages.k, s, 0, p + steps) - kt).abs() <= torch.finfo(T16[dtype]).eps / 2 * kt.abs() * 1.001 + tol + 2.0 ** -25).all())
        assert torch.equal(pages.get(pages.v, s, 0, p + steps), vals[s].double())
    last = torch.tensor([p + steps for p in prompts])
    ref, _, tol, _ = attention_ref(pages, out["q"], last.tolist(), [0, 1, 2], hd ** -0.5)
    half = torch.finfo(T16[dtype]).eps / 2
    assert bool(((out["o"].double() - ref).abs() <= half * ref.abs() * 1.001 + tol + 2.0 ** -25).all())
    x = out["o"].double().flatten(1) @ w.double().T
    assert (logits.double() - x).abs().max() < H * hd * 2.0 ** -24 * (out["o"].double().flatten(1).abs() @ w.double().abs().T).max()
    assert torch.equal(out["lp"].top_ids.long(), logits.sort(dim=-1, descending=True, stable=True).indices[:, :5])


@gpu
def test_pages_of_a_models_cache_and_its_score():
    """A model's cache copied into pages gives the contiguous cache's decode attention; score() reads the model's logits."""
    s = ki.CONFIGS["C0"]
    model = kr.KrakenModel(kr.make_config(s), ki.make_weights(s, 0, DEV), DEV)
    L = 100
    tok = ki.uniform_tokens(1, s.vocab, 1, L, DEV)
    model.prefill(tok)
    H, hd = s.n_head, s.head_dim
    kc, vc = model.kv_view(0, 1, 0)[:, :, :L], model.kv_view(0, 1, 1)[:, :, :L]
    pages = Pages(70, [L], H, hd, 16, "bf16", fill=False)
    where = torch.arange(L, dtype=torch.int32, device=DEV)
    kr.op_paged_append(kc[0].transpose(0, 1), vc[0].transpose(0, 1), pages.k, pages.v, pages.table, where, row_seq=torch.zeros_like(where))
    assert torch.equal(pages.get(pages.k, 0, 0, L), kc[0].transpose(0, 1).double())
    q = normal(71, 1, H, hd).to(torch.bfloat16)
    n = torch.tensor([L], dtype=torch.int32, device=DEV)
    out, _ = check_attention(pages, q, n)
    other = kr.op_decode_attention(q.view(1, 1, H * hd), model.kv_view(0, 1, 0)[None], model.kv_view(0, 1, 1)[None], L)
    assert (other.view(1, H, hd) - out).abs().max() <= 2.0 ** -7 * out.abs().max()
    got = model.score(tok, top=3)
    logits = model.prefill_all_logits(tok)[0]
    ref = torch.log_softmax(logits.double(), -1)
    assert (got.logprob[:-1].double() - ref[:-1].gather(1, tok[0, 1:, None].long())[:, 0]).abs().max() < 1e-4 and got.logprob[-1] == 0
    assert torch.equal(got.top_ids.long(), logits.sort(dim=-1, descending=True, stable=True).indices[:, :3])
    model.close()


# ---------------------------------------------------------------------------------------------------- refusals (no GPU)

def cache_args(**over):
    f = dict(k=1 << 20, v=1 << 21, page_table=1 << 22, page_stride=2048, head_stride=1024, slot_stride=64, table_stride=4, n_pages=8,
             page_size=16, n_kv_head=2, head_dim=64, n_seqs=3, max_pages=4)
    f.update(over)
    return kr.PagedCacheArgs(**f)


CACHE_REFUSALS = [
    (dict(k=None), kr.EINVAL), (dict(v=None), kr.EINVAL), (dict(page_table=None), kr.EINVAL), (dict(n_pages=0), kr.EINVAL),
    (dict(page_size=0), kr.EINVAL), (dict(n_kv_head=0), kr.EINVAL), (dict(n_seqs=0), kr.EINVAL), (dict(max_pages=0), kr.EINVAL),
    (dict(table_stride=3), kr.EINVAL), (dict(page_stride=-8), kr.EINVAL), (dict(max_pages=1 << 20, table_stride=1 << 20, page_size=1 << 12), kr.EINVAL),
    (dict(head_dim=80), kr.EUNSUPPORTED), (dict(k=(1 << 20) + 8), kr.EUNSUPPORTED), (dict(v=(1 << 20) + 2), kr.EUNSUPPORTED),
    (dict(page_stride=2044), kr.EUNSUPPORTED), (dict(head_stride=1020), kr.EUNSUPPORTED), (dict(slot_stride=66), kr.EUNSUPPORTED),
]


def append_args(**over):
    f = dict(k=1 << 20, v=1 << 20, k_row_stride=128, k_head_stride=64, v_row_stride=128, v_head_stride=64, q=1 << 20, q_row_stride=128,
             q_head_stride=64, q_out=1 << 20, q_out_row_stride=128, q_out_head_stride=64, row_seq=1 << 20, row_pos=1 << 20,
             inv_freq=1 << 20, rows=2, n_head=4, rot_dim=64)
    f.update(over)
    return kr.PagedAppendArgs(**f)


def attention_args(**over):
    f = dict(q=1 << 20, q_row_stride=256, q_head_stride=64, out=1 << 20, out_row_stride=256, out_head_stride=64, n_keys=1 << 20,
             row_seq=1 << 20, workspace=1 << 20, workspace_bytes=1 << 30, scale=0.125, rows=2, n_head=4)
    f.update(over)
    return kr.PagedAttentionArgs(**f)


def logprob_args(**over):
    f = dict(logits=1 << 20, row_stride=100, targets=1 << 20, logprob=1 << 20, entropy=1 << 20, lse=1 << 20, top_ids=1 << 20,
             top_logprobs=1 << 20, rows=2, vocab=100, dtype=0, top=5, scale=1.0)
    f.update(over)
    return kr.LogprobsArgs(**f)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_refusals_before_the_device_is_touched(dtype):
    L = kr.lib(dtype)

    def append(c, a):
        return L.kraken_op_paged_append(c and C.byref(c), a and C.byref(a), None, None)

    def attend(c, a):
        return L.kraken_op_paged_attention(c and C.byref(c), a and C.byref(a), None, None)

    def score(a):
        return L.kraken_op_token_logprobs(a and C.byref(a), None, None)

    for over, code in CACHE_REFUSALS:
        assert append(cache_args(**over), append_args()) == code, over
        assert attend(cache_args(**over), attention_args()) == code, over
    assert append(None, append_args()) == append(cache_args(), None) == kr.EINVAL
    assert attend(None, attention_args()) == attend(cache_args(), None) == score(None) == kr.EINVAL
    for over, code in [(dict(rows=-1), kr.EINVAL), (dict(k=None), kr.EINVAL), (dict(v=None), kr.EINVAL), (dict(row_pos=None), kr.EINVAL),
                       (dict(inv_freq=None), kr.EINVAL), (dict(q_out=None), kr.EINVAL), (dict(n_head=0), kr.EINVAL),
                       (dict(row_seq=None, rows=4), kr.EINVAL), (dict(rot_dim=-8), kr.EINVAL), (dict(rot_dim=12), kr.EUNSUPPORTED),
                       (dict(rot_dim=72), kr.EUNSUPPORTED), (dict(k=(1 << 20) + 4), kr.EUNSUPPORTED), (dict(v_row_stride=65), kr.EUNSUPPORTED),
                       (dict(q=(1 << 20) + 8), kr.EUNSUPPORTED), (dict(q_out_head_stride=4), kr.EUNSUPPORTED),
                       (dict(q_out_row_stride=0), kr.EINVAL), (dict(q_out_head_stride=0), kr.EINVAL)]:
        assert append(cache_args(), append_args(**over)) == code, over
    for over in (dict(page_stride=0), dict(head_stride=0), dict(slot_stride=0)):      # nothing to write to twice
        assert append(cache_args(**over), append_args()) == kr.EINVAL, over
    assert append(cache_args(), append_args(rows=0)) == kr.OK
    for over, code in [(dict(rows=-1), kr.EINVAL), (dict(q=None), kr.EINVAL), (dict(out=None), kr.EINVAL), (dict(n_keys=None), kr.EINVAL),
                       (dict(n_head=3), kr.EINVAL), (dict(n_head=0), kr.EINVAL), (dict(window=-1), kr.EINVAL), (dict(scale=math.nan), kr.EINVAL),
                       (dict(score_cap=-1.0), kr.EINVAL), (dict(score_cap=math.inf), kr.EINVAL), (dict(row_seq=None, rows=4), kr.EINVAL),
                       (dict(out_row_stride=0), kr.EINVAL), (dict(out_head_stride=0), kr.EINVAL), (dict(lse=1 << 20), kr.EINVAL),
                       (dict(workspace=None), kr.ECAPACITY), (dict(workspace_bytes=1000), kr.ECAPACITY), (dict(workspace=(1 << 20) + 8), kr.EINVAL),
                       (dict(q=(1 << 20) + 2), kr.EUNSUPPORTED), (dict(out_row_stride=252), kr.EUNSUPPORTED)]:
        assert attend(cache_args(), attention_args(**over)) == code, over
    assert attend(cache_args(), attention_args(rows=0)) == kr.OK
    for over, code in [(dict(rows=-1), kr.EINVAL), (dict(logits=None), kr.EINVAL), (dict(vocab=0), kr.EINVAL), (dict(row_stride=-1), kr.EINVAL),
                       (dict(dtype=2), kr.EINVAL), (dict(top=-1), kr.EINVAL), (dict(top=6, vocab=5), kr.EINVAL), (dict(scale=0.0), kr.EINVAL),
                       (dict(scale=math.inf), kr.EINVAL), (dict(targets=None), kr.EINVAL), (dict(top_ids=None, top_logprobs=None), kr.EINVAL),
                       (dict(top=33), kr.EUNSUPPORTED), (dict(logits=(1 << 20) + 2), kr.EUNSUPPORTED)]:
        assert score(logprob_args(**over)) == code, over
    assert score(logprob_args(rows=0)) == kr.OK
    n = C.c_size_t(0)
    assert L.kraken_paged_attention_workspace(4, 2, 64, None) == kr.EINVAL
    assert L.kraken_paged_attention_workspace(4, 3, 64, C.byref(n)) == kr.EINVAL
    assert L.kraken_paged_attention_workspace(4, 2, 80, C.byref(n)) == kr.EUNSUPPORTED


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scales_and_caps_that_leave_the_type_are_refused(dtype):
    """scale * log2(e) and 1 / score_cap are taken in 32 bits: where one of them is infinite, a score of 0 became NaN."""
    L = kr.lib(dtype)
    for over in (dict(score_cap=1e-39), dict(score_cap=1e-45), dict(scale=2.4e38), dict(scale=-3.4e38)):
        a = attention_args(**over)
        assert L.kraken_op_paged_attention(C.byref(cache_args()), C.byref(a), None, None) == kr.EINVAL, over
    assert L.kraken_op_token_logprobs(C.byref(logprob_args(scale=2.4e38)), None, None) == kr.EINVAL


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attention_more_rows_than_its_counters_hold_are_refused(dtype):
    """Tiles and rows are added up in one 64-bit number, 40 and 23 bits of it."""
    L = kr.lib(dtype)
    wide = dict(max_pages=1 << 15, table_stride=1 << 15, page_size=1 << 15, slot_stride=64, head_stride=1 << 21, page_stride=1 << 22)
    for cache, rows in ((cache_args(), 1 << 23), (cache_args(), (1 << 31) - 1), (cache_args(**wide), 1 << 16)):
        a = attention_args(rows=rows)
        assert L.kraken_op_paged_attention(C.byref(cache), C.byref(a), None, None) == kr.EUNSUPPORTED, rows
    # one row less is taken, as far as its workspace
    a = attention_args(rows=(1 << 23) - 1, workspace_bytes=0)
    assert L.kraken_op_paged_attention(C.byref(cache_args()), C.byref(a), None, None) == kr.ECAPACITY


def test_struct_sizes():
    assert C.sizeof(kr.PagedCacheArgs) == 7 * 8 + 6 * 4
    assert C.sizeof(kr.PagedAppendArgs) == 15 * 8 + 4 * 4
    assert C.sizeof(kr.PagedAttentionArgs) == 13 * 8 + 2 * 4 + 3 * 4 + 4
    assert C.sizeof(kr.LogprobsArgs) == 8 * 8 + 5 * 4 + 4


def test_wrappers_refuse_what_does_not_fit():
    """The binding's own checks come before any call (CPU tensors are refused)."""
    z = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    cache = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table, pos = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        kr.op_paged_append(z, z, cache, cache, table, pos)
    with pytest.raises(ValueError):
        kr.op_paged_decode_attention(z, cache, cache, table, pos)
    with pytest.raises(ValueError):
        kr.op_token_logprobs(torch.zeros(2, 5))


@gpu
def test_wrappers_refuse_on_the_device():
    z = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device=DEV)
    cache = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
    table, pos = torch.zeros(2, 2, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    for bad in (dict(k=z[:, :1]), dict(k=z[..., :32]), dict(k=z.half()), dict(v=z[:1]), dict(v_cache=cache[:3]), dict(page_table=table.long()),
                dict(positions=pos.long()), dict(positions=pos[:1]), dict(positions=None), dict(row_seq=pos[:1]), dict(q=z[:1]),
                dict(q=z, q_out=z[:1]), dict(inv_freq=torch.zeros(32, dtype=torch.float64, device=DEV)), dict(k=z.transpose(0, 2).contiguous().transpose(0, 2)),
                dict(status=torch.zeros(1)), dict(positions=pos.cpu())):
        with pytest.raises(ValueError):
            kr.op_paged_append(**{**dict(k=z, v=z, k_cache=cache, v_cache=cache, page_table=table, positions=pos), **bad})
    for bad in (dict(q=z[..., :32]), dict(n_keys=pos.long()), dict(n_keys=None), dict(out=z[:1]), dict(lse=torch.zeros(2, 3, device=DEV)),
                dict(slopes=torch.zeros(3, device=DEV)), dict(row_seq=pos.cpu())):
        with pytest.raises(ValueError):
            kr.op_paged_decode_attention(**{**dict(q=z, k_cache=cache, v_cache=cache, page_table=table, n_keys=pos), **bad})
    with pytest.raises(kr.KrakenError) as e:
        kr.op_paged_decode_attention(z[:, :1], cache, cache, table, pos)       # one query head, two key/value heads
    assert e.value.status == kr.EINVAL
    x = torch.zeros(2, 50, device=DEV)
    for bad in (dict(logits=x.double()), dict(logits=x.T), dict(targets=pos.long()), dict(targets=pos[:1])):
        with pytest.raises(ValueError):
            kr.op_token_logprobs(**{**dict(logits=x), **bad})
    with pytest.raises(kr.KrakenError) as e:
        kr.op_token_logprobs(x, top=40)
    assert e.value.status == kr.EUNSUPPORTED

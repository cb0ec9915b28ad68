"""Attention of chunks over pages: what a row's result may depend on, to the last bit, and scores at the ends of their range.

A row's result follows from its own query, the keys and values that it sees, and how the call's lengths cut the work.  So calls that
differ in anything else are compared bit for bit; the others against 64 bits with the tolerances of test_paged_chunk.
"""
import ctypes as C
import math

import pytest
import torch

import paper_2408_07802_b200 as kr
from test_paged_chunk import cache_args, check_chunk, chunk_args, int32
from test_paged_ops import DEV, T16, Pages, normal

gpu = pytest.mark.gpu


def starts_of(spans, first=0):
    starts = [first]
    for _, n in spans:
        starts.append(starts[-1] + n)
    return starts


@gpu
@pytest.mark.parametrize("H,Hkv,hd,dtype,window", [(8, 2, 128, "bf16", 0), (4, 4, 64, "f16", 0), (16, 2, 104, "bf16", 333)])
def test_copies_by_lanes_give_the_same_bits(H, Hkv, hd, dtype, window):
    """Pages of 100 slots go by the lanes' copies, pages of 16 by the copy engine; the tiles are the same."""
    spans = [(1500, 300), (700, 700), (0, 513), (90, 1), (1, 2), (640, 128)]
    lens, starts = [p + n for p, n in spans], starts_of(spans)
    q = normal(5, starts[-1], H, hd).to(T16[dtype])
    got = []
    for page in (16, 100, 1):
        pages = Pages(40, lens, Hkv, hd, page, dtype)
        for _ in range(2):
            status = torch.zeros(1, dtype=torch.int32, device=DEV)
            got.append(kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, int32(starts), int32(lens), window=window, status=status))
            assert int(status) == 0
    for out, lse in got[1:]:
        assert bool((out == got[0][0]).all()) and bool((lse == got[0][1]).all())


@gpu
def test_chunks_on_one_another_beyond_all_counting():
    """q_start that goes back and forth over all rows: every second chunk is one that exists, and all of them together have more than
    2^32 tiles.  Nothing is done, and the status word says so."""
    rows, keys, page, chunks = 1 << 17, 1 << 18, 256, 1 << 14
    q = torch.zeros(rows, 1, 64, dtype=torch.bfloat16, device=DEV)
    k = torch.zeros(1, 1, page, 64, dtype=torch.bfloat16, device=DEV)
    table = torch.zeros(1, keys // page, dtype=torch.int32, device=DEV)
    pairs, tiles = rows // 256, (keys - rows // 2) // 128
    assert chunks // 2 * pairs * tiles > 2 ** 32
    starts = torch.zeros(chunks + 1, dtype=torch.int32, device=DEV)
    starts[1::2] = rows
    out, lse = torch.full_like(q, 7.0), torch.full((rows, 1), 7.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    zeros = torch.zeros(chunks, dtype=torch.int32, device=DEV)
    kr.op_paged_chunk_attention(q, k, k, table, starts, torch.full_like(zeros, keys), chunk_seq=zeros, out=out, lse=lse, status=status)
    assert int(status) == kr.STATUS_BAD_PAGE
    assert bool((out == 7).all()) and bool((lse == 7).all())
    # one that goes back once: the chunk with the rows from 20 to 10 does not exist, the others do
    status.zero_()
    kr.op_paged_chunk_attention(q[:30], k, k, table, int32([0, 20, 10, 30]), int32([40, 40, 40]), chunk_seq=int32([0, 0, 0]), out=out[:30],
                                lse=lse[:30], status=status)
    assert int(status) == kr.STATUS_BAD_PAGE and bool((out[:30] == 0).all()) and bool((out[30:] == 7).all())


def call(pages, q, starts, lens, **kw):
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    kr.op_paged_chunk_attention(q, pages.k, pages.v, pages.table, int32(starts), int32(lens), out=out, lse=lse, **kw)
    return out, lse


# ------------------------------------------------------------------ a row and what is none of its business

def leave_in_shared_memory(value, dtype):
    """A call with 4 query heads a key/value head fills all rows of its query tiles, on every SM."""
    pages = Pages(41, [128], 1, 128, 16, dtype, fill=False)
    pages.k[:], pages.v[:] = 1.0, 1.0
    q = torch.full((148 * 64, 4, 128), value, dtype=T16[dtype], device=DEV)
    call(pages, q, [64 * i for i in range(149)], [128] * 148, chunk_seq=int32([0] * 148))


@gpu
@pytest.mark.parametrize("cap,scale", [(0.0, None), (30.0, 0.125), (4.0, 0.125)])
@pytest.mark.parametrize("H,Hkv,hd,page,dtype", [(3, 1, 64, 16, "bf16"), (10, 2, 128, 16, "f16"), (65, 1, 64, 16, "bf16"), (4, 1, 128, 16, "bf16"),
                                                 (6, 2, 72, 100, "bf16"), (7, 1, 128, 100, "f16")])
def test_a_row_follows_from_what_it_sees_alone(H, Hkv, hd, page, dtype, cap, scale):
    """The same to the last bit whatever the other chunks' queries, padding rows, slots behind the sequences, keys and values behind
    a token and what an earlier call left in shared memory: also where these would choose another way to the same number."""
    spans, big = [(200, 50), (90, 40)], 1e30 if dtype == "bf16" else 6e4
    lens, starts = [p + n for p, n in spans], starts_of(spans, 3)
    kw = dict(score_cap=cap, scale=scale)
    pages = Pages(42, lens, Hkv, hd, page, dtype)
    q = normal(6, starts[-1] + 20, H, hd).to(T16[dtype])
    leave_in_shared_memory(0.0, dtype)
    out, lse = call(pages, q, starts, lens, **kw)
    mine = slice(starts[0], starts[1])
    same = lambda got, rows: bool((got[0][rows] == out[rows]).all()) and bool((got[1][rows] == lse[rows]).all())  # noqa: E731
    for value in (1.0, big, math.inf, math.nan):
        leave_in_shared_memory(value, dtype)
        assert same(call(pages, q, starts, lens, **kw), slice(None)), value
    for factor in (0.0, 300.0, big):
        other = q.clone()
        other[starts[1]:] = (other[starts[1]:].float() * factor).to(q.dtype)
        other[:starts[0]] = other[starts[2]:] = big
        assert same(call(pages, other, starts, lens, **kw), mine), factor
    for value in (0.0, 500.0, big):
        for cache in (pages.k, pages.v):
            cache.nan_to_num_(nan=value)
        assert same(call(pages, q, starts, lens, **kw), slice(None)), value
    # the last token's key, which no other row sees
    pages = Pages(42, lens, Hkv, hd, page, dtype)
    for value in (500.0, big, math.nan):
        pages.k[pages.table[0, (lens[0] - 1) // page].item(), :, (lens[0] - 1) % page] = value
        assert same(call(pages, q, starts, lens, **kw), slice(starts[0], starts[1] - 1)), value


# ------------------------------------------------------------------ scores that come near their cap

@gpu
@pytest.mark.parametrize("cap,size", [(15.0, 8.0), (15.0, 40.0), (50.0, 20.0), (0.7, 1.0)])
@pytest.mark.parametrize("H,Hkv,hd,page,dtype", [(3, 1, 64, 16, "bf16"), (8, 2, 128, 64, "f16"), (4, 4, 104, 100, "bf16")])
def test_scores_near_the_cap(H, Hkv, hd, page, dtype, cap, size):
    """Scores with a deviation of `size`; every third token's are a hundredth of that, so that small and large rows share a warp."""
    spans = [(300, 90), (0, 130), (700, 1)]
    lens, starts = [p + n for p, n in spans], starts_of(spans)
    pages = Pages(43, lens, Hkv, hd, page, dtype)
    q = normal(7, starts[-1], H, hd) * size
    q[::3] *= 0.01
    slopes = torch.linspace(0.5, 0.01, H, device=DEV) if size == 20.0 else None
    check_chunk(pages, q.to(T16[dtype]), starts, lens, cap=cap, slopes=slopes, window=200 if size == 40.0 else 0)


@gpu
@pytest.mark.parametrize("page", [16, 100])
@pytest.mark.parametrize("scale,cap", [(1e15, 1e-18), (1.0, 1e-5), (1.0, 1e-38), (1e-30, 1e8), (0.125, 1e30), (0.125, 3e38), (-1e15, 1e-15)])
@pytest.mark.parametrize("size", [0.0, 1.0])
def test_scale_and_cap_far_apart(scale, cap, size, page):
    """Each of the two fits 32 bits; their quotient, or its powers, need not.  Scores of at most `cap` (and of 0 for queries of 0)
    leave all keys the same weight, or are those without a cap where that is far away."""
    n, new = 200, 40
    pages = Pages(44, [n], 1, 64, page, "bf16")
    q = (normal(8, new, 3, 64) * size).to(torch.bfloat16)
    out, lse = call(pages, q, [0, new], [n], scale=scale, score_cap=cap)
    if cap < 1 or scale < 1e-20 or size == 0:
        v = pages.get(pages.v, 0, 0, n)[:, 0]
        for i in range(new):
            seen = n - new + 1 + i
            # weights of e^(+-1e-5) at most, rounded to 16 bits; half a step of the output; sums over 200 keys
            assert bool(((out[i].double() - v[:seen].mean(0)).abs() <= 2.0 ** -8 * (v[:seen].abs().mean(0) + v[:seen].mean(0).abs()) + 3e-5).all())
            assert bool(((lse[i].double() - math.log(seen)).abs() <= 3e-5).all())
    else:
        want, want_lse = call(pages, q, [0, new], [n], scale=scale)
        assert (out.float() - want.float()).abs().max() <= 2.0 ** -6 and (lse - want_lse).abs().max() <= 1e-5


@gpu
@pytest.mark.parametrize("page", [16, 100])
@pytest.mark.parametrize("cap,size", [(1e6, 8e4), (1e4, 800.0), (3e-3, 4e-4)])
def test_caps_of_every_size(cap, size, page):
    """Scores up to about a third of a cap that is large or small."""
    pages = Pages(45, [333, 64], 2, 64, page, "bf16")
    q = (normal(9, 80, 4, 64) * size).to(torch.bfloat16)
    check_chunk(pages, q, [0, 60, 80], [333, 64], cap=cap)


@pytest.mark.parametrize("scale,cap,code", [(1e20, 1e-20, kr.EINVAL), (-1e20, 1e-20, kr.EINVAL), (2.0, 1e-38, kr.EINVAL), (1e20, 1e-45, kr.EINVAL),
                                            (2e38, 1.0, kr.EINVAL), (1e20, 1e-17, kr.ECAPACITY), (0.0, 1e-38, kr.ECAPACITY), (1e-38, 3e38, kr.ECAPACITY)])
def test_scale_over_cap_refusals(scale, cap, code):
    """Too far apart for 32 bits: refused; the others are taken (and then refused for want of a workspace)."""
    args = chunk_args(scale=scale, score_cap=cap, workspace=None)
    assert kr.lib().kraken_op_paged_chunk_attention(C.byref(cache_args()), C.byref(args), None, None) == code

"""Attention of chunks over pages: what a row's result may depend on, to the last bit, and scores at the ends of their range.

A row's result follows from its own query, the keys and values that it sees, and how the call's lengths cut the work.  So calls that
differ in anything else are compared bit for bit; the others against 64 bits with the tolerances of test_paged_chunk.
"""
import math

import pytest
import torch

import paper_2408_07802_b200 as kr
from test_paged_chunk import check_chunk, int32
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

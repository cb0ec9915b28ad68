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

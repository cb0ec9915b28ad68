"""Drawing tokens: rows that CTAs share, rows with few tokens left, weights between the windows, temperatures at the ends of fp32.

What is compared exactly (ids of a temperature of 0, of rows with one answer) has no tolerance; the others derive theirs beside
the comparison.
"""
import math

import pytest
import torch

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

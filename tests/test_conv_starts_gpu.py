"""Sequences of a packed convolution in any order and with gaps: `starts` that
descend (an end before its begin is an empty sequence), as zeros behind the last
sequence of a padded batch do."""
import numpy as np
import pytest
import torch

import oracle
from layer_testutil import check
from paper_2608_02560_amd import precog as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BAR = 2.0 ** -19  # as test_conv_gpu.py derives it


@pytest.mark.parametrize("T,starts", [
    (40, [0, 10, 30] + [0] * 6),                # zeros behind the last sequence
    (40, [0, 10, 30] + [-1] * 6),
    (300, [0, 100, 300] + [0] * 130),           # more entries than a wave has lanes
    (40, [30, 10, 40]),                         # an empty one, then tokens behind and before its begin
    (90, [50, 90, 0, 50]),                      # the later tokens first
    (200, [150, 200, 100, 130, 0, 100]),
    (70, [70, 70, 0, 0, 70, 5]),                # empty ones on all sides of the whole axis
    (64, [64, 20, 21, 22, 5, 6, 20]),           # rows in no sequence between them
    (33, [33, 0, 33, 0]),
    (40, [100, 7, 1000]),                       # clamped
    (50, [20])])
@pytest.mark.parametrize("in_place", [False, True])
def test_any_order(T, starts, in_place):
    D, W, B = 520, 4, len(starts) - 1
    gen = torch.Generator().manual_seed(T)
    x, w = torch.randn((T, D), generator=gen).bfloat16(), torch.randn((D, W), generator=gen) * 0.5
    tails = torch.randn((B, W - 1, D), generator=gen).bfloat16()
    y = torch.full((T, D), 9.0, device=DEV)
    tail0 = tails.to(DEV)
    tailT = tail0 if in_place else torch.full_like(tail0, 5.0)
    P.conv_encode(P.conv_desc(B, T, D, W, P.BF16, P.F32), x.to(DEV), w.to(DEV), None,
                  torch.tensor(starts, dtype=torch.int32, device=DEV), tail0=tail0, y=y, tailT=tailT)
    ry, at = np.full((T, D), 9.0), np.clip(starts, 0, T)
    for b in range(B):
        n = max(at[b + 1] - at[b], 0)
        ry[at[b]:at[b] + n], rt = oracle.conv(x[at[b]:at[b] + n], w, None, tails[b])
        assert torch.equal(tailT[b].cpu().double(), torch.tensor(rt)), b
    check(y, ry, BAR)

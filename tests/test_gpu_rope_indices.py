"""Rows of several positions, each with channel pairs of its own: one call in place for each of them."""
import numpy as np
import pytest
import torch

import paper_2605_23163_amd as F
from tests import paged_ref as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_three_positions(dtype, interleaved):
    D, rows, parts = 128, 50, (16, 24, 24)      # pairs of time, row and column
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, 7, D, generator=g, device="cuda").to(DT[dtype])
    table = F.fdd_rope_table(D, base=1e6, interleaved=interleaved, scaling="parts", stretch=4.0, original=4096)
    w, m = R.frequencies(D, 1e6, "parts", 4.0, 4096)
    pos = np.stack([np.full(rows, 70000), 70000 + np.arange(rows) // 9, 70000 + np.arange(rows) % 9])
    y, want, at = x.clone(), x.double().cpu().numpy(), 0
    for i, n in enumerate(parts):
        mine = np.zeros(D // 2, dtype=bool)
        mine[at:at + n] = True
        at += n
        turns = torch.where(torch.from_numpy(mine).cuda(), table.turns, torch.zeros_like(table.turns))
        F.fdd_rope(y, torch.from_numpy(pos[i].astype(np.int32)).cuda(), F.RopeTable(turns, interleaved, m if i == 2 else 1.0), out=y)
        want = R.rotate(want, pos[i], np.where(mine, w, 0.0), m if i == 2 else 1.0, interleaved)
    # a pair is turned in one call; the last one's magnitude rounds the other pairs once more (and the first rounding by half a step of itself)
    bound = R.rotate_bound(x.double().cpu().numpy(), w, m, interleaved, dtype == "bf16", want)
    assert np.all(np.abs(y.double().cpu().numpy() - want) <= bound * (2 + 2.0 ** -7))

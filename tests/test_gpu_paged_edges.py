"""Inputs of the paged-cache calls where an answer hangs on one step of a kernel, against the 64-bit oracle."""
import itertools

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2511_12201_amd import binding as ob
from test_gpu_paged import BF16, F32, U32, Cache, Guarded, check_eviction, host, ints, rand, within

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ eviction

def border_weights(rng, kind, n, border):
    if kind == "spread":
        return (border * (1 + 1e-3 * rng.standard_normal(n))).astype(np.float32)
    low, close = {"few": (200, 100), "many": (200, 200)}[kind]
    w = np.full(n, border, dtype=np.float32)
    w[:low] = 0.97 * border
    w[low:low + close] = np.nextafter(np.float32(border), np.float32(0))
    return w[rng.permutation(n)]


@pytest.mark.parametrize("rows,pages", [(2300, 36), (4096, 64), (7000, 128), (8192, 128), (12000, 256), (16384, 256), (17000, 266)])
@pytest.mark.parametrize("kind", ["few", "many", "spread"])
def test_eviction_cuts_below_a_border_of_the_bins(rows, pages, kind):
    """Weights on both sides of a step of a key's upper 11 bits (the pairs' are 0.875 and 1), the cut a few rows off the number of
    those above it; pools of every way to hold the keys."""
    rng = np.random.default_rng(rows)
    cache = Cache(rng, 1, 2, pages, 64, 64, BF16)
    acc = np.stack([np.concatenate([border_weights(rng, kind, rows, b), np.zeros(cache.cap - rows, np.float32)]) for b in (0.875, 1.0)])
    acc = torch.from_numpy(acc[None]).cuda()
    pos = torch.arange(cache.cap, device="cuda").int().expand(1, 2, -1).contiguous()
    above = int((acc[0, 1, :rows] >= 1).sum())
    for i, budget in enumerate((above - 1, above, above + 1, above + 50, above + 101)):
        check_eviction(cache, budget, 0, 0, [cache.cap + 1], [[rows, rows]], pos.clone(), acc.clone(), i % 2 == 0)


@pytest.mark.parametrize("pages", [128, 256, 257])
def test_eviction_below_a_border_stays_inside_its_scratch(pages):
    """Few rows leave from among many: what is listed has to be no more than what moves."""
    rng = np.random.default_rng(pages)
    cache, ws = Cache(rng, 1, 2, pages, 64, 64, BF16), Guarded()
    n = cache.cap
    acc = torch.from_numpy(np.stack([border_weights(rng, "many", n, 1.0) for _ in range(2)])[None]).cuda()
    pos = torch.arange(n, device="cuda").int().expand(1, 2, -1).contiguous()
    for budget in (n - 300, n - 399, n - 350):
        outs = [torch.full((2 * n + 256,), -7, dtype=dt, device="cuda") for dt in (torch.int32, torch.float32)]
        ob.omni_paged_evict(cache.pool, budget, 0, 0, ints([n + 1]), ints([[n, n]]), pos, acc, ws=ws,
                            row_pos_out=outs[0][:-256].view(1, 2, n), acc_out=outs[1][:-256].view(1, 2, n))
        ws.check()
        assert all((x[-256:] == -7).all() for x in outs)

"""GPU: pages among a group's shared ones that none of its rows sees may hold anything, their scales included
(daf_cache_attn_shared): a step planned for a longer prefix, an empty sequence, rows at early positions."""
from __future__ import annotations

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
CFGS = [(BF16, 128, 28, 4), (BF16, 64, 6, 1), (F32, 128, 4, 2), (F32, 64, 16, 16)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import paper_2607_21599_amd as daf
    daf.lib()
    yield
    torch.cuda.synchronize()


def _spoil(p, pages, value):
    """NaN codes under scales of `value`."""
    at = torch.as_tensor(sorted(pages), device="cuda")
    for n in "kv":
        p.t[n].view(torch.uint8)[:, at] = 0x7F
        p.t[n + "_scale"][:, at] = value


def _entries_past_the_end(p, seq, lens, value):
    """The tables' entries past the sequences' lengths name pages that were never taken, the same for all."""
    free = (p.t["refs"] == 0).nonzero()[:, 0]
    _spoil(p, free.tolist(), value)
    width = p.t["table"].shape[1]
    for s, n in zip(seq, lens):
        have = -(-n // 64)
        p.t["table"][s, have:] = free[torch.arange(have, width, device="cuda") % len(free)].int()


VALUES = [float("nan"), float("inf"), 2.0 ** 100]


@pytest.mark.parametrize("dtype,d,hq,heads", CFGS)
@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("groups,shared,promise,nq", [
    ([3], [2300], [3800], [1, 1, 1]),             # a decode step of forks without tokens of their own
    ([1], [2300], [3800], [70]),                  # one request of many rows
    ([4], [100], [3200], [1, 5, 0, 70]),          # few of the promised pages
    ([2, 3], [0, 2240], [2624, 4000], [1, 2, 1, 1, 3])])  # empty sequences, and a full last page
def test_promise_above_the_lengths(dtype, d, hq, heads, value, groups, shared, promise, nq):
    from test_gpu_cache_shared import _check, _cu, _forked
    p, _, seq, lens = _forked(groups, shared, [0] * sum(groups), hq, heads, d, dtype, seed=3)
    # _forked's table is as wide as the lengths need: a wider one
    wide = torch.full((p.t["table"].shape[0], max(promise) // 64 + 2), -1, dtype=torch.int32, device="cuda")
    wide[:, :p.t["table"].shape[1]] = p.t["table"]
    p.t["table"] = wide
    import paper_2607_21599_amd as daf
    p.c = daf.Cache.from_tensors(p.t)
    _entries_past_the_end(p, seq, lens, value)
    _check(p, 0, _cu(nq), seq, groups, promise)


@pytest.mark.parametrize("dtype,d,hq,heads", CFGS)
@pytest.mark.parametrize("value", VALUES)
def test_rows_before_the_last_pages(dtype, d, hq, heads, value):
    from test_gpu_cache_shared import _check, _cu, _forked
    p, rng, seq, lens = _forked([3], [3000], [9, 70, 1], hq, heads, d, dtype, seed=4)
    nq = [2, 30, 1]
    pos = np.concatenate([rng.integers(-1, 700, n) for n in nq])
    _spoil(p, p.t["table"][seq[0], 11:46].tolist(), value)
    _check(p, 0, _cu(nq), seq, [3], [3000], pos)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", VALUES)
def test_more_pages_of_a_split_than_lanes(dtype, value):
    """Rows that fill the device with few splits, each of more than 64 pages, of which a row sees the first ones."""
    import paper_2607_21599_amd as daf
    from cache_pair import dev
    from test_gpu_cache_shared import _attn, _cu, _forked
    p, _, seq, lens = _forked([4], [300], [0] * 4, 16, 16, 64, dtype, seed=5)
    pages = 330
    wide = torch.full((p.t["table"].shape[0], pages), -1, dtype=torch.int32, device="cuda")
    wide[:, :p.t["table"].shape[1]] = p.t["table"]
    p.t["table"] = wide
    p.c = daf.Cache.from_tensors(p.t)
    _entries_past_the_end(p, seq, lens, value)
    nq = [256] * 4
    rows, g = daf.CacheRows(_cu(nq), dev(seq)), daf.CacheGroups([0, 4], [pages * 64])
    block = 128 if dtype == BF16 else 64
    size = daf.daf_cache_attn_shared_workspace_size(p.cfg, p.c, rows, g, pages * 64)
    splits = (size / 4 / 65 - 1024 * 16) / (1024 * 16)  # of 1024 rows and 16 heads, which fill their blocks
    assert 1024 % block == 0 and 1 <= splits < pages / 66, splits
    q = torch.randn(1024, 16, 64, generator=torch.Generator().manual_seed(6)).to(dtype)
    o, lse = _attn(p, 0, _cu(nq), seq, q.cuda(), [4], [pages * 64], max_len=pages * 64)
    few = torch.arange(0, 1024, 31).tolist()  # the oracle on some of the rows, each at its position
    at = [lens[0] - 256 + i % 256 for i in few]
    cu = _cu([sum(i // 256 == b for i in few) for b in range(4)])
    p.within_bounds(o[few], lse[:, few].contiguous(), 0, cu, seq, q[few], at)
    assert o.isfinite().all()

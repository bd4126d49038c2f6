"""GPU: groups of daf_cache_attn_shared in which some sequences, the first ones among them, are empty or shorter than
the shared pages, as a batch has them whose slots are kept when a request ends."""
from __future__ import annotations

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import paper_2607_21599_amd as daf
    daf.lib()
    yield
    torch.cuda.synchronize()


def _shorten(p, s, n):
    """The first n tokens of a sequence stay; the table names no page past them."""
    p.t["len"][s] = p.o.len[s] = n
    p.t["table"][s, -(-n // 64):] = p.o.table[s, -(-n // 64):] = -1


@pytest.mark.parametrize("dtype,d,hq,heads", [(BF16, 128, 28, 4), (F32, 64, 6, 1)])
@pytest.mark.parametrize("n,gone", [(2, [0]), (5, [0, 1, 3]), (5, [0, 1, 2, 3]), (70, [0, 1]), (70, list(range(69))),
                                    (130, list(range(66)) + [129])])
@pytest.mark.parametrize("varied", [False, True])
def test_freed_sequences_of_a_group(dtype, d, hq, heads, n, gone, varied):
    """The others against 64 bits: to the last bit they need not be what they were before. References of rows of
    one wave are raised together, by whole numbers; an exponent's argument s - m is rounded to 2^-24 of itself, so
    other rows' references change weights by a rounding, which the bound of a result has."""
    from test_gpu_cache_shared import _check, _cu, _forked
    p, _, seq, _ = _forked([n], [2300], [1 + i % 70 for i in range(n)], hq, heads, d, dtype, seed=21)
    nq = [1 + (varied and i % 3 == 1) - (varied and i == 2) for i in range(n)]
    p.free([seq[i] for i in gone])
    o, lse = _check(p, 0, _cu(nq), seq, [n], [2300], seed=6)
    there = torch.as_tensor(np.repeat([i not in gone for i in range(n)], nq), device="cuda")
    assert (o[~there] == 0).all() and (lse[:, ~there] == -torch.inf).all() and lse[:, there].isfinite().all()


@pytest.mark.parametrize("dtype,d,hq,heads", [(BF16, 128, 28, 4), (F32, 64, 6, 1)])
@pytest.mark.parametrize("lens", [[100, 2300, 2240, 2368], [2239, 2240, 70, 2400], [0, 2100, 2239, 64], [64, 1, 2300, 0]])
@pytest.mark.parametrize("promise", [2240, 3500])
def test_sequences_shorter_than_the_shared_pages(dtype, d, hq, heads, lens, promise):
    """The longest one's pages where none reaches the promise."""
    from test_gpu_cache_shared import _check, _cu, _forked
    p, _, seq, _ = _forked([4], [2240], [128, 200, 130, 128], hq, heads, d, dtype, seed=22)
    wide = torch.full((p.t["table"].shape[0], 60), -1, dtype=torch.int32, device="cuda")
    wide[:, :p.t["table"].shape[1]] = p.t["table"]
    p.t["table"] = wide
    p.o.table = wide.cpu().numpy().astype(p.o.table.dtype)
    import paper_2607_21599_amd as daf
    p.c = daf.Cache.from_tensors(p.t)
    for s, L in zip(seq, lens):
        _shorten(p, s, L if promise == 2240 else min(L, 2240))
    for nq in ([1] * 4, [3, 1, 20, 2]):
        _check(p, 0, _cu(nq), seq, [4], [promise])


def test_without_a_list_of_sequences_the_first_is_empty():
    from test_gpu_cache_shared import _attn, _forked
    p, _, seq, _ = _forked([3], [2420], [5, 60, 1], 8, 2, 64, BF16, seed=23)
    for n in ("table", "len"):
        p.t[n][:3] = p.t[n][torch.as_tensor(seq).cuda()].clone()
    q = torch.randn(3, 8, 64, generator=torch.Generator().manual_seed(5)).to(BF16).cuda()
    good, _ = _attn(p, 0, [0, 1, 2, 3], None, q, [3], [2420])
    p.t["len"][0], p.t["table"][0] = 0, -1
    o, _ = _attn(p, 0, [0, 1, 2, 3], None, q, [3], [2420])
    assert torch.equal(o[1:], good[1:]) and (o[0] == 0).all()

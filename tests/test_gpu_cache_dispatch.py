"""GPU: what an attention call over the paged cache must cope with, through each of the
kernels that it may take: NaN where no row looks, pages that are not there, other softmax
scales; and the reload of page ids where a workgroup has more than its lanes hold."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from cache_pair import f64
from test_gpu_cache import BF16, F32, _fill, _pair

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import paper_2607_21599_amd as daf
    daf.lib()
    yield
    torch.cuda.synchronize()


# keys and rows: one workgroup per head, a line of pages, row blocks without and with splits
CALLS = [(300, 3), (4000, 3), (300, 50), (3000, 50)]
TYPES = [(BF16, 128), (F32, 64), (BF16, 64), (F32, 128)]


def _nan_pool(keys, d, dtype, seed, seqs=1):
    p = _pair(pages=seqs * (keys // 64 + 2), heads=2, d=d, hq=8, n_seqs=seqs, max_seq_pages=keys // 64 + 2, dtype=dtype)
    for n in "kv":
        p.t[n].view(torch.uint8).fill_(0x7F)
        p.o.code[n][:] = np.nan
    return p, np.random.default_rng(seed)


def _nan_from(p, seq, at, end):
    """Tokens at .. end - 1 of a sequence become NaN codes."""
    for t in range(at, end):
        page, slot = int(p.o.table[seq, t // 64]), t % 64
        p.t["k"].view(torch.uint8)[0, page, :, slot] = 0x7F
        p.t["v"].view(torch.uint8)[0, page, :, :, slot] = 0xFF
        for n in "kv":
            p.o.code[n][0, page, :, slot] = np.nan


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("keys,rows", CALLS)
def test_nan_where_no_row_looks(dtype, d, keys, rows):
    p, rng = _nan_pool(keys, d, dtype, keys + rows + d)
    _fill(p, rng, [0], [keys])
    q = torch.from_numpy(rng.standard_normal((rows, 8, d))).float()
    _nan_from(p, 0, keys, -(-keys // 64) * 64)  # past the last token
    p.check_attn(0, [0, rows], [0], q)
    top = keys - 70  # past the largest position, inside a page that rows see
    _nan_from(p, 0, top + 1, keys)
    pos = rng.integers(0, top + 1, rows)
    pos[rows // 2], pos[0] = top, -1
    o, lse = p.check_attn(0, [0, rows], [0], q, pos.tolist())
    assert not o[0].any() and torch.isneginf(lse[:, 0]).all() and o.isfinite().all()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("keys,rows", CALLS)
def test_pages_that_are_not_there(dtype, d, keys, rows):
    p, rng = _nan_pool(keys, d, dtype, keys + rows + d + 1)
    _fill(p, rng, [0], [keys])
    last = -(-keys // 64) - 1
    _nan_from(p, 0, keys, (last + 1) * 64)
    q = torch.from_numpy(rng.standard_normal((rows, 8, d))).float()
    pos = rng.integers(0, keys, rows).tolist()
    keep = p.o.table.copy()
    for gone in ([0], [last], [1, 3], [i for i in range(last + 1) if i % 3], list(range(last)), list(range(last + 1))):
        p.o.table[0, gone] = [(-1, p.t["refs"].numel(), 2 ** 31 - 1, -2 ** 31)[i % 4] for i in gone]
        p.t["table"].copy_(torch.from_numpy(p.o.table).int())
        p.check_attn(0, [0, rows], [0], q)
        p.check_attn(0, [0, rows], [0], q, pos)
        p.o.table[:] = keep


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("keys,rows", CALLS)
@pytest.mark.parametrize("times", [2.0 ** -10, 0.25, 4.0, 64.0])
def test_softmax_scales(dtype, d, keys, rows, times):
    """A scale of `times` the default one is the default one on q times that. Large scales
    leave features of rows whose one weighty key has a 0 there, so that bf16 rows beside
    others (more than 64 per head) show the steps of their fp16 weights: half a step, 2^-25,
    where a row's largest weight is 2^10 or more, is 2^-35 of that weight per key, times
    values of at most 448 times a scale at most 16 times the least."""
    import paper_2607_21599_amd as daf
    p, rng = _nan_pool(keys, d, dtype, keys + rows + d + 2)
    _fill(p, rng, [0], [keys])
    q = torch.from_numpy(rng.standard_normal((rows, 8, d))).to(dtype)
    p.cfg = daf.AttnCfg(8, 2, d, p.cfg.dtype, times / d ** 0.5)
    o, lse = p.attn(0, [0, rows], [0], q.cuda())
    if dtype == BF16 and rows * 4 > 64:
        want, _, _, _ = p.o.attn(0, [0, rows], [0], None, f64(q * times), 1 / d ** 0.5)
        step = keys * 2.0 ** -35 * 448 * 16 * p.o.scale["v"][0, p.o.table[0, :-(-keys // 64)]].min()
        off = f64(o) - want
        o = torch.from_numpy(want + np.sign(off) * np.maximum(np.abs(off) - step, 0))
    p.within_bounds(o, lse, 0, [0, rows], [0], q * times, None)


@pytest.mark.parametrize("heads,rows,lens", [(1, [9, 70, 200], [1500, 40, 900]), (3, [65, 1, 0, 130], [700, 64, 0, 1300]),
                                             (5, [300], [2000]), (8, [40, 40, 33], [64, 3000, 500]), (9, [17, 80], [400, 1])])
def test_every_row_block_and_split(heads, rows, lens):
    """Numbers of (head, split) pairs and row blocks that do not divide by each other, planned
    for the lengths and for far longer ones."""
    p = _pair(pages=sum(-(-n // 64) for n in lens) + 2, heads=heads, d=64, hq=heads * 8, n_seqs=len(lens),
              max_seq_pages=400)
    rng = np.random.default_rng(heads)
    _fill(p, rng, list(range(len(lens))), lens)
    q = torch.from_numpy(rng.standard_normal((sum(rows), heads * 8, 64))).float()
    cu = [0] + np.cumsum(rows).tolist()
    for max_len in (max(lens), 5000, 25600):
        p.check_attn(0, cu, list(range(len(lens))), q, max_len=max_len)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_more_pages_than_a_waves_lanes_hold(dtype):
    """Few rows, many heads, a long sequence: 4 workgroups per head, of 65 pages a wave. Some
    pages are not there. Against the formula in 64 bits, some of the heads."""
    import paper_2607_21599_amd as daf
    from cache_pair import dev
    from paper_2607_21599_amd.tensors import cache_tensors
    heads, d, pages = 64, 64, 1045
    keys = pages * 64 - 13
    t = cache_tensors(1, pages, heads, d, 1, pages)
    c = daf.Cache.from_tensors(t)
    gen = torch.Generator(device="cuda").manual_seed(5)
    for n in "kv":
        x = torch.randint(0, 256, t[n].shape, generator=gen, device="cuda", dtype=torch.uint8)
        x[(x & 0x7F) > 0x68] &= 0x37  # magnitudes up to 32, no NaN
        t[n].view(torch.uint8).copy_(x)
        t[n + "_scale"].copy_(torch.exp2(torch.randint(-4, -2, (1, pages, heads), generator=gen, device="cuda").float()))
    rng = np.random.default_rng(5)
    ids = rng.permutation(pages)
    gone = [0, 255, 256, 300, 777, 1044]
    ids[gone] = -1
    t["table"].copy_(dev(ids)[None])
    t["len"].fill_(keys)
    cfg = daf.AttnCfg(heads, heads, d, daf.DAF_BF16 if dtype == BF16 else daf.DAF_F32)
    q = (torch.randn(2, heads, d, generator=gen, device="cuda") * 0.25).to(dtype)
    rows = daf.CacheRows([0, 2], dev([0]), dev([keys - 1, 40000]))
    size = daf.daf_cache_attn_workspace_size(cfg, c, rows, keys)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    # 4 workgroups per head: two partial results of 16 rows each
    assert size < 2 * 4 * heads * 16 * (d + 1) * 4 + 4096 and pages > 4 * 4 * 64
    o, lse = torch.zeros_like(q), torch.zeros(heads, 2, device="cuda")
    daf.daf_cache_attn(cfg, c, 0, rows, keys, q, o, lse, ws, size)
    there = torch.from_numpy(ids >= 0).repeat_interleave(64)[:keys].cuda()
    at = torch.from_numpy(np.maximum(ids, 0)).long().cuda()
    for h in (0, 1, 31, 63):
        k = (t["k"][0, at, h].double() * t["k_scale"][0, at, h, None, None].double()).reshape(-1, d)[:keys]
        v = (t["v"][0, at, h].double() * t["v_scale"][0, at, h, None, None].double()).transpose(1, 2).reshape(-1, d)[:keys]
        for r, last in enumerate((keys - 1, 40000)):
            see = there & (torch.arange(keys, device="cuda") <= last)
            x = (k[see] @ q[r, h].double()) / d ** 0.5
            w = torch.exp(x - x.max())
            want, mean = w @ v[see] / w.sum(), w @ v[see].abs() / w.sum()
            # the bounds of the roundings as for every other case (cache_pair)
            size_ = float((k[see].abs() @ q[r, h].double().abs()).max()) / d ** 0.5
            e = 2.0 ** -24 * ((d + 12) * size_ + keys + 64)
            half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -23
            tol = (2 * e * mean + half * mean) * (1 + half) + half * want.abs()
            assert ((o[r, h].double() - want).abs() <= tol).all(), (h, r)
            full = float(x.max() + w.sum().log())
            assert abs(float(lse[h, r]) - full) <= e + 2.0 ** -22 * (1 + abs(full))

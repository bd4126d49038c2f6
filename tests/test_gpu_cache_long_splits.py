"""GPU: many rows over many pages, where a workgroup walks more pages than it has ids in
its lanes: 64 at a time, with gaps and other scales among them."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from test_gpu_cache import BF16, F32, _fill, _pair

pytestmark = pytest.mark.gpu

KEYS, PAGES = 12700, 199


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import paper_2607_21599_amd as daf
    daf.lib()
    yield
    torch.cuda.synchronize()


def _case(heads, hq, d, dtype, seed):
    p = _pair(pages=PAGES + 3, heads=heads, d=d, hq=hq, n_seqs=2, max_seq_pages=PAGES + 2, dtype=dtype)
    rng = np.random.default_rng(seed)
    for n in "kv":  # what nobody writes is NaN
        p.t[n].view(torch.uint8).fill_(0x7F)
        p.o.code[n][:] = np.nan
    _fill(p, rng, [1], [KEYS])
    # past the last token, too
    page, tail = int(p.o.table[1, PAGES - 1]), KEYS % 64
    p.t["k"].view(torch.uint8)[0, page, :, tail:] = 0x7F
    p.t["v"].view(torch.uint8)[0, page, :, :, tail:] = 0x7F
    return p, rng


def _check(p, rng, rows, pos, some, mark=""):
    q = torch.from_numpy(rng.standard_normal((rows, p.hq, p.d))).to(p.dtype)
    o, lse = p.attn(0, [0, rows], [1], q.cuda(), pos)
    assert o.isfinite().all() and not lse.isnan().any()
    at = [KEYS - rows + j for j in some] if pos is None else [pos[j] for j in some]
    p.within_bounds(o[some], lse[:, some], 0, [0, len(some)], [1], q[some], at)


# 3 and 1 splits of 12700 keys
@pytest.mark.parametrize("heads,hq,rows", [(16, 128, 1040), (32, 128, 2080)])
@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F32, 64), (BF16, 128)])
def test_pages_64_at_a_time(heads, hq, rows, dtype, d):
    p, rng = _case(heads, hq, d, dtype, heads + d)
    _check(p, rng, rows, None, [0, rows // 2, rows - 1])
    pos = np.sort(rng.choice(KEYS, rows, replace=False)).tolist()
    pos[0], pos[1], pos[-2], pos[-1] = -1, 4095, KEYS - 1, 63
    _check(p, rng, rows, pos, [0, 1, rows // 2, rows - 2, rows - 1])
    # pages that are not there: at the ends of the runs of 64, a run of its own, the last one
    gone = [0, 63, 64, *range(67, 131), 133, 134, PAGES - 1]
    p.o.table[1, gone] = -1
    p.t["table"].copy_(torch.from_numpy(p.o.table).int())
    _check(p, rng, rows, pos, [0, 1, rows // 2, rows - 2, rows - 1])
    _check(p, rng, rows, None, [0, rows - 1])
    p.o.table[1, :131] = -1
    p.t["table"].copy_(torch.from_numpy(p.o.table).int())
    _check(p, rng, rows, pos, [0, 1, rows // 2, rows - 2, rows - 1])


@pytest.mark.parametrize("heads,hq,rows", [(16, 128, 1040), (32, 128, 2080)])
def test_a_scale_far_from_the_others(heads, hq, rows):
    """Past the first 64 pages, so that the way of the weights follows from all of them."""
    p, rng = _case(heads, hq, 64, BF16, 7)
    for page, far in ((131, 2.0 ** 9), (150, 2.0 ** -30)):
        id = int(p.o.table[1, page])
        p.t["v_scale"][0, id] *= far
        p.o.scale["v"][0, id] *= far
    _check(p, rng, rows, None, [0, 300, rows - 1])
    pos = np.sort(rng.choice(KEYS, rows, replace=False)).tolist()
    _check(p, rng, rows, pos, [0, 300, 600, rows - 1])

"""GPU: NaN and infinities in a row's q, and NaN in a key, through every kernel that an
attention call over the paged cache may take: a result is NaN, never that of a row that
sees no key, nor one that leaves keys out."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from test_gpu_cache import BF16, F32, _cu, _fill, _pair

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import paper_2607_21599_amd as daf
    daf.lib()
    yield
    torch.cuda.synchronize()


# keys and rows: one workgroup per head, a line of pages, row blocks without and with splits
CALLS = [(300, 3), (4000, 3), (70, 30), (3000, 30)]


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64), (BF16, 64), (F32, 128)])
@pytest.mark.parametrize("keys,rows", CALLS)
def test_of_a_row(dtype, d, keys, rows):
    p = _pair(pages=70, heads=2, d=d, hq=8, n_seqs=1, max_seq_pages=64, dtype=dtype)
    rng = np.random.default_rng(keys + d)
    _fill(p, rng, [0], [keys])
    q = torch.from_numpy(rng.standard_normal((rows, 8, d))).float()
    good = torch.ones(rows, dtype=torch.bool)
    bad = q.clone()
    for row, head, value in [(0, 1, float("nan")), (rows - 1, 6, float("inf")), (rows - 1, 2, -float("inf"))]:
        bad[row, head, 5] = value
        good[row] = False
    o, lse = p.attn(0, [0, rows], [0], bad.to(dtype).cuda())
    for row, head in [(0, 1), (rows - 1, 6), (rows - 1, 2)]:
        assert o[row, head].isnan().all() and lse[head, row].isnan(), (row, head)
    assert int(lse.isnan().sum()) == 3 and int(o.isnan().any(-1).sum()) == 3
    some = good.nonzero()[:, 0]
    at = [keys - rows + int(r) for r in some]
    p.within_bounds(o[some], lse[:, some], 0, [0, len(some)], [0], q[some].to(dtype), at)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
@pytest.mark.parametrize("keys,rows", CALLS)
def test_of_a_key(dtype, d, keys, rows):
    """Rows that see a key with a NaN are NaN, those before it are not."""
    p = _pair(pages=70, heads=2, d=d, hq=8, n_seqs=1, max_seq_pages=64, dtype=dtype)
    rng = np.random.default_rng(keys + d + 1)
    _fill(p, rng, [0], [keys])
    where = keys // 2
    k = torch.ones(1, 2, d)
    k[0, 1, 3] = float("nan")
    p.write(0, [0, 1], [0], k, torch.ones(1, 2, d), [where])
    pos = [where - 1 - j if j % 2 else keys - 1 - j for j in range(rows)]
    q = torch.from_numpy(rng.standard_normal((rows, 8, d))).float()
    o, lse = p.attn(0, [0, rows], [0], q.to(dtype).cuda(), pos)
    sees = torch.tensor([at >= where for at in pos])
    assert lse[4:, sees].isnan().all() and o[sees][:, 4:].isnan().all()
    assert lse[:4].isfinite().all() and lse[:, ~sees].isfinite().all()
    assert o[:, :4].isfinite().all() and o[~sees].isfinite().all()


@pytest.mark.parametrize("keys,rows", CALLS)
def test_no_key_beside_a_nan(keys, rows):
    """A row that sees no key stays 0 and -infinity, with its q NaN too."""
    p = _pair(pages=70, heads=1, d=64, hq=4, n_seqs=1, max_seq_pages=64)
    rng = np.random.default_rng(keys + 2)
    _fill(p, rng, [0], [keys])
    q = torch.from_numpy(rng.standard_normal((rows, 4, 64))).to(BF16).cuda()
    q[1] = float("nan")
    q[2] = float("nan")
    pos = [keys - 1] * rows
    pos[0] = pos[1] = -1
    o, lse = p.attn(0, [0, rows], [0], q, pos)
    assert not o[:2].any() and torch.isneginf(lse[:, :2]).all()
    assert o[2].isnan().all() and lse[:, 2].isnan().all()
    assert o[3:].isfinite().all() and lse[:, 3:].isfinite().all()

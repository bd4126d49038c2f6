"""GPU: how exactly bf16 rows take their weights: closer than bf16 holds them."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from cache_pair import f64
from test_gpu_cache import BF16, _fill, _pair

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import paper_2607_21599_amd as daf
    daf.lib()
    yield
    torch.cuda.synchronize()


def close(p, o, q, pos, seq=0):
    """A weight is off by at most 2^-11 of itself (11 bits, to nearest), as is their sum, or
    by 2^-35 of the row's largest one where it is held in fp16, times a value of at most 448
    times a scale that is 16 times the least. 2^-24 (d + 12) of the largest |q||k| for the
    score, twice, and of the number of keys for the sums. The output's rounding is half a
    step, 2^-8."""
    want, _, mean, size = p.o.attn(0, [0, len(pos)], [seq], pos, f64(q), 1 / p.d ** 0.5)
    keys = int(p.o.len[seq])
    scales = p.o.scale["v"][0, p.o.table[seq, :-(-keys // 64)]]  # [pages][heads]
    least = np.where(scales > 0, scales, np.inf).min(0).repeat(p.hq // p.heads)[:, None]  # [hq][1]
    e = 2.0 ** -24 * ((p.d + 12) * size + 2 * keys + 64)
    tol = (2.0 ** -10 + 2 * e.T[..., None]) * mean * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    tol += keys * 2.0 ** -35 * 448 * 16 * least
    err = np.abs(f64(o) - want)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("d,heads,hq", [(128, 2, 14), (64, 1, 4)])
@pytest.mark.parametrize("keys,rows", [(9, 1), (16, 4), (9, 40), (16, 64)])
def test_few_keys(d, heads, hq, keys, rows):
    """Where a weight's rounding shows most: few keys of like weight, whose values cancel."""
    p = _pair(pages=4, heads=heads, d=d, hq=hq, n_seqs=1, max_seq_pages=2)
    rng = np.random.default_rng(keys + rows)
    _fill(p, rng, [0], [keys])
    q = torch.from_numpy(rng.standard_normal((rows, hq, d)) * 0.3).to(BF16)
    pos = [keys - 1] * rows
    o, _ = p.attn(0, [0, rows], [0], q.cuda(), pos)
    close(p, o, q, pos)


@pytest.mark.parametrize("d,heads,hq", [(128, 1, 7), (64, 2, 16)])
@pytest.mark.parametrize("rows,keys", [(1, 200), (2, 3000), (40, 200), (40, 3000)])
@pytest.mark.parametrize("spread", [0, 4, 5, 16, 40, 100])
def test_pages_of_other_scales(d, heads, hq, rows, keys, spread):
    """One page whose values are 2^spread times those of the others, and whose keys the rows
    all but ignore: the others' values, down to the smallest codes, still make the result.
    One page of zeros among them."""
    p = _pair(pages=50, heads=heads, d=d, hq=hq, n_seqs=1, max_seq_pages=48)
    rng = np.random.default_rng(spread + rows)
    _fill(p, rng, [0], [keys])
    n = -(-keys // 64)
    big, none = int(p.o.table[0, n - 2]), int(p.o.table[0, 1])
    for page in p.o.table[0, :n].tolist():
        top = 2.0 ** -20
        if page == none:
            top = 0.0
        elif page == big:
            top *= 2.0 ** spread
        p.o.scale["v"][0, page] = top
        p.t["v_scale"][0, page] = top
    # codes of every size, the smallest ones too
    codes = torch.from_numpy(rng.integers(0, 256, (50, heads, d, 64))).to(torch.uint8)
    codes[(codes & 0x7F) == 0x7F] = 1
    codes[none] = 0
    p.t["v"].view(torch.uint8)[0] = codes.cuda()
    p.o.code["v"][0] = codes.view(torch.float8_e4m3fn).double().numpy().swapaxes(-1, -2)
    # scores of the page of large values: at least 2^-150 below the others
    k = p.t["k"].view(torch.uint8)
    k[0, big, :, :, 0] = 0xFE  # -448
    p.o.code["k"][0, big, :, :, 0] = -448
    at = 448 * p.o.scale["k"][0, big].min() / d ** 0.5
    q = torch.from_numpy(rng.standard_normal((rows, hq, d))).to(BF16)
    q[:, :, 0] = 130 / at
    for page in p.o.table[0, :n].tolist():
        if page != big:
            k[0, page, :, :, 0] = 0
            p.o.code["k"][0, page, :, :, 0] = 0
    pos = [keys - 1 - j for j in range(rows)]
    o, _ = p.attn(0, [0, rows], [0], q.cuda(), pos)
    close(p, o, q, pos)


@pytest.mark.parametrize("rows", [1, 40])
def test_many_small_weights(rows):
    """One large weight and thousands of small ones that together make half of the row."""
    p = _pair(pages=130, heads=1, d=64, hq=4, n_seqs=1, max_seq_pages=128)
    keys = 8000
    rng = np.random.default_rng(3)
    assert p.extend([0], [keys]) == 0
    k = torch.zeros(keys, 1, 64)
    k[4321, 0, 0] = 8.0  # score 9 with q of 9: e^9 = 8103 times the others
    p.write(0, [0, keys], [0], k, torch.from_numpy(rng.standard_normal((keys, 1, 64)) + 1).float())
    q = torch.zeros(rows, 4, 64, dtype=BF16)
    q[:, :, 0] = 9.0
    q[:, 1, 0] = 16.0  # e^16: 1100 times all others together
    q[:, 2, 0] = 0.0
    pos = [keys - 1] * rows
    o, _ = p.attn(0, [0, rows], [0], q.cuda(), pos)
    close(p, o, q, pos)


@pytest.mark.parametrize("d,hq", [(128, 7), (64, 16)])
def test_references_that_rise(d, hq):
    """Scores that rise by more than a reference allows, in steps inside a page and between
    pages, with weights in flight that still count."""
    p = _pair(pages=40, heads=1, d=d, hq=hq, n_seqs=1, max_seq_pages=32)
    keys = 2000
    rng = np.random.default_rng(4)
    assert p.extend([0], [keys]) == 0
    k = torch.from_numpy(rng.standard_normal((keys, 1, d)) * 0.1).float()
    k[:, 0, 0] = torch.linspace(0, 60, keys).floor()
    p.write(0, [0, keys], [0], k, torch.from_numpy(rng.standard_normal((keys, 1, d))).float())
    q = torch.from_numpy(rng.standard_normal((40, hq, d))).to(BF16)
    q[:, :, 0] = d ** 0.5 * torch.tensor([0.25, 0.5, 1, 2, 4] * 8).view(40, 1)
    pos = [keys - 1 - 37 * j for j in range(40)]
    for rows in (40, 2):
        o, _ = p.attn(0, [0, rows], [0], q[:rows].cuda(), pos[:rows])
        close(p, o, q[:rows], pos[:rows])

"""GPU: the bits of a decode row's weights through daf_cache_attn_shared and daf_cache_attn, where two large
values of V cancel and the roundings of their weights are what is left."""
from __future__ import annotations

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

SHARED, TAILS = 2240, [70, 1, 200]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import paper_2607_21599_amd as daf
    daf.lib()
    yield
    torch.cuda.synchronize()


def _cache(hq, heads, d, at_b):
    """Keys 3 and at_b of the sequences have K of nearly the same score and V of 1 and -1; all others are zeros."""
    from test_gpu_cache_shared import _cu, _pair
    n = len(TAILS)
    p = _pair(pages=120, heads=heads, d=d, n_seqs=n + 1, max_seq_pages=40, hq=hq)
    seq = list(range(n))

    def rows(lo, counts):
        k, v = (torch.zeros(sum(counts), heads, d) for _ in range(2))
        for first in _cu(counts)[:-1]:
            for at, sign in ((3, 1.0), (at_b, -1.0)):
                if lo <= at < lo + counts[0]:
                    k[first + at - lo, :, 0], k[first + at - lo, :, 1], v[first + at - lo] = 8.0, 0.25 * (sign < 0), sign
        return k, v

    assert p.extend([n], [SHARED]) == 0
    p.write(0, [0, SHARED], [n], *rows(0, [SHARED]))
    assert p.fork([n] * n, seq) == 0
    assert p.extend(seq, TAILS) == 0
    for s, t in zip(seq, TAILS):
        p.write(0, [0, t], [s], *rows(SHARED, [t]))
    return p, seq


@pytest.mark.parametrize("hq,heads,d", [(28, 4, 128), (6, 1, 64)])
@pytest.mark.parametrize("at_b", [40, 20 * 64 + 7, SHARED])  # in one page, in two splits, in the rest of each sequence
def test_weights_of_decode_rows(hq, heads, d, at_b):
    """o = (w_a - w_b) / sum: two weights of at most half the sum, each in two bf16 terms (2^-17 of it). Scores are
    sums of two products, off by at most 16 roundings of 2^-24 of their size with the exponents' arguments, the
    split's LSE and the join; 64 more for exponentials, products and quotients. Then half a step of the output."""
    from cache_pair import f64
    from test_gpu_cache_shared import _attn
    p, seq = _cache(hq, heads, d, at_b)
    gen = torch.Generator().manual_seed(d + at_b)
    q = torch.zeros(3, hq, d)
    q[..., 0] = 16 + 8 * torch.rand(3, hq, generator=gen)
    q[..., 1] = 0.3 * torch.randn(3, hq, generator=gen)
    q = q.to(torch.bfloat16)
    cu = [0, 1, 2, 3]
    want, _, mean, size = p.o.attn(0, cu, seq, None, f64(q), 1 / d ** 0.5)
    e = (2.0 ** -17 + 2.0 ** -24 * (16 * size.T[..., None] + 64)) * mean
    tol = e + 2.0 ** -8 * (np.abs(want) + e)
    assert np.abs(want).max() < 0.02 and mean.min() > 0.9  # they cancel
    for name, o in (("daf_cache_attn", p.attn(0, cu, seq, q.cuda())[0]),
                    ("daf_cache_attn_shared", _attn(p, 0, cu, seq, q.cuda(), [3], [SHARED])[0])):
        err = np.abs(f64(o) - want)
        assert (err <= tol).all(), (name, float((err / tol).max()))

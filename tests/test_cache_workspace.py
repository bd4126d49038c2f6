"""CPU: the attention's workspace stays bounded, however many the rows and keys are."""
import itertools

import numpy as np
import pytest

import paper_2607_21599_amd as daf
from test_cache_checks import FAKE

# partial results of at most 8192 workgroups: 128 rows of D values and an LSE in fp32 each
MOST = {d: 8192 * 128 * (d + 1) * 4 + 256 for d in (64, 128)}


def _size(rows, max_len, hq=28, hkv=4, d=128, dtype=daf.DAF_BF16):
    c = daf.Cache(1, 10, hkv, d, 64, 1 << 20, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE)
    cu = np.concatenate([[0], np.cumsum(rows)])
    assert int(cu[-1]) * hq < 2 ** 31
    return daf.daf_cache_attn_workspace_size(daf.AttnCfg(hq, hkv, d, dtype), c, daf.CacheRows(cu), max_len)


def test_of_many_rows():
    assert _size([32768], 32768) == 0  # the device is full without splits
    assert 0 < _size([4915], 32768) <= 220 << 20
    assert 0 < _size([4096], 131072) <= 240 << 20
    assert 0 < _size([128], 32896) <= 32 << 20
    # many sequences of few rows, any of which may be the only long one
    assert 0 < _size([10] * 128, 131072) <= 520 << 20


@pytest.mark.parametrize("dtype", [daf.DAF_BF16, daf.DAF_F32])
@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (4, 1, 64), (16, 16, 128), (64, 8, 64), (7, 7, 64)])
def test_over_the_range(dtype, hq, hkv, d):
    for rows, requests, keys in itertools.product((1, 2, 5, 17, 40, 128, 777, 4915, 32768), (1, 3, 32),
                                                  (0, 63, 1500, 8000, 32768, 131072, 1 << 20, 1 << 26)):
        assert _size([rows] * requests, keys, hq, hkv, d, dtype) <= MOST[d], (rows, requests, keys)

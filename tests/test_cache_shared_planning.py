"""CPU: what planning a call of daf_cache_attn_shared takes of the host, which every call of every layer pays."""
import time

import pytest

import paper_2607_21599_amd as daf
from test_cache_checks import _cache


def _call(hq, hkv, groups, shared):
    cfg, n = daf.AttnCfg(hq, hkv, 128, daf.DAF_BF16), sum(groups)
    cu = [0]
    for x in groups:
        cu.append(cu[-1] + x)
    c = _cache(n_kv_heads=hkv, head_dim=128, n_seqs=n, max_seq_pages=1 << 13)
    rows, g = daf.CacheRows(list(range(n + 1))), daf.CacheGroups(cu, shared)
    return lambda: daf.daf_cache_attn_shared_workspace_size(cfg, c, rows, g, 140000)


@pytest.mark.parametrize("hq,hkv", [(32, 8), (32, 32)])
@pytest.mark.parametrize("others", [[640] * 127, [640 + 64 * i for i in range(127)], [131072 - 64 * i for i in range(127)]])
def test_many_groups_are_planned_at_once(hq, hkv, others):
    """128 groups of two, one of them with a long prefix: a few us more than a call takes anyway."""
    size = _call(hq, hkv, [2] * 128, [131072] + others)
    took = []
    for _ in range(200):
        t = time.perf_counter()
        assert size() > 0
        took.append(time.perf_counter() - t)
    assert min(took) < 100e-6, min(took)

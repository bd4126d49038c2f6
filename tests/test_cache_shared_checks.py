"""CPU: refusals and workspace sizes of daf_cache_attn_shared."""
import pytest

import paper_2607_21599_amd as daf
from test_cache_checks import ALIGN, FAKE, INVALID, UNSUPPORTED, WORKSPACE, _cache, _cfg, _status

ROWS = daf.CacheRows([0, 1, 2, 3])


def _args(**change):
    a = dict(cfg=_cfg(), cache=_cache(max_seq_pages=600), layer=0, rows=ROWS, groups=daf.CacheGroups([0, 3], [3200]),
             max_len=4000, q=FAKE, o=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 40, stream=0)
    a.update(change)
    return a.values()


def _size(**change):
    a = list(_args(**change))
    return daf.daf_cache_attn_shared_workspace_size(a[0], a[1], a[3], a[4], a[5])


@pytest.mark.parametrize("change,status", [
    (dict(cfg=_cfg(head_dim=64)), INVALID), (dict(cfg=_cfg(dtype=9)), UNSUPPORTED), (dict(layer=2), INVALID),
    (dict(cache=_cache(table=None)), INVALID), (dict(max_len=-1), INVALID), (dict(max_len=600 * 64 + 1), INVALID),
    (dict(q=None), INVALID), (dict(o=None), INVALID), (dict(q=FAKE + 8), ALIGN), (dict(o=FAKE + 8), ALIGN),
    (dict(lse=FAKE + 4), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws=FAKE + 8), ALIGN),
    (dict(rows=daf.CacheRows([0, 2, 1, 3])), INVALID),
    (dict(groups=daf.CacheGroups([0, 2], [320])), INVALID), (dict(groups=daf.CacheGroups([0, 4], [320])), INVALID),
    (dict(groups=daf.CacheGroups([1, 3], [320])), INVALID), (dict(groups=daf.CacheGroups([0, 2, 1, 3], [1, 2, 3])), INVALID),
    (dict(groups=daf.CacheGroups([0, 3], [-1])), INVALID), (dict(groups=daf.CacheGroups([0], [])), INVALID)])
def test_bad_calls(change, status):
    assert _status(daf.daf_cache_attn_shared, *_args(**change)) == status
    if status == INVALID and not {"layer", "q", "o"} & set(change):
        assert _size(**change) == 0


def test_groups_without_lengths():
    g = daf.CacheGroups([0, 3], [320])
    g.shared = None
    assert _status(daf.daf_cache_attn_shared, *_args(groups=g)) == INVALID
    g = daf.CacheGroups([0, 3], [320])
    g.cu = None
    assert _status(daf.daf_cache_attn_shared, *_args(groups=g)) == INVALID
    g.n = -1
    assert _status(daf.daf_cache_attn_shared, *_args(groups=g)) == INVALID
    assert _status(daf.daf_cache_attn_shared, *_args(groups=None)) == INVALID
    with pytest.raises(ValueError):
        daf.CacheGroups([0, 3], [1, 2])


def test_workspace_sizes():
    need = _size()
    assert need > 0
    assert _status(daf.daf_cache_attn_shared, *_args(ws_bytes=need - 1)) == WORKSPACE
    # nothing shared, or few pages: that of daf_cache_attn
    a = list(_args())
    assert _size(groups=daf.CacheGroups([0, 3], [640]), max_len=800) == daf.daf_cache_attn_workspace_size(a[0], a[1], a[3], 800)
    for g in (daf.CacheGroups([0, 3], [63]), daf.CacheGroups([0, 1, 2, 3], [320, 320, 320]), daf.CacheGroups([0, 3], [0])):
        a = list(_args())
        assert _size(groups=g) == daf.daf_cache_attn_workspace_size(a[0], a[1], a[3], a[5])
    assert _size(rows=daf.CacheRows([0, 0, 0, 0])) == 0


@pytest.mark.parametrize("hq,hkv,d,dtype", [(28, 4, 128, daf.DAF_BF16), (4, 1, 64, daf.DAF_BF16), (32, 32, 128, daf.DAF_F32),
                                            (64, 1, 64, daf.DAF_F32)])
def test_workspace_bound(hq, hkv, d, dtype):
    """As the header has it, over numbers of rows, requests, groups and lengths."""
    cfg = daf.AttnCfg(hq, hkv, d, dtype)
    c = _cache(n_kv_heads=hkv, head_dim=d, n_seqs=3000, max_seq_pages=1 << 15)
    for n_req, rows in ((2, 1), (2, 3000), (40, 1), (40, 64), (256, 1), (256, 130), (1500, 3)):
        r = daf.CacheRows([rows * i for i in range(n_req + 1)])
        for groups in {1, min(2, n_req // 2), n_req // 2}:  # of two requests or more
            cu = [n_req * i // groups for i in range(groups + 1)]
            for shared, max_len in ((64, 128), (4096, 5000), (131072, 140000), (1 << 17, 1 << 18), (64, 1 << 18)):
                g = daf.CacheGroups(cu, [shared] * groups)
                size = daf.daf_cache_attn_shared_workspace_size(cfg, c, r, g, max_len)
                most = min(n_req, 256) * rows
                per_group = 512 * (d + 1) * hkv * min(groups, 128)
                assert 0 <= size <= 8 * (d + 1) * most * hq + per_group + 544e6, (n_req, rows, groups, shared, size)
                assert size > 0 or shared == 64  # those may go daf_cache_attn's way


def test_too_many_rows():
    c = _cache(n_seqs=2, max_seq_pages=(1 << 25) - 1)
    r, g = daf.CacheRows([0, 40_000_000, 76_000_000]), daf.CacheGroups([0, 2], [3200])
    assert _status(daf.daf_cache_attn_shared, *_args(cache=c, rows=r, groups=g)) == UNSUPPORTED
    long = daf.CacheRows([0, 1_000_000, 2_000_000])
    assert _status(daf.daf_cache_attn_shared, *_args(cache=c, rows=long, groups=g, max_len=(1 << 31) - 100)) == UNSUPPORTED

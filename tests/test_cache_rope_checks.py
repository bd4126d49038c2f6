"""CPU: refusals of daf_cache_write_rope, which come before anything touches the GPU."""
import pytest

import paper_2607_21599_amd as daf
from test_cache_checks import ALIGN, FAKE, INVALID, UNSUPPORTED, _cache, _cfg, _status

GOOD = dict(cfg=None, cache=None, layer=1, rows=None, theta=1e6, q=FAKE, q_stride=28 * 128, k=FAKE, v=FAKE,
            kv_stride=512, q_out=2 * FAKE, stream=0)


def _args(**change):
    a = dict(GOOD, cfg=_cfg(), cache=_cache(), rows=daf.CacheRows([0, 3, 8]))
    a.update(change)
    return a.values()


@pytest.mark.parametrize("change,status", [
    (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(theta=0.0), INVALID), (dict(theta=-1.0), INVALID),
    (dict(theta=float("nan")), INVALID), (dict(theta=float("inf")), INVALID), (dict(q=None), INVALID),
    (dict(q_out=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(q_stride=28 * 128 - 8), INVALID),
    (dict(kv_stride=504), INVALID), (dict(kv_stride=-512), INVALID), (dict(kv_stride=516), ALIGN),
    (dict(q_stride=28 * 128 + 4), ALIGN), (dict(q=FAKE + 8), ALIGN), (dict(k=FAKE + 8), ALIGN), (dict(v=FAKE + 8), ALIGN),
    (dict(q_out=FAKE + 8), ALIGN), (dict(q_out=FAKE, q_stride=6000), INVALID), (dict(kv_stride=1 << 40), UNSUPPORTED)])
def test_bad_calls(change, status):
    assert _status(daf.daf_cache_write_rope, *_args(**change)) == status


def test_bad_cfg_cache_and_rows():
    for change, status in ((dict(cfg=_cfg(head_dim=64)), INVALID), (dict(cfg=_cfg(dtype=5)), UNSUPPORTED),
                           (dict(cache=_cache(n_pages=0)), INVALID), (dict(cache=_cache(k=FAKE + 8)), ALIGN),
                           (dict(rows=daf.CacheRows([0, 5, 3])), INVALID), (dict(rows=daf.CacheRows([1, 5])), INVALID)):
        assert _status(daf.daf_cache_write_rope, *_args(**change)) == status
    wide = [0, (1 << 31) - 1]  # more workgroups than a launch takes
    assert _status(daf.daf_cache_write_rope, *_args(rows=daf.CacheRows(wide, None, FAKE))) == UNSUPPORTED


def test_no_rows_are_no_work():
    daf.daf_cache_write_rope(*_args(rows=daf.CacheRows([0, 0]), q=None, q_out=None, k=None, v=None))

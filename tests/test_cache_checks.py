"""CPU: the paged cache's plain implementation, and the calls' refusals, which come
before anything touches the GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2607_21599_amd as daf
from oracle.cache import CacheOracle, e4m3, scale_for

FAKE = 0x10000  # an aligned non-null address; never dereferenced on these paths


def _cfg(**kw):
    return daf.AttnCfg(**dict(dict(n_q_heads=28, n_kv_heads=4, head_dim=128), **kw))


def _cache(**kw):
    a = dict(n_layers=2, n_pages=10, n_kv_heads=4, head_dim=128, n_seqs=3, max_seq_pages=5, k=FAKE, v=FAKE,
             k_scale=FAKE, v_scale=FAKE, table=FAKE, len=FAKE, refs=FAKE)
    a.update(kw)
    return daf.Cache(*a.values())


def _status(fn, *args):
    with pytest.raises(daf.DafError) as e:
        fn(*args)
    assert daf.daf_last_error()
    return e.value.status


INVALID, ALIGN, UNSUPPORTED, WORKSPACE = (daf.DAF_ERR_INVALID_ARG, daf.DAF_ERR_ALIGNMENT, daf.DAF_ERR_UNSUPPORTED,
                                          daf.DAF_ERR_WORKSPACE)
ROWS = daf.CacheRows([0, 3, 8])
BIG = 1 << 30


def _calls(cfg, c, rows=ROWS):
    """Every call with good arguments otherwise."""
    yield daf.daf_cache_write, (cfg, c, 0, rows, FAKE, FAKE, 0)
    yield daf.daf_cache_read, (cfg, c, 0, rows, FAKE, FAKE, 0)
    yield daf.daf_cache_attn, (cfg, c, 0, rows, 100, FAKE, FAKE, FAKE, FAKE, BIG, 0)


def _page_calls(c):
    yield daf.daf_pages_extend, (c, 1, FAKE, FAKE, FAKE, 0)
    yield daf.daf_pages_fork, (c, 1, FAKE, FAKE, FAKE, FAKE, BIG, 0)
    yield daf.daf_pages_unshare, (c, ROWS, FAKE, FAKE, BIG, 0)
    yield daf.daf_pages_free, (c, 1, FAKE, 0)
    yield daf.daf_pages_copy, (c, 1, FAKE, FAKE, 0)
    yield daf.daf_pages_compact, (c, FAKE, FAKE, BIG, 0)


@pytest.mark.parametrize("change,status", [
    (dict(n_layers=0), INVALID), (dict(n_pages=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(n_seqs=-1), INVALID),
    (dict(max_seq_pages=0), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(n_kv_heads=2000), UNSUPPORTED),
    (dict(max_seq_pages=1 << 25), UNSUPPORTED),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k_scale=None), INVALID), (dict(v_scale=None), INVALID),
    (dict(table=None), INVALID), (dict(len=None), INVALID), (dict(refs=None), INVALID),
    (dict(k=FAKE + 8), ALIGN), (dict(v_scale=FAKE + 4), ALIGN), (dict(table=FAKE + 4), ALIGN),
    (dict(len=FAKE + 4), ALIGN), (dict(refs=FAKE + 4), ALIGN)])
def test_bad_caches(change, status):
    c = _cache(**change)
    for fn, args in [*_calls(_cfg(), c), *_page_calls(c)]:
        assert _status(fn, *args) == status, fn.__name__
    assert daf.daf_pages_workspace_size(c) == 0
    assert daf.daf_cache_attn_workspace_size(_cfg(), c, ROWS, 300) == 0


@pytest.mark.parametrize("cfg,status", [
    (dict(n_kv_heads=2), INVALID), (dict(head_dim=64), INVALID), (dict(n_q_heads=30), INVALID),
    (dict(n_q_heads=2048), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(softmax_scale=float("inf")), INVALID),
    (dict(softmax_scale=-1.0), INVALID)])
def test_configurations_that_do_not_fit(cfg, status):
    for fn, args in _calls(_cfg(**cfg), _cache()):
        assert _status(fn, *args) == status, fn.__name__


def test_bad_rows():
    c = _cache()
    for rows, status in [(daf.CacheRows([1, 3]), INVALID), (daf.CacheRows([0, 3, 2]), INVALID),
                         (daf.CacheRows([0, 3], FAKE + 4), ALIGN), (daf.CacheRows([0, 3], None, FAKE + 8), ALIGN)]:
        for fn, args in [*_calls(_cfg(), c, rows), (daf.daf_pages_unshare, (c, rows, FAKE, FAKE, BIG, 0))]:
            assert _status(fn, *args) == status, fn.__name__
    bad = daf.CacheRows([0, 1])
    bad.n = -1
    none = daf.CacheRows([0, 1])
    none.cu = ctypes.POINTER(ctypes.c_int32)()
    for rows in (bad, none):
        for fn, args in _calls(_cfg(), c, rows):
            assert _status(fn, *args) == INVALID
    many = daf.CacheRows(np.arange(258))
    assert _status(daf.daf_pages_unshare, c, many, FAKE, FAKE, BIG, 0) == UNSUPPORTED


def test_bad_arguments():
    c, cfg = _cache(), _cfg()
    for layer in (-1, 2):
        for fn, args in _calls(cfg, c):
            assert _status(fn, args[0], args[1], layer, *args[3:]) == INVALID
    assert _status(daf.daf_cache_write, cfg, c, 0, ROWS, None, FAKE, 0) == INVALID
    assert _status(daf.daf_cache_write, cfg, c, 0, ROWS, FAKE, FAKE + 2, 0) == ALIGN
    assert _status(daf.daf_cache_read, cfg, c, 0, ROWS, FAKE + 2, None, 0) == ALIGN
    attn = daf.daf_cache_attn
    assert _status(attn, cfg, c, 0, ROWS, -1, FAKE, FAKE, None, FAKE, BIG, 0) == INVALID
    assert _status(attn, cfg, c, 0, ROWS, 321, FAKE, FAKE, None, FAKE, BIG, 0) == INVALID
    assert _status(attn, cfg, c, 0, ROWS, 320, None, FAKE, None, FAKE, BIG, 0) == INVALID
    assert _status(attn, cfg, c, 0, ROWS, 320, FAKE, None, None, FAKE, BIG, 0) == INVALID
    assert _status(attn, cfg, c, 0, ROWS, 320, FAKE, FAKE, FAKE + 4, FAKE, BIG, 0) == ALIGN
    assert _status(attn, cfg, c, 0, daf.CacheRows([0, 2 ** 31 - 1]), 64, FAKE, FAKE, None, FAKE, BIG, 0) == UNSUPPORTED
    wide = _cache(n_kv_heads=1024)
    for fn in (daf.daf_cache_write, daf.daf_cache_read):
        assert _status(fn, _cfg(n_q_heads=1024, n_kv_heads=1024), wide, 0, daf.CacheRows([0, 2 ** 31 - 1]), FAKE, FAKE,
                       0) == UNSUPPORTED
    long = _cache(max_seq_pages=2048)
    # 2^25 workgroups of 256: more threads than a launch has
    assert _status(attn, cfg, long, 0, daf.CacheRows([0, 2 ** 31 // cfg.n_q_heads - 1]), 131072, FAKE, FAKE, None, FAKE,
                   2 ** 62, 0) == UNSUPPORTED
    assert _status(daf.daf_pages_free, c, 2 ** 23 + 1, FAKE, 0) == UNSUPPORTED
    one = daf.CacheRows([0, 1])
    need = daf.daf_cache_attn_workspace_size(cfg, long, one, 131072)
    assert need > 0
    for ws, size, status in [(None, need, WORKSPACE), (FAKE, need - 1, WORKSPACE), (FAKE + 4, need, ALIGN)]:
        assert _status(attn, cfg, long, 0, one, 131072, FAKE, FAKE, None, ws, size, 0) == status
    need = daf.daf_pages_workspace_size(c)
    for ws, size, status in [(None, need, WORKSPACE), (FAKE, need - 1, WORKSPACE), (FAKE + 4, need, ALIGN)]:
        assert _status(daf.daf_pages_fork, c, 1, FAKE, FAKE, FAKE, ws, size, 0) == status
        assert _status(daf.daf_pages_unshare, c, ROWS, FAKE, ws, size, 0) == status
        assert _status(daf.daf_pages_compact, c, FAKE, ws, size, 0) == status
    for n, status in [(-1, INVALID), (4097, UNSUPPORTED)]:
        assert _status(daf.daf_pages_extend, c, n, FAKE, FAKE, FAKE, 0) == status
        assert _status(daf.daf_pages_fork, c, n, FAKE, FAKE, FAKE, FAKE, BIG, 0) == status
    assert _status(daf.daf_pages_free, c, -1, FAKE, 0) == INVALID
    assert _status(daf.daf_pages_copy, c, -1, FAKE, FAKE, 0) == INVALID
    assert _status(daf.daf_pages_copy, c, 1, None, FAKE, 0) == INVALID
    assert _status(daf.daf_pages_fork, c, 1, FAKE, None, FAKE, FAKE, BIG, 0) == INVALID
    assert _status(daf.daf_pages_extend, c, 1, FAKE, FAKE, None, 0) == INVALID
    assert _status(daf.daf_pages_extend, c, 1, FAKE + 4, FAKE, FAKE, 0) == ALIGN
    assert _status(daf.daf_pages_compact, c, None, FAKE, BIG, 0) == INVALID
    assert daf.lib().daf_cache_write(None, None, 0, None, None, None, None) == INVALID
    assert daf.lib().daf_cache_attn(None, None, 0, None, 0, None, None, None, None, 0, None) == INVALID
    assert daf.lib().daf_pages_extend(None, 0, None, None, None, None) == INVALID


def test_nothing_to_do_is_no_error():
    c, cfg = _cache(), _cfg()
    none = daf.CacheRows([0, 0, 0])
    daf.daf_cache_write(cfg, c, 0, none, None, None, 0)
    daf.daf_cache_read(cfg, c, 0, none, None, None, 0)
    daf.daf_cache_read(cfg, c, 0, ROWS, None, None, 0)
    daf.daf_cache_attn(cfg, c, 0, none, 320, None, None, None, None, 0, 0)
    assert daf.daf_cache_attn_workspace_size(cfg, c, none, 320) == 0
    daf.daf_pages_free(c, 0, None, 0)
    daf.daf_pages_copy(c, 0, None, None, 0)


def test_cache_of_tensors():
    from paper_2607_21599_amd.tensors import cache_tensors
    t = cache_tensors(2, 6, 3, 128, 4, 5, device="cpu")
    c = daf.Cache.from_tensors(t)
    assert (c.n_layers, c.n_pages, c.n_kv_heads, c.head_dim, c.n_seqs, c.max_seq_pages) == (2, 6, 3, 128, 4, 5)
    assert (t["table"] == -1).all() and not t["len"].any() and not t["refs"].any()
    for name, x in [("v", t["k"]), ("refs", t["refs"][:5]), ("k_scale", t["k_scale"].double()),
                    ("table", t["table"].t()), ("k", t["k"][:, ::2])]:
        with pytest.raises(ValueError):
            daf.Cache.from_tensors(dict(t, **{name: x}))


def test_e4m3_of_the_plain_form():
    """Against torch's conversion over every code and the borders between them."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    codes = codes[codes.isfinite()]
    v = codes.sort().values
    mid = (v[1:] + v[:-1]) / 2
    for x in (v, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20)):
        want = x.float().to(torch.float8_e4m3fn).double().numpy()
        assert np.array_equal(e4m3(x.float().double().numpy()), want)


def test_scale_of_the_plain_form():
    for top, want in [(0, 0), (448, 1), (448.0001, 2), (1, 2.0 ** -8), (0.875, 2.0 ** -9), (1e-38, 2.0 ** -100),
                      (3.4e38, 2.0 ** 120), (449 * 2.0 ** 50, 2.0 ** 51)]:
        assert scale_for(top) == want


def test_plain_cache_by_hand():
    o = CacheOracle(1, 5, 1, 2, 3, 3)
    assert o.extend([1, 0], [65, 1]) == 0 and o.table[1].tolist() == [0, 1, -1] and o.table[0, 0] == 2
    assert o.fork([1], [2]) == 0 and o.table[2].tolist() == [0, 3, -1] and o.refs.tolist() == [2, 1, 1, 1, 0]
    k = np.arange(130.0).reshape(65, 1, 2)
    o.write(0, [0, 65], [1], None, k, -k, 1e38)
    assert o.scale["k"][0, 0, 0] == 0.5 and o.scale["k"][0, 1, 0] == 0.5
    assert o.read(0, [0, 2], [1], [3, 64])[0].tolist() == [[[6, 7]], [[128, 128]]]
    x = o.attn(0, [0, 1], [1], [1], np.zeros((1, 1, 2)), 1.0)
    assert x[0].tolist() == [[[-1, -2]]] and np.isclose(x[1][0, 0], np.log(2))
    assert o.unshare([0, 1], [2], [5]) == 0 and o.table[2, 0] == 4 and o.refs.tolist() == [1, 1, 1, 1, 1]
    o.free([1])
    assert o.compact() == 3 and o.table[2].tolist() == [1, 0, -1] and o.table[0, 0] == 2 and o.len.tolist() == [1, 0, 65]

"""GPU: daf_cache_write_rope against the rotation in 64 bits and oracle/cache.py."""
from __future__ import annotations

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import paper_2607_21599_amd as daf
    daf.lib()
    yield
    torch.cuda.synchronize()


def _cu(n):
    return [0] + np.cumsum(n).tolist()


def _turned(x, at, theta):
    """x [rows][heads][d] float64 at positions `at`; and the magnitudes that went into each value."""
    half = x.shape[-1] // 2
    angle = np.asarray(at, np.float64)[:, None] * float(theta) ** (-2.0 * np.arange(half) / (2 * half))
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = x[..., :half], x[..., half:]
    size = np.abs(a) + np.abs(b)
    return np.concatenate([a * c - b * s, b * c + a * s], -1), np.concatenate([size, size], -1)


def _call(p, theta, layer, cu, seq, q, k, v, pos=None, joint=True, stream=None, in_place=False):
    """q, k, v: tensors of p.dtype on the GPU, [rows][heads][d]; joint: as parts of one row with a gap behind it."""
    import paper_2607_21599_amd as daf
    from cache_pair import dev
    n, d = k.shape[0], p.d
    rows = daf.CacheRows(cu, None if seq is None else dev(seq), None if pos is None else dev(pos))
    out = torch.full((n + 1, p.hq, d), 77.0, dtype=p.dtype, device="cuda")
    if joint:
        pitch = (p.hq + 2 * p.heads) * d + 8
        row = torch.full((n, pitch), torch.nan, dtype=p.dtype, device="cuda")
        row[:, :-8] = torch.cat([q.reshape(n, -1), k.reshape(n, -1), v.reshape(n, -1)], 1)
        q, k, v = row[:, :p.hq * d], row[:, p.hq * d:(p.hq + p.heads) * d], row[:, (p.hq + p.heads) * d:]
        qs = ks = pitch
    else:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        qs, ks = p.hq * d, p.heads * d
        if in_place:
            out[:n] = q
            q = out
    daf.daf_cache_write_rope(p.cfg, p.c, layer, rows, theta, q, qs, k, v, ks, out, stream)
    torch.cuda.synchronize()
    assert (out[n] == 77).all()
    return out[:n]


def _positions(p, cu, seq, pos):
    at = np.zeros(cu[-1], np.int64)
    for b in range(len(cu) - 1):
        n, L = cu[b + 1] - cu[b], int(p.o.len[seq[b]]) if 0 <= seq[b] < len(p.o.len) else 0
        at[cu[b]:cu[b + 1]] = np.arange(L - n, L) if pos is None else pos[cu[b]:cu[b + 1]]
    return at


def _check_q(p, out, q, at, theta):
    """Two fp32 products and a sum of turned values, sines of half a step: 4 roundings of 2^-24 of the
    magnitudes; the fp64 angle's error is below 2^-24 for positions below 2^21. Then the output's."""
    from cache_pair import f64
    want, size = _turned(f64(q), at, theta)
    half = 2.0 ** -8 if p.dtype == BF16 else 2.0 ** -24
    tol = 6 * 2.0 ** -24 * size * (1 + half) + half * np.abs(want)
    err = np.abs(f64(out) - want)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())


def _write(p, theta, layer, cu, seq, q, k, v, pos=None, **kw):
    """The call on both caches, and their comparison: V and what lies beside the new rows bit for bit, K
    within the rotation's fp32 error of half a step of its code."""
    from cache_pair import MOST, f64
    out = _call(p, theta, layer, cu, seq, q, k, v, pos, **kw)
    at = _positions(p, cu, seq, pos)
    _check_q(p, out, q, at, theta)
    want, size = _turned(f64(k), at, theta)
    inside = [b for b in range(len(cu) - 1) if 0 <= seq[b] < len(p.o.len)]
    for b in inside:  # one request at a time: the oracle takes those of sequences that exist
        lo, hi = cu[b], cu[b + 1]
        p.o.write(layer, [0, hi - lo], [seq[b]], None if pos is None else pos[lo:hi], want[lo:hi], f64(v)[lo:hi],
                  MOST[F32])
    for n in "kv":
        assert np.array_equal(f64(p.t[n + "_scale"]), p.o.scale[n]), n
    code = {n: f64(p.t[n].float()) for n in "kv"}
    assert np.array_equal(code["v"].swapaxes(-1, -2), p.o.code["v"], equal_nan=True)
    differ = code["k"] != p.o.code["k"]
    for b in inside:
        for i in range(cu[b], cu[b + 1]):
            page = p.o.page(seq[b], at[i] // 64) if 0 <= at[i] < p.o.len[seq[b]] else None
            if page is None:
                continue
            scale = p.o.scale["k"][layer, page][:, None]
            with np.errstate(divide="ignore", invalid="ignore"):
                x, e = np.where(scale > 0, want[i] / scale, 0), np.where(scale > 0, size[i] / scale, 0) * 6 * 2.0 ** -24
            step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(x) + e, 2.0 ** -6))), -6) - 3)
            got = code["k"][layer, page, :, at[i] % 64]
            assert (np.abs(got - x) <= step / 2 + e).all()
            differ[layer, page, :, at[i] % 64] = False
    assert not differ.any(), "codes beside the new rows"
    # the oracle follows what was rounded the other way, so that later writes compare
    p.o.code["k"] = code["k"]
    return out


def _pair(**kw):
    from cache_pair import Pair
    return Pair(**kw)


def _rows(rng, p, n, size=1.0):
    def one(heads):
        x = rng.standard_normal((n, heads, p.d)) * size * np.exp2(rng.integers(-3, 4, (n, 1, 1)))
        return torch.from_numpy(x).to(p.dtype).cuda()
    return one(p.hq), one(p.heads), one(p.heads)


CFGS = [(BF16, 128, 4, 28), (BF16, 64, 1, 4), (F32, 64, 3, 6), (F32, 128, 2, 2)]


@pytest.mark.parametrize("dtype,d,heads,hq", CFGS)
@pytest.mark.parametrize("joint", [True, False])
def test_appends_of_every_length(dtype, d, heads, hq, joint):
    p = _pair(layers=2, pages=40, heads=heads, hq=hq, d=d, n_seqs=5, max_seq_pages=10, dtype=dtype)
    rng = np.random.default_rng(d + heads)
    seq = [3, 0, 4]
    for step, n in enumerate([(1, 63, 0), (64, 1, 129), (0, 65, 7), (200, 2, 1), (1, 1, 1)]):
        assert p.extend(seq, n) == 0
        for la in (1, 0):
            _write(p, 1e4, la, _cu(n), seq, *_rows(rng, p, sum(n), 2.0 ** step), joint=joint)


@pytest.mark.parametrize("dtype,d,heads,hq", CFGS)
@pytest.mark.parametrize("share", [0.02, 0.3, 1.0])
def test_rows_at_positions(dtype, d, heads, hq, share):
    p = _pair(pages=24, heads=heads, hq=hq, d=d, n_seqs=3, max_seq_pages=9, dtype=dtype)
    rng = np.random.default_rng(int(share * 100) + d)
    seq, lens = [2, 0], [517, 300]
    assert p.extend(seq, lens) == 0
    _write(p, 1e6, 0, _cu(lens), seq, *_rows(rng, p, sum(lens)))
    for size in (0.1, 30.0):
        pos = [np.sort(rng.choice(n, max(1, int(n * share)), replace=False)) for n in lens]
        cu = _cu([len(x) for x in pos])
        _write(p, 1e6, 0, cu, seq, *_rows(rng, p, cu[-1], size), np.concatenate(pos), joint=size < 1, in_place=size > 1)


def test_position_zero_is_daf_cache_write():
    """No rotation: the bits of K, V and the scales, and q itself."""
    for dtype, d in ((BF16, 128), (F32, 64)):
        a, b = (_pair(pages=6, heads=2, hq=4, d=d, n_seqs=4, dtype=dtype) for _ in range(2))
        rng = np.random.default_rng(d)
        for x in (a, b):
            assert x.extend([0, 1, 2], [1, 1, 1]) == 0
        q, k, v = _rows(rng, a, 3)
        out = _call(a, 1e6, 0, [0, 1, 2, 3], None, q, k, v)
        b.write(0, [0, 1, 2, 3], [0, 1, 2], k.float().cpu(), v.float().cpu())
        assert torch.equal(out, q)
        for n in ("k", "v", "k_scale", "v_scale"):
            assert torch.equal(a.t[n].view(torch.uint8), b.t[n].view(torch.uint8)), n


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_far_positions(dtype):
    """Around 2^20 and 2,000,000, in sequences whose other pages are not there."""
    p = _pair(pages=8, heads=2, hq=4, d=128, n_seqs=2, max_seq_pages=32768, dtype=dtype)
    lens, rng = [2_000_001, (1 << 20) + 5], np.random.default_rng(1)
    for s, L in enumerate(lens):
        for i in range(2):
            pg = (L - 1) // 64 - i
            p.o.table[s, pg] = 2 * s + i
            p.t["table"][s, pg] = 2 * s + i
        p.o.len[s] = L
        p.t["len"][s] = L
    for theta in (1e4, 1e6, 1.0, 0.5):
        _write(p, theta, 0, [0, 70, 130], [0, 1], *_rows(rng, p, 130))
    pos = np.array([5, 1_999_990, 2_000_000, 0, (1 << 20) + 1])  # 5 and 0: their pages are not there
    _write(p, 1e6, 0, [0, 3, 5], [0, 1], *_rows(rng, p, 5), pos)


def test_rows_that_go_nowhere():
    """Before the sequence's start, positions outside, sequences out of range: the cache stays, q is turned."""
    p = _pair(pages=6, heads=1, hq=3, d=64, n_seqs=2, max_seq_pages=3)
    rng = np.random.default_rng(3)
    assert p.extend([0, 1], [70, 3]) == 0
    _write(p, 1e4, 0, [0, 70, 73], [0, 1], *_rows(rng, p, 73))
    before = {n: p.t[n].clone() for n in ("k", "v", "k_scale", "v_scale")}
    at = np.array([-70, -1, 70, 500, 2, 9])
    _write(p, 1e4, 0, [0, 4, 6], [0, 7], *_rows(rng, p, 6), at)
    for n, x in before.items():
        assert torch.equal(p.t[n].view(torch.uint8), x.view(torch.uint8)), n
    _write(p, 1e4, 0, [0, 9, 9, 12], [1, -1, 0], *_rows(rng, p, 12))  # more rows than tokens
    _write(p, 1e4, 0, [0, 5], [-1], *_rows(rng, p, 5))


def test_infinities_and_nan_of_k():
    p = _pair(pages=4, heads=1, hq=1, d=64, n_seqs=1, max_seq_pages=3)
    assert p.extend([0], [3]) == 0
    k = torch.ones(3, 1, 64, dtype=BF16, device="cuda")
    k[0, 0, 5], k[1, 0, 7], k[2, 0, 40] = torch.nan, torch.inf, -torch.inf
    q = torch.ones(3, 1, 64, dtype=BF16, device="cuda")
    _call(p, 1e4, 0, [0, 3], [0], q, k, q)
    page = int(p.t["table"][0, 0])
    code = p.t["k"][0, page, 0].float()
    assert code[0, 5].isnan() and code[0, 37].isnan() and int(code[0].isnan().sum()) == 2
    # position 1, angle 1 * theta^(-7/32) in the first quarter: infinite, as the largest finite value
    assert code[1, 7] == 256 and code[1, 39] == 256 and float(p.t["k_scale"][0, page, 0]) == 2.0 ** 120
    # position 2, angle 2 * theta^(-8/32) = 0.2 of -infinity in the upper half: + sine, - cosine
    assert code[2, 8] == 256 and code[2, 40] == -256


def test_more_requests_than_a_launch_takes():
    p = _pair(pages=700, heads=1, hq=2, d=64, n_seqs=600, max_seq_pages=2)
    rng = np.random.default_rng(4)
    n = [1 + i % 3 for i in range(600)]
    assert p.extend(list(range(600)), n) == 0
    _write(p, 1e4, 0, _cu(n), list(range(600)), *_rows(rng, p, sum(n)))


def test_keys_and_values_alone():
    import paper_2607_21599_amd as daf
    a, b = (_pair(pages=6, heads=2, hq=4, d=128, n_seqs=2) for _ in range(2))
    rng = np.random.default_rng(5)
    for x in (a, b):
        assert x.extend([1], [90]) == 0
    q, k, v = _rows(rng, a, 90)
    _call(a, 1e4, 0, [0, 90], [1], q, k, v)
    from cache_pair import dev
    daf.daf_cache_write_rope(b.cfg, b.c, 0, daf.CacheRows([0, 90], dev([1])), 1e4, None, 0, k, v, 256, None)
    for n in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(a.t[n].view(torch.uint8), b.t[n].view(torch.uint8)), n


def test_a_graph_follows_the_lengths():
    """A captured append, replayed after each extend, as a decode loop has it."""
    import paper_2607_21599_amd as daf
    from cache_pair import dev
    a, b = (_pair(pages=12, heads=2, hq=4, d=128, n_seqs=3) for _ in range(2))
    rng = np.random.default_rng(6)
    for x in (a, b):
        assert x.extend([0, 1, 2], [60, 1, 130]) == 0
    start = _rows(rng, a, 191)
    for x in (a, b):
        _call(x, 1e4, 0, [0, 60, 61, 191], [0, 1, 2], *start)
    q, k, v = (torch.zeros(3, h, 128, dtype=BF16, device="cuda") for h in (4, 2, 2))
    out, seq, rows = torch.zeros_like(q), dev([0, 1, 2]), [0, 1, 2, 3]
    cr = daf.CacheRows(rows, seq)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        daf.daf_cache_write_rope(a.cfg, a.c, 0, cr, 1e4, q, 512, k, v, 256, out)
    for _ in range(6):
        new = _rows(rng, a, 3)
        for x in (a, b):
            assert x.extend([0, 1, 2], [1, 1, 1]) == 0
        for to, x in zip((q, k, v), new):
            to.copy_(x)
        out.fill_(9)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, _call(b, 1e4, 0, rows, [0, 1, 2], *new))
        for n in ("k", "v", "k_scale", "v_scale"):
            assert torch.equal(a.t[n].view(torch.uint8), b.t[n].view(torch.uint8)), n

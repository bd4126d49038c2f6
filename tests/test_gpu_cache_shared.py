"""GPU: attention of groups that share their first pages (daf_cache_attn_shared) against
oracle/cache.py (64 bits) and daf_cache_attn."""
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


def _pair(**kw):
    from cache_pair import Pair
    return Pair(**kw)


def _rows(rng, n, heads, d, size=1.0):
    x = rng.standard_normal((n, heads, d)) * size
    x *= np.exp2(rng.integers(-3, 4, (n, 1, 1)))
    return torch.from_numpy(x).float()


def _cu(n):
    return [0] + np.cumsum(n).tolist()


def _forked(groups, shared, tails, hq, heads, d, dtype, seed=0, layers=1, size=1.0):
    """A cache in which the sequences of each group share their first pages, as forks of a
    prefix that are then lengthened; the sequences in the order of the requests."""
    n = sum(groups)
    lens = [s + t for s, t in zip(np.repeat(shared, groups).tolist(), tails)]
    pages = sum(-(-x // 64) for x in lens) + sum(-(-s // 64) for s in shared) + len(groups) + 4
    p = _pair(layers=layers, pages=pages, heads=heads, d=d, n_seqs=n + len(groups), max_seq_pages=max(lens) // 64 + 2,
              hq=hq, dtype=dtype)
    rng = np.random.default_rng(seed)
    order = rng.permutation(n + len(groups)).tolist()
    seq, stems = order[:n], order[n:]

    def write(which, m):
        cu = _cu(m)
        for la in range(layers):
            p.write(la, cu, which, _rows(rng, cu[-1], heads, d, size), _rows(rng, cu[-1], heads, d, size))

    assert p.extend(stems, shared) == 0
    write(stems, shared)
    assert p.fork(np.repeat(stems, groups).tolist(), seq) == 0
    assert p.extend(seq, tails) == 0
    write(seq, tails)
    return p, rng, seq, lens


def _attn(p, layer, cu, seq, q, groups, shared, pos=None, max_len=None, lse=True, stream=None, ws_fill=0xFF):
    import paper_2607_21599_amd as daf
    from cache_pair import dev
    max_len = p.t["table"].shape[1] * 64 if max_len is None else max_len
    rows = daf.CacheRows(cu, None if seq is None else dev(seq), None if pos is None else dev(pos))
    g = daf.CacheGroups(_cu(groups), shared)
    whole = torch.full((q.shape[0] + 1, *q.shape[1:]), 77.0, dtype=p.dtype, device="cuda")
    le = torch.full((p.hq, q.shape[0]), 77.0, device="cuda") if lse else None
    size = daf.daf_cache_attn_shared_workspace_size(p.cfg, p.c, rows, g, max_len)
    ws = torch.full((max(size, 16),), ws_fill, dtype=torch.uint8, device="cuda")  # NaN in every word
    daf.daf_cache_attn_shared(p.cfg, p.c, layer, rows, g, max_len, q, whole, le, ws, size, stream)
    torch.cuda.synchronize()
    assert (whole[-1] == 77).all()
    return whole[:-1], le


def _check(p, layer, cu, seq, groups, shared, pos=None, max_len=None, seed=1):
    gen = torch.Generator().manual_seed(seed)
    q = torch.randn(cu[-1], p.hq, p.d, generator=gen).to(p.dtype)
    o, lse = _attn(p, layer, cu, seq, q.cuda(), groups, shared, pos, max_len)
    p.within_bounds(o, lse, layer, cu, seq, q, pos)
    return o, lse


CFGS = [(BF16, 128, 28, 4), (BF16, 64, 6, 1), (F32, 128, 4, 2), (F32, 64, 16, 16)]


@pytest.mark.parametrize("dtype,d,hq,heads", CFGS)
@pytest.mark.parametrize("far", [0, 2112])  # few pages go daf_cache_attn's way
@pytest.mark.parametrize("groups,shared", [
    ([2], [64]), ([5], [130]), ([3, 1, 4], [640, 200, 63]), ([1, 1, 1], [500, 64, 0]), ([12], [1500]),
    ([2, 9, 2], [64, 1, 900])])
def test_decode_steps(dtype, d, hq, heads, groups, shared, far):
    n, shared = sum(groups), [s + far for s in shared]
    rng = np.random.default_rng(n)
    tails = rng.integers(1, 200, n).tolist()
    p, _, seq, lens = _forked(groups, shared, tails, hq, heads, d, dtype)
    _check(p, 0, list(range(n + 1)), seq, groups, shared)
    _check(p, 0, list(range(n + 1)), seq, groups, shared, max_len=max(lens))
    # a promise of fewer common tokens, or of none, and rows beyond those of the sequences
    _check(p, 0, list(range(n + 1)), seq, groups, [s - s // 8 for s in shared])
    _check(p, 0, list(range(n + 1)), seq, groups, [0] * len(groups))


@pytest.mark.parametrize("dtype,d,hq,heads", CFGS)
@pytest.mark.parametrize("shared,nq", [(2200, [40, 1, 7, 0, 64]), (2300, [3, 2, 1, 20, 5]), (2176, [0, 0, 130, 0, 1]),
                                       (128, [0, 0, 130, 0, 1])])
def test_questions(dtype, d, hq, heads, shared, nq):
    """Several rows per request, some with none; some rows lie before the shared pages' end."""
    tails = [max(n - 3, 0) for n in nq]
    p, _, seq, _ = _forked([5], [shared], tails, hq, heads, d, dtype, seed=2)
    _check(p, 0, _cu(nq), seq, [5], [shared])


@pytest.mark.parametrize("dtype,d,hq,heads,groups,shared,nq", [
    (BF16, 128, 28, 4, [3], [2200], [60, 50, 64]),                       # a few partial results of each row
    (F32, 128, 16, 16, [3, 2], [4416, 200], [60, 64, 40, 50, 51]),       # more of them
    (BF16, 64, 16, 16, [2, 4], [3200, 100], [70, 60, 40, 30, 30, 31]),
    (F32, 64, 16, 16, [2, 4], [6400, 100], [2, 2, 70, 64, 70, 64]),
    (BF16, 128, 16, 16, [2, 4], [6400, 100], [2, 2, 70, 64, 70, 64])])
def test_more_pairs_than_a_join_helps(dtype, d, hq, heads, groups, shared, nq):
    """Rows and heads that fill the device by themselves: their joins by one, two or four teams of lanes."""
    assert sum(nq) * hq >= 4096
    p, _, seq, _ = _forked(groups, shared, [n + 5 for n in nq], hq, heads, d, dtype, seed=17)
    _check(p, 0, _cu(nq), seq, groups, shared)


@pytest.mark.parametrize("dtype,d,hq,heads", CFGS)
def test_rows_at_positions(dtype, d, hq, heads):
    """Anywhere in their sequences, in no order, before the first token and past the last."""
    p, rng, seq, lens = _forked([3, 2], [2300, 700], [10, 1, 90, 200, 64], hq, heads, d, dtype, seed=3)
    nq = [9, 4, 30, 1, 12]
    pos = np.concatenate([rng.integers(-2, L + 40, n) for n, L in zip(nq, lens)])
    _check(p, 0, _cu(nq), seq, [3, 2], [2300, 700], pos)


def test_without_a_list_of_sequences():
    p, _, seq, _ = _forked([4], [2420], [5, 60, 1, 200], 28, 4, 128, BF16, seed=4)
    order = np.argsort(seq)  # request b is sequence b: move the table's rows
    for n in ("table", "len"):
        rows = p.t[n][torch.as_tensor(seq).cuda()].clone()
        p.t[n][:4] = rows
        setattr(p.o, n, np.concatenate([rows.cpu().numpy(), getattr(p.o, n)[4:]]).astype(getattr(p.o, n).dtype))
    assert len(order) == 4
    gen = torch.Generator().manual_seed(5)
    q = torch.randn(4, 28, 128, generator=gen).to(BF16)
    o, lse = _attn(p, 0, [0, 1, 2, 3, 4], None, q.cuda(), [4], [2420])
    p.within_bounds(o, lse, 0, [0, 1, 2, 3, 4], [0, 1, 2, 3], q, None)


def test_other_layers_and_no_lse():
    p, _, seq, _ = _forked([3], [2200], [7, 70, 1], 8, 2, 64, BF16, layers=3)
    for la in (2, 0):
        o, _ = _check(p, la, [0, 1, 2, 3], seq, [3], [2200])
    q = torch.randn(3, 8, 64, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    alone, _ = _attn(p, 0, [0, 1, 2, 3], seq, q, [3], [2200], lse=False)
    assert torch.equal(alone, o)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_long_tails_are_split(dtype):
    """Rests of thousands of keys beside short ones: pieces of the line."""
    p, _, seq, _ = _forked([3, 2], [2240, 64], [3000, 1, 65, 5000, 9], 8, 2, 64, dtype, seed=6)
    _check(p, 0, list(range(6)), seq, [3, 2], [2240, 64])
    _check(p, 0, _cu([5, 1, 1, 9, 2]), seq, [3, 2], [2240, 64])


def test_more_requests_than_a_launch_takes():
    """Groups on both sides of a launch's border, and one that it cuts."""
    groups, shared = [200, 100, 1, 13], [2230, 64, 10, 200]
    tails = [1 + i % 5 for i in range(sum(groups))]
    p, _, seq, _ = _forked(groups, shared, tails, 4, 1, 64, BF16, seed=7)
    _check(p, 0, list(range(len(seq) + 1)), seq, groups, shared)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("varied", [False, True])
def test_more_groups_than_lanes(dtype, varied):
    """Over a hundred groups of one to three requests, long and short prefixes, with none among them."""
    groups = [2, 1, 3] * 34
    shared = [2200 + i if i in (0, 50, 63, 64, 65, 101) else 64 * (i % 4) + i % 5 for i in range(102)]
    nq = [1 + (i % 3 if varied else 0) - (varied and i % 11 == 0) for i in range(sum(groups))]
    p, _, seq, _ = _forked(groups, shared, [3 + i % 7 for i in range(sum(groups))], 6, 1, 64, dtype, seed=18)
    _check(p, 0, _cu(nq), seq, groups, shared)


def test_sequences_and_pages_that_are_not_there():
    """Sequences out of range see nothing; pages out of range hold no keys, for the whole group."""
    p, _, seq, _ = _forked([3], [2220], [30, 5, 64], 4, 2, 64, BF16, seed=8)
    for s in seq:
        p.t["table"][s, 2] = p.o.table[s, 2] = -1
        p.t["table"][s, 4] = p.o.table[s, 4] = 10 ** 6
    _check(p, 0, [0, 1, 2, 3], seq, [3], [2220])
    q = torch.randn(3, 4, 64, generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    bad = list(seq)
    bad[1] = 99
    o, lse = _attn(p, 0, [0, 1, 2, 3], bad, q, [3], [2220])
    good, good_lse = _attn(p, 0, [0, 1, 2, 3], seq, q, [3], [2220])
    assert torch.equal(o[[0, 2]], good[[0, 2]]) and (o[1] == 0).all() and (lse[:, 1] == -torch.inf).all()
    assert torch.equal(lse[:, [0, 2]], good_lse[:, [0, 2]])
    # the group's pages are those of its first sequence: without it they are not there
    bad = [-5] + seq[1:]
    o, lse = _attn(p, 0, [0, 1, 2, 3], bad, q, [3], [2220])
    assert (o[0] == 0).all() and (lse[:, 0] == -torch.inf).all()
    assert o.isfinite().all() and not lse.isnan().any()


@pytest.mark.parametrize("n", [5, 70])
def test_padded_groups(n):
    """Requests whose sequence is out of range, with and without rows, at a group's head: the others read the
    group's pages as if it were not there."""
    p, _, seq, _ = _forked([n], [2300], [1 + i % 70 for i in range(n)], 4, 2, 64, BF16, seed=16)
    q = torch.randn(n, 4, 64, generator=torch.Generator().manual_seed(6)).to(BF16).cuda()
    cu = list(range(n + 1))
    good, good_lse = _attn(p, 0, cu, seq, q, [n], [2300])
    for gone in ([0], [0, 1], list(range(n - 1))):
        bad = [(-1 if i % 2 else 1 << 30) if i in gone else x for i, x in enumerate(seq)]
        o, lse = _attn(p, 0, cu, bad, q, [n], [2300])
        assert (o[:len(gone)] == 0).all() and (lse[:, :len(gone)] == -torch.inf).all()
        assert torch.equal(o[len(gone):], good[len(gone):]) and torch.equal(lse[:, len(gone):], good_lse[:, len(gone):])
    # the first has no rows either
    nq = [0] + [1] * (n - 1)
    want, want_lse = _attn(p, 0, _cu(nq), seq, q[1:].contiguous(), [n], [2300])
    o, lse = _attn(p, 0, _cu(nq), [-1] + seq[1:], q[1:].contiguous(), [n], [2300])
    assert torch.equal(o, want) and torch.equal(lse, want_lse)
    # none is there
    o, lse = _attn(p, 0, cu, [-1] * n, q, [n], [2300])
    assert (o == 0).all() and (lse == -torch.inf).all()


def test_empty_sequences_and_rows_without_keys():
    p = _pair(pages=8, heads=1, hq=4, d=64, n_seqs=4, max_seq_pages=60)
    q = torch.randn(9, 4, 64, generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    o, lse = _attn(p, 0, [0, 3, 6, 9], [0, 1, 2], q, [3], [2656])
    assert (o == 0).all() and (lse == -torch.inf).all()


def test_nan_beside_the_keys_and_nan_scores():
    """NaN codes that no row sees stay out; a NaN in q stays in its row and head."""
    p, _, seq, lens = _forked([3], [2112], [3, 70, 1], 8, 2, 64, BF16, seed=9)
    for s, L in zip(seq, lens):
        pg, slot = (L - 1) // 64, L % 64
        page = int(p.t["table"][s, pg])
        if slot:
            p.t["k"].view(torch.uint8)[:, page, :, slot:] = 0x7F
            p.t["v"].view(torch.uint8)[:, page, :, :, slot:] = 0x7F
    _check(p, 0, [0, 1, 2, 3], seq, [3], [2112])
    q = torch.randn(3, 8, 64, generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    good, good_lse = _attn(p, 0, [0, 1, 2, 3], seq, q, [3], [2112])
    q[1, 3, 5] = torch.nan
    o, lse = _attn(p, 0, [0, 1, 2, 3], seq, q, [3], [2112])
    assert o[1, 3].isnan().all() and lse[3, 1].isnan()
    keep = torch.ones(3, 8, dtype=torch.bool, device="cuda")
    keep[1, 3] = False
    assert torch.equal(o[keep], good[keep]) and torch.equal(lse.t()[keep], good_lse.t()[keep])


def test_shared_pages_that_some_rows_do_not_see():
    """Positions inside the shared pages, with NaN codes past the last row of all."""
    p, _, seq, lens = _forked([4], [2280], [1, 1, 1, 1], 28, 4, 128, BF16, seed=10)
    page = int(p.t["table"][seq[0], 5])
    p.t["k"].view(torch.uint8)[:, page, :, 40:] = 0x7F
    p.t["v"].view(torch.uint8)[:, page, :, :, 40:] = 0x7F
    at = np.array([5 * 64 + 39, 17, 0, 200])
    _check(p, 0, [0, 1, 2, 3, 4], seq, [4], [2280], at)


def test_values_of_other_sizes():
    """Scales of V far apart, so that weights take two bf16 terms."""
    for size in (1e-6, 1.0, 1e6):
        p, _, seq, _ = _forked([6], [2700], [1, 2, 3, 4, 5, 6], 28, 4, 128, BF16, seed=11, size=size)
        _check(p, 0, list(range(7)), seq, [6], [2700])


def test_scores_far_apart():
    """Rows whose maximum lies in the shared pages, in the rest, or far from all others."""
    p, _, seq, _ = _forked([3], [2400], [100, 3, 9], 4, 1, 64, F32, seed=12, size=4.0)
    _check(p, 0, [0, 1, 2, 3], seq, [3], [2400])


def test_as_daf_cache_attn():
    """The same rows without groups: both within half a step of the output and the sums' roundings of the exact
    result, so within twice that of each other; lse to the last bits of fp32."""
    import paper_2607_21599_amd as daf
    from cache_pair import dev
    p, _, seq, _ = _forked([8], [2200], [1 + 9 * i for i in range(8)], 28, 4, 128, BF16, seed=13)
    q = torch.randn(8, 28, 128, generator=torch.Generator().manual_seed(3)).to(BF16).cuda()
    cu = list(range(9))
    a, al = _attn(p, 0, cu, seq, q, [8], [2200])
    b, bl = p.attn(0, cu, seq, q)
    size = b.double().abs().mean()
    assert ((a.double() - b.double()).abs() <= 2.0 ** -7 * (b.double().abs() + size)).all()
    assert ((al - bl).abs() <= 1e-4).all()
    # groups of one request and few rows are that call itself
    c, cl = _attn(p, 0, cu, seq, q, [1] * 8, [2200] * 8)
    assert torch.equal(c, b) and torch.equal(cl, bl)
    rows = daf.CacheRows(cu, dev(seq))
    top = p.t["table"].shape[1] * 64
    assert (daf.daf_cache_attn_shared_workspace_size(p.cfg, p.c, rows, daf.CacheGroups(cu, [2200] * 8), top)
            == daf.daf_cache_attn_workspace_size(p.cfg, p.c, rows, top))


def test_results_do_not_depend_on_the_workspace_or_the_stream():
    p, _, seq, _ = _forked([6, 2], [2900, 128], [1 + 40 * i for i in range(8)], 28, 4, 128, BF16, seed=14)
    q = torch.randn(8, 28, 128, generator=torch.Generator().manual_seed(4)).to(BF16).cuda()
    cu = list(range(9))
    want, want_lse = _attn(p, 0, cu, seq, q, [6, 2], [2900, 128])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for fill, stream in ((0, None), (0x7F, side), (0xFF, side)):
        o, lse = _attn(p, 0, cu, seq, q, [6, 2], [2900, 128], ws_fill=fill, stream=stream)
        assert torch.equal(o, want) and torch.equal(lse, want_lse)


def test_a_graph_follows_the_lengths():
    """A captured decode step of beams, replayed as their sequences grow over a page's end."""
    import paper_2607_21599_amd as daf
    from cache_pair import dev
    p, rng, seq, lens = _forked([4], [2300], [50, 1, 20, 60], 28, 4, 128, BF16, seed=15)
    max_len = p.t["table"].shape[1] * 64
    cu, g = [0, 1, 2, 3, 4], daf.CacheGroups([0, 4], [2300])
    rows = daf.CacheRows(cu, dev(seq))
    size = daf.daf_cache_attn_shared_workspace_size(p.cfg, p.c, rows, g, max_len)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    q = torch.randn(4, 28, 128, generator=torch.Generator().manual_seed(5)).to(BF16)
    qd, o, lse = q.cuda(), torch.zeros(4, 28, 128, dtype=BF16, device="cuda"), torch.zeros(28, 4, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        daf.daf_cache_attn_shared(p.cfg, p.c, 0, rows, g, max_len, qd, o, lse, ws, size)
    for _ in range(5):
        assert p.extend(seq, [3] * 4) == 0
        p.write(0, _cu([3] * 4), seq, _rows(rng, 12, 4, 128), _rows(rng, 12, 4, 128))
        o.fill_(9)
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        p.within_bounds(o, lse, 0, cu, seq, q, None)

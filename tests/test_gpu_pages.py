"""GPU: the page calls of the paged cache against oracle/cache.py, alone, in long
random runs, together with the rows and the attention, and in captured graphs."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from test_gpu_cache import BF16, F32, _cu, _fill, _pair, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import paper_2607_21599_amd as daf
    daf.lib()
    yield
    torch.cuda.synchronize()


def test_extend_is_all_or_nothing():
    p = _pair(pages=10, heads=1, n_seqs=5, max_seq_pages=6)
    assert p.extend([1, 3], [0, 64]) == 0
    assert p.extend([3, 0, 1], [1, 200, 63]) == 0
    p.same()
    for seq, n in [([2], [320]), ([4, 2], [130, 129])]:  # 3 pages are left
        assert p.extend(seq, n) > 0
        p.same()
    for seq, n in [([5], [1]), ([-1], [1]), ([2, 2], [1, 1]), ([2], [-1]), ([0], [185]), ([0], [2 ** 31 - 1]),
                   ([2, 4, 2 ** 30], [1, 1, 0])]:
        assert p.extend(seq, n) == -1
        p.same()
    assert p.extend([4, 2], [128, 64]) == 0  # to the last page
    assert p.extend([4], [1]) == 1
    p.same()
    assert p.extend([], []) == 0
    import paper_2607_21599_amd as daf
    p.free([4])
    daf.daf_pages_extend(p.c, 2, None, None, p.status)  # sequences 0 and 1, one token each
    assert p.o.extend([0, 1], [1, 1]) == int(p.status) == 0
    p.same()


def test_fork_shares_and_copies():
    p = _pair(layers=3, pages=22, heads=2, d=128, n_seqs=12, max_seq_pages=6)
    rng = np.random.default_rng(1)
    _fill(p, rng, [0, 1, 2], [200, 128, 1], layers=3)
    assert p.fork([0, 0, 1, 2, 3], [4, 5, 6, 7, 8]) == 0  # 3 is empty
    p.same()
    for src, dst in [([0], [4]), ([0, 1], [9, 9]), ([0, 9], [9, 10]), ([12], [9]), ([0], [-1]), ([0], [12]),
                     ([9], [9])]:
        assert p.fork(src, dst) == -1
        p.same()
    # the copies of a last page are of their own, the full pages are one
    assert p.extend([4, 0], [1, 1]) == 0
    for s in (4, 0):
        p.write(1, [0, 1], [s], _rows(rng, 1, 2, 128, 9.0), _rows(rng, 1, 2, 128, 9.0))
    p.same()
    while p.extend([9], [64]) == 0:  # use up the pool
        if p.o.len[9] == 6 * 64:
            break
    left = len(p.o.free_ids())
    assert p.extend([10], [64 * left - 40]) == 0 and not p.o.free_ids()
    assert p.fork([0, 4], [11, 3]) == 2 and p.fork([1], [11]) == 0
    p.same()
    p.free([11, 11, 0, 40, -3, 4, 5])
    p.same()
    assert p.fork([], []) == 0


def test_fork_of_a_last_page_that_is_not_there():
    p = _pair(pages=10, heads=1, d=64, n_seqs=6, max_seq_pages=3)
    _fill(p, np.random.default_rng(6), [0, 1], [130, 70])
    p.o.table[0, 2] = -1
    p.t["table"].copy_(torch.from_numpy(p.o.table).int())
    assert p.fork([0, 1, 0], [2, 3, 4]) == 0
    p.same()
    assert p.o.table[2, 2] == -1 and p.o.table[3, 1] >= 0


def test_unshare_copies_what_the_rows_touch():
    p = _pair(layers=2, pages=40, heads=3, d=64, n_seqs=8, max_seq_pages=10)
    rng = np.random.default_rng(2)
    _fill(p, rng, [0, 1], [600, 130], layers=2)
    assert p.fork([0, 0, 1], [2, 3, 4]) == 0
    pos = [0, 63, 64, 300, 301, 599, 5, 6, 129]
    assert p.unshare([0, 6, 9], [2, 4], pos) == 0
    p.same()
    assert p.unshare([0, 6, 9], [2, 4], pos) == 0  # of their own already
    p.same()
    # both owners of a page at once: each gets a copy and the old one is free
    assert p.fork([1], [5]) == 0
    before = len(p.o.free_ids())
    assert p.unshare([0, 1, 2], [1, 5], [10, 10]) == 0
    assert len(p.o.free_ids()) == before - 1
    p.same()
    assert p.unshare([0, 2, 2, 5], [3, 0, 5]) == 0  # last rows
    p.same()
    for cu, seq, at in [([0, 2], [0], [5, 5]), ([0, 2], [0], [70, 5]), ([0, 1, 2], [0, 0], [1, 2]),
                        ([0, 1], [8], [1]), ([0, 1], [-1], [1])]:
        assert p.unshare(cu, seq, at) == -1
        p.same()
    assert p.unshare([0, 3], [0], [-2 ** 31, 700, 2 ** 31 - 1]) == 0  # positions of no token
    while len(p.o.free_ids()) > 1:
        assert p.extend([7 if p.o.len[7] < 600 else 6], [64]) == 0
    assert p.unshare([0, 10], [3], [i * 60 for i in range(10)]) > 1
    p.same()


@pytest.mark.parametrize("heads,d", [(1, 64), (3, 64), (5, 128)])
def test_copy_of_pages(heads, d):
    p = _pair(layers=2, pages=16, heads=heads, d=d, n_seqs=2, max_seq_pages=8)
    rng = np.random.default_rng(3)
    _fill(p, rng, [0, 1], [300, 200], layers=2)
    p.copy([0, 0, 3, 2, -1, 5, 16, 1, 2 ** 31 - 1], [10, 11, 12, 2, 13, 16, 14, 15, 9])
    p.same()
    p.copy([], [])


def test_compact_of_scattered_pools():
    for seed in range(4):
        rng = np.random.default_rng(seed)
        pages = int(rng.integers(20, 60))
        p = _pair(layers=2, pages=pages, heads=2, d=64, n_seqs=14, max_seq_pages=6)
        seqs = list(range(10))
        for s in seqs:
            n = int(rng.integers(0, 250))
            if -(-n // 64) <= len(p.o.free_ids()):
                _fill(p, rng, [s], [n], layers=2)
        p.free([int(s) for s in rng.choice(10, 4, replace=False)])
        if len(p.o.free_ids()) > 3:
            assert p.fork([seqs[0], seqs[1]], [11, 12]) == 0
        p.free([0, 3])
        p.compact()
        p.same()
        p.compact()  # nothing to move
        p.same()
        p.free(list(range(14)))
        p.compact()  # nothing left
        p.same()


@pytest.mark.parametrize("n", [4096, 1500])
def test_many_sequences(n):
    """As many sequences as a call takes; a pool that takes several steps to scan."""
    p = _pair(pages=3 * n + 7, heads=1, n_seqs=2 * n, max_seq_pages=3)
    rng = np.random.default_rng(n)
    seq = rng.permutation(n).tolist()
    assert p.extend(seq, rng.integers(0, 130, n).tolist()) == 0
    assert p.fork(seq, (np.arange(n) + n).tolist()) == 0
    p.free(seq[::2])
    p.compact()
    assert p.extend(seq, rng.integers(0, 60, n).tolist()) == 0
    assert p.extend([seq[0], seq[1], seq[0]], [1, 1, 1]) == -1
    p.same()


def test_random_runs():
    """Every call in any order, everything compared after each step."""
    for seed in range(3):
        rng = np.random.default_rng(100 + seed)
        p = _pair(layers=2, pages=30, heads=2, d=64, hq=6, n_seqs=6, max_seq_pages=8,
                  dtype=BF16 if seed % 2 else F32)
        seen = set()
        for _ in range(60):
            act = rng.choice(["append", "append", "rows", "fork", "free", "compact", "attn"])
            some = [s for s in range(6) if p.o.len[s] > 0]
            none = [s for s in range(6) if p.o.len[s] == 0]
            if act == "append":
                seq = [int(s) for s in rng.choice(6, 2, replace=False)]
                n = [int(x) for x in rng.integers(0, 150, 2)]
                if p.extend(seq, n) == 0:
                    # a page that a fork shares is full, so that no append touches it
                    for la in range(2):
                        p.write(la, _cu(n), seq, _rows(rng, sum(n), 2, 64), _rows(rng, sum(n), 2, 64))
            elif act == "rows" and some:
                seq = [int(s) for s in rng.permutation(some)[:2]]
                pos = [np.sort(rng.choice(p.o.len[s], min(int(p.o.len[s]), 9), replace=False)) for s in seq]
                cu = _cu([len(x) for x in pos])
                pos = np.concatenate(pos)
                if p.unshare(cu, seq, pos) == 0:
                    p.write(1, cu, seq, _rows(rng, cu[-1], 2, 64, 5.0), _rows(rng, cu[-1], 2, 64, 5.0), pos)
            elif act == "fork" and some and none:
                p.fork([int(rng.choice(some))], [none[0]])
            elif act == "free" and some:
                p.free([int(rng.choice(some))])
            elif act == "compact":
                p.compact()
            elif act == "attn" and some:
                n = [min(3, int(p.o.len[s])) for s in some]
                p.check_attn(1, _cu(n), some, torch.from_numpy(rng.standard_normal((sum(n), 6, 64))).float())
            else:
                continue
            seen.add(act)
            p.same()
        assert len(seen) == 6


def test_a_request_from_documents_to_decode():
    """The calls as a server makes them: a document set enters the cache once; each
    request forks it, takes its own copy of the pages it writes, puts its recomputed
    rows in, appends and asks its question and decodes; the documents stay as they were."""
    import paper_2607_21599_amd as daf
    heads, hq, d = 2, 14, 128
    p = _pair(layers=2, pages=60, heads=heads, d=d, hq=hq, n_seqs=4, max_seq_pages=20)
    rng = np.random.default_rng(11)
    _fill(p, rng, [0], [1000], layers=2)
    stored = p.read(1, [0, 1000], [0])
    assert p.fork([0, 0], [1, 2]) == 0
    for r, s in enumerate((1, 2)):
        idx = np.sort(rng.choice(1000, 150, replace=False))
        assert p.unshare([0, 150], [s], idx) == 0
        for la in range(2):
            p.write(la, [0, 150], [s], _rows(rng, 150, heads, d), _rows(rng, 150, heads, d), idx)
    assert p.extend([1, 2], [33, 17]) == 0
    for la in range(2):
        p.write(la, [0, 33, 50], [1, 2], _rows(rng, 50, heads, d), _rows(rng, 50, heads, d))
        p.check_attn(la, [0, 33, 50], [1, 2], torch.from_numpy(rng.standard_normal((50, hq, d))).float())
    for step in range(5):
        assert p.extend([1, 2], [1, 1]) == 0
        for la in range(2):
            p.write(la, [0, 1, 2], [1, 2], _rows(rng, 2, heads, d), _rows(rng, 2, heads, d))
            p.check_attn(la, [0, 1, 2], [1, 2], torch.from_numpy(rng.standard_normal((2, hq, d))).float())
        if step == 2:
            p.free([1])
            p.compact()
            assert p.fork([0], [1]) == 0
    p.same()
    for a, b in zip(stored, p.read(1, [0, 1000], [0])):
        assert torch.equal(a, b)
    # the selection takes what the cache holds: no deviation where nothing was recomputed
    cached, _ = p.read(1, [0, 1000], [0])
    scores = torch.zeros(1000, device="cuda")
    idx = torch.zeros(10, dtype=torch.int32, device="cuda")
    fresh = cached.clone()
    fresh[::100] += 1
    daf.daf_select_important(p.cfg, daf.Batch.single(1000, 0, 10), [fresh], [cached], scores, idx)
    assert idx.tolist() == list(range(0, 1000, 100))


def test_captured_decode_steps():
    """A decode step (extend, write, attention) as a graph: lengths and tables live on
    the device, so replays go on; each is compared with an eager run of the same steps
    beside it, with other work between the replays. Two graphs share their workspaces."""
    import paper_2607_21599_amd as daf
    from cache_pair import dev
    heads, hq, d = 2, 6, 64
    rng = np.random.default_rng(12)
    pairs = [_pair(layers=1, pages=90, heads=heads, d=d, hq=hq, n_seqs=3, max_seq_pages=40) for _ in range(2)]
    for p in pairs:
        r = np.random.default_rng(13)
        _fill(p, r, [0, 1, 2], [1500, 63, 700])
    q, k, v = (torch.from_numpy(rng.standard_normal((3, n, d))).to(BF16).cuda() for n in (hq, heads, heads))
    rows = daf.CacheRows([0, 1, 2, 3])
    size = daf.daf_cache_attn_workspace_size(pairs[0].cfg, pairs[0].c, rows, 2560)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    outs = [(torch.zeros(3, hq, d, dtype=BF16, device="cuda"), torch.zeros(hq, 3, device="cuda")) for _ in pairs]

    def step(p, out):
        daf.daf_pages_extend(p.c, 3, None, None, p.status)
        daf.daf_cache_write(p.cfg, p.c, 0, rows, k, v)
        daf.daf_cache_attn(p.cfg, p.c, 0, rows, 2560, q, out[0], out[1], ws, size)

    side = torch.cuda.Stream()
    graphs = []
    for _ in range(2):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(pairs[0], outs[0])
        graphs.append(g)
    for i in range(70):  # past the ends of pages
        k.copy_(torch.from_numpy(rng.standard_normal((3, heads, d))).to(BF16))
        q.mul_(0.99)
        graphs[i % 2].replay()
        step(pairs[1], outs[1])
        if i % 10 == 0:
            torch.cuda.synchronize()
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]), i
    for n in ("k", "v", "k_scale", "v_scale", "table", "len", "refs"):
        a, b = (p.t[n].view(torch.uint8) if n in ("k", "v") else p.t[n] for p in pairs)
        assert torch.equal(a, b), n
    assert int(pairs[0].t["len"][1]) == 133


def test_captured_page_calls():
    """Fork, unshare, compact and free in a graph, replayed on changing states."""
    import paper_2607_21599_amd as daf
    from cache_pair import dev
    pairs = [_pair(layers=2, pages=40, heads=2, d=64, n_seqs=6, max_seq_pages=10) for _ in range(2)]
    for p in pairs:
        _fill(p, np.random.default_rng(14), [0, 1], [500, 130], layers=2)
    src, dst = dev([0, 1, 0]), dev([2, 3, 4])
    pos = dev([3, 70, 499, 0, 129])
    rows = daf.CacheRows([0, 3, 5], dev([4, 3]), pos)
    live = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(p):
        daf.daf_pages_free(p.c, 3, dst)
        daf.daf_pages_fork(p.c, 3, src, dst, p.status, p.ws, p.ws_size)
        daf.daf_pages_unshare(p.c, rows, p.status, p.ws, p.ws_size)
        daf.daf_pages_free(p.c, 1, src)
        daf.daf_pages_compact(p.c, live, p.ws, p.ws_size)
        daf.daf_pages_free(p.c, 1, src)
        daf.daf_pages_fork(p.c, 1, dst, src, p.status, p.ws, p.ws_size)

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(pairs[0])
    for i in range(5):
        g.replay()
        step(pairs[1])
        torch.cuda.synchronize()
        for n in ("k", "v", "k_scale", "v_scale", "table", "len", "refs", "status"):
            a, b = (p.status if n == "status" else p.t[n].view(torch.uint8) if n in ("k", "v") else p.t[n]
                    for p in pairs)
            assert torch.equal(a, b), (i, n)
        assert int(pairs[0].status) == 0


def test_calls_on_another_stream():
    """Every call takes the stream that it is given, or the current one."""
    import paper_2607_21599_amd as daf
    p = _pair(layers=1, pages=40, heads=2, d=64, hq=4, n_seqs=3, max_seq_pages=30)
    rng = np.random.default_rng(15)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _fill(p, rng, [0], [1800])
        assert p.fork([0], [1]) == 0
        p.check_attn(0, [0, 2], [1], torch.from_numpy(rng.standard_normal((2, 4, 64))).float())
        p.compact()
    s.synchronize()
    p.same()
    q = torch.from_numpy(rng.standard_normal((2, 4, 64))).to(BF16).cuda()
    torch.cuda.synchronize()
    want, _ = p.attn(0, [0, 2], [0], q)
    torch.cuda.synchronize()
    got, _ = p.attn(0, [0, 2], [0], q, stream=s)
    s.synchronize()
    assert torch.equal(want, got)

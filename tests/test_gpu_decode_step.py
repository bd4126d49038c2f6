"""GPU: decode steps of a small model over shared documents, as a server runs them: per layer

    s += delta;  h = norm(s) in 8 bits;  q, k, v = h Wqkv + b in 4-bit weights;  rotation
    and append;  attention of groups;  s += o Wo;  h = norm(s);  SiLU(h Wg) * h Wu;  ... Wd

Each call's results are checked on its own inputs against 64 bits, then the same steps run
from a graph, token after token, against the eager ones."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_21599_amd as daf
from oracle import step as orc

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
HIDDEN, INTER, HQ, HKV, D, LAYERS, THETA, EPS = 384, 640, 8, 2, 64, 2, 1e4, 1e-6
GROUPS, SHARED, TAILS = [5, 1, 3], [2144, 64, 130], [3, 61, 64, 1, 127, 30, 2, 5, 62]
N = len(TAILS)
QKV = (HQ + 2 * HKV) * D


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    daf.lib()
    yield
    torch.cuda.synchronize()


class Server:
    """Weights, a cache whose groups of sequences are forks of one prefix each, and the buffers of a step."""

    def __init__(self, seed):
        from cache_pair import Pair, dev
        from paper_2607_21599_amd.tensors import mx_weights
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def randn(*shape, size=1.0):
            return (torch.randn(shape, generator=gen, device="cuda") * size).to(BF16)

        def weights(n, k):
            return [t.contiguous() for t in mx_weights(randn(n, k, size=k ** -0.5))]

        self.w = [dict(norm1=1 + randn(HIDDEN, size=0.1), qkv=weights(QKV, HIDDEN), bias=randn(QKV, size=0.1),
                       o=weights(HIDDEN, HQ * D), norm2=1 + randn(HIDDEN, size=0.1), gu=weights(2 * INTER, HIDDEN),
                       d=weights(HIDDEN, INTER)) for _ in range(LAYERS)]
        lens = [s + t for s, t in zip(np.repeat(SHARED, GROUPS).tolist(), TAILS)]
        self.p = Pair(layers=LAYERS, pages=sum(-(-x // 64) for x in lens) + 2 * N + 16, heads=HKV, d=D, n_seqs=N + len(GROUPS),
                      max_seq_pages=max(lens) // 64 + 3, hq=HQ)
        rng = np.random.default_rng(seed)
        order = rng.permutation(N + len(GROUPS)).tolist()
        self.seq, stems = order[:N], order[N:]

        def fill(which, m):
            assert self.p.extend(which, m) == 0
            cu = [0] + np.cumsum(m).tolist()
            for la in range(LAYERS):
                k, v = (torch.from_numpy(rng.standard_normal((cu[-1], HKV, D))).float() for _ in range(2))
                self.p.write(la, cu, which, k, v)

        fill(stems, SHARED)
        assert self.p.fork(np.repeat(stems, GROUPS).tolist(), self.seq) == 0
        fill(self.seq, TAILS)
        self.seqs = dev(self.seq)
        self.rows = daf.CacheRows(list(range(N + 1)), self.seqs)
        self.groups = daf.CacheGroups([0] + np.cumsum(GROUPS).tolist(), SHARED)
        self.max_len = self.p.t["table"].shape[1] * 64
        size = max([daf.daf_cache_attn_shared_workspace_size(self.p.cfg, self.p.c, self.rows, self.groups, self.max_len)]
                   + [daf.daf_linear_mx_workspace_size(N, n, k) for n, k in
                      ((QKV, HIDDEN), (HIDDEN, HQ * D), (2 * INTER, HIDDEN), (HIDDEN, INTER))])
        self.size, self.ws = size, torch.full((max(size, 16),), 0xFF, dtype=torch.uint8, device="cuda")

        def buf(*shape, dtype=BF16):
            return torch.zeros(shape, dtype=dtype, device="cuda")

        self.b = dict(x=buf(N, HIDDEN), s=buf(N, HIDDEN), delta=buf(N, HIDDEN), codes=buf(N, HIDDEN, dtype=torch.float8_e4m3fn),
                      scales=buf(N, HIDDEN // 32, dtype=torch.uint8), qkv=buf(N, QKV), q=buf(N, HQ, D), o=buf(N, HQ, D),
                      lse=buf(HQ, N, dtype=torch.float32), gu=buf(N, 2 * INTER), act=buf(N, INTER), out=buf(N, HIDDEN))

    def linear(self, n, k, a, scales, w, bias, c):
        daf.daf_linear_mx(N, n, k, a, scales, w[0], w[1], bias, None, c, self.ws, self.size)

    def step(self, seen=lambda *a: None):
        """One token of every sequence: from x to out."""
        b, p = self.b, self.p
        daf.daf_pages_extend(p.c, N, self.seqs, None, p.status)
        b["s"].copy_(b["x"])
        delta = None
        for la, w in enumerate(self.w):
            for half in range(2):
                x = b["s"].clone() if seen.__name__ == "seen" else None
                d = None if delta is None else delta.clone()
                daf.daf_add_rmsnorm(daf.DAF_BF16, N, HIDDEN, b["s"], delta, w[f"norm{half + 1}"], EPS,
                                    None if delta is None else b["s"], None, b["codes"], b["scales"])
                seen("norm", la, half, x, d)
                delta = b["delta"]
                if half == 0:
                    self.linear(QKV, HIDDEN, b["codes"], b["scales"], w["qkv"], w["bias"], b["qkv"])
                    seen("qkv", la)
                    q, k, v = b["qkv"].split([HQ * D, HKV * D, HKV * D], 1)
                    daf.daf_cache_write_rope(p.cfg, p.c, la, self.rows, THETA, q, QKV, k, v, QKV, b["q"])
                    seen("rope", la)
                    daf.daf_cache_attn_shared(p.cfg, p.c, la, self.rows, self.groups, self.max_len, b["q"], b["o"],
                                              b["lse"], self.ws, self.size)
                    seen("attn", la)
                    self.linear(HIDDEN, HQ * D, b["o"], None, w["o"], None, b["delta"])
                    seen("o", la)
                else:
                    self.linear(2 * INTER, HIDDEN, b["codes"], b["scales"], w["gu"], None, b["gu"])
                    seen("gu", la)
                    daf.daf_silu_mul(N, INTER, b["gu"], b["act"])
                    self.linear(HIDDEN, INTER, b["act"], None, w["d"], None, b["delta"])
                    seen("d", la)
        b["out"].copy_(b["s"] + b["delta"])


def _near_linear(a, w, bias, c):
    want, size = orc.linear(a, orc.mx_values(orc.e2m1_values(w[0]), w[1]), bias)
    e = (a.shape[1] + 16) * 2.0 ** -24 * size
    assert ((c.double() - want).abs() <= e + 2.0 ** -8 * (want.abs() + e)).all()


def test_every_call_of_a_step():
    from test_gpu_cache_rope import _turned
    s = Server(1)
    b, p = s.b, s.p
    b["x"].copy_(torch.randn(N, HIDDEN, generator=torch.Generator().manual_seed(2)))

    def seen(what, la, half=0, x=None, d=None):
        torch.cuda.synchronize()
        w = s.w[la]
        rows = orc.mx_values(b["codes"].double(), b["scales"])
        if what == "norm":
            if d is not None:
                want = x.double() + d.double()
                assert ((b["s"].double() - want).abs() <= 2.0 ** -8 * want.abs() * (1 + 2.0 ** -15)).all()
            want = orc.rmsnorm(b["s"], w[f"norm{half + 1}"], EPS)
            scale = orc.scales_of(b["scales"]).repeat_interleave(32, 1)
            # half a step of a code, and the fp32 arithmetic
            assert ((rows - want).abs() <= torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * scale) + 2.0 ** -18 * want.abs()).all()
        elif what in ("qkv", "gu"):
            _near_linear(rows, w[what], w["bias"] if what == "qkv" else None, b[what])
        elif what in ("o", "d"):
            _near_linear((b["o"].view(N, -1) if what == "o" else b["act"]).double(), w[what], None, b["delta"])
        elif what == "rope":
            p.o.len[:] = p.t["len"].cpu().numpy()  # as extend has left them
            p.o.table[:] = p.t["table"].cpu().numpy()
            at = p.o.len[s.seq] - 1
            x = b["qkv"].double().cpu().numpy().reshape(N, HQ + 2 * HKV, D)
            want, size = _turned(x[:, :HQ + HKV], at, THETA)
            e = 6 * 2.0 ** -24 * size
            off = np.abs(b["q"].double().cpu().numpy() - want[:, :HQ])
            assert (off <= e[:, :HQ] * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want[:, :HQ])).all()
            k, v = p.t["k"][la].double().cpu().numpy(), p.t["v"][la].double().cpu().numpy()
            ks, vs = p.t["k_scale"][la].double().cpu().numpy(), p.t["v_scale"][la].double().cpu().numpy()
            for i, t in enumerate(at):
                page, slot = p.o.table[s.seq[i], t // 64], t % 64
                for got, sc, val, err in ((k[page, :, slot] * ks[page][:, None], ks, want[i, HQ:], e[i, HQ:]),
                                          (v[page, :, :, slot] * vs[page][:, None], vs, x[i, HQ + HKV:], 0)):
                    half_step = np.maximum(2.0 ** -4 * np.abs(val), 2.0 ** -10 * sc[page][:, None])
                    assert (np.abs(got - val) <= half_step + 2 * err).all()
            # what the attention reads: codes and scales as they are
            for n in "kv":
                code = p.t[n].double().cpu().numpy()
                p.o.code[n] = code.swapaxes(-1, -2) if n == "v" else code
                p.o.scale[n] = p.t[n + "_scale"].double().cpu().numpy()
        elif what == "attn":
            p.within_bounds(b["o"], b["lse"], la, list(range(N + 1)), s.seq, b["q"], None)

    for _ in range(3):
        s.step(seen)
        assert int(p.status) == 0


def test_steps_from_a_graph():
    a, e = Server(3), Server(3)
    gen = torch.Generator().manual_seed(4)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.step()
    for i in range(6):  # over ends of pages
        x = torch.randn(N, HIDDEN, generator=gen).to(BF16)
        for s in (a, e):
            s.b["x"].copy_(x)
        e.step()
        for n in ("codes", "scales", "qkv", "q", "o", "gu", "act", "out", "delta"):
            a.b[n].view(torch.uint8).fill_(0x7F)
        a.ws.fill_(0xFF)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert int(a.p.status) == 0 and int(e.p.status) == 0
        for n in ("out", "lse", "q"):
            assert torch.equal(a.b[n], e.b[n]), (i, n)
        for n in ("k", "v", "k_scale", "v_scale", "table", "len", "refs"):
            assert torch.equal(a.p.t[n].view(torch.uint8), e.p.t[n].view(torch.uint8)), (i, n)


def test_steps_of_two_servers_at_once():
    """On a stream each, with workspaces of their own."""
    alone, both = [Server(5), Server(6)], [Server(5), Server(6)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    x = torch.randn(N, HIDDEN, generator=torch.Generator().manual_seed(7)).to(BF16).cuda()
    for s in alone + both:
        s.b["x"].copy_(x)
    for s in alone:
        for _ in range(3):
            s.step()
    torch.cuda.synchronize()
    for _ in range(3):
        for s, stream in zip(both, streams):
            with torch.cuda.stream(stream):
                s.step()
    torch.cuda.synchronize()
    for s, t in zip(alone, both):
        assert torch.equal(s.b["out"], t.b["out"]) and torch.equal(s.p.t["k"].view(torch.uint8), t.p.t["k"].view(torch.uint8))

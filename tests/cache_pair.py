"""A paged cache on the GPU beside the plain one of oracle/cache.py: the same calls
on both, and their comparison."""
from __future__ import annotations

import numpy as np
import torch

import paper_2607_21599_amd as daf
from oracle.cache import CacheOracle
from paper_2607_21599_amd.tensors import cache_tensors

MOST = {torch.bfloat16: float(torch.finfo(torch.bfloat16).max), torch.float32: float(torch.finfo(torch.float32).max)}


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a)).to(dtype).cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


class Pair:
    def __init__(self, layers=1, pages=16, heads=2, d=64, n_seqs=4, max_seq_pages=8, hq=None, dtype=torch.bfloat16):
        self.heads, self.d, self.dtype = heads, d, dtype
        self.hq = hq or heads
        self.cfg = daf.AttnCfg(self.hq, heads, d, daf.DAF_BF16 if dtype == torch.bfloat16 else daf.DAF_F32)
        self.t = cache_tensors(layers, pages, heads, d, n_seqs, max_seq_pages)
        for n in ("k", "v"):  # a known pool, so that whole pools can be compared
            self.t[n].view(torch.uint8).zero_()
            self.t[n + "_scale"].zero_()
        self.c = daf.Cache.from_tensors(self.t)
        self.o = CacheOracle(layers, pages, heads, d, n_seqs, max_seq_pages)
        self.status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
        self.ws_size = daf.daf_pages_workspace_size(self.c)
        self.ws = torch.full((self.ws_size,), 0xA5, dtype=torch.uint8, device="cuda")

    # -- page calls, each checked on its status -----------------------------------
    def _status(self, want):
        assert int(self.status) == want, (int(self.status), want)
        return want

    def extend(self, seq, n_new):
        daf.daf_pages_extend(self.c, len(seq), dev(seq), dev(n_new), self.status)
        return self._status(self.o.extend(seq, n_new))

    def fork(self, src, dst):
        daf.daf_pages_fork(self.c, len(src), dev(src), dev(dst), self.status, self.ws, self.ws_size)
        return self._status(self.o.fork(src, dst))

    def unshare(self, cu, seq, pos=None):
        rows = daf.CacheRows(cu, dev(seq), None if pos is None else dev(pos))
        daf.daf_pages_unshare(self.c, rows, self.status, self.ws, self.ws_size)
        return self._status(self.o.unshare(cu, seq, pos))

    def free(self, seq):
        daf.daf_pages_free(self.c, len(seq), dev(seq))
        self.o.free(seq)

    def copy(self, src, dst):
        daf.daf_pages_copy(self.c, len(src), dev(src), dev(dst))
        self.o.copy(src, dst)

    def compact(self):
        n = torch.full((1,), -5, dtype=torch.int32, device="cuda")
        daf.daf_pages_compact(self.c, n, self.ws, self.ws_size)
        assert int(n) == self.o.compact()

    # -- rows ------------------------------------------------------------------------
    def write(self, layer, cu, seq, k, v, pos=None):
        """k, v: float tensors [rows][heads][d] on the CPU."""
        k, v = k.to(self.dtype), v.to(self.dtype)
        rows = daf.CacheRows(cu, dev(seq), None if pos is None else dev(pos))
        daf.daf_cache_write(self.cfg, self.c, layer, rows, k.cuda(), v.cuda())
        self.o.write(layer, cu, seq, pos, f64(k), f64(v), MOST[self.dtype])

    def read(self, layer, cu, seq, pos=None):
        rows = daf.CacheRows(cu, dev(seq), None if pos is None else dev(pos))
        k, v = (torch.full((cu[-1], self.heads, self.d), 77.0, dtype=self.dtype, device="cuda") for _ in range(2))
        daf.daf_cache_read(self.cfg, self.c, layer, rows, k, v)
        want = self.o.read(layer, cu, seq, pos)
        for name, x, y in zip("kv", (k, v), want):
            assert np.array_equal(f64(x), y, equal_nan=True), name
        return k, v

    def same(self):
        """Everything, the slots that hold no token included."""
        torch.cuda.synchronize()
        for n in ("table", "len", "refs"):
            assert np.array_equal(self.t[n].cpu().numpy(), getattr(self.o, n)), n
        for n in "kv":
            code = f64(self.t[n].float())
            code = code.swapaxes(-1, -2) if n == "v" else code
            assert np.array_equal(f64(self.t[n + "_scale"]), self.o.scale[n]), n
            assert np.array_equal(code, self.o.code[n], equal_nan=True), n

    def attn(self, layer, cu, seq, q, pos=None, max_len=None, lse=True, stream=None):
        top = self.t["table"].shape[1] * daf.DAF_PAGE_TOKENS
        max_len = top if max_len is None else max_len
        rows = daf.CacheRows(cu, dev(seq) if seq is not None else None, None if pos is None else dev(pos))
        o = torch.full(q.shape, 77.0, dtype=self.dtype, device="cuda")
        le = torch.full((self.hq, q.shape[0]), 77.0, device="cuda") if lse else None
        size = daf.daf_cache_attn_workspace_size(self.cfg, self.c, rows, max_len)
        ws = torch.full((max(size, 16),), 0xFF, dtype=torch.uint8, device="cuda")  # NaN in every word
        daf.daf_cache_attn(self.cfg, self.c, layer, rows, max_len, q, o, le, ws, size, stream)
        return o, le

    def check_attn(self, layer, cu, seq, q, pos=None, max_len=None):
        """The GPU's result within the bounds of its roundings of the exact one.

        A score of d terms is off by at most (d + 8) 2^-24 of sum |q||k| scale (fp32
        sums and products) plus 2^-22 of itself (the exponent's argument); a weight by
        twice that (numerator, denominator) plus one part per key of the sums, each
        2^-24. bf16 adds half a step (2^-8) for the weight's rounding and one for the
        output's, fp32 2^-24 for the output and 2^-23 for the three-term weight.
        """
        q = q.to(self.dtype)
        o, lse = self.attn(layer, cu, seq, q.cuda(), pos, max_len)
        self.within_bounds(o, lse, layer, cu, list(range(len(cu) - 1)) if seq is None else seq, q, pos)
        return o, lse

    def within_bounds(self, o, lse, layer, cu, seq, q, pos):
        """check_attn's comparison of given results, of rows of q that are in the dtype."""
        d, hq = self.d, self.hq
        want, want_lse, mean, size = self.o.attn(layer, cu, seq, pos, f64(q), 1 / d ** 0.5)
        keys = max([int(self.o.len[s]) for s in seq] + [1])
        e = 2.0 ** -24 * ((d + 8) * size + 4 * size + keys + 64)  # [hq][rows]
        tol = 2 * e.T[..., None] * mean
        half = 2.0 ** -8 if self.dtype == torch.bfloat16 else 2.0 ** -23
        tol = (tol + half * mean) * (1 + half) + half * np.abs(want) + 1e-30
        err = np.abs(f64(o) - want)
        assert (err <= tol).all(), (float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
        none = np.isneginf(want_lse)
        got = f64(lse)
        assert np.array_equal(np.isneginf(got), none)
        some = ~none
        off = np.abs(got[some] - want_lse[some])
        lim = e[some] + 2.0 ** -22 * (1 + np.abs(want_lse[some]))
        assert (off <= lim).all(), float((off / lim).max())

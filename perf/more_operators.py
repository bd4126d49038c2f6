"""Operators of a decode step over stored documents, with their plain forms and exact results.

A server that has forked a document set for many requests runs, per layer and step:

* norm: the residual's addition and the RMS norm of the sum, written in the rows' type
  and, for the projections in few bits, as e4m3 codes with one power-of-two scale per
  32 values;
* linear: projections of few rows (in bf16, or the norm's codes) with weights in 4 bits:
  e2m1 codes, two per byte, with one power-of-two scale per 32 of a row;
* append: the rotary position embedding of q and k, and the rotated K and the V into the
  paged 8-bit cache, from the rows of the joint projection;
* shared: attention over that cache for groups of requests whose first pages are the
  same ones.

The scale of 32 values is the smallest power of two >= 2^-100 under which their largest
magnitude is at most 448, and is held as its exponent + 127 in a byte. That of a page
and head of the cache is the same (0 if all are zeros), and not less than the present
one while a row of the page stays.

A case is a dict of plain values. ``nq`` are the rows of each request and ``lens`` the
tokens of its sequence, the rows included (separated by blanks); ``groups`` the requests
of each group and ``shared`` the tokens that its sequences have in common.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 64
BLOCK = 32      # values per scale outside of the cache
MIN_EXP = -100  # exponent of the smallest scale
THETA = 1e6
EPS = 1e-6
WIDE = dict(hq=28, hkv=4, d=128, dtype="bf16")  # this repository's model widths
HIDDEN, INTER = 3584, 18944
RAGGED32 = ("8192 4097 64 1 2500 777 8000 5121 300 129 6400 1023 4096 65 2048 3333 "
            "7001 12 513 1900 8191 63 128 1500 4444 2222 999 6000 31 3500 250 7777")


def _norm(rows, width, out, dtype="bf16", add=True):
    return dict(kind="norm", rows=rows, width=width, out=out, dtype=dtype, add=add)


def _linear(m, n, k, a, bias=False, residual=False):
    return dict(kind="linear", m=m, n=n, k=k, a=a, bias=bias, residual=residual)


def _append(lens, nq, at="tail", **kw):
    return dict(dict(kind="append", lens=lens, nq=nq, at=at, **WIDE), **kw)


def _shared(groups, shared, tails, nq, **kw):
    """tails: the tokens of each request after the shared ones."""
    g, s, t = (_ints(x) for x in (groups, shared, tails))
    lens = [a + b for a, b in zip(np.repeat(s, g).tolist(), t)]
    return dict(dict(kind="shared", groups=groups, shared=shared, lens=_text(lens), nq=nq, at="tail", **WIDE), **kw)


def _ints(text):
    return [int(x) for x in text.split()]


def _text(numbers):
    return " ".join(map(str, numbers))


def listed():
    cases = [
        # one token between two projections in bf16: latency only
        ("norm_1", _norm(1, HIDDEN, "y")),
        # the recomputed and question rows of the benchmark's layer, for projections of either kind
        ("norm_5043", _norm(5043, HIDDEN, "both")),
        # q, k and v of one token of one conversation, from the norm's codes
        ("qkv_1", _linear(1, 4608, HIDDEN, "mx", bias=True)),
        # the gate and up projections of a serving batch's decode step
        ("gate_up_32", _linear(32, 2 * INTER, HIDDEN, "mx")),
        # the down projection of a smaller batch, onto the residual stream
        ("down_12", _linear(12, HIDDEN, INTER, "bf16", residual=True)),
        # a decode step of a ragged serving batch: one new row per sequence
        ("append_32", _append(RAGGED32, _text([1] * 32))),
        # the recomputed rows of a request (15% of 32k) over the offline ones
        ("hybrid_32k", _append("32768", "4915", at="pos")),
        # a document enters the cache
        ("document_16k", _append("16384", "16384")),
        # beam search over a short conversation: latency
        ("beams_4", _shared("4", "777", "1 9 64 130", "1 1 1 1")),
        # a decode step of 32 answers over one document set
        ("answers_32k", _shared("32", "32768", _text([1 + 37 * i % 700 for i in range(32)]), _text([1] * 32))),
        # the question rows of 8 requests over one document set
        ("questions_32k", _shared("8", "32768", "40 33 64 25 40 7 52 40", "40 33 64 25 40 7 52 40")),
        # a decode step over five document sets of different lengths, with requests that share nothing
        ("sets_5", _shared("8 3 1 12 1", "9000 4096 100 1984 5000", _text([1 + 61 * i % 900 for i in range(25)]),
                           _text([1] * 25), hq=8, hkv=2, d=64, dtype="f32")),
    ]
    return [dict(c, name=n) for n, c in cases]


def draw(rng):
    def log(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))

    kind = rng.choice(["norm", "linear", "linear", "append", "append", "shared", "shared", "shared"])
    if kind == "norm":
        out = rng.choice(["y", "mx", "both"])
        width = log(1, 512) * 8 if out == "y" else log(1, 256) * BLOCK
        return _norm(log(1, 5043 * HIDDEN // max(width, 1024)), width, out, rng.choice(["bf16", "bf16", "f32"]),
                     rng.random() < 0.7)
    if kind == "linear":
        m, n, k = log(1, 128), log(16, 2 * INTER), log(1, INTER // BLOCK) * BLOCK
        most = 2 * INTER * HIDDEN * 32
        n = max(1, min(n, most // (k * max(m, 32))))
        return _linear(m, n, k, rng.choice(["mx", "bf16"]), rng.random() < 0.4, rng.random() < 0.4)
    hq, hkv = rng.choice([(28, 4), (28, 4), (8, 2), (4, 1), (16, 16), (6, 1), (32, 8), (20, 4)])
    kw = dict(hq=hq, hkv=hkv, d=rng.choice([64, 128, 128]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
              at=rng.choice(["tail", "tail", "pos"]))
    if kind == "append":
        b = log(1, 64)
        most = 16384 * 4 // max(hkv, 4) // (1 if kw["dtype"] == "bf16" else 2)
        lens = [log(1, most // b) for _ in range(b)]
        nq = [log(1, max(1, n // 4)) if kw["at"] == "pos" else n if b < 4 else min(n, log(1, 8)) for n in lens]
        return _append(_text(lens), _text(nq), **kw)
    n_groups = rng.choice([1, 1, 1, 2, 3, 6])
    groups = [log(1, 32 // n_groups) for _ in range(n_groups)]
    b = sum(groups)
    top = 32768 * 4 * 32 // max(hkv, 4) // max(b, 4) // 4 if kw["dtype"] == "f32" else 32768 * 4 // max(hkv, 4)
    shared = [log(1, min(top, 32768)) for _ in groups]
    tails = [log(1, 1000) for _ in range(b)]
    # pairs of rows and keys no more than the listed questions' (a third of them in fp32)
    pairs = 300 * 32768 * 28 // hq // (1 if kw["dtype"] == "bf16" else 3)
    rows = max(1, min(64, pairs // (b * (max(shared) + 1000))))
    nq = [1] * b if rng.random() < 0.5 else [min(n, log(1, rows)) for n in tails]
    return _shared(_text(groups), _text(shared), _text(tails), _text(nq), **kw)


# ---- cases in numbers ------------------------------------------------------------
def _pages(n):
    return -(-n // PAGE)


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def work(case):
    kind = case["kind"]
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        a = k * 2 if case["a"] == "bf16" else k + k // BLOCK
        return {"bytes": n * (k // 2 + k // BLOCK) + m * a + 2 * n * case["bias"] + 2 * m * n * (1 + case["residual"]),
                "flops": 2 * m * n * k}
    el = 2 if case["dtype"] == "bf16" else 4
    if kind == "norm":
        rows, width = case["rows"], case["width"]
        moved = el * (3 if case["add"] else 1) + (el if case["out"] != "mx" else 0)
        if case["out"] != "y":
            moved += 1 + 1 / BLOCK
        return {"bytes": rows * width * moved + width * el, "flops": 8 * rows * width}
    lens, nq = _ints(case["lens"]), _ints(case["nq"])
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    rows, row8 = sum(nq), 2 * hkv * d  # one token's K and V in the cache
    if kind == "append":
        return {"bytes": rows * ((2 * hq + 2 * hkv) * d * el + row8), "flops": 6 * rows * (hq + hkv) * d}
    groups, shared = _ints(case["groups"]), _ints(case["shared"])
    keys = sum(lens) - sum((g - 1) * (s // PAGE * PAGE) for g, s in zip(groups, shared))
    if case["at"] == "tail":
        pairs = sum(n * L - n * (n - 1) // 2 for n, L in zip(nq, lens))
    else:
        pairs = sum(n * (L + 1) // 2 for n, L in zip(nq, lens))
    return {"bytes": keys * row8 + keys // PAGE * 8 * hkv + 2 * rows * hq * d * el + 4 * rows * hq,
            "flops": 4 * pairs * hq * d}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def randint(lo, hi, *shape, dtype=torch.uint8):
        return torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=dtype)

    kind, s = case["kind"], {"case": case}
    if kind == "norm":
        rows, width, dt = case["rows"], case["width"], _dt(case)
        # a residual stream: rows of different sizes, a few features far larger than the others
        outlier = torch.where(torch.rand(width, generator=gen, device="cuda") < 0.01, 30.0, 1.0)
        s["x"] = (randn(rows, width) * torch.exp(randn(rows, 1)) * outlier).to(dt)
        s["delta"] = randn(rows, width).to(dt) if case["add"] else None
        s["w"] = (1 + 0.2 * randn(width)).to(dt)
        s["sum"] = torch.zeros_like(s["x"]) if case["add"] else None
        s["y"] = torch.zeros_like(s["x"]) if case["out"] != "mx" else None
        if case["out"] != "y":
            s["codes"] = torch.zeros(rows, width, dtype=torch.float8_e4m3fn, device="cuda")
            s["scales"] = torch.zeros(rows, width // BLOCK, dtype=torch.uint8, device="cuda")
    elif kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        # weights of about 1 / sqrt(k): codes of all 16 values, scales of a few sizes
        s["w"] = randint(0, 256, n, k // 2)
        s["w_scales"] = randint(0, 3, n, k // BLOCK) + (126 - round(math.log2(3 * k ** 0.5)))
        if case["a"] == "mx":
            s["a"] = (randn(m, k) * 112).clamp_(-448, 448).to(torch.float8_e4m3fn)
            s["a_scales"] = randint(118, 122, m, k // BLOCK)
        else:
            s["a"], s["a_scales"] = randn(m, k).to(torch.bfloat16), None
        s["bias"] = randn(n).to(torch.bfloat16) if case["bias"] else None
        s["residual"] = randn(m, n).to(torch.bfloat16) if case["residual"] else None
        s["c"] = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    else:
        _prepare_cache(case, seed, s, randn, randint)
    if own:
        s["h"] = _handle(s)
    return s


def _prepare_cache(case, seed, s, randn, randint):
    rng = np.random.default_rng(seed)
    lens, nq = _ints(case["lens"]), _ints(case["nq"])
    hq, hkv, d, dt = case["hq"], case["hkv"], case["d"], _dt(case)
    groups = _ints(case["groups"]) if case["kind"] == "shared" else [1] * len(lens)
    common = np.repeat(_ints(case["shared"]), groups) // PAGE if case["kind"] == "shared" else [0] * len(lens)
    first = np.repeat(np.cumsum([0] + groups)[:-1], groups)  # of each request's group
    n_seqs, n_pages = len(lens) + 1, sum(map(_pages, lens)) + 5

    def codes(*shape):
        return (randn(*shape) * 112).clamp_(-448, 448).to(torch.float8_e4m3fn)

    def scales():
        return torch.exp2(randint(-9, -7, 1, n_pages, hkv, dtype=torch.int32).float())

    s.update(k=codes(1, n_pages, hkv, PAGE, d), v=codes(1, n_pages, hkv, d, PAGE), k_scale=scales(), v_scale=scales())
    # sequences lie in shuffled pages, and their table rows in shuffled order
    ids, seq = rng.permutation(n_pages).astype(np.int32), rng.permutation(n_seqs)[:len(lens)].astype(np.int32)
    table = np.full((n_seqs, max(map(_pages, lens)) + 1), -1, np.int32)
    length, refs, at = np.zeros(n_seqs, np.int32), np.zeros(n_pages, np.int32), 0
    for i, n in enumerate(lens):
        have = int(common[i]) if first[i] != i else 0  # pages of the group's first request
        table[seq[i], :have] = table[seq[first[i]], :have]
        table[seq[i], have:_pages(n)] = ids[at:at + _pages(n) - have]
        at += _pages(n) - have
        np.add.at(refs, table[seq[i], :_pages(n)], 1)
        length[seq[i]] = n
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    s.update(table=dev(table), len=dev(length), refs=dev(refs), seq=dev(seq), pos=None, max_len=max(lens),
             cu=np.concatenate([[0], np.cumsum(nq)]).astype(np.int32))
    if case["at"] == "pos":
        s["pos"] = dev(np.concatenate([np.sort(rng.choice(L, n, replace=False)) for n, L in zip(nq, lens)])
                       .astype(np.int32))
    total = sum(nq)
    if case["kind"] == "append":
        # rows of the joint projection; a few of larger values, so that scales differ and grow
        big = torch.where(randint(0, 50, total, 1) == 0, 8.0, 0.5)
        s["qkv"] = (randn(total, (hq + 2 * hkv) * d) * big).to(dt)
        s["q_out"] = torch.zeros(total, hq, d, dtype=dt, device="cuda")
        return
    s["group_cu"] = np.concatenate([[0], np.cumsum(groups)]).astype(np.int32)
    s["group_shared"] = np.array(_ints(case["shared"]), np.int32)
    s["q"] = randn(total, hq, d).to(dt)
    s["o"] = torch.zeros(total, hq, d, dtype=dt, device="cuda")
    s["lse"] = torch.zeros(hq, total, device="cuda")


def _handle(s):
    """What a program that uses the library keeps: descriptors and a workspace."""
    import paper_2607_21599_amd as daf
    c, h, size = s["case"], {"daf": daf}, 0
    if c["kind"] == "norm":
        h["dtype"] = daf.DAF_BF16 if c["dtype"] == "bf16" else daf.DAF_F32
        return h
    if c["kind"] == "linear":
        size = daf.daf_linear_mx_workspace_size(c["m"], c["n"], c["k"])
    else:
        h["cfg"] = daf.AttnCfg(c["hq"], c["hkv"], c["d"], daf.DAF_BF16 if c["dtype"] == "bf16" else daf.DAF_F32)
        h["cache"] = daf.Cache.from_tensors({n: s[n] for n in ("k", "v", "k_scale", "v_scale", "table", "len", "refs")})
        h["rows"] = daf.CacheRows(s["cu"], s["seq"], s["pos"])
        if c["kind"] == "shared":
            h["groups"] = daf.CacheGroups(s["group_cu"], s["group_shared"])
            size = daf.daf_cache_attn_shared_workspace_size(h["cfg"], h["cache"], h["rows"], h["groups"], s["max_len"])
    h["size"], h["ws"] = size, torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    return h


def _run_own(s):
    c, h = s["case"], s["h"]
    daf, kind = h["daf"], c["kind"]
    if kind == "norm":
        daf.daf_add_rmsnorm(h["dtype"], c["rows"], c["width"], s["x"], s["delta"], s["w"], EPS, s["sum"], s["y"],
                            s.get("codes"), s.get("scales"))
        return _norm_out(s)
    if kind == "linear":
        daf.daf_linear_mx(c["m"], c["n"], c["k"], s["a"], s["a_scales"], s["w"], s["w_scales"], s["bias"],
                          s["residual"], s["c"], h["ws"], h["size"])
        return {"c": s["c"]}
    if kind == "append":
        hq, hkv, d = c["hq"], c["hkv"], c["d"]
        q, k, v = s["qkv"].split([hq * d, hkv * d, hkv * d], 1)
        pitch = (hq + 2 * hkv) * d
        daf.daf_cache_write_rope(h["cfg"], h["cache"], 0, h["rows"], THETA, q, pitch, k, v, pitch, s["q_out"])
        return _append_out(s)
    daf.daf_cache_attn_shared(h["cfg"], h["cache"], 0, h["rows"], h["groups"], s["max_len"], s["q"], s["o"], s["lse"],
                              h["ws"], h["size"])
    return {"o": s["o"], "lse": s["lse"]}


def _norm_out(s):
    out = {n: s[n] for n in ("sum", "y", "codes") if s.get(n) is not None}
    if "scales" in s:
        out["scales"] = s["scales"].view(torch.float8_e8m0fnu)
    return out


def _append_out(s):
    return {"q": s["q_out"], "k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "norm":
        return _plain_norm(state)
    if kind == "linear":
        return _plain_linear(state)
    return _plain_append(state) if kind == "append" else _plain_attn(state)


# ---- plain forms -----------------------------------------------------------------
def _exponent(top):
    """Of the smallest power of two (>= 2^MIN_EXP) under which top is at most 448."""
    m, e = torch.frexp(top)  # m in [0.5, 1)
    return torch.where(top > 0, torch.clamp(e - 9 + (m > 0.875).int(), min=MIN_EXP), MIN_EXP)


def _plain_norm(s):
    dt, h = _dt(s["case"]), s["x"].float()
    if s["delta"] is not None:
        s["sum"].copy_(h + s["delta"].float())
        h = s["sum"].float()
    y = h * (1 / torch.sqrt(h.square().mean(-1, keepdim=True) + EPS)) * s["w"].float()
    if s["y"] is not None:
        s["y"].copy_(y.to(dt))
    if "codes" in s:
        y = y.view(len(y), -1, BLOCK)
        e = _exponent(y.abs().amax(-1))
        s["codes"].copy_(torch.ldexp(y, -e[..., None]).view(s["codes"].shape).to(torch.float8_e4m3fn))
        s["scales"].copy_(e + 127)
    return _norm_out(s)


def _plain_linear(s):
    values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    code = torch.stack([s["w"] & 15, s["w"] >> 4], -1).view(len(s["w"]), -1, BLOCK)
    w = torch.ldexp(values[code.int()], s["w_scales"].int()[..., None] - 127).view(len(s["w"]), -1)
    a = s["a"].float()
    if s["a_scales"] is not None:
        a = torch.ldexp(a.view(len(a), -1, BLOCK), s["a_scales"].int()[..., None] - 127).view(a.shape)
    c = a @ w.t()
    if s["bias"] is not None:
        c = c + s["bias"].float()
    if s["residual"] is not None:
        c = c + s["residual"].float()
    s["c"].copy_(c.to(torch.bfloat16))
    return {"c": s["c"]}


def _row_map(s):
    """Per row: its request, its place in the request, its position; per request: its rows, its tokens."""
    cu = torch.from_numpy(s["cu"]).cuda().long()
    n = cu[1:] - cu[:-1]
    req = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n)
    j = torch.arange(len(req), device="cuda") - cu[req]
    have = s["len"].long()[s["seq"].long()]
    return req, j, (have - n)[req] + j if s["pos"] is None else s["pos"].long(), n, have


def _rotated(x, at):
    half = x.shape[-1] // 2
    angle = at[:, None].double() * THETA ** (-torch.arange(half, device="cuda").double() / half)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain_append(s):
    c, width = s["case"], s["table"].shape[1]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    req, _, at, n, have = _row_map(s)
    q, k, v = s["qkv"].float().split([hq * d, hkv * d, hkv * d], 1)
    s["q_out"].copy_(_rotated(q.view(-1, hq, d), at).to(_dt(c)))
    k, v = _rotated(k.view(-1, hkv, d), at), v.view(-1, hkv, d)
    entry, slot = req * width + at // PAGE, at % PAGE
    used, where = torch.unique(entry, return_inverse=True)  # the touched (request, page) pairs
    e_req, e_page = used // width, used % width
    page = s["table"].long()[s["seq"].long()[e_req], e_page]
    # rows that held a token before and are not written now
    old = have[e_req] if s["pos"] is not None else (have - n)[e_req]
    held = torch.arange(PAGE, device="cuda") < (old - e_page * PAGE)[:, None]
    hit = torch.zeros(len(used), PAGE, dtype=torch.bool, device="cuda")
    hit[where, slot] = True
    kept = (held & ~hit).any(1)
    _put(s, "k", k, page, where, slot, hit, kept)
    _put(s, "v", v, page, where, slot, hit, kept)
    return _append_out(s)


def _put(s, name, x, page, where, slot, hit, kept):
    hkv = x.shape[1]
    top = torch.zeros(len(page), hkv, device="cuda")
    top.scatter_reduce_(0, where[:, None].expand(-1, hkv), x.abs().amax(-1), "amax")
    present = torch.where(kept[:, None], s[name + "_scale"][0][page], 0.0)
    scale = torch.maximum(present, torch.where(top > 0, torch.exp2(_exponent(top).float()), 0.0))
    safe = torch.where(scale > 0, scale, 1.0)
    pool = s[name][0].view(torch.uint8)
    block = pool[page].view(torch.float8_e4m3fn).float()  # [pages][hkv][64][d] or its transpose
    block = block.transpose(2, 3) if name == "v" else block
    keep = kept[:, None, None, None] & ~hit[:, None, :, None]
    block = torch.where(keep, block * (present / safe)[..., None, None], 0.0).to(torch.float8_e4m3fn)
    block = block.view(torch.uint8).permute(0, 2, 1, 3).contiguous()  # [pages][64][hkv][d]
    block[where, slot] = (x / safe[where][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    block = block.permute(0, 2, 1, 3)
    pool[page] = block.transpose(2, 3).contiguous() if name == "v" else block.contiguous()
    s[name + "_scale"][0][page] = scale


def _plain_attn(s):
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    req, j, limit, n, _ = _row_map(s)
    b, rows, most = len(n), int(np.max(np.diff(s["cu"]))), _pages(s["max_len"])
    ids = s["table"].long()[s["seq"].long()][:, :most].clamp(min=0)  # past a sequence's pages: hidden below
    k = s["k"][0].view(torch.uint8)[ids].view(torch.float8_e4m3fn).float() * s["k_scale"][0][ids][..., None, None]
    v = s["v"][0].view(torch.uint8)[ids].view(torch.float8_e4m3fn).float() * s["v_scale"][0][ids][..., None, None]
    k = k.permute(0, 2, 4, 1, 3).reshape(b, hkv, d, most * PAGE)
    v = v.permute(0, 2, 1, 4, 3).reshape(b, hkv, most * PAGE, d)
    q = torch.zeros(b, rows, hq, d, device="cuda")
    q[req, j] = s["q"].float()
    lim = torch.full((b, rows), -1, device="cuda")
    lim[req, j] = limit
    g = hq // hkv
    q = q.view(b, rows, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, rows * g, d)
    x = (q @ k) * (1 / math.sqrt(d))
    hide = torch.arange(most * PAGE, device="cuda") > lim[..., None]  # [b][rows][keys]
    x = x.view(b, hkv, rows, g, -1).masked_fill_(hide[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[..., 0]
    p = p / torch.where(total == 0, 1.0, total)
    o = (p.reshape(b, hkv, rows * g, -1) @ v).view(b, hkv, rows, g, d)
    s["o"].copy_(o.permute(0, 2, 1, 3, 4).reshape(b, rows, hq, d)[req, j].to(_dt(c)))
    s["lse"].copy_(lse.permute(0, 2, 1, 3).reshape(b, rows, hq)[req, j].t())
    return {"o": s["o"], "lse": s["lse"]}


# ---- exact results, from the definitions ------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        return _exact_norm(case, s)
    if kind == "linear":
        return _exact_linear(case, s)
    return _exact_append(case, s) if kind == "append" else _exact_attn(case, s)


def _exact_e4m3(x):
    """The nearest e4m3 value (ties to even) of float64 values of at most 448."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_scale(top, zero):
    """Of a tensor of largest magnitudes; `zero` where they are 0."""
    e = torch.full_like(top, MIN_EXP)
    e = torch.maximum(e, torch.ceil(torch.log2(top.clamp(min=2.0 ** -200) / 448)))
    e = torch.where((e > MIN_EXP) & (top <= 448 * torch.exp2(e - 1)), e - 1, e)  # of a rounded logarithm
    e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
    return torch.where(top == 0, zero, torch.exp2(e))


def _exact_norm(case, s):
    h, out = s["x"].double(), {}
    if case["add"]:
        out["sum"] = h + s["delta"].double()
        h = out["sum"].to(_dt(case)).double()  # the norm is that of the rounded sum
    y = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["width"] + EPS) * s["w"].double()
    if case["out"] != "mx":
        out["y"] = y
    if case["out"] != "y":
        y = y.reshape(case["rows"], -1, BLOCK)
        scale = _exact_scale(y.abs().amax(2), 2.0 ** MIN_EXP)
        out["codes"] = _exact_e4m3(y / scale[..., None]).reshape(case["rows"], -1)
        out["scales"] = scale
    return out


def _exact_linear(case, s):
    def e2m1(c):  # two exponent bits, one mantissa bit
        e, m = (c >> 1 & 3).double(), (c & 1).double()
        return torch.where(e == 0, m / 2, torch.exp2(e - 1) * (1 + m / 2)) * (1 - 2 * (c >> 3).double())

    n, k = case["n"], case["k"]
    w = torch.empty(n, k, dtype=torch.float64, device="cuda")
    w[:, 0::2], w[:, 1::2] = e2m1(s["w"] % 16), e2m1(s["w"] // 16)
    w *= torch.exp2(s["w_scales"].double() - 127).repeat_interleave(BLOCK, 1)
    a = s["a"].double()
    if case["a"] == "mx":
        a = a * torch.exp2(s["a_scales"].double() - 127).repeat_interleave(BLOCK, 1)
    c = torch.mm(a, w.t().contiguous())
    if case["bias"]:
        c += s["bias"].double()
    if case["residual"]:
        c += s["residual"].double()
    return {"c": c}


def _exact_append(case, s):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    lens, cu, seq = _ints(case["lens"]), s["cu"].tolist(), s["seq"].tolist()
    table = s["table"].cpu().numpy()
    pos = None if s["pos"] is None else s["pos"].cpu().numpy()
    at = [np.arange(L - cu[b + 1] + cu[b], L) if pos is None else pos[cu[b]:cu[b + 1]] for b, L in enumerate(lens)]
    rows = s["qkv"].double().view(-1, hq + 2 * hkv, d)
    # features i and i + d/2 as a complex number, turned by its angle
    angle = np.concatenate(at)[:, None] * np.power(THETA, -np.arange(d // 2) * 2.0 / d)
    turn = torch.from_numpy(np.exp(1j * angle)).cuda()[:, None]
    z = torch.complex(rows[:, :hq + hkv, :d // 2], rows[:, :hq + hkv, d // 2:]) * turn
    z = torch.cat([z.real, z.imag], -1)
    out = {"q": z[:, :hq]}
    for name, x in (("k", z[:, hq:]), ("v", rows[:, hq + hkv:])):
        code, scale = s[name].double(), s[name + "_scale"].double()
        code = code.transpose(3, 4).contiguous() if name == "v" else code  # [1][pages][hkv][64][d]
        for b, L in enumerate(lens):
            before = L if pos is not None else L - len(at[b])
            for p in np.unique(at[b] // PAGE).tolist():
                here = np.nonzero(at[b] // PAGE == p)[0]
                slots = at[b][here] - p * PAGE
                stay = np.setdiff1d(np.arange(max(0, min(PAGE, before - p * PAGE))), slots)
                page, new = int(table[seq[b], p]), x[torch.from_numpy(cu[b] + here).cuda()].transpose(0, 1)
                sc = _exact_scale(new.abs().amax((1, 2)), 0.0)
                block = torch.zeros_like(code[0, page])
                if len(stay):
                    sc = torch.maximum(sc, scale[0, page])
                    ratio = torch.where(sc > 0, scale[0, page] / sc, 0.0)
                    block = _exact_e4m3(code[0, page] * ratio[:, None, None])
                block[:, torch.from_numpy(slots).cuda()] = _exact_e4m3(new / torch.where(sc > 0, sc, 1.0)[:, None, None])
                code[0, page], scale[0, page] = block, sc
        out[name] = code.transpose(3, 4).contiguous() if name == "v" else code
        out[name + "_scale"] = scale
    return out


def _exact_attn(case, s):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    seq, cu, lens = s["seq"].long(), s["cu"].tolist(), _ints(case["lens"])
    out = torch.zeros(cu[-1], hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(hq, cu[-1], dtype=torch.float64, device="cuda")
    for b, L in enumerate(lens):
        pages = s["table"][seq[b], :_pages(L)].long()
        n = cu[b + 1] - cu[b]
        last = torch.arange(L - n, L, device="cuda") if s["pos"] is None else s["pos"][cu[b]:cu[b + 1]].long()
        unseen = torch.arange(L, device="cuda")[None] > last[:, None]
        kk, vv = s["k"][0].view(torch.uint8)[pages], s["v"][0].view(torch.uint8)[pages]
        for h in range(hkv):
            ks, vs = s["k_scale"][0, pages, h].double(), s["v_scale"][0, pages, h].double()
            k = (kk[:, h].contiguous().view(torch.float8_e4m3fn).double() * ks[:, None, None]).reshape(-1, d)[:L]
            v = vv[:, h].transpose(1, 2).contiguous().view(torch.float8_e4m3fn).double() * vs[:, None, None]
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            q = s["q"][cu[b]:cu[b + 1], heads].double().transpose(0, 1).reshape(-1, d)
            x = (torch.mm(q, k.t().contiguous()) / d ** 0.5).view(-1, n, L).masked_fill(unseen, -math.inf)
            z = torch.logsumexp(x, 2)
            lse[heads, cu[b]:cu[b + 1]] = z
            w = torch.exp(x - z[..., None]).view(-1, L)
            out[cu[b]:cu[b + 1], heads] = torch.mm(w, v.reshape(-1, d)[:L].contiguous()).view(-1, n, d).transpose(0, 1)
    return {"o": out, "lse": lse}

"""GPU: daf_linear_mx against oracle/step.py (64 bits)."""
from __future__ import annotations

import pytest
import torch

import paper_2607_21599_amd as daf
from oracle import step as orc

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    daf.lib()
    yield
    torch.cuda.synchronize()


def _inputs(m, n, k, mx, seed, spread=3):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def bytes_(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=torch.uint8)

    t = {"w": bytes_(0, 256, n, k // 2), "ws": bytes_(120, 120 + spread, n, k // 32), "as": None}
    x = torch.randn(m, k, generator=gen, device="cuda")
    if mx:
        t["a"], t["as"] = (x * 112).clamp(-448, 448).to(E4M3), bytes_(118, 118 + spread, m, k // 32)
    else:
        t["a"] = x.to(BF16)
    t["bias"] = torch.randn(n, generator=gen, device="cuda").to(BF16)
    t["res"] = torch.randn(m, n, generator=gen, device="cuda").to(BF16)
    return t


def _values(t):
    a = t["a"].double() if t["as"] is None else orc.mx_values(t["a"].double(), t["as"])
    return a, orc.mx_values(orc.e2m1_values(t["w"]), t["ws"])


def _run(t, bias=False, residual=False, stream=None, into=None):
    m, n, k = t["a"].shape[0], t["w"].shape[0], 2 * t["w"].shape[1]
    size = daf.daf_linear_mx_workspace_size(m, n, k)
    ws = torch.full((max(size, 16),), 0xFF, dtype=torch.uint8, device="cuda")  # NaN in every word
    whole = torch.full((m * n + 64,), 77.0, dtype=BF16, device="cuda")
    c = whole[:m * n].view(m, n) if into is None else into
    daf.daf_linear_mx(m, n, k, t["a"], t["as"], t["w"], t["ws"], t["bias"] if bias else None,
                      t["res"] if residual else None, c, ws, size, stream)
    torch.cuda.synchronize()
    assert (whole[m * n:] == 77).all()
    return c


def _check(t, c, bias=False, residual=False):
    """Exact products, K + 2 fp32 sums in any order, half a step of bf16."""
    want, size = orc.linear(*_values(t), t["bias"] if bias else None, t["res"] if residual else None)
    e = (t["a"].shape[1] + 16) * 2.0 ** -24 * size
    tol = e + 2.0 ** -8 * (want.abs() + e)
    err = (c.double() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())


SHAPES = [(1, 1, 32), (1, 16, 256), (2, 5, 64), (3, 17, 288), (16, 64, 512), (17, 33, 96), (31, 1, 4096),
          (33, 130, 1056), (64, 100, 2080), (65, 48, 4128), (130, 257, 512), (1, 4608, 3584), (12, 96, 18944),
          (40, 200, 9472), (8, 20000, 256), (20, 16400, 288), (48, 16390, 96), (100, 1024, 1024)]


@pytest.mark.parametrize("mx", [True, False])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_shapes(m, n, k, mx):
    t = _inputs(m, n, k, mx, m + n + k)
    _check(t, _run(t))
    _check(t, _run(t, True, True), True, True)


@pytest.mark.parametrize("mx", [True, False])
@pytest.mark.parametrize("m,n,k", [(1, 100, 4096), (9, 300, 18944), (16, 48, 544), (30, 64, 2048), (70, 33, 1024),
                                   (5, 17000, 320)])
def test_whole_numbers_are_exact(m, n, k, mx):
    """Products of whole numbers whose sums stay below 2^8: every output is exact."""
    gen = torch.Generator(device="cuda").manual_seed(k + m)
    t = _inputs(m, n, k, mx, 1)
    # at most 40 values of a row are not 0, and of size 1: at most 40 * 6
    a = torch.zeros(m, k, device="cuda")
    at = torch.randint(0, k, (m, 40), generator=gen, device="cuda")
    a.scatter_(1, at, torch.randint(0, 2, (m, 40), generator=gen, device="cuda").float() * 2 - 1)
    t["a"] = a.to(E4M3 if mx else BF16)
    if mx:
        t["as"].fill_(127)
    whole = torch.tensor([0, 2, 4, 5, 6, 7, 8, 10, 12, 13, 14, 15], device="cuda", dtype=torch.uint8)
    pick = torch.randint(0, len(whole), (n, k), generator=gen, device="cuda")
    t["w"] = (whole[pick[:, 0::2]] | whole[pick[:, 1::2]] << 4).contiguous()
    t["ws"].fill_(127)
    want, _ = orc.linear(*_values(t))
    assert torch.equal(_run(t).double(), want)


def test_every_code_and_scale():
    """W's 16 codes under every scale byte against one value 1 of A: the output is the weight, rounded to bf16."""
    k, n = 32, 256 * 16
    code = torch.arange(16, device="cuda", dtype=torch.uint8).repeat(256)
    t = {"w": torch.zeros(n, k // 2, dtype=torch.uint8, device="cuda"), "as": None,
         "ws": torch.arange(256, device="cuda").repeat_interleave(16).to(torch.uint8)[:, None].contiguous(),
         "a": torch.zeros(2, k, dtype=BF16, device="cuda")}
    t["w"][:, 5] = code | code << 4
    t["a"][0, 10], t["a"][1, 11] = 1, 1
    a, w = _values(t)
    want = torch.where(torch.isnan(w).any(1), torch.nan, w[:, 10])
    c = _run(t)
    for row in c.double():
        assert torch.equal(row.isnan(), want.isnan())
        assert torch.equal(row[~want.isnan()], want[~want.isnan()])


def test_every_code_and_scale_of_a():
    """A's 256 codes under every scale byte against a weight 1."""
    k, m = 32, 256
    t = {"a": torch.zeros(m, k, dtype=torch.uint8, device="cuda"), "w": torch.zeros(7, k // 2, dtype=torch.uint8,
                                                                                      device="cuda"),
         "ws": torch.full((7, 1), 127, dtype=torch.uint8, device="cuda")}
    t["w"][:, 8] = 2  # 1 at k = 16
    t["a"][:, 16] = torch.arange(256, device="cuda").to(torch.uint8)
    t["a"] = t["a"].view(E4M3)
    for b in (0, 1, 26, 27, 28, 100, 127, 200, 246, 247, 248, 254, 255):
        t["as"] = torch.full((m, 1), b, dtype=torch.uint8, device="cuda")
        a, w = _values(t)
        want = a[:, 16].to(BF16).double()  # 448 * 2^120 is beyond bf16: infinite
        c = _run(t).double()
        for j in range(7):
            assert torch.equal(c[:, j].isnan(), want.isnan()) and torch.equal(c[:, j].nan_to_num(), want.nan_to_num()), b


def test_nan_and_infinity_stay_in_their_rows():
    t = _inputs(20, 70, 416, False, 5)
    clean = _run(t)
    t["a"][3, 400], t["a"][17, 0] = torch.nan, torch.inf  # in the last block, and where the lanes past the end look
    t["w"][:, 0] = (t["w"][:, 0] & 0xF0) | 2
    c = _run(t)
    assert c[3].isnan().all() and (c[17] == torch.inf).all()
    t2 = dict(t, a=t["a"].clone())
    t2["a"][3, 400], t2["a"][17, 0] = 0, 0
    ok = [i for i in range(20) if i not in (3, 17)]
    assert torch.equal(c[ok], _run(t2)[ok])
    assert clean.isfinite().all()


@pytest.mark.parametrize("m,n,k", [(5, 37, 416), (20, 33, 4128), (3, 16, 32)])
def test_scales_of_any_alignment(m, n, k):
    """Scales from every byte of a word on, to the last byte of their allocation, between bytes of other scales."""
    t = _inputs(m, n, k, True, 21)
    want = _run(t)
    for off in (1, 2, 3):
        u = dict(t)
        for name in ("ws", "as"):
            whole = torch.full((t[name].numel() + off,), 255, dtype=torch.uint8, device="cuda")  # NaN
            whole[off:] = t[name].flatten()
            u[name] = whole[off:].view(t[name].shape)
            assert u[name].data_ptr() % 4 == off
        assert torch.equal(_run(u), want)
        between = torch.full((t["ws"].numel() + 8,), 255, dtype=torch.uint8, device="cuda")
        between[off:off + t["ws"].numel()] = t["ws"].flatten()
        u["ws"] = between[off:off + t["ws"].numel()].view(n, k // 32)
        assert torch.equal(_run(u), want)


@pytest.mark.parametrize("m,n,k", [(3, 65, 512), (12, 96, 18944)])
def test_residual_in_place(m, n, k):
    t = _inputs(m, n, k, True, 8)
    want = _run(t, True, True)
    into = t["res"]
    assert torch.equal(_run(t, True, True, into=into), want)


@pytest.mark.parametrize("m,n,k", [(4, 4608, 3584), (12, 96, 18944)])
def test_another_stream_and_a_graph(m, n, k):
    t = _inputs(m, n, k, True, 11)
    want = _run(t, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(_run(t, True, stream=side), want)
    size = daf.daf_linear_mx_workspace_size(m, n, k)
    ws, c = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda"), torch.zeros(m, n, dtype=BF16, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        daf.daf_linear_mx(m, n, k, t["a"], t["as"], t["w"], t["ws"], t["bias"], None, c, ws, size)
    for i in range(3):
        c.fill_(-1)
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c, want), i

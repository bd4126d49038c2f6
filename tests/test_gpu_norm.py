"""GPU: daf_add_rmsnorm against oracle/step.py (64 bits)."""
from __future__ import annotations

import pytest
import torch

import paper_2607_21599_amd as daf
from oracle import step as orc

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    daf.lib()
    yield
    torch.cuda.synchronize()


def _inputs(rows, width, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, width, generator=gen, device="cuda") * torch.exp(
        2 * torch.randn(rows, 1, generator=gen, device="cuda"))
    delta = torch.randn(rows, width, generator=gen, device="cuda")
    w = 1 + torch.randn(width, generator=gen, device="cuda") / 2
    return x.to(dtype), delta.to(dtype), w.to(dtype)


def _guarded(rows, width, dtype):
    """Rows with a row of a known value before and after them."""
    whole = torch.full((rows + 2, width), 77.0, device="cuda").to(dtype)
    return whole, whole[1:-1]


def _ran(x, delta, w, eps=EPS, y=True, codes=True, into=None, stream=None):
    """The call on guarded outputs; sum, y, codes, scales, or None where not wanted."""
    rows, width = x.shape
    whole = {"sum": _guarded(rows, width, x.dtype) if delta is not None else None,
             "y": _guarded(rows, width, x.dtype) if y else None,
             "codes": _guarded(rows, width, torch.float8_e4m3fn) if codes else None,
             "scales": _guarded(rows, width // 32, torch.uint8) if codes else None}
    out = {n: v[1] if v else None for n, v in whole.items()}
    # a row before them, so that its end need not be aligned to 16 bytes: copies where it is not
    for n in ("sum", "y", "codes"):
        if out[n] is not None and out[n].data_ptr() % 16:
            whole[n] = None
            out[n] = out[n].clone()
    if into:
        out.update(into)
    daf.daf_add_rmsnorm(daf.DAF_BF16 if x.dtype == BF16 else daf.DAF_F32, rows, width, x, delta, w, eps, out["sum"],
                        out["y"], out["codes"], out["scales"], stream)
    torch.cuda.synchronize()
    for n, v in whole.items():
        if v is not None:
            ends = v[0][[0, -1]].float()
            assert torch.equal(ends, torch.full_like(ends, 77.0).to(v[0].dtype).float()), n
    return out


def _check(x, delta, w, out, eps=EPS):
    """fp32 arithmetic: a thread's chain of the sum of squares has at most width / 64 + 8 terms, the
    joins 14 more; the root halves their error; 8 roundings follow. Then half a step of the output."""
    rows, width = x.shape
    e = ((width / 64 + 24) / 2 + 8) * 2.0 ** -24
    half = 2.0 ** -8 if x.dtype == BF16 else 2.0 ** -24
    s = x
    if delta is not None:
        s = out["sum"]
        want = x.double() + delta.double()
        assert ((s.double() - want).abs() <= (half + 2.0 ** -24) * want.abs()).all()
    want = orc.rmsnorm(s, w, eps)
    if out["y"] is not None:
        assert ((out["y"].double() - want).abs() <= (e + half) * want.abs() + 1e-44).all()
    if out["codes"] is None:
        return
    top = want.view(rows, -1, 32).abs().amax(2)
    b = out["scales"].double()
    assert ((b >= 27) & (b <= 247)).all()
    scale = torch.exp2(b - 127)
    assert (top * (1 - e) <= 448 * scale).all()
    assert ((b == 27) | (top * (1 + e) >= 224 * scale)).all(), "a smaller scale would do"
    scale = scale.repeat_interleave(32, 1)
    got = out["codes"].double() * scale
    tol = torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * scale) + 2 * e * want.abs()
    assert ((got - want).abs() <= tol).all(), float(((got - want).abs() / tol).max())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,width", [(1, 8), (1, 32), (3, 64), (2, 3584), (7, 4096), (5, 4128), (33, 8192),
                                        (2, 32768), (3, 40000), (1500, 96), (1025, 3584), (1100, 4096), (1030, 4128)])
def test_rows_of_every_width(rows, width, dtype):
    x, delta, w = _inputs(rows, width, dtype, rows + width)
    for d in (delta, None):
        for y, codes in ((True, width % 32 == 0), (False, True), (True, False)):
            if codes and width % 32:
                continue
            _check(x, d, w, _ran(x, d, w, y=y, codes=codes))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [512, 544, 1024, 1056, 2048, 2080, 4096, 4128, 8224, 16384, 16416])
def test_nothing_is_written_past_the_last_row(width, dtype):
    """Every number of waves per row, with every number of rows in the last workgroup: inputs, and eight rows
    before and behind each output, stay."""
    for rows in range(1, 10):
        x, delta, w = _inputs(rows, width, dtype, rows)
        kept = [v.clone() for v in (x, delta, w)]
        whole = {}
        for n, cols, t in (("sum", width, dtype), ("y", width, dtype), ("codes", width, torch.float8_e4m3fn), ("scales", width // 32, torch.uint8)):
            whole[n] = torch.full((rows + 16, cols), 77.0, device="cuda").to(t)
        out = {n: v[8:-8] for n, v in whole.items()}
        daf.daf_add_rmsnorm(daf.DAF_BF16 if dtype == BF16 else daf.DAF_F32, rows, width, x, delta, w, EPS, out["sum"], out["y"],
                            out["codes"], out["scales"])
        torch.cuda.synchronize()
        for n, v in whole.items():
            ends = torch.cat([v[:8], v[-8:]]).float()
            assert torch.equal(ends, torch.full_like(ends, 77.0).to(v.dtype).float()), (n, rows)
        assert all(torch.equal(a, b) for a, b in zip(kept, (x, delta, w)))
        _check(x, delta, w, out)


def test_codes_are_those_of_the_rounding_of_y():
    """Both outputs of one call, and those of a call each, are the same bits."""
    x, delta, w = _inputs(40, 3584, BF16, 3)
    both = _ran(x, delta, w)
    one, other = _ran(x, delta, w, codes=False), _ran(x, delta, w, y=False)
    assert torch.equal(both["y"], one["y"]) and torch.equal(both["sum"], one["sum"])
    assert torch.equal(both["codes"].view(torch.uint8), other["codes"].view(torch.uint8))
    assert torch.equal(both["scales"], other["scales"])


def test_without_delta_as_daf_rmsnorm():
    """fp32 rounding apart: half a step and the arithmetic of both."""
    x, _, w = _inputs(65, 3584, BF16, 4)
    y = torch.empty_like(x)
    daf.daf_rmsnorm(65, 3584, x, w, EPS, y)
    got = _ran(x, None, w, codes=False)["y"]
    assert ((got.double() - y.double()).abs() <= 2.0 ** -7 * y.double().abs()).all()


@pytest.mark.parametrize("rows,width", [(3, 96), (1100, 512), (2, 40000)])
def test_outputs_in_place(rows, width):
    x, delta, w = _inputs(rows, width, BF16, width)
    want = _ran(x, delta, w, codes=False)
    for sum_in, y_in in (("x", None), ("delta", None), ("x", "delta"), ("delta", "x"), (None, "x"), (None, "delta")):
        t = {"x": x.clone(), "delta": delta.clone()}
        into = {}
        if sum_in:
            into["sum"] = t[sum_in]
        if y_in:
            into["y"] = t[y_in]
        if not sum_in:
            into["sum"] = None
        out = _ran(t["x"], t["delta"], w, codes=False, into=into)
        assert torch.equal(out["y"], want["y"]), (sum_in, y_in)
        if sum_in:
            assert torch.equal(out["sum"], want["sum"]), (sum_in, y_in)


def test_zeros_infinities_and_nan():
    x = torch.ones(6, 64, device="cuda")
    x[0] = 0                # zeros: y 0, codes 0, the smallest scale
    x[1, 3] = torch.inf     # mean infinite: 1 / inf = 0, inf * 0 = NaN there, 0 elsewhere
    x[2, 40] = torch.nan    # a row with NaN is NaN
    x[3] = 1e-30            # below eps
    w = torch.ones(64, device="cuda")
    w[5] = torch.inf
    out = _ran(x, None, w, eps=EPS)
    y, codes, scales = out["y"], out["codes"].float(), out["scales"]
    inf_at = torch.arange(64, device="cuda") == 5
    assert (y[0][~inf_at] == 0).all() and y[0, 5].isnan()  # 0 * inf
    assert codes[0, 5].isnan() and (codes[0][~inf_at] == 0).all() and scales[0].tolist() == [27, 27]
    assert y[1, 3].isnan() and codes[1, 3].isnan() and (y[1][[0, 1, 63]] == 0).all()
    assert y[2].isnan().all() and codes[2].isnan().all()
    assert scales[2].tolist() == [27, 27]  # NaN does not count
    assert y[4, 5] == torch.inf
    # infinity counts as the largest finite value: 2^128 (1 - 2^-24) <= 448 * 2^120
    assert scales[4, 0] == 247 and codes[4, 5] == 256 and scales[4, 1] == 119  # 1 = 256 * 2^-8


def test_another_stream_and_a_graph():
    x, delta, w = _inputs(33, 3584, BF16, 9)
    want = _ran(x, delta, w)
    side = torch.cuda.Stream()
    out = {n: torch.zeros_like(v) for n, v in want.items()}

    def call(stream=None):
        daf.daf_add_rmsnorm(daf.DAF_BF16, 33, 3584, x, delta, w, EPS, out["sum"], out["y"], out["codes"],
                            out["scales"], stream)

    def same():
        return all(torch.equal(out[n].view(torch.uint8), want[n].view(torch.uint8)) for n in want)

    side.wait_stream(torch.cuda.current_stream())
    call(side)
    torch.cuda.synchronize()
    assert same()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(3):
        for v in out.values():
            v.view(torch.uint8).fill_(1)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert same()

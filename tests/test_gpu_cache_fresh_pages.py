"""GPU: pages that extend has just taken. Whatever their last owner, or the memory of a
new pool, left in them does not count for the rows that are written there."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from test_gpu_cache import BF16, F32, _cu, _pair, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import paper_2607_21599_amd as daf
    daf.lib()
    yield
    torch.cuda.synchronize()


def _leave(p, scale, codes=None):
    """What memory may hold where a pool is made: the same in every page, of both sides."""
    for n in "kv":
        p.t[n + "_scale"].fill_(scale)
        p.o.scale[n][:] = scale
        if codes is not None:
            p.t[n].view(torch.uint8).fill_(codes)
            p.o.code[n][:] = float(torch.tensor([codes], dtype=torch.uint8).view(torch.float8_e4m3fn).float())


@pytest.mark.parametrize("dtype,d,heads", [(BF16, 128, 2), (F32, 64, 3)])
@pytest.mark.parametrize("scale", [float("inf"), float("nan"), 1.5, 2.0 ** 100, -1.0])
def test_two_calls_fill_what_one_would(dtype, d, heads, scale):
    """Two documents' rows written by a call each, into pages of which one has rows of both,
    beside the same rows in one call on a clean pool."""
    rng = np.random.default_rng(d)
    n = [100, 150]
    k, v = (torch.from_numpy(rng.standard_normal((250, heads, d))).float().clamp(-3, 3) for _ in "kv")
    for x in (k, v):  # the first document has the largest magnitude, so that no scale grows
        x[::5, :, 0] = 4.0
        x[n[0]:, :, 0] = 0.0
    seen = []
    for halves in (True, False):
        p = _pair(layers=2, pages=6, heads=heads, d=d, n_seqs=2, max_seq_pages=5, dtype=dtype)
        if halves:
            _leave(p, scale, 0x7F)
        assert p.extend([1], [250]) == 0
        for layer in (1, 0):
            if halves:
                p.write(layer, [0, 100], [1], k[:100], v[:100], np.arange(100))
                p.write(layer, [0, 150], [1], k[100:], v[100:], np.arange(100, 250))
            else:
                p.write(layer, [0, 250], [1], k, v)
            seen.append(p.read(layer, [0, 250], [1]))
        if halves:  # the free pages too, which keep what they held
            for name in "kv":
                code = p.t[name].double().cpu().numpy()
                code = code.swapaxes(-1, -2) if name == "v" else code
                assert np.array_equal(p.t[name + "_scale"].cpu().numpy(), p.o.scale[name], equal_nan=True)
                assert np.array_equal(code, p.o.code[name], equal_nan=True)
    for two, one in zip(seen[:2], seen[2:]):
        for a, b in zip(two, one):
            assert torch.equal(a, b)
            assert not a.isnan().any()


def test_pages_of_a_freed_sequence():
    """A request with large values goes; the next one's small rows, which come in two
    calls, keep their precision."""
    p = _pair(layers=1, pages=5, heads=2, d=64, n_seqs=3, max_seq_pages=4)
    rng = np.random.default_rng(1)
    assert p.extend([0, 2], [200, 30]) == 0
    p.write(0, [0, 200, 230], [0, 2], _rows(rng, 230, 2, 64, 1e4), _rows(rng, 230, 2, 64, 1e4))
    p.free([0])
    assert p.extend([1], [130]) == 0
    x = torch.from_numpy(rng.uniform(0.25, 0.5, (130, 2, 64))).float()
    for at in (range(0, 50), range(50, 130)):
        p.write(0, [0, len(at)], [1], x[list(at)], -x[list(at)], list(at))
        p.same()
    k, v = p.read(0, [0, 130], [1])
    # half a step of the bf16 input and of a normal code
    assert ((k.float().cpu() - x).abs() <= x * (2.0 ** -4 + 2.0 ** -8)).all() and torch.equal(v, -k)
    # the last pages of sequences that go on keep their scales, those that they take start anew
    assert p.extend([1, 2], [30, 40]) == 0
    p.same()
    for i, s in ((2, 1), (0, 2)):
        assert p.t["k_scale"][0, int(p.o.table[s, i])].min() > 0
    assert not p.t["k_scale"][0, int(p.o.table[2, 1])].any()


def test_fresh_pages_past_the_list_in_shared_memory():
    """More new pages in one call than the plan lists, of several heads and layers."""
    n = 5000
    p = _pair(layers=2, pages=n + 40, heads=3, d=64, n_seqs=3, max_seq_pages=n)
    _leave(p, 7.0)
    assert p.extend([0], [64 * 30]) == 0
    assert p.extend([1, 0, 2], [64 * 4800 - 5, 1, 64 * 100]) == 0
    for name in ("table", "len", "refs"):
        assert np.array_equal(p.t[name].cpu().numpy(), getattr(p.o, name)), name
    for name in "kv":
        s = p.t[name + "_scale"].cpu().numpy()
        assert np.array_equal(s, p.o.scale[name])
        assert (s[:, p.o.refs > 0] == 0).all() and (s[:, p.o.refs == 0] == 7).all()

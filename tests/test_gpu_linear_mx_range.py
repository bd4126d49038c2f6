"""GPU: daf_linear_mx at both ends of its range, where values of codes or their products leave bf16's or fp32's."""
from __future__ import annotations

import pytest
import torch

import paper_2607_21599_amd as daf

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    daf.lib()
    yield
    torch.cuda.synchronize()


def _one(a_code, a_byte, w_code, w_byte, k=64):
    """C of rows with one code of A (a float) each at k = 3 and weights of one code (a nibble) each there; the sizes
    of both are broadcast to [m] and [n]."""
    m, n = len(a_code), len(w_code)
    a = torch.zeros(m, k, device="cuda")
    a[:, 3] = torch.tensor(a_code, device="cuda")
    w = torch.zeros(n, k // 2, dtype=torch.uint8, device="cuda")
    w[:, 1] = torch.tensor(w_code, device="cuda").to(torch.uint8) << 4
    a_s = torch.tensor(a_byte, device="cuda").to(torch.uint8)[:, None].expand(m, k // 32).contiguous()
    w_s = torch.tensor(w_byte, device="cuda").to(torch.uint8)[:, None].expand(n, k // 32).contiguous()
    c = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    daf.daf_linear_mx(m, n, k, a.to(E4M3), a_s, w, w_s, None, None, c, None, 0)
    return c.double()


def test_an_infinity_from_the_norm():
    """x / rms is infinite where w is; its code is 256 * 2^120, which is no bf16 value: infinite with a weight, NaN
    with a weight of 0."""
    x = torch.ones(2, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    w[5] = torch.inf
    codes, scales = torch.zeros(2, 64, dtype=E4M3, device="cuda"), torch.zeros(2, 2, dtype=torch.uint8, device="cuda")
    daf.daf_add_rmsnorm(daf.DAF_F32, 2, 64, x, None, w, 1e-6, None, None, codes, scales)
    assert codes[0, 5].float() == 256 and scales[0, 0] == 247
    wt = torch.zeros(3, 32, dtype=torch.uint8, device="cuda")
    wt[0, 2], wt[1, 2] = 2 << 4, 10 << 4  # 1, -1 and 0 at k = 5
    c = torch.zeros(2, 3, dtype=torch.bfloat16, device="cuda")
    daf.daf_linear_mx(2, 3, 64, codes, scales, wt, torch.full((3, 2), 127, dtype=torch.uint8, device="cuda"), None, None,
                      c, None, 0)
    assert (c[:, 0] == torch.inf).all() and (c[:, 1] == -torch.inf).all() and c[:, 2].isnan().all()


def test_the_largest_values_that_are_finite():
    """240 * 2^120 times a weight of 0.5 and 1 is below 2^128; 256 and 448 are infinite."""
    c = _one([240.0, 256.0, 448.0, -448.0], [247] * 4, [1, 2], [127, 127])
    assert c[0].tolist() == [120.0 * 2.0 ** 120, 240.0 * 2.0 ** 120]
    assert (c[1:3] == torch.inf).all() and (c[3] == -torch.inf).all()


def test_small_products():
    """Exact from 2^-126 on; what lies below may be lost, but is no more than 2^-126."""
    code, bytes_ = [2.0 ** -9, 1.0, 448.0], [27, 60, 90]
    for b in bytes_:
        for wb in (27, 40, 64, 101):
            c = _one(code, [b] * 3, [1, 7, 10], [wb] * 3)
            want = torch.tensor(code, dtype=torch.float64)[:, None] * torch.tensor([0.5, 6.0, -1.0], dtype=torch.float64)
            want = (want * 2.0 ** (b - 127) * 2.0 ** (wb - 127)).cuda()
            normal = want.abs() >= 2.0 ** -126
            near = (c - want).abs() <= 2.0 ** -8 * want.abs()  # the output's rounding
            assert (near | ~normal).all() and ((c - want).abs() <= 2.0 ** -126)[~normal].all(), (b, wb)

"""CPU: weights in 4 bits (tensors.mx_weights) against the nearest values by search."""
import pytest
import torch

from oracle.step import E2M1, e2m1_values, mx_values
from paper_2607_21599_amd.tensors import mx_weights

VALUES = torch.tensor(E2M1, dtype=torch.float64)


def _check(w):
    codes, scales = mx_weights(w)
    n, k = w.shape
    assert codes.shape == (n, k // 2) and scales.shape == (n, k // 32) and codes.dtype == scales.dtype == torch.uint8
    x = w.double().view(n, -1, 32)
    top, s = x.abs().amax(2), torch.exp2(scales.double() - 127)
    assert ((scales >= 27) & (scales <= 247)).all()
    assert ((top <= 6 * s) | (scales == 247)).all() and ((scales == 27) | (top > 3 * s)).all()
    got = mx_values(e2m1_values(codes), scales).view(n, -1, 32)
    off = ((x.abs() / s[..., None])[..., None] - VALUES).abs().amin(3) * s[..., None]  # from the nearest value
    assert torch.equal((got - x).abs(), off)
    assert (got * x >= 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_random_weights(dtype):
    g = torch.Generator().manual_seed(1)
    for size in (1e-35, 1e-3, 1.0, 1e30):
        _check((torch.randn(17, 320, generator=g) * size * torch.exp(torch.randn(17, 1, generator=g))).to(dtype))


def test_values_between_codes_and_borders_of_scales():
    mid = (VALUES[1:] + VALUES[:-1]) / 2
    row = torch.cat([VALUES, mid, -VALUES, -mid, torch.tensor([5.999, 6.0])])[:32]
    w = torch.stack([row * 2.0 ** e for e in (-20, 0, 7)] + [torch.full((32,), x) for x in (6.0, 6.0001, 3.0, 3.0001, 0.0)])
    codes, scales = mx_weights(w.double())
    _check(w.double())
    got = mx_values(e2m1_values(codes), scales)
    # ties go to the code without the lowest bit: 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4
    assert got[1, 8:15].tolist() == [0, 1, 1, 2, 2, 4, 4]
    assert scales[3:, 0].tolist() == [127, 128, 126, 127, 27]


def test_rows_that_are_not_whole_blocks():
    with pytest.raises(ValueError):
        mx_weights(torch.zeros(4, 48))

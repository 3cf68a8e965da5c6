"""How far elements of 4 and 8 bits are off, element by element: half the spacing of the
elements at their magnitude, in groups that the largest scale holds; others saturate."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as qo


def groups(rng, low, high, n=4000):
    x = rng.standard_normal((n, 32)) * np.exp2(rng.integers(low, high, (n, 1)))
    x[::7, rng.integers(0, 32)] *= 64          # one above the others
    return torch.tensor(x).to(torch.bfloat16).double().numpy()


def held(x, bits):
    codes, scales = qo.quantise(x, bits)
    v = qo.values(codes, scales, bits)
    step = np.exp2(scales.astype(float) - 127)
    return v, step


@pytest.mark.parametrize("bits", (4, 8))
def test_half_a_step_at_their_magnitude(bits):
    rng = np.random.default_rng(3)
    grid = qo.elements(bits)[:2 ** (bits - 1)]
    grid = grid[np.isfinite(grid)]
    _, _, fits, most = qo.FORMATS[bits]
    for low, high in ((-3, 3), (-130, 125), (-140, -100), (100, 127)):
        x = groups(rng, low, high)
        x = x[np.isfinite(x).all(-1) & (np.abs(x).max(-1) <= fits * 2.0 ** most)]
        v, step = held(x, bits)
        y = np.abs(x) / step
        at = np.clip(np.searchsorted(grid, y, side="right"), 1, len(grid) - 1)
        spacing = grid[at] - grid[at - 1]      # beyond the largest element: that below it
        assert (np.abs(v / step - x / step) <= spacing / 2).all()
        assert len(x) > 100


@pytest.mark.parametrize("bits,largest", [(4, 6.0), (8, 448.0)])
def test_groups_beyond_the_largest_scale_saturate(bits, largest):
    _, _, fits, most = qo.FORMATS[bits]
    x = np.zeros((3, 32))
    top = (2 - 2.0 ** -7) * 2.0 ** 127         # the largest bf16
    x[0, 3], x[1, 4] = top, -top
    x[2, 5] = fits * 2.0 ** most * (1 + 2.0 ** -6)
    v, step = held(x, bits)
    assert (step == 2.0 ** most).all()
    assert v[0, 3] == largest * 2.0 ** most == -v[1, 4] == v[2, 5]
    half = (2.0 if bits == 4 else 32.0) / 2 * 2.0 ** most
    assert abs(v[0, 3] - top) > half           # half a step does not hold for these


def test_the_largest_of_a_group_in_8_bits():
    """The least power of two that leaves no magnitude beyond the largest element: those that
    would round to it from above, up to 464, take the next."""
    x = np.zeros((3, 32))
    x[0, 0], x[1, 0], x[2, 0] = 448.0, 450.0, 464.0
    codes, scales = qo.quantise(x, 8)
    assert (scales[:, 0].astype(int) - 127).tolist() == [0, 1, 1]
    assert qo.values(codes, scales, 8)[:, 0].tolist() == [448.0, 448.0, 448.0]

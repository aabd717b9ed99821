"""The token operators' GELU where 1 + erf cancels: far on the negative side it
keeps its relative accuracy."""
import math

import pytest
import torch

from oracle import tokens as plain
from paper_1912_03203_amd import dynconv as dc
from tests.test_gpu_tokens import DEV, TYPES, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dc.load()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [20, 500])
def test_gelu_on_the_negative_side(dtype, rows):
    """Products with the identity, so that the value before the activation is exact.
    With z = v / sqrt 2 off by 2^-23 (its constant and its product), erfc(z) moves by at
    most (2 z^2 + 1) times as much; 16 steps of 2^-23 for erfc itself, two roundings."""
    v = torch.linspace(-8.0, 3.0, rows * 16).view(rows, 16).to(dtype)
    y = torch.empty_like(v, device=DEV)
    starts = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    w = torch.eye(16, dtype=dtype)[None]
    got = dc.grouped_linear(dev(v), y, dev(w), None, starts, act=dc.ACT_GELU).cpu().double()
    x = v.double()
    want = 0.5 * x * torch.erfc(-x / math.sqrt(2))
    fp32 = (x * x + 1 + 16 + 1) * 2.0 ** -23 * want.abs()
    assert bool(((got - want).abs() <= plain.stored(want, fp32, dtype)).all())

"""Products with 4-bit weights: calls at the edges of what their documentation allows."""
import numpy as np
import pytest
import torch

from paper_2505_13544_b200 import binding as M

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [0x7F800001, 0x7F80FFFF, 0x7FC00000, 0x7FFFFFFF, -0x7FFFFF, -1])
@pytest.mark.parametrize("n", [3, 20])
def test_every_nan_stays_one(n, bits):
    """fp32 rows are split into terms of 16 bits: a NaN with all of its fraction in the lower half is no infinity."""
    g = torch.Generator(device="cuda").manual_seed(n)
    packed = M.mtla_qweight_pack(torch.randn(256, 40, device="cuda", generator=g))
    x = torch.randn(n, 256, device="cuda", generator=g)
    want = M.mtla_qweight_product(packed, x, 40)
    x[1].view(torch.int32)[77] = bits
    assert torch.isnan(x[1, 77])
    y = M.mtla_qweight_product(packed, x, 40)
    assert torch.isnan(y[1]).all()
    keep = [i for i in range(n) if i != 1]
    assert torch.equal(y[keep], want[keep])

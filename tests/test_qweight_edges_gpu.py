"""Products with 4-bit weights: calls at the edges of what their documentation allows."""
import time

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


@pytest.mark.parametrize("n,n_in,n_out", [(20, 4096, 300), (32, 1024, 129), (40, 128, 1000), (9, 512, 5000), (70, 2048, 20000)])
def test_a_wait_that_runs_out_gives_no_result(n, n_in, n_out):
    """Rows of x that never arrive, for a cluster's CTAs (8, 2) and for CTAs by themselves: every result is NaN, also of the
    CTAs that others' sums are added to; the call after it is an ordinary one."""
    g = torch.Generator(device="cuda").manual_seed(n)
    packed = M.mtla_qweight_pack(torch.randn(n_in, n_out, device="cuda", generator=g))
    x = torch.randn(n, n_in, device="cuda", generator=g).bfloat16()
    want = M.mtla_qweight_product(packed, x, n_out)
    assert torch.isfinite(want).all()
    out = torch.full((n + 1, n_out), 7.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    M.mtla_selftest_qweight_timeout(packed, x, out[:n])
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 1.0
    assert torch.isnan(out[:n]).all() and (out[n:] == 7).all()
    assert torch.equal(M.mtla_qweight_product(packed, x, n_out), want)

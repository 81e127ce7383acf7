"""Attention over the 4-bit pool: every kernel that a call can reach, replayed graphs, overlapping streams."""
import numpy as np
import pytest
import torch

from oracle import qpool_oracle as Q
from paper_2505_13544_b200 import binding as M
from tests.test_operators_gpu import attend_setup, bound, check_attend, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dr", [32, 64])
@pytest.mark.parametrize("heads", [1, 16, 17, 31, 32])
@pytest.mark.parametrize("lens", [[1, 64, 65, 130, 0, 7], [1000], [3] * 60])
def test_the_smallest_batches(lens, heads, dr):
    """r 64 and at most 148 table entries take the warp-level kernel, a wider table the tensor-core kernel: on the
    same batch both stay within the bound, hence within twice the bound of each other."""
    cfg, pages, table, slots, q, seqs = attend_setup(lens, heads, 64, dr, "bf16", 60 + heads)
    assert table.numel() <= 148
    small = check_attend(cfg, pages, table, slots, q, seqs, 0.125, "bf16", lens)
    wide = torch.full((len(lens), 149), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    large = check_attend(cfg, pages, wide, slots, q, seqs, 0.125, "bf16", lens)
    for b, n in enumerate(lens):
        if n:
            want, _, mean_abs = Q.attend(host(q[b]), seqs[b][:, :64], seqs[b][:, 64:], 0.125)
            tol, _ = bound(host(q[b]), seqs[b], 0.125, mean_abs, want, "bf16", 64)
            assert (np.abs(host(small[0][b]) - host(large[0][b])) <= 2 * tol).all()


@pytest.mark.parametrize("r,dr,heads", [(192, 64, 8), (256, 32, 32), (384, 64, 17), (512, 64, 8), (512, 64, 32)])
@pytest.mark.parametrize("batch", [1022, 1023, 4096])
def test_batches_at_the_limits_of_the_tensor_core_kernel(batch, r, dr, heads):
    """1022 sequences are the most whose lists that kernel holds; a few slots each, one longer."""
    rng = np.random.default_rng(batch + r + heads)
    lens = [int(v) for v in rng.choice([0, 1, 2, 3, 5], batch)]
    lens[batch // 2], lens[-1] = 300, 65
    cfg, pages, table, slots, q, seqs = attend_setup(lens, heads, r, dr, "bf16", 70)
    out, lse = M.mtla_qpool_attend(cfg, pages, table, slots, q.cuda(), scale=0.125)
    got, got_lse = out.cpu(), lse.cpu()
    for b in sorted({*range(0, batch, 41), batch // 2, batch - 1}):
        if lens[b] == 0:
            assert (got[b] == 0).all() and torch.isneginf(got_lse[b]).all()
            continue
        want, want_lse, mean_abs = Q.attend(host(q[b]), seqs[b][:, :r], seqs[b][:, r:], 0.125)
        tol, tol_lse = bound(host(q[b]), seqs[b], 0.125, mean_abs, want, "bf16", r)
        assert (np.abs(host(got[b]) - want) <= tol).all(), (b, lens[b])
        assert (np.abs(host(got_lse[b]) - want_lse) <= tol_lse + 2.0 ** -23 * np.abs(want_lse)).all(), b
    none = torch.tensor(lens) == 0
    assert torch.isfinite(got.float()).all() and (got[none] == 0).all()
    assert torch.isneginf(got_lse[none]).all() and torch.isfinite(got_lse[~none]).all()

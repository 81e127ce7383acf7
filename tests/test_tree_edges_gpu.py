"""Drafted trees over the 4-bit pool: what a failure inside leaves, and calls at the edges of what their documentation
allows.  Oracle and tolerances are those of test_tree_gpu.py."""
import ctypes
import time

import numpy as np
import pytest
import torch

from oracle import tree_oracle as T
from paper_2505_13544_b200 import binding as M
from tests.test_operators_gpu import DT, host
from tests.test_tree_gpu import check_tree, dev, pool_of, starts_of, tree_setup

pytestmark = pytest.mark.gpu


def call_args(s):
    return (*s[:5], s[5].cuda(), dev(s[6], torch.int64), s[7].cuda())


# slots, nodes, heads, r, type: up to 2 columns an SM, up to 8, more; more than 148 groups of 64 columns.
JOINS = [([300, 0], [3, 2], 4, 128, "bf16"), ([300, 0, 70], [20, 9, 4], 16, 192, "bf16"),
         ([300, 0, 70], [20, 9, 16], 31, 256, "bf16"), ([130, 0, 64, 1, 300], [64] * 5, 32, 64, "bf16"),
         ([300, 0], [3, 2], 4, 128, "fp32"), ([300, 0, 70], [20, 9, 4], 16, 192, "fp32"),
         ([300, 0, 70], [20, 9, 16], 31, 256, "fp32")]


@pytest.mark.parametrize("case", range(len(JOINS)))
def test_a_wait_that_runs_out_gives_no_result(case):
    """A bounded wait that gives up leaves the list of parts unwritten.  Here it says that every group has 200 parts (which
    the workspace does have room for): all nodes get NaN whatever it says, nodes of no request stay as they were, and
    the next call on the same workspace is an ordinary one."""
    lens, counts, heads, r, dtype = JOINS[case]
    s = tree_setup(lens, counts, heads, r, 32, dtype, case, front=1, pad=2)
    args, n = call_args(s), sum(counts)
    ws = torch.zeros(M.mtla_qpool_tree_workspace_bytes(s[0], len(lens), n + 3), dtype=torch.uint8, device="cuda")
    out = torch.full((n + 3, heads, r), 7.0, dtype=DT[dtype], device="cuda")
    lse = torch.full((n + 3, heads), 7.0, device="cuda")
    for parts in (0, 200 << 32):                             # none; the first 200
        ws.view(torch.int64).fill_(parts)
        out.fill_(7), lse.fill_(7)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        M.mtla_selftest_tree_timeout(*args, scale=0.125, out=out, lse=lse, workspace=ws)
        torch.cuda.synchronize()
        assert time.perf_counter() - t0 < 1.0
        for t in (out, lse):
            assert torch.isnan(t[1:n + 1]).all() and (t[:1] == 7).all() and (t[n + 1:] == 7).all()
    check_tree(s, 0.125, dtype, lens, nodes=set(range(0, n + 3, 5)), workspace=ws)


@pytest.mark.parametrize("heads,count", [(4, 3), (32, 2), (16, 9)])
def test_first_slots_whose_scores_are_minus_infinity(heads, count):
    """Keys of minus infinity (of bf16 queries with a positive element there) take their slots out, also where a CTA's
    share begins with whole tiles of them: the scores behind them set the references."""
    r, dr, batch = 128, 32, 200
    lens, hidden = [[500, 130, 700, 129][b % 4] for b in range(batch)], [[256, 129, 300, 128][b % 4] for b in range(batch)]
    cfg, pages, table, slots, starts, rows, seen, q, seqs, host_starts = tree_setup(lens, [count] * batch, heads, r, dr, "bf16", 31)
    q[..., r] = q[..., r].abs() + 0.5
    q *= 4
    table_h = table.cpu()
    at = torch.cat([table_h[b, torch.arange(n) // 64].long() * 64 + torch.arange(n) % 64 for b, n in enumerate(hidden)])
    holes = torch.cat([torch.from_numpy(v[:n]).float() for v, n in zip(seqs, hidden)])
    holes[:, r] = -float("inf")
    M.mtla_qpool_write(cfg, pages, holes.cuda(), at.cuda())
    s = (cfg, pages, table, slots, starts, rows, seen, q, [v[n:] for v, n in zip(seqs, hidden)], host_starts)
    check_tree(s, 0.125, "bf16", [n - h for n, h in zip(lens, hidden)], nodes=set(range(0, batch * count, 7)))


def test_sums_that_are_set_down_twice():
    """344 tiles a group and 372 a CTA: segments of over 256 tiles, whose sums leave tensor memory twice and are added up.
    At tile 250 the scores rise by 5.8, a little more than what a reference may stay behind (8 log 2 = 5.55), so that
    the sums of the first 128 tiles have to be brought to another reference at the second time, and still weigh
    128 e^-5.8 / (94 + 250 e^-5.8) = 0.4 % of the result.  Latents of one sign, so the mean of the relative errors shows what is lost or counted too much: a probability's rounding, 2^-11
    at most; what the matrix unit cuts off in the 1024 products of 128 tiles, less than 2^-22 each (a quarter of 2^-10); the
    results' rounding to bf16, which cancels out over 2048 of them (4 standard deviations are 4 * 2^-8 / sqrt(12 * 2048), a
    quarter of 2^-10): together below 2^-10 + 2^-11."""
    n, heads, r, dr, scale = 44000, 32, 64, 32, 0.5
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randn(n, r + dr, device="cuda", generator=g)
    rows[:, :r] = rows[:, :r].abs() + 0.5
    rows[:, r] = 5.8 / scale * (torch.arange(n, device="cuda") // (250 * 128))
    cfg, pages, order, seq = pool_of(rows, heads, r, dr)
    counts, lens = [64] * 5, [n, n - 5, n - 700, n - 128, n]
    q = torch.randn(320, heads, r + dr, device="cuda", generator=g) * 0.01
    q[..., r] = 1.0
    mine = torch.randn(320, r + dr, device="cuda", generator=g).bfloat16()
    s = (cfg, pages, order[None].repeat(5, 1).contiguous(), dev(lens), dev(starts_of(counts)), mine.cpu(), [0] * 320,
         q.bfloat16().cpu(), [seq] * 5, starts_of(counts))
    nodes = {0, 20, 63, 64, 130, 200, 319}
    out, _ = check_tree(s, scale, "bf16", lens, nodes=nodes)
    for i in nodes:
        want, _, _ = T.attend_node(host(s[7][i]), seq[:lens[i // 64]], np.zeros((0, r + dr)), 0, scale, r)
        assert abs((host(out[i]) / want - 1).mean()) <= 2.0 ** -10 + 2.0 ** -11, i


@pytest.mark.parametrize("case", range(len(JOINS)))
def test_attend_tree_without_the_logarithm(case):
    """A NULL lse: the same outputs, through each of the joins."""
    lens, counts, heads, r, dtype = JOINS[case]
    args = call_args(tree_setup(lens, counts, heads, r, 32, dtype, case, front=1, pad=2))
    cfg, pages, table, slots, starts, rows, seen, q = args
    n = sum(counts)
    want, _ = M.mtla_qpool_attend_tree(*args, scale=0.125)
    out = torch.full((n + 3, heads, r), 7.0, dtype=DT[dtype], device="cuda")
    ws = torch.empty(M.mtla_qpool_tree_workspace_bytes(cfg, len(lens), n + 3), dtype=torch.uint8, device="cuda")
    status = M.load_library().mtla_qpool_attend_tree(
        ctypes.byref(cfg), pages.data_ptr(), table.data_ptr(), table.shape[1], slots.data_ptr(), starts.data_ptr(), len(lens),
        rows.data_ptr(), r + 32, seen.data_ptr(), q.data_ptr(), n + 3, 1 if dtype == "bf16" else 0, 0.125, out.data_ptr(), None,
        ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert status == 0
    torch.cuda.synchronize()
    assert torch.equal(out[1:n + 1], want[1:n + 1]) and (out[:1] == 7).all() and (out[n + 1:] == 7).all()

"""Attention over the 4-bit pool: every kernel that a call can reach, replayed graphs, overlapping streams."""
import numpy as np
import pytest
import torch

from oracle import qpool_oracle as Q
from paper_2505_13544_b200 import binding as M
from tests.test_operators_gpu import attend_setup, bound, check_attend, host, rope_bound

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


def test_a_captured_step_follows_the_lengths():
    """One graph of all four calls, replayed while requests grow on the device, over pages whose visible slots
    all hold finite rows: every output against the oracle, from buffers filled with something else before."""
    heads, r, dr, stride, batch, width, n_pages = 16, 64, 32, 2, 2, 5, 40
    cfg = M.make_qpool_config(n_heads=heads, latent_rank=r, rope_dim=dr, n_pages=n_pages)
    pages, rope, freq = M.make_qpool(cfg), M.make_rope_config(rope_dim=dr), Q.rope_frequencies(dr)
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    table, held, fresh = torch.full((batch, width), -1, **i32), torch.zeros(batch, **i32), torch.ones(batch, **i32)
    free, m = torch.arange(20, **i32), M.make_slot_map(batch, batch)
    rows = torch.randn(batch, r + dr, device="cuda", generator=g).bfloat16()
    q = torch.randn(batch, heads, r + dr, device="cuda", generator=g).bfloat16()
    turned = torch.empty_like(rows)
    out, lse = torch.empty(batch, heads, r, dtype=q.dtype, device="cuda"), torch.empty(batch, heads, device="cuda")
    ws = torch.empty(M.mtla_qpool_workspace_bytes(cfg, batch), dtype=torch.uint8, device="cuda")

    def step():
        M.mtla_slot_map(held, fresh, free, table, stride=stride, out=m)
        M.mtla_rope(rope, [rows[:, None]], m.position, first=r, out=[turned[:, None]])
        M.mtla_qpool_write(cfg, pages, turned, m.store)
        M.mtla_qpool_attend(cfg, pages, table, m.slots, q, scale=0.125, out=out, lse=lse, workspace=ws)

    everything = torch.arange(n_pages * 64, device="cuda")
    stored = torch.randn(n_pages * 64, r + dr, device="cuda", generator=g).bfloat16()
    M.mtla_qpool_write(cfg, pages, stored, everything)
    clean = pages.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([0, 0], [1, 0], [5, 6], [126, 127], [127, 300], [128, 129], [255, 2], [300, 511]):
        o_table = [[-1] * width for _ in range(batch)]
        for b, h in enumerate(lens):                  # the pages that the held tokens have
            for p in range(-(-(-(-h // stride)) // 64)):
                o_table[b][p] = 39 - p - 8 * b
        table.copy_(torch.tensor(o_table))
        held.copy_(torch.tensor(lens))
        pages.copy_(clean)
        for t in (out, lse, turned):
            t.fill_(-123.0)
        for t in (m.starts, m.seq, m.position, m.slot, m.store, m.slots, m.taken):
            t.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        want = Q.slot_map(lens, [1] * batch, stride, o_table, list(range(20)))
        assert table.tolist() == o_table and m.taken.item() == want["taken"] and m.slots.tolist() == want["slots"]
        assert m.store.tolist() == want["store"] and m.position.tolist() == lens
        turn = Q.rope(host(rows[:, None]), lens, freq, "interleaved", r)
        tol = rope_bound(rows[:, None], turn, r, dr, "interleaved", 1.0, "bf16")
        assert (np.abs(host(turned[:, None]) - turn) <= tol).all()
        now = host(M.mtla_qpool_read(cfg, pages, everything, dtype=torch.float32))
        byte, code = Q.quantise(host(turned)[:, :r])
        for b in range(batch):
            row = now[want["store"][b]]
            assert np.array_equal(row[:r], Q.dequantise(byte, code)[b]) and np.array_equal(row[r:], host(turned[b, r:]))
            n = want["slots"][b]
            seq = now[[o_table[b][j // 64] * 64 + j % 64 for j in range(n)]]
            exact, exact_lse, mean_abs = Q.attend(host(q[b]), seq[:, :r], seq[:, r:], 0.125)
            tol, tol_lse = bound(host(q[b]), seq, 0.125, mean_abs, exact, "bf16", r)
            assert (np.abs(host(out[b]) - exact) <= tol).all(), (lens, b)
            assert (np.abs(host(lse[b]) - exact_lse) <= tol_lse + 2.0 ** -23 * np.abs(exact_lse)).all(), (lens, b)


@pytest.mark.parametrize("captured", [False, True])
def test_two_streams_with_a_workspace_each_and_different_batches(captured):
    """Calls that overlap on two streams, each with its own workspace, kept until the end, and its own lengths and
    queries, so that partials of one that reached the other would change a result."""
    cfg, pages, table, slots, q, _ = attend_setup([5000, 40, 700, 0], 8, 256, 32, "bf16", 80)
    calls = []
    for i, lens in enumerate(([5000, 40, 700, 0], [3, 0, 1, 0])):
        t, n, x = table.clone(), torch.tensor(lens, dtype=torch.int32, device="cuda"), (q.cuda() * (1 + i)).contiguous()
        ws = torch.empty(M.mtla_qpool_workspace_bytes(cfg, 4), dtype=torch.uint8, device="cuda")
        want = M.mtla_qpool_attend(cfg, pages, t, n, x, scale=0.125, workspace=ws)
        results = [tuple(torch.full_like(w, 9.0) for w in want) for _ in range(20)]
        calls.append((t, n, x, ws, want, results, torch.cuda.Stream()))
    torch.cuda.synchronize()

    def run(i, k):
        t, n, x, ws, _, results, stream = calls[i]
        M.mtla_qpool_attend(cfg, pages, t, n, x, scale=0.125, workspace=ws, out=results[k][0], lse=results[k][1],
                            stream=torch.cuda.current_stream() if captured else stream)

    if captured:
        graphs = []
        for i in range(2):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[i]):
                for k in range(20):
                    run(i, k)
        for i in range(2):
            with torch.cuda.stream(calls[i][6]):
                graphs[i].replay()
    else:
        for k in range(20):
            for i in range(2):
                run(i, k)
    torch.cuda.synchronize()
    for _, _, _, _, want, results, _ in calls:
        for out, lse in results:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])

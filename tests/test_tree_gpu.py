"""Drafted trees over the 4-bit pool on the GPU against their 64-bit oracle.

Tolerances are sums of the roundings that the kernels make; see test_operators_gpu.bound() for the context's part
and tree_bound() for what the join adds.  Maps have to agree exactly."""
import math

import numpy as np
import pytest
import torch

from oracle import tree_oracle as T
from paper_2505_13544_b200 import binding as M
from tests.test_operators_gpu import DT, attend_setup, bound, half_step, host

pytestmark = pytest.mark.gpu


def dev(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def random_parents(rng, count, reach=5):
    return [int(rng.integers(max(-1, i - reach), i)) for i in range(count)]


def starts_of(counts, front=0):
    return [int(v) for v in np.cumsum([front] + list(counts))]


# ------------------------------------------------------------------------------ maps

def check_map(held, starts, parents, stride):
    n = len(parents)
    m = M.mtla_tree_map(dev(held), dev(starts), dev(parents), stride=stride)
    want = T.tree_map(held, starts, parents, stride, n)
    for name in ("seq", "position", "seen", "slots"):
        assert getattr(m, name).tolist() == want[name], name


@pytest.mark.parametrize("stride", [1, 2, 3, 5])
@pytest.mark.parametrize("counts,front,pad", [([1], 0, 0), ([64], 0, 0), ([0, 0], 0, 3), ([33, 0, 1, 64, 17], 2, 9),
                                              ([5] * 300, 0, 40), ([0, 31, 32, 63], 1, 0)])
def test_tree_map(counts, front, pad, stride):
    rng = np.random.default_rng(sum(counts) * 8 + stride)
    parents = [0] * front + [p for c in counts for p in random_parents(rng, c)] + [7] * pad
    held = [int(v) for v in rng.integers(0, 5000, len(counts))]
    check_map(held, starts_of(counts, front), parents, stride)


@pytest.mark.parametrize("stride", [1, 2, 7])
def test_tree_map_of_chains_and_stars(stride):
    check_map([0, 13], [0, 64, 128], list(range(-1, 63)) + [-1] * 64, stride)


def test_tree_map_of_the_largest_batch():
    rng = np.random.default_rng(2)
    counts = [int(v) for v in rng.integers(0, 9, 4096)]
    parents = [p for c in counts for p in random_parents(rng, c)] + [0] * 5
    check_map([int(v) for v in rng.integers(0, 1 << 30, 4096)], starts_of(counts), parents, 2)


def test_tree_map_refuses_on_the_device():
    chain = list(range(-1, 4))
    check_map([7, -1, 2], [0, 5, 10, 15], chain * 3, 2)                       # negative
    check_map([7, 2 ** 31 - 5, 2 ** 31 - 4], [0, 5, 10, 15], chain * 3, 2)    # last position fits; does not
    check_map([7, 7, 7], [0, 5, 10, 15], chain + [-1, 0, 1, 3, 2] + chain, 2)  # a parent behind its node
    check_map([7, 7], [0, 5, 10], chain + [-2, 0, 1, 2, 3], 2)
    check_map([3, 3], [0, 65, 70], list(range(-1, 64)) + chain, 1)            # 65 nodes
    check_map([3, 3, 3], [0, 6, 4, 10], chain * 2, 1)                         # starts fall
    check_map([3, 3], [0, 6, 11], chain * 2, 1)                               # or leave the nodes
    check_map([3, 3], [-1, 6, 10], chain * 2, 1)


def test_tree_map_without_requests():
    m = M.mtla_tree_map(dev([]), dev([0]), dev([1, 2]), stride=2)
    assert m.seq.tolist() == [-1, -1] and m.position.tolist() == [0, 0] and m.seen.tolist() == [0, 0]


# ------------------------------------------------------------------------------ attention

def tree_bound(q, seq, scale, mean_abs, out, dtype, r, merges):
    """The context's bound over everything that the node sees, and for every drafted row and every part that is
    joined one rescaling of the sums: an exponential, 2^-22, and two roundings of 2^-24."""
    tol, tol_lse = bound(q, seq, scale, mean_abs, out, dtype, r)
    more = merges * (2.0 ** -22 + 2.0 ** -23)
    return tol + 2 * more * mean_abs, tol_lse + more


def tree_setup(lens, counts, heads, r, dr, dtype, seed, masks="tree", front=0, pad=0, **kw):
    cfg, pages, table, slots, _, seqs = attend_setup(lens, heads, r, dr, dtype, seed, **kw)
    rng = np.random.default_rng(seed + 1000)
    n = front + sum(counts) + pad
    starts = starts_of(counts, front)
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(n, heads, r + dr, generator=g).to(DT[dtype])
    rows = torch.randn(n, r + dr, generator=g).to(DT[dtype])
    if masks == "tree":
        parents = [0] * front + [p for c in counts for p in random_parents(rng, c)] + [0] * pad
        seen = T.tree_map([2 * v + 1 for v in lens], starts, parents, 2, n)["seen"]
    else:
        seen = [int(v) for v in rng.integers(-2 ** 63, 2 ** 63, n)]
    return cfg, pages, table, slots, dev(starts), rows, seen, q, seqs, starts


def check_tree(s, scale, dtype, lens, nodes=None, **kw):
    cfg, pages, table, slots, starts_d, rows, seen, q, seqs, starts = s
    r, heads = cfg.latent_rank, cfg.n_heads
    out, lse = M.mtla_qpool_attend_tree(cfg, pages, table, slots, starts_d, rows.cuda(), dev(seen, torch.int64),
                                        q.cuda(), scale=scale, **kw)
    got, got_lse, rows64, q64 = host(out), host(lse), host(rows), host(q)
    for b, n in enumerate(lens):
        context, mine = seqs[b][:max(n, 0)], rows64[starts[b]:starts[b + 1]]
        for i in range(starts[b], starts[b + 1]):
            if nodes is not None and i not in nodes:
                continue
            want, want_lse, mean_abs = T.attend_node(q64[i], context, mine, seen[i], scale, r)
            picked = [mine[j] for j in range(min(64, len(mine))) if seen[i] >> j & 1]
            both = np.concatenate([context, np.array(picked).reshape(-1, r + cfg.rope_dim)])
            if len(both) == 0:
                assert (got[i] == 0).all() and np.isneginf(got_lse[i]).all(), i
                continue
            tol, tol_lse = tree_bound(q64[i], both, scale, mean_abs, want, dtype, r, len(picked) + n // 64 + 2)
            assert np.isfinite(got[i]).all(), i
            worst = (np.abs(got[i] - want) / tol).max()
            assert worst <= 1, (b, i, worst)
            assert (np.abs(got_lse[i] - want_lse) <= tol_lse + 2.0 ** -23 * np.abs(want_lse)).all(), (b, i)
    return out, lse


TREE_CASES = [
    # slots, nodes, heads, r, d_R
    ([1], [1], 1, 64, 32), ([64], [2], 4, 64, 64), ([65, 3], [7, 1], 8, 256, 32), ([63, 0, 129], [5, 4, 0], 16, 512, 64),
    ([0, 0], [3, 1], 3, 128, 32), ([5, 700, 1, 0, 64, 128], [1, 9, 0, 2, 16, 33], 17, 192, 32), ([1000], [3], 32, 512, 64),
    ([300] * 3, [11, 2, 64], 31, 448, 32), ([2, 3, 4], [1, 2, 3], 9, 320, 64), ([1, 0, 2000, 17], [2, 2, 5, 1], 24, 384, 64),
    ([40] * 40, [2] * 40, 5, 128, 64), ([4500], [13], 16, 256, 64), ([127, 128, 129, 191, 192, 193], [4] * 6, 12, 256, 32),
    ([257, 130], [64, 40], 8, 128, 32), ([3000, 10], [1, 40], 2, 512, 32), ([511], [21], 3, 512, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(TREE_CASES)))
def test_attend_tree(case, dtype):
    lens, counts, heads, r, dr = TREE_CASES[case]
    check_tree(tree_setup(lens, counts, heads, r, dr, dtype, case), 1 / math.sqrt(64), dtype, lens)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_masks_of_any_bits(dtype):
    """Random bits, those behind the request's nodes among them; more than 64 nodes, of which 64 can be seen."""
    lens, counts = [100, 0, 5], [70, 9, 1]
    check_tree(tree_setup(lens, counts, 5, 128, 32, dtype, 3, masks="any"), -0.2, dtype, lens)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_nodes_that_see_nothing(dtype):
    lens, counts = [0, 70, 0], [3, 2, 2]
    s = list(tree_setup(lens, counts, 4, 64, 32, dtype, 8))
    s[6] = [0, 2, 0, 0, 1, 0, 0]
    check_tree(s, 0.125, dtype, lens)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_that_are_not_seen_hold_anything(dtype, bad):
    """Nodes 1 and 3 of the first request hold no numbers: whoever does not see them is as before."""
    lens, counts = [90, 10], [5, 2]
    s = list(tree_setup(lens, counts, 6, 128, 64, dtype, 9))
    s[6] = [1, 2, 5, 8 + 1, 16 + 4, 1, 3]
    s[5] = s[5].clone()
    s[5][1] = bad
    s[5][3, 5] = bad
    clean = {0, 2, 4, 5, 6}
    out, lse = check_tree(s, 0.125, dtype, lens, nodes=clean)
    assert torch.isnan(out[1]).any() and not torch.isfinite(out[3].float()).all()


def test_nodes_of_no_request_are_left_as_they_were():
    lens, counts = [70, 3], [3, 4]
    s = tree_setup(lens, counts, 8, 128, 32, "bf16", 4, front=2, pad=3)
    out = torch.full((12, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((12, 8), 7.0, device="cuda")
    check_tree(s, 0.125, "bf16", lens, out=out, lse=lse)
    for t in (out, lse):
        assert (t[:2] == 7).all() and (t[9:] == 7).all() and not (t[2:9] == 7).any()


@pytest.mark.parametrize("starts", [[0, 5, 3], [0, 3, 9], [-1, 3, 7]])
def test_starts_out_of_order_give_nan(starts):
    s = list(tree_setup([70, 3], [3, 4], 8, 128, 32, "bf16", 4))
    out, lse = M.mtla_qpool_attend_tree(*s[:4], dev(starts), s[5].cuda(), dev(s[6], torch.int64), s[7].cuda(), scale=1.0)
    assert torch.isnan(out).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pages_outside_the_pool_are_left_out(dtype):
    lens, counts = [200, 64], [3, 2]
    s = list(tree_setup(lens, counts, 4, 128, 32, dtype, 5))
    s[2] = s[2].clone()
    s[2][0, 1], s[2][1, 0] = s[0].n_pages, -5
    seqs = list(s[8])
    seqs[0] = np.concatenate([seqs[0][:64], seqs[0][128:]])
    seqs[1] = seqs[1][:0]
    s[8] = seqs
    check_tree(s, 0.125, dtype, [136, 0])


def test_slots_past_the_table_count_as_the_table():
    lens, counts = [64, 128], [3, 2]
    s = list(tree_setup(lens, counts, 4, 128, 32, "bf16", 5))
    s[2] = s[2][:, :1].contiguous()
    s[3] = dev([1 << 30, 2 ** 31 - 1])
    check_tree(s, 0.125, "bf16", [64, 64])
    s[3] = dev([-3, -2 ** 31])
    check_tree(s, 0.125, "bf16", [-3, -1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_with_a_stride(dtype):
    lens, counts = [70], [6]
    s = list(tree_setup(lens, counts, 4, 128, 32, dtype, 5))
    wide = torch.full((6, 200), math.nan, dtype=DT[dtype], device="cuda")
    wide[:, 8:168] = s[5].cuda()
    cfg, pages, table, slots, starts_d, rows, seen, q, seqs, starts = s
    want = M.mtla_qpool_attend_tree(cfg, pages, table, slots, starts_d, rows.cuda(), dev(seen, torch.int64), q.cuda(), scale=1.0)
    got = M.mtla_qpool_attend_tree(cfg, pages, table, slots, starts_d, wide[:, 8:168], dev(seen, torch.int64), q.cuda(), scale=1.0)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_node_is_one_query(dtype):
    """Trees of one node that sees only the context are the attention of one query per sequence."""
    lens = [900, 64, 1, 333]
    s = list(tree_setup(lens, [1] * 4, 16, 512, 64, dtype, 6))
    s[6] = [0] * 4
    check_tree(s, 0.125, dtype, lens)


def test_large_values_and_large_scores():
    """Scores whose maxima rise through the whole context and again in the drafted rows."""
    lens, counts = [500], [4]
    s = list(tree_setup(lens, counts, 4, 128, 32, "bf16", 11, size=30.0))
    check_tree(s, 0.01, "bf16", lens)


def test_results_repeat_and_follow_the_lengths_in_a_graph():
    lens, counts = [700, 64, 129, 5], [12, 1, 30, 4]
    cfg, pages, table, slots, starts, rows, seen, q, seqs, host_starts = tree_setup(lens, counts, 8, 256, 32, "bf16", 12)
    rows, q, seen_d = rows.cuda(), q.cuda(), dev(seen, torch.int64)
    n = q.shape[0]
    kw = dict(scale=0.125, out=torch.empty(n, 8, 256, dtype=torch.bfloat16, device="cuda"), lse=torch.empty(n, 8, device="cuda"),
              workspace=torch.empty(M.mtla_qpool_tree_workspace_bytes(cfg, 4, n), dtype=torch.uint8, device="cuda"))
    first = [t.clone() for t in M.mtla_qpool_attend_tree(cfg, pages, table, slots, starts, rows, seen_d, q, **kw)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        M.mtla_qpool_attend_tree(cfg, pages, table, slots, starts, rows, seen_d, q, **kw)
    for _ in range(3):
        kw["out"].fill_(9), kw["lse"].fill_(9), kw["workspace"].fill_(255)
        graph.replay()
        assert torch.equal(kw["out"], first[0]) and torch.equal(kw["lse"], first[1])
    slots.copy_(dev([650, 0, 128, 3]))
    graph.replay()
    out, lse = kw["out"].clone(), kw["lse"].clone()
    check = check_tree((cfg, pages, table, slots, starts, rows, seen, q, seqs, host_starts), 0.125, "bf16", [650, 0, 128, 3])
    assert torch.equal(check[0], out) and torch.equal(check[1], lse)


def test_another_stream_and_two_calls_at_once():
    lens, counts = [2000, 900], [20, 9]
    s = tree_setup(lens, counts, 16, 256, 64, "bf16", 13)
    args = (*s[:5], s[5].cuda(), dev(s[6], torch.int64), s[7].cuda())
    want = M.mtla_qpool_attend_tree(*args, scale=0.125)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [M.mtla_qpool_attend_tree(*args, scale=0.125, stream=st) for _ in range(5) for st in streams]
    torch.cuda.synchronize()
    for out, lse in got:
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_a_verification_step():
    """The operators as a serving loop runs them: a map, products with 4-bit weights, rotations at the nodes' positions,
    attention, the accepted path into the pool; then a plain step over the grown cache sees what the path saw."""
    heads, r, dr, stride, n_pages, d = 4, 128, 32, 1, 8, 64
    cfg = M.make_qpool_config(n_heads=heads, latent_rank=r, rope_dim=dr, n_pages=n_pages)
    pages, rope = M.make_qpool(cfg), M.make_rope_config(rope_dim=dr)
    pages.zero_()
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    held, parents, counts = [100, 3], [-1, 0, 0, 1, 3, -1, 0, 1], [5, 3]
    table = dev([[3, 1, 6], [0, 5, 2]])
    cache = [rand(h, r + dr) for h in held]
    for b, h in enumerate(held):
        at = torch.tensor([int(table[b, j // 64]) * 64 + j % 64 for j in range(h)], device="cuda")
        M.mtla_qpool_write(cfg, pages, cache[b], at)
    m = M.mtla_tree_map(dev(held), dev([0, 5, 8]), dev(parents), stride=stride)
    assert m.slots.tolist() == held
    w_q = M.mtla_qweight_pack(rand(d, heads * (r + dr)) / 8)
    w_c = M.mtla_qweight_pack(rand(d, r + dr) / 8)
    x = rand(8, d)
    q = M.mtla_qweight_product(w_q, x, heads * (r + dr)).view(8, heads, r + dr)
    rows = M.mtla_qweight_product(w_c, x, r + dr)
    q, rows = [t.clone() for t in M.mtla_rope(rope, [q, rows.view(8, 1, r + dr)], m.position, first=r)]
    rows = rows.view(8, r + dr)
    out, lse = M.mtla_qpool_attend_tree(cfg, pages, table, m.slots, dev([0, 5, 8]), rows, m.seen, q, scale=0.1)
    # Path 0, 1, 3 of the first request and 0, 1 of the second are accepted.
    path = {0: [0, 1, 3], 1: [5, 6]}
    index = [-1] * 8
    for b, nodes in path.items():
        for k, i in enumerate(nodes):
            slot = held[b] + k
            index[i] = int(table[b, slot // 64]) * 64 + slot % 64
    M.mtla_qpool_write(cfg, pages, rows, dev(index, torch.int64))
    last = torch.tensor([3, 6], device="cuda")
    again, lse2 = M.mtla_qpool_attend(cfg, pages, table, dev([103, 5]), q[last].contiguous(), scale=0.1)
    # The path's rows are now in 4 bits: at most 3/16 of their group's largest latent off.
    stored = M.mtla_qpool_read(cfg, pages, dev([v for v in index if v >= 0], torch.int64), dtype=torch.float32)
    off = (stored - rows[[0, 1, 3, 5, 6]]).abs().max().item()
    top = rows[:, :r].abs().max().item()
    assert off <= 3 / 16 * top
    for k, (b, nodes) in enumerate(path.items()):
        context = host(M.mtla_qpool_read(cfg, pages, torch.tensor(
            [int(table[b, j // 64]) * 64 + j % 64 for j in range(held[b])], device="cuda"), dtype=torch.float32))
        want, want_lse, mean_abs = T.attend_node(host(q[nodes[-1]]), context, host(rows[nodes]), (1 << len(nodes)) - 1, 0.1, r)
        both = np.concatenate([context, host(rows[nodes])])
        tol, tol_lse = tree_bound(host(q[nodes[-1]]), both, 0.1, mean_abs, want, "fp32", r, len(nodes) + 4)
        assert (np.abs(host(out[nodes[-1]]) - want) <= tol).all()
        shift = np.abs(host(q[nodes[-1]])[:, :r]).sum(-1) * 0.1 * off          # of a path row's score
        assert (np.abs(host(lse2[k]) - host(lse[nodes[-1]])) <= shift + 1e-4).all()


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")
def test_on_another_gpu_than_the_current_one():
    s = tree_setup([100], [5], 4, 64, 32, "bf16", 1)
    args = [s[0]] + [t.cuda() for t in (s[1], s[2], s[3], s[4], s[5], dev(s[6], torch.int64), s[7])]
    want = M.mtla_qpool_attend_tree(*args, scale=1.0)
    with torch.cuda.device(1):
        got = M.mtla_qpool_attend_tree(*args, scale=1.0)
    torch.cuda.synchronize(0)
    assert torch.equal(want[0], got[0])


# ------------------------------------------------------------------------------ many columns, long contexts

def pool_of(rows, heads, r, dr, junk=0xFF):
    """A pool of one sequence's rows (as stored) and its table row."""
    n = rows.shape[0]
    n_pages = -(-n // 64) + 1
    cfg = M.make_qpool_config(n_heads=heads, latent_rank=r, rope_dim=dr, n_pages=n_pages)
    pages = torch.full((n_pages, M.mtla_qpool_page_bytes(cfg)), junk, dtype=torch.uint8, device="cuda")
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(n))[:-(-n // 64)].int().cuda()
    j = torch.arange(n, device="cuda")
    index = order[j // 64].long() * 64 + j % 64
    M.mtla_qpool_write(cfg, pages, rows, index)
    return cfg, pages, order, host(M.mtla_qpool_read(cfg, pages, index, dtype=torch.float32))


@pytest.mark.parametrize("masks", ["tree", "any"])
@pytest.mark.parametrize("r,dr", [(64, 32), (192, 64), (512, 32)])
def test_many_columns(r, dr, masks):
    """More than 148 groups of columns: the drafted rows go through matrix products."""
    lens, counts = [130, 0, 64, 1, 300], [64, 63, 80, 64, 65]
    s = tree_setup(lens, counts, 32, r, dr, "bf16", r, masks=masks, front=3, pad=2)
    out = torch.full((sum(counts) + 5, 32, r), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((sum(counts) + 5, 32), 7.0, device="cuda")
    nodes = {*range(3, 3 + sum(counts), 13), 66, 67, 129, 130, 2 + sum(counts)}
    check_tree(s, 0.125, "bf16", lens, nodes=nodes, out=out, lse=lse)
    for t in (out, lse):
        assert (t[:3] == 7).all() and (t[-2:] == 7).all() and torch.isfinite(t).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_many_columns_and_rows_that_hold_anything(bad):
    """Whoever sees such a row gets NaN, the others are as they were without it, bit by bit."""
    lens, counts = [130, 0, 64, 1, 300], [64, 64, 64, 64, 64]
    s = list(tree_setup(lens, counts, 32, 128, 32, "bf16", 2))
    args = lambda rows: (*s[:5], rows.cuda(), dev(s[6], torch.int64), s[7].cuda())
    clean, clean_lse = M.mtla_qpool_attend_tree(*args(s[5]), scale=0.125)
    rows = s[5].clone()
    rows[5, 3], rows[64 + 17, 130], rows[256] = bad, bad, bad
    out, lse = M.mtla_qpool_attend_tree(*args(rows), scale=0.125)
    sees = torch.tensor([bool((i // 64 == 0 and s[6][i] >> 5 & 1) or (i // 64 == 1 and s[6][i] >> 17 & 1)
                              or (i // 64 == 4 and s[6][i] & 1)) for i in range(320)], device="cuda")
    assert sees.any() and torch.isnan(out[sees]).all() and torch.isnan(lse[sees]).all()
    # (Zeros in the place of the row's numbers: nothing else of a sum changes.)
    assert torch.equal(out[~sees], clean[~sees]) and torch.equal(lse[~sees], clean_lse[~sees])


def test_many_columns_that_see_nothing_and_a_refused_batch():
    lens, counts = [0] * 5, [64] * 5
    s = list(tree_setup(lens, counts, 32, 64, 32, "bf16", 2))
    s[6] = [0 if i % 3 else s[6][i] for i in range(320)]
    check_tree(s, 0.125, "bf16", lens, nodes=set(range(0, 320, 7)))
    out, lse = M.mtla_qpool_attend_tree(*s[:4], dev([0, 64, 32, 192, 256, 320]), s[5].cuda(), dev(s[6], torch.int64),
                                        s[7].cuda(), scale=1.0)
    assert torch.isnan(out).all() and torch.isnan(lse).all()


def test_sums_over_many_tiles():
    """Segments of more than 128 tiles, latents of one sign: the sums leave tensor memory in between, so what the matrix
    unit cuts off does not grow with the length.  Five requests share the pages."""
    n, heads, r, dr = 25600 + 77, 32, 64, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randn(n, r + dr, device="cuda", generator=g)
    rows[:, :r] = rows[:, :r].abs() + 0.5
    cfg, pages, order, seq = pool_of(rows, heads, r, dr)
    counts, lens = [64] * 5, [n, n - 5, 25600, 20000, n]
    q = (torch.randn(320, heads, r + dr, device="cuda", generator=g) * 0.3).bfloat16()
    mine = torch.randn(320, r + dr, device="cuda", generator=g).bfloat16()
    seen = [1 << (i % 64) for i in range(320)]
    s = (cfg, pages, order[None].repeat(5, 1).contiguous(), dev(lens), dev(starts_of(counts)), mine.cpu(),
         [v - (1 << 64) if v >> 63 else v for v in seen], q.cpu(), [seq] * 5, starts_of(counts))
    check_tree(s, 0.125, "bf16", lens, nodes={0, 63, 64, 130, 200, 319})


@pytest.mark.parametrize("heads,count", [(4, 3), (32, 7)])
def test_scores_that_rise_from_tile_to_tile(heads, count):
    """Every tile's largest score exceeds the one before by more than 2^8: references rise and sums are rescaled, in one
    CTA's share and across shares; then the drafted rows exceed them again, or fall far short."""
    n, r, dr = 700, 128, 32
    g = torch.Generator().manual_seed(4)
    q = torch.randn(count, heads, r + dr, generator=g).bfloat16()
    rows = torch.randn(n, r + dr, generator=g) * 0.1
    rows[::50] += q[0, 0].float()[None] * torch.linspace(0.05, 1.0, len(rows[::50]))[:, None]
    cfg, pages, order, seq = pool_of(rows.cuda(), heads, r, dr)
    mine = torch.stack([q[i, 0].float() * f for i, f in zip(range(count), [1.2, 0.01, 0.5, 1.5, 1.0, 0.7, 0.1])]).bfloat16()
    for batch in (1, 200):                             # few and many tiles in a share
        counts, lens = [count] * batch, [n - 3 * (i % 60) for i in range(batch)]
        s = (cfg, pages, order[None].repeat(batch, 1).contiguous(), dev(lens), dev(starts_of(counts)),
             mine.repeat(batch, 1), [(1 << (i % count)) | 1 for i in range(count * batch)], q.repeat(batch, 1, 1),
             [seq] * batch, starts_of(counts))
        check_tree(s, 2.0, "bf16", lens, nodes={*range(count), count * batch - 1, count * batch // 2})


def test_many_requests_and_few_slots():
    """A segment every tile, groups of all widths, requests without slots or nodes between them."""
    rng = np.random.default_rng(8)
    lens = [int(v) for v in rng.choice([0, 1, 70, 128, 129, 200], 300)]
    counts = [int(v) for v in rng.choice([0, 1, 2, 5, 9], 300)]
    for heads, r in ((8, 64), (31, 128), (16, 256)):
        s = tree_setup(lens, counts, heads, r, 32, "bf16", heads)
        check_tree(s, 0.125, "bf16", lens, nodes=set(range(0, sum(counts), 9)))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_most_requests(dtype):
    """4096 requests of one node."""
    lens, counts = [3] * 4096, [1] * 4096
    s = tree_setup(lens, counts, 2, 64, 32, dtype, 5)
    check_tree(s, 0.125, dtype, lens, nodes={0, 1, 31, 32, 2047, 4095})


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("dtype,count,heads", [("bf16", 3, 5), ("bf16", 64, 32), ("fp32", 20, 16)])
def test_a_query_that_is_not_finite_reaches_no_other(dtype, count, heads, bad):
    lens, counts = [300, 65, 200, 1, 130], [count] * 5
    s = list(tree_setup(lens, counts, heads, 128, 32, dtype, 21))
    whole, _ = M.mtla_qpool_attend_tree(*s[:4], s[4], s[5].cuda(), dev(s[6], torch.int64), s[7].cuda(), scale=0.125)
    s[7][1, 2, 7], s[7][count, 0, 130] = bad, bad
    out, lse = M.mtla_qpool_attend_tree(*s[:4], s[4], s[5].cuda(), dev(s[6], torch.int64), s[7].cuda(), scale=0.125)
    keep = torch.ones(5 * count, heads, dtype=torch.bool)
    keep[1, 2] = keep[count, 0] = False
    assert torch.isfinite(lse.cpu()[keep]).all() and torch.isnan(out.cpu()[~keep]).any(-1).all()
    # Rescaling of sums goes by what a warp's columns need together, so the others may move by a few roundings.
    d = (out.cpu()[keep].double() - whole.cpu()[keep].double()).abs().max().item()
    assert d <= 2 * whole.abs().max().item() * (half_step(DT[dtype]) + 2.0 ** -11)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_offsets_past_32_bits(dtype):
    """More than 2^31 elements in the queries, the results and the parts; the requests share their pages."""
    heads, r, dr, batch = 32, 512, 64, 2055
    n = batch * 64
    assert n * heads * r > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(6)
    cfg, pages, order, seq = pool_of(torch.randn(65, r + dr, device="cuda", generator=g), heads, r, dr)
    lens = [65 - i % 3 for i in range(batch)]
    q = torch.empty(n, heads, r + dr, dtype=DT[dtype], device="cuda").normal_(generator=g)
    rows = torch.randn(n, r + dr, device="cuda", generator=g).to(DT[dtype])
    seen = [(1 << i % 64) | 1 for i in range(n)]
    seen = torch.tensor([v - (1 << 64) if v >> 63 else v for v in seen], device="cuda")
    starts = starts_of([64] * batch)
    out, lse = M.mtla_qpool_attend_tree(cfg, pages, order[None].repeat(batch, 1).contiguous(), dev(lens), dev(starts),
                                        rows, seen, q, scale=0.125)
    for i in (0, 63, 64, n // 2 - 1, 2 ** 31 // (heads * (r + dr)), 2 ** 31 // (heads * r) + 1, n - 64, n - 1):
        b = i // 64
        q64, mine, context = host(q[i]), host(rows[64 * b:64 * b + 64]), seq[:lens[b]]
        bits = int(seen[i])
        want, want_lse, mean_abs = T.attend_node(q64, context, mine, bits, 0.125, r)
        both = np.concatenate([context, mine[[j for j in range(64) if bits >> j & 1]]])
        tol, tol_lse = tree_bound(q64, both, 0.125, mean_abs, want, dtype, r, 5)
        assert (np.abs(host(out[i]) - want) <= tol).all(), i
        assert (np.abs(host(lse[i]) - want_lse) <= tol_lse + 2.0 ** -23 * np.abs(want_lse)).all(), i
    assert all(torch.isfinite(out[i:i + 4096]).all() for i in range(0, n, 4096))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pages_past_32_bits(dtype):
    heads, r, dr, n = 8, 512, 64, 200
    size = M.mtla_qpool_page_bytes(M.make_qpool_config(n_heads=heads, latent_rank=r, rope_dim=dr, n_pages=1))
    n_pages = 2 ** 31 // size + 9
    cfg = M.make_qpool_config(n_heads=heads, latent_rank=r, rope_dim=dr, n_pages=n_pages)
    pages = torch.full((n_pages, size), 0xFF, dtype=torch.uint8, device="cuda")
    order = torch.tensor([n_pages - 1, 3, n_pages - 7, n_pages - 2], dtype=torch.int32, device="cuda")
    j = torch.arange(n, device="cuda")
    index = order[j // 64].long() * 64 + j % 64
    g = torch.Generator(device="cuda").manual_seed(9)
    M.mtla_qpool_write(cfg, pages, torch.randn(n, r + dr, device="cuda", generator=g), index)
    seq = host(M.mtla_qpool_read(cfg, pages, index, dtype=torch.float32))
    q = torch.randn(7, heads, r + dr, device="cuda", generator=g).to(DT[dtype])
    rows = torch.randn(7, r + dr, device="cuda", generator=g).to(DT[dtype])
    check_tree((cfg, pages, order[None].repeat(2, 1).contiguous(), dev([n, 65]), dev([0, 4, 7]), rows.cpu(),
                [1, 2, 5, 9, 1, 3, 7], q.cpu(), [seq, seq], [0, 4, 7]), 0.125, dtype, [n, 65])

"""Verification steps with chunks of several tokens: the operators over drafted trees as a serving loop runs them, against
the layer's own incremental decoding (Form I of the oracle, and the decode step of a layer handle)."""
import copy

import numpy as np
import pytest
import torch

from oracle import mtla_oracle as O
from oracle import qpool_oracle as Q
from oracle import tree_oracle as T
from paper_2505_13544_b200 import binding as M
from paper_2505_13544_b200 import synth
from tests import helpers as H
from tests.test_operators_gpu import bound, host
from tests.test_tree_gpu import dev, starts_of

pytestmark = pytest.mark.gpu

# A chain, and a tree whose second branch forks below its first level.
PARENTS = [[-1, 0, 1, 2, 3], [-1, -1, 0, 1, 3, 3, 5]]
ACCEPTED = [[0, 1, 2, 3], [1, 3, 5, 6]]


def layer_of(stride, held):
    return synth.Workload(name="drafted", dtype="fp32", batch=1, d_model=128, n_heads=4, head_dim=64, latent_rank=128,
                          rope_dim=32, hyper_dim=32, stride=stride, prefill_tokens=0, context_tokens=held, decode_steps=8,
                          seed=23)


@pytest.mark.parametrize("held", [[7, 8], [130, 129], [1, 192], [0, 2]])
@pytest.mark.parametrize("stride", [2, 3])
def test_a_step_sees_what_the_layers_decoding_sees(stride, held):
    w = layer_of(stride, max(held))
    weights = synth.make_weights(w)
    p = H.oracle_params(w, weights)
    r, dr, heads, dh = p.latent_rank, p.rope_dim, p.n_heads, p.head_dim
    rng = np.random.default_rng(stride * 1000 + held[0])
    cfg = M.make_qpool_config(n_heads=heads, latent_rank=r, rope_dim=dr, n_pages=8)
    pages, rope = M.make_qpool(cfg), M.make_rope_config(rope_dim=dr)
    table, free = dev([[-1] * 4] * 2), dev([5, 2, 7, 0, 3, 1])

    # Prompts: a chunk's row goes to where the map says, with the chunk's last token.
    m = M.mtla_slot_map(dev([0, 0]), dev(held), free, table, stride=stride, n_tokens=sum(held))
    rows = rng.standard_normal((sum(held), r + dr)).astype(np.float32)
    M.mtla_qpool_write(cfg, pages, torch.from_numpy(rows).cuda(), m.store)
    taken = int(m.taken)

    def slots_of(b, n):
        at = torch.tensor([int(table[b, j // 64]) * 64 + j % 64 for j in range(n)], dtype=torch.int64, device="cuda")
        return host(M.mtla_qpool_read(cfg, pages, at, dtype=torch.float32)).reshape(n, r + dr)

    cache = [slots_of(b, -(-held[b] // stride)) for b in range(2)]
    # Drafts: Form I along every path gives the nodes' rows and queries (not rotated yet) and the outputs.
    counts, starts = [len(v) for v in PARENTS], starts_of([len(v) for v in PARENTS])
    x = rng.standard_normal((sum(counts), p.d_model)).astype(np.float32)
    states, want, row, query = [], [], [], []
    for b, parents in enumerate(PARENTS):
        for i, parent in enumerate(parents):
            st = copy.deepcopy(states[starts[b] + parent]) if parent >= 0 else O.state_from_cache(cache[b], held[b], p)
            xi = x[starts[b] + i].astype(np.float64)
            want.append(O.decode_step(p, st, xi))
            states.append(st)
            row.append(np.concatenate([st.c_hat[-1], xi @ p.w_kr]))
            absorbed = np.einsum("hd,rhd->hr", (xi @ p.w_q).reshape(heads, dh), p.w_k.reshape(r, heads, dh))
            query.append(np.concatenate([absorbed, (xi @ p.w_qr).reshape(heads, dr)], 1))
    n = sum(counts)
    m = M.mtla_tree_map(dev(held), dev(starts), dev([v for parents in PARENTS for v in parents]), stride=stride)
    assert m.slots.tolist() == [h // stride for h in held]
    assert m.position.tolist() == [st.tokens - 1 for st in states]
    q, rows = (torch.from_numpy(np.stack(v)).float().cuda() for v in (query, row))
    q, rows = M.mtla_rope(rope, [q, rows.view(n, 1, r + dr)], m.position, first=r)
    rows = rows.reshape(n, r + dr)
    out, _ = M.mtla_qpool_attend_tree(cfg, pages, table, m.slots, dev(starts), rows, m.seen, q, scale=dh ** -0.5)
    y = np.einsum("nhr,rhd->nhd", host(out), p.w_v.reshape(r, heads, dh)).reshape(n, -1) @ p.w_o
    H.assert_close(torch.from_numpy(y), np.stack(want), "fp32", "nodes")
    # The layer's own steps along the accepted paths.
    for b, path in enumerate(ACCEPTED):
        h = H.gpu_handle(w, weights, max_prefill_tokens=0)
        try:
            if held[b]:
                M.mtla_cache_import(h, torch.from_numpy(cache[b]).float().cuda()[None].contiguous(), held[b])
            for i in path:
                got = M.mtla_decode_step(h, torch.from_numpy(x[starts[b] + i]).cuda()[None])
                assert np.abs(host(got)[0] - y[starts[b] + i]).max() <= 2 * H.FP32_MAX_ABS, (b, i)
        finally:
            M.mtla_destroy(h)

    # The accepted paths go into the pool; what later plain steps see are their states.
    nodes = [starts[b] + i for b, path in enumerate(ACCEPTED) for i in path]
    m = M.mtla_slot_map(dev(held), dev([len(v) for v in ACCEPTED]), free[taken:].contiguous(), table, stride=stride,
                        n_tokens=len(nodes))
    M.mtla_qpool_write(cfg, pages, rows[nodes], m.store)
    last = [starts[b] + path[-1] for b, path in enumerate(ACCEPTED)]
    assert m.slots.tolist() == [len(states[i].c_hat) for i in last]
    seqs = [slots_of(b, len(states[i].c_hat)) for b, i in enumerate(last)]
    for b, i in enumerate(last):
        closed = held[b] // stride
        assert np.array_equal(seqs[b][:closed], cache[b][:closed])
        fresh = O.cache_array(states[i])[closed:]
        # A stored latent is at most half the step between the largest codes, a sixth of the scale's reach and the
        # scale's own rounding up, an eighth, off: 3/16 of the group's largest one.  Keys are rounded to bf16.
        groups = fresh[:, :r].reshape(-1, 32)
        off = np.abs(seqs[b][closed:, :r].reshape(-1, 32) - groups).max(-1)
        assert (off <= 3 / 16 * np.abs(groups).max(-1) + 1e-5).all()
        assert np.abs(seqs[b][closed:, r:] - fresh[:, r:]).max() <= 2.0 ** -8 * np.abs(fresh[:, r:]).max() + 1e-5
    again, lse = M.mtla_qpool_attend(cfg, pages, table, m.slots, q[last].contiguous(), scale=dh ** -0.5)
    for b, i in enumerate(last):
        q64 = host(q[i])
        w_out, w_lse, mean_abs = Q.attend(q64, seqs[b][:, :r], seqs[b][:, r:], dh ** -0.5)
        tol, tol_lse = bound(q64, seqs[b], dh ** -0.5, mean_abs, w_out, "fp32", r)
        assert (np.abs(host(again[b]) - w_out) <= tol).all()
        assert (np.abs(host(lse[b]) - w_lse) <= tol_lse + 2.0 ** -23 * np.abs(w_lse)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_tree_that_the_map_refuses_sees_the_context_alone(dtype):
    """A refused tree's nodes have seq -1 and see no drafted row.  Its request keeps its slots, so that a plain step
    over the same map still finds its context, and the attention answers with the softmax over it."""
    heads, r, dr, n_slots = 4, 64, 32, [70, 40]
    cfg = M.make_qpool_config(n_heads=heads, latent_rank=r, rope_dim=dr, n_pages=4)
    pages = M.make_qpool(cfg)
    g = torch.Generator(device="cuda").manual_seed(2)
    M.mtla_qpool_write(cfg, pages, torch.randn(256, r + dr, device="cuda", generator=g), torch.arange(256, device="cuda"))
    table, starts = dev([[0, 1], [2, 3]]), dev([0, 3, 6])
    m = M.mtla_tree_map(dev([2 * n_slots[0] + 1, 2 * n_slots[1]]), starts, dev([-1, 2, 0, -1, 0, 1]), stride=2)
    assert m.seq.tolist() == [-1] * 3 + [1] * 3 and m.seen.tolist()[:3] == [0] * 3 and m.slots.tolist() == n_slots
    q = torch.randn(6, heads, r + dr, device="cuda", generator=g).to(dtype)
    rows = torch.randn(6, r + dr, device="cuda", generator=g).to(dtype)
    out, lse = M.mtla_qpool_attend_tree(cfg, pages, table, m.slots, starts, rows, m.seen, q, scale=0.2)
    context = host(M.mtla_qpool_read(cfg, pages, torch.arange(n_slots[0], device="cuda"), dtype=torch.float32))
    for i in range(3):
        want, want_lse, mean_abs = T.attend_node(host(q[i]), context, host(rows[:3]), 0, 0.2, r)
        tol, tol_lse = bound(host(q[i]), context, 0.2, mean_abs, want, "bf16" if dtype is torch.bfloat16 else "fp32", r)
        more = 4 * (2.0 ** -22 + 2.0 ** -23)                 # joining two parts
        assert (np.abs(host(out[i]) - want) <= tol + 2 * more * mean_abs).all()
        assert (np.abs(host(lse[i]) - want_lse) <= tol_lse + more + 2.0 ** -23 * np.abs(want_lse)).all()

"""Drafted trees and 4-bit weights: pins of their oracle, and what the calls refuse (host checks only)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import qpool_oracle as Q
from oracle import tree_oracle as T
from paper_2505_13544_b200 import binding as M

A = 1 << 20          # an aligned address that no refused call reads


def pool_config(**kw):
    return M.make_qpool_config(**{**dict(n_heads=8, latent_rank=256, rope_dim=32, n_pages=4), **kw})


BAD_POOLS = (dict(n_heads=0), dict(n_heads=33), dict(latent_rank=96), dict(latent_rank=576), dict(latent_rank=0),
             dict(rope_dim=16), dict(rope_dim=128), dict(n_pages=0))


def test_a_chain_sees_what_a_sequence_sees():
    """A drafted chain on `held` tokens: node i has the slots that a sequence of held + i + 1 tokens has."""
    for stride in (1, 2, 3, 4):
        for held in range(9):
            m = T.tree_map([held], [0, 6], [-1, 0, 1, 2, 3, 4], stride, 6)
            for i in range(6):
                assert m["slots"][0] + bin(m["seen"][i]).count("1") == -(-(held + i + 1) // stride)
                assert m["position"][i] == held + i and m["seen"][i] >> i & 1


def test_tree_map_oracle_on_a_worked_example():
    # held 3, stride 2: roots stand at 3 and close the open chunk; their children open one.
    m = T.tree_map([3], [0, 5], [-1, -1, 0, 1, 2], 2, 7)
    assert m["slots"] == [1] and m["position"] == [3, 3, 4, 4, 5, 0, 0]
    assert m["seen"] == [1, 2, 1 | 4, 2 | 8, 1 | 16, 0, 0] and m["seq"] == [0] * 5 + [-1] * 2


def test_weight_layout_round_trip():
    rng = np.random.default_rng(3)
    w = rng.standard_normal((136, 19))
    back = T.unpack_weight(T.pack_weight(w), 136, 19)
    full = np.zeros((160, 19))
    full[:136] = w
    assert np.array_equal(back, Q.dequantise(*Q.quantise(full.T)).T[:136])
    assert len(T.pack_weight(w)) == M.mtla_qweight_bytes(136, 19)


# ------------------------------------------------------------------------------ refusals

def test_tree_map_refuses():
    lib = M.load_library()

    def call(held=A, starts=A, parents=A, B=2, stride=2, n=5, null=False, **kw):
        o = M.mtla_tree_map_out(**{**dict(seq=A, position=A, seen=A, slots=A), **kw})
        return lib.mtla_tree_map(held, starts, parents, B, stride, None if null else ctypes.byref(o), n, None)

    for bad in (dict(held=None), dict(starts=None), dict(parents=None), dict(B=0), dict(stride=0), dict(n=-1),
                dict(null=True), dict(seq=None), dict(position=None), dict(seen=None), dict(slots=None),
                dict(seen=A + 4), dict(held=A + 1), dict(parents=A + 2)):
        assert call(**bad) == -1, bad
    assert call(B=4097) == -2


def test_attend_tree_refuses():
    lib = M.load_library()
    need = M.mtla_qpool_tree_workspace_bytes(pool_config(), 3, 20)
    assert need > 0

    def call(pages=A, table=A, width=2, slots=A, starts=A, B=3, rows=A, stride=288, seen=A, q=A, n=20, dtype=1,
             scale=0.125, out=A, lse=None, ws=A, ws_bytes=need, **kw):
        c = pool_config(**kw)
        return lib.mtla_qpool_attend_tree(ctypes.byref(c), pages, table, width, slots, starts, B, rows, stride, seen, q,
                                          n, dtype, scale, out, lse, ws, ws_bytes, None)

    for bad in (dict(pages=None), dict(table=None), dict(slots=None), dict(starts=None), dict(rows=None),
                dict(seen=None), dict(q=None), dict(out=None), dict(ws=None), dict(width=0), dict(B=0), dict(n=-1),
                dict(dtype=3), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(q=A + 8),
                dict(out=A + 2), dict(ws=A + 128), dict(table=A + 2), dict(lse=A + 2), dict(seen=A + 4),
                dict(rows=A + 8), dict(stride=280), dict(stride=292), dict(dtype=0, stride=290)):
        assert call(**bad) == -1, bad
    for bad in BAD_POOLS + (dict(B=4097), dict(width=1 << 30), dict(n=1 << 29)):
        assert call(**bad) == -2, bad
    assert call(ws_bytes=need - 1) == -3
    assert lib.mtla_qpool_attend_tree(None, A, A, 1, A, A, 1, A, 288, A, A, 1, 1, 1.0, A, None, A, need, None) == -2
    assert M.mtla_qpool_tree_workspace_bytes(pool_config(), 0, 1) == 0
    assert M.mtla_qpool_tree_workspace_bytes(pool_config(), 1, -1) == 0
    assert lib.mtla_qpool_tree_workspace_bytes(None, 1, 1) == 0


def test_qweight_refuses():
    lib = M.load_library()
    for n_in, n_out in ((0, 1), (7, 1), (12, 4), (8, 0), (-8, 4), ((1 << 16) + 8, 1), ((1 << 22) + 8, 1), (8, (1 << 22) + 1)):
        assert M.mtla_qweight_bytes(n_in, n_out) == 0
        assert lib.mtla_qweight_pack(A, 1 << 23, 1, n_in, n_out, A, None) == -2
        assert lib.mtla_qweight_unpack(A, n_in, n_out, A, 1 << 23, 1, None) == -2
        assert lib.mtla_qweight_product(A, n_in, n_out, A, 1 << 23, 1, A, 1 << 23, 1, None) == -2
    for bad in (dict(w=None), dict(packed=None), dict(dtype=2), dict(packed=A + 8), dict(w=A + 1), dict(stride=15)):
        a = {**dict(w=A, packed=A, dtype=1, stride=16), **bad}
        assert lib.mtla_qweight_pack(a["w"], a["stride"], a["dtype"], 128, 16, a["packed"], None) == -1, bad
        assert lib.mtla_qweight_unpack(a["packed"], 128, 16, a["w"], a["stride"], a["dtype"], None) == -1, bad
    for bad in (dict(p=None), dict(x=None), dict(y=None), dict(n=-1), dict(dtype=5), dict(p=A + 8), dict(x=A + 8),
                dict(y=A + 1), dict(xs=120), dict(xs=132), dict(ys=15), dict(dtype=0, xs=130), dict(dtype=0, y=A + 2)):
        a = {**dict(p=A, x=A, xs=128, n=2, y=A, ys=16, dtype=1), **bad}
        assert lib.mtla_qweight_product(a["p"], 128, 16, a["x"], a["xs"], a["n"], a["y"], a["ys"], a["dtype"],
                                        None) == -1, bad
    assert lib.mtla_qweight_product(A, 128, 16, A, 128, (1 << 19) + 1, A, 16, 1, None) == -2


def test_calls_for_nothing_take_empty_buffers():
    lib = M.load_library()
    cfg = pool_config()
    need = M.mtla_qpool_tree_workspace_bytes(cfg, 2, 0)
    assert lib.mtla_qpool_attend_tree(ctypes.byref(cfg), A, A, 1, A, A, 2, None, 0, None, None, 0, 1, 1.0, None, None, A,
                                      need, None) == 0
    assert lib.mtla_qweight_product(A, 128, 16, None, 128, 0, None, 16, 1, None) == 0


def test_host_tensors_are_refused_by_the_binding():
    i32 = dict(dtype=torch.int32)
    with pytest.raises(TypeError):
        M.mtla_tree_map(torch.zeros(1, **i32), torch.zeros(2, **i32), torch.zeros(1, **i32), stride=1)
    cfg = pool_config()
    pages = torch.zeros(4, M.mtla_qpool_page_bytes(cfg), dtype=torch.uint8)
    with pytest.raises(TypeError):
        M.mtla_qpool_attend_tree(cfg, pages, torch.zeros(1, 1, **i32), torch.zeros(1, **i32), torch.zeros(2, **i32),
                                 torch.zeros(1, 288), torch.zeros(1, dtype=torch.int64), torch.zeros(1, 8, 288), scale=1.0)
    with pytest.raises(TypeError):
        M.mtla_qweight_pack(torch.zeros(128, 16))
    with pytest.raises(TypeError):
        M.mtla_qweight_unpack(torch.zeros(1088, dtype=torch.uint8), 128, 16, dtype=torch.float16)
    with pytest.raises(TypeError):
        M.mtla_qweight_product(torch.zeros(1088, dtype=torch.uint8), torch.zeros(1, 128), 16)

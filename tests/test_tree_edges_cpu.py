"""Drafted trees and 4-bit weights: what the self-tests of waits refuse, and the order in which the attention's roles may
come to the ends of segments (host checks only)."""
import ctypes
import os
import re

import pytest

from paper_2505_13544_b200 import binding as M
from tests.test_tree_cpu import A, BAD_POOLS, pool_config


def test_selftest_of_the_tree_attentions_wait_refuses():
    lib = M.load_library()
    need = M.mtla_qpool_tree_workspace_bytes(pool_config(), 3, 20)

    def call(pages=A, slots=A, B=3, rows=A, stride=288, n=20, dtype=1, out=A, ws=A, ws_bytes=need, **kw):
        c = pool_config(**kw)
        return lib.mtla_selftest_tree_timeout(ctypes.byref(c), pages, A, 2, slots, A, B, rows, stride, A, A, n, dtype,
                                              0.125, out, None, ws, ws_bytes, None)

    for bad in (dict(pages=None), dict(slots=None), dict(rows=None), dict(out=None), dict(ws=None), dict(B=0), dict(n=-1),
                dict(dtype=3), dict(out=A + 2), dict(ws=A + 128), dict(stride=280)):
        assert call(**bad) == -1, bad
    for bad in BAD_POOLS + (dict(B=4097),):
        assert call(**bad) == -2, bad
    assert call(ws_bytes=need - 1) == -3


def test_selftest_of_the_products_wait_refuses():
    lib = M.load_library()
    for bad in (dict(p=None), dict(x=None), dict(y=None), dict(n=-1), dict(p=A + 8), dict(x=A + 8), dict(y=A + 1),
                dict(xs=120), dict(xs=132), dict(ys=15)):
        a = {**dict(p=A, x=A, xs=128, n=2, y=A, ys=16), **bad}
        assert lib.mtla_selftest_qweight_timeout(a["p"], 128, 16, a["x"], a["xs"], a["n"], a["y"], a["ys"], None) == -1, bad
    assert lib.mtla_selftest_qweight_timeout(A, 12, 16, A, 128, 1, A, 16, None) == -2


# ------------------------------------------------------------------------------ ends of segments

def ways_into_a_standstill(ring, stages, lengths):
    """The softmax warps, the warp that issues the value products and the value warps over segments of `lengths` tiles,
    with `stages` probability tiles and `ring` barriers for the ends of segments: every order in which they may go on.  A
    wait asks for a phase's parity only, so it misses a phase when the one after it completes too."""
    tiles = [(s, i == 0, i == n - 1) for s, n in enumerate(lengths) for i in range(n)]
    softmax, issuer, value = [], [], []
    for n, (seg, first, last) in enumerate(tiles):
        st, rnd = n % stages, n // stages
        softmax += [("wait", ("p_empty", st), rnd - 1), ("arrive", ("p_full", st), 0)]
        value += [("arrive", ("unit", n), 0)]
        issuer += [("wait", ("p_full", st), rnd)]
        if first and seg:
            issuer += [("wait", ("o_empty", 0), seg - 1)]
        issuer += [("wait", ("unit", n), 0), ("arrive", ("p_empty", st), 0)]
        if last:
            softmax += [("arrive", ("end_full", seg % ring), 0)]
            issuer += [("arrive", ("o_full", seg & 1), 0)]
            value += [("wait", ("end_full", seg % ring), seg // ring), ("wait", ("o_full", seg & 1), seg >> 1),
                      ("arrive", ("o_empty", 0), 0)]
    programs = (softmax, issuer, value)
    done = [{} for _ in programs]                        # completed phases of a barrier before every step of its arriver
    for steps, counts in zip(programs, done):
        for bar in {b for what, b, _ in steps if what == "arrive"}:
            total, counts[bar] = 0, [0]
            for what, b, _ in steps:
                total += what == "arrive" and b == bar
                counts[bar].append(total)
    arriver = {bar: k for k, counts in enumerate(done) for bar in counts}
    stuck, seen, todo = [], {(0, 0, 0)}, [(0, 0, 0)]
    while todo:
        at = todo.pop()
        moved = False
        for k, steps in enumerate(programs):
            if at[k] == len(steps):
                continue
            what, bar, phase = steps[at[k]]
            if what == "wait":
                count = done[arriver[bar]][bar][at[arriver[bar]]]
                if count & 1 == phase & 1:
                    continue
                assert count > phase, "a wait that passes before its phase is complete"
            moved = True
            after = (*at[:k], at[k] + 1, *at[k + 1:])
            if after not in seen:
                seen.add(after)
                todo.append(after)
        if not moved and any(i < len(steps) for i, steps in zip(at, programs)):
            stuck.append(at)
    return stuck


def end_ring():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "paper_2505_13544_b200", "csrc", "tree_attn_tc.cuh")) as f:
        text = f.read()
    rings = re.findall(r"end_full\[(\w+)\]", text)
    assert rings
    return int(rings[0]) if rings[0].isdigit() else int(re.search(r"constexpr int %s = (\d+);" % rings[0], text).group(1))


@pytest.mark.parametrize("stages", [1, 2])
@pytest.mark.parametrize("lengths", [[1] * 9, [1, 1, 2, 1, 1, 1, 3, 1], [2] * 5, [3, 1, 1, 1, 1, 2]])
def test_no_order_of_the_roles_misses_the_end_of_a_segment(lengths, stages):
    assert ways_into_a_standstill(end_ring(), stages, lengths) == []


def test_two_barriers_for_the_ends_would_miss_one():
    assert ways_into_a_standstill(2, 2, [1] * 5)

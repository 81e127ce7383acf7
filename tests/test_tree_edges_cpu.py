"""Drafted trees: what the self-test of a wait refuses (host checks only)."""
import ctypes

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

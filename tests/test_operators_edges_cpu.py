"""Operators around the 4-bit pool: what the calls refuse at the edges of their documentation (host checks only)."""
import ctypes

from paper_2505_13544_b200 import binding as M

A = 1 << 20          # an aligned address that no refused call reads


def test_selftest_of_the_pool_attentions_wait_refuses():
    lib = M.load_library()
    cfg = M.make_qpool_config(n_heads=2, latent_rank=64, rope_dim=32, n_pages=1)
    need = M.mtla_qpool_workspace_bytes(cfg, 3)

    def call(slots=A, B=3, dtype=1, out=A, lse=A, ws=A, ws_bytes=need, c=cfg):
        return lib.mtla_selftest_qpool_timeout(ctypes.byref(c), slots, B, dtype, out, lse, ws, ws_bytes, None)

    for bad in (dict(slots=None), dict(out=None), dict(ws=None), dict(B=0), dict(dtype=2), dict(out=A + 8), dict(lse=A + 2),
                dict(ws=A + 16), dict(slots=A + 1)):
        assert call(**bad) == -1, bad
    assert call(B=4097) == -2
    assert call(c=M.make_qpool_config(n_heads=0, latent_rank=64, rope_dim=32, n_pages=1)) == -2
    assert call(ws_bytes=need - 1) == -3

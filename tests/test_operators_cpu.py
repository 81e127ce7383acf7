"""Operators around the 4-bit pool: pins of their oracle, and what the calls refuse (host checks only)."""
import ctypes

import numpy as np
import pytest

from oracle import qpool_oracle as Q
from paper_2505_13544_b200 import binding as M

A = 1 << 20          # an aligned address that no refused call reads


def test_scale_grid_is_the_top_of_half_precision():
    bits = (np.arange(len(Q.SCALES), dtype=np.uint16) << 7).view(np.float16).astype(np.float64)
    assert np.array_equal(bits, Q.SCALES)
    assert Q.SCALES[-1] == 10240.0 and np.isnan(np.array([255 << 7], dtype=np.uint16).view(np.float16)[0])


def test_quantise_is_within_half_a_step_and_idempotent():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((6, 64)) * np.exp(rng.uniform(-6, 6, (6, 1)))
    byte, code = Q.quantise(x)
    y = Q.dequantise(byte, code)
    s = np.repeat(Q.SCALES[byte], 32, axis=1)
    assert (np.abs(x) <= 6 * s).all()                       # the scale reaches
    assert (np.abs(x - y) <= s).all()                       # the widest step is 2 s
    small = np.abs(x) <= 2 * s
    assert (np.abs(x - y)[small] <= 0.25 * s[small]).all()
    byte2, code2 = Q.quantise(y)
    assert np.array_equal(Q.dequantise(byte2, code2), y)


def test_quantise_ties_specials_and_saturation():
    s = 0.25
    v = np.zeros((1, 64))
    v[0, :8] = np.array([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]) * s
    v[0, 32:34] = [1e6, 3.0]
    byte, code = Q.quantise(v)
    assert Q.SCALES[byte[0, 0]] == s
    assert list(code[0, :8]) == [7, 0, 2, 2, 4, 4, 6, 6]
    assert Q.dequantise(byte, code)[0, 32] == 61440.0
    v[0, 40] = np.inf
    byte, code = Q.quantise(v)
    back = Q.dequantise(byte, code)
    assert np.isnan(back[0, 32:]).all() and np.isfinite(back[0, :32]).all()


@pytest.mark.parametrize("r,dr", [(64, 32), (192, 64), (256, 32), (512, 64)])
def test_page_round_trip(r, dr):
    rng = np.random.default_rng(r)
    byte = rng.integers(0, 226, (64, r // 32), dtype=np.uint8)
    codes = rng.integers(0, 16, (64, r), dtype=np.uint8)
    keys = rng.integers(0, 1 << 16, (64, dr), dtype=np.uint16)
    page = Q.pack_page(byte, codes, keys)
    assert len(page) == M.mtla_qpool_page_bytes(M.make_qpool_config(n_heads=1, latent_rank=r, rope_dim=dr, n_pages=1))
    got = Q.unpack_page(page, r, dr)
    for a, b in zip(got, (byte, codes, keys)):
        assert np.array_equal(a, b)


def test_rope_oracle_turns_back_and_keeps_inner_products():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 12))
    f = Q.rope_frequencies(8, scaling="ramp", factor=4.0, low=1.0, high=4.0, train_tokens=64)
    for layout in ("interleaved", "half"):
        y = Q.rope(x, [5, 70, 123456], f, layout, 2)
        assert np.allclose(Q.rope(y, [5, 70, 123456], f, layout, 2, inverse=True), x, atol=1e-10)
        # The score of a query and a key depends on the distance of their positions alone.
        q, k = rng.standard_normal((2, 1, 1, 12))
        a = (Q.rope(q, [40], f, layout, 2) * Q.rope(k, [31], f, layout, 2)).sum()
        b = (Q.rope(q, [109], f, layout, 2) * Q.rope(k, [100], f, layout, 2)).sum()
        assert abs(a - b) < 1e-12


def test_slot_map_oracle_on_a_worked_example():
    table = [[7, -1], [-1, -1]]
    m = Q.slot_map([126, 0], [3, 3], 2, table, [4, 9, 11])
    assert m["slots"] == [65, 2] and m["taken"] == 2 and table == [[7, 4], [9, -1]]
    assert m["slot"] == [7 * 64 + 63, 7 * 64 + 63, 4 * 64, 9 * 64, 9 * 64, 9 * 64 + 1]
    assert m["store"] == [-1, 7 * 64 + 63, 4 * 64, -1, 9 * 64, 9 * 64 + 1]


# ------------------------------------------------------------------------------ refusals

def test_slot_map_refuses():
    lib = M.load_library()

    def call(held=A, fresh=A, B=2, stride=2, table=A, width=3, free=A, n_free=4, n=5, **kw):
        o = dict(starts=A, seq=A, position=A, slot=A, store=A, slots=A, taken=A)
        o.update(kw)
        return lib.mtla_slot_map(held, fresh, B, stride, table, width, free, n_free,
                                 ctypes.byref(M.mtla_slot_map_out(**o)), n, None)

    for bad in (dict(held=None), dict(fresh=None), dict(table=None), dict(B=0), dict(stride=0), dict(width=0),
                dict(n_free=-1), dict(n=-1), dict(free=None), dict(starts=None), dict(slots=None), dict(taken=None),
                dict(seq=None), dict(store=None), dict(slot=A + 4), dict(held=A + 1)):
        assert call(**bad) == -1, bad
    assert call(B=16385) == -2
    assert lib.mtla_slot_map(A, A, 1, 1, A, 1, A, 1, None, 1, None) == -1


def test_rope_refuses():
    lib = M.load_library()

    def call(n_tensors=1, dtype=1, positions=A, n=4, cfg=None, **kw):
        c = M.make_rope_config(**{**dict(rope_dim=32), **(cfg or {})})
        t = dict(x=A, y=2 * A, x_token_stride=128, x_head_stride=64, y_token_stride=128, y_head_stride=64,
                 n_heads=2, width=64, first=32)
        t.update(kw)
        arr = (M.mtla_rope_tensor * 5)(*[M.mtla_rope_tensor(**t) for _ in range(5)])
        return lib.mtla_rope(ctypes.byref(c), arr, n_tensors, dtype, positions, n, 0, None)

    for bad in (dict(x=None), dict(y=None), dict(positions=None), dict(n=-1), dict(n_tensors=0), dict(dtype=7),
                dict(first=-1), dict(x=A + 1), dict(x_token_stride=-1), dict(y_head_stride=32),
                dict(y_token_stride=64), dict(y_token_stride=0), dict(y=A, y_token_stride=256),
                dict(cfg=dict(theta=-1.0)), dict(cfg=dict(factor=float("inf"))),
                dict(cfg=dict(scaling="ramp", train_tokens=0)),
                dict(cfg=dict(scaling="ramp", train_tokens=8, ramp_low=2.0, ramp_high=2.0))):
        assert call(**bad) == -1, bad
    for bad in (dict(n_tensors=5), dict(cfg=dict(rope_dim=31)), dict(cfg=dict(rope_dim=258)),
                dict(cfg=dict(rope_dim=0)), dict(first=33)):
        assert call(**bad) == -2, bad
    assert call(n=0) == 0                                    # nothing to do
    # heads outermost is a valid order of the result
    assert call(n=0, y_token_stride=64, y_head_stride=64 * 7) == 0


def pool_config(**kw):
    return M.make_qpool_config(**{**dict(n_heads=8, latent_rank=256, rope_dim=32, n_pages=4), **kw})


BAD_POOLS = (dict(n_heads=0), dict(n_heads=33), dict(latent_rank=32), dict(latent_rank=576), dict(latent_rank=96),
             dict(rope_dim=16), dict(rope_dim=0), dict(rope_dim=96), dict(n_pages=0))


def test_pool_rows_refuse():
    lib = M.load_library()

    def write(pages=A, rows=A, stride=288, dtype=1, index=A, n=3, **kw):
        c = pool_config(**kw)
        w = lib.mtla_qpool_write(ctypes.byref(c), pages, rows, stride, dtype, index, n, None)
        assert lib.mtla_qpool_read(ctypes.byref(c), pages, index, n, rows, stride, dtype, None) == w
        return w

    for bad in (dict(pages=None), dict(rows=None), dict(index=None), dict(n=-1), dict(dtype=2), dict(stride=287),
                dict(stride=292), dict(pages=A + 8), dict(rows=A + 8), dict(index=A + 4)):
        assert write(**bad) == -1, bad
    for bad in BAD_POOLS:
        assert write(**bad) == -2, bad
        assert M.mtla_qpool_page_bytes(pool_config(**bad)) == 0
    assert write(n=0) == 0
    assert M.mtla_qpool_page_bytes(pool_config()) == 64 * (128 + 8 + 64)


def test_attend_refuses():
    lib = M.load_library()
    need = M.mtla_qpool_workspace_bytes(pool_config(), 3)
    assert need > 0

    def call(pages=A, table=A, width=2, slots=A, B=3, q=A, dtype=1, scale=0.125, out=A, lse=None, ws=A,
             ws_bytes=need, **kw):
        c = pool_config(**kw)
        return lib.mtla_qpool_attend(ctypes.byref(c), pages, table, width, slots, B, q, dtype, scale, out, lse, ws,
                                     ws_bytes, None)

    for bad in (dict(pages=None), dict(table=None), dict(slots=None), dict(q=None), dict(out=None), dict(ws=None),
                dict(width=0), dict(B=0), dict(dtype=3), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(q=A + 8), dict(out=A + 2), dict(ws=A + 128), dict(table=A + 2), dict(lse=A + 2)):
        assert call(**bad) == -1, bad
    for bad in BAD_POOLS + (dict(B=4097), dict(width=1 << 30)):
        assert call(**bad) == -2, bad
    assert call(ws_bytes=need - 1) == -3
    assert M.mtla_qpool_workspace_bytes(pool_config(), 0) == 0
    assert M.mtla_qpool_workspace_bytes(pool_config(), 4097) == 0


def test_null_configs_are_refused():
    lib = M.load_library()
    assert lib.mtla_qpool_page_bytes(None) == 0 and lib.mtla_qpool_workspace_bytes(None, 1) == 0
    assert lib.mtla_qpool_write(None, A, A, 288, 1, A, 1, None) == -2
    assert lib.mtla_rope(None, None, 1, 1, A, 1, 0, None) == -1


def test_host_tensors_are_refused_by_the_binding():
    import torch
    cfg = pool_config()
    pages = torch.zeros(4, M.mtla_qpool_page_bytes(cfg), dtype=torch.uint8)
    with pytest.raises(TypeError):
        M.mtla_qpool_write(cfg, pages, torch.zeros(1, 288), torch.zeros(1, dtype=torch.int64))
    with pytest.raises(TypeError):
        M.mtla_slot_map(torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                        torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32), stride=1,
                        out=M.make_slot_map(1, 1, "cpu"))


def test_calls_for_nothing_take_empty_buffers():
    """An empty tensor's address is NULL."""
    lib = M.load_library()
    cfg, rope = pool_config(), M.make_rope_config(rope_dim=32)
    for call in (lib.mtla_qpool_write, lambda c, p, r, s, d, i, n, st: lib.mtla_qpool_read(c, p, i, n, r, s, d, st)):
        assert call(ctypes.byref(cfg), A, None, 288, 1, None, 0, None) == 0
        assert call(ctypes.byref(cfg), None, None, 288, 1, None, 0, None) == -1
    t = M.mtla_rope_tensor(None, None, 128, 64, 64, 64 * 7, 2, 64, 32)        # another order of the result
    assert lib.mtla_rope(ctypes.byref(rope), ctypes.byref(t), 1, 1, None, 0, 0, None) == 0
    assert lib.mtla_rope(ctypes.byref(rope), ctypes.byref(t), 1, 1, A, 1, 0, None) == -1


def test_attend_refuses_a_scale_that_overflows_in_base_two():
    cfg = pool_config()
    need = M.mtla_qpool_workspace_bytes(cfg, 1)
    assert M.load_library().mtla_qpool_attend(ctypes.byref(cfg), A, A, 1, A, 1, A, 1, 3e38, A, None, A, need, None) == -1

"""Operators around the 4-bit pool: calls at the edges of what their documentation allows."""
import ctypes
import time

import numpy as np
import pytest
import torch

from oracle import qpool_oracle as Q
from paper_2505_13544_b200 import binding as M
from tests.test_operators_gpu import host, rope_bound

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("side_stream", [False, True])
@pytest.mark.parametrize("n_tokens", [0, 5])
def test_slot_map_of_no_requests(n_tokens, side_stream):
    """A loop whose last request has ended: no page is taken, every token is behind the last one."""
    none, table = torch.empty(0, **I32), torch.empty(0, 4, **I32)
    stream = torch.cuda.Stream() if side_stream else None
    out = M.make_slot_map(0, n_tokens)
    for t in (out.starts, out.seq, out.position, out.slot, out.store, out.taken):
        t.fill_(77)
    torch.cuda.synchronize()
    for kw in (dict(out=out), dict(n_tokens=n_tokens)):
        m = M.mtla_slot_map(none, none, torch.arange(3, **I32), table, stride=2, stream=stream, **kw)
        torch.cuda.synchronize()
        assert m.starts.tolist() == [0] and m.taken.tolist() == [0] and m.slots.tolist() == []
        assert m.position.tolist() == [0] * n_tokens
        assert m.seq.tolist() == m.slot.tolist() == m.store.tolist() == [-1] * n_tokens
    with pytest.raises(M.MTLAError):
        M.mtla_slot_map(none, none, none, table, stride=0, n_tokens=0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_of_no_sequences(dtype):
    cfg = M.make_qpool_config(n_heads=3, latent_rank=64, rope_dim=32, n_pages=2)
    pages = M.make_qpool(cfg)
    q = torch.empty(0, 3, 96, dtype=dtype, device="cuda")
    out, lse = M.mtla_qpool_attend(cfg, pages, torch.empty(0, 2, **I32), torch.empty(0, **I32), q, scale=1.0)
    assert out.shape == (0, 3, 64) and out.dtype is dtype and lse.shape == (0, 3)
    with pytest.raises(TypeError):
        M.mtla_qpool_attend(cfg, pages, torch.empty(0, 2, **I32), torch.empty(1, **I32), q, scale=1.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch", [3, 300])
def test_a_wait_that_runs_out_gives_no_result(batch, dtype):
    """A bounded wait that gives up: every output is NaN, those of sequences without slots too, and the next
    call on the same workspace is an ordinary one."""
    cfg = M.make_qpool_config(n_heads=5, latent_rank=192, rope_dim=32, n_pages=2)
    pages = M.make_qpool(cfg)
    M.mtla_qpool_write(cfg, pages, torch.randn(128, 224, device="cuda"), torch.arange(128, device="cuda"))
    slots = torch.arange(batch, **I32) % 100                    # the first one has none
    table = torch.zeros(batch, 2, **I32)
    q = torch.randn(batch, 5, 224, device="cuda").to(dtype)
    ws = torch.full((M.mtla_qpool_workspace_bytes(cfg, batch),), 0x5A, dtype=torch.uint8, device="cuda")
    want, want_lse = M.mtla_qpool_attend(cfg, pages, table, slots, q, scale=0.1, workspace=ws)
    out, lse = torch.zeros_like(want), torch.zeros_like(want_lse)
    for fill in (0, 0xFF):
        ws.fill_(fill)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        M.mtla_selftest_qpool_timeout(cfg, slots, out, lse, ws)
        torch.cuda.synchronize()
        assert time.perf_counter() - t0 < 1.0                   # it returned at the budget
        assert torch.isnan(out).all() and torch.isnan(lse).all()
    again, again_lse = M.mtla_qpool_attend(cfg, pages, table, slots, q, scale=0.1, workspace=ws)
    assert torch.equal(again, want) and torch.equal(again_lse, want_lse)
    assert torch.isfinite(want.float()).all() and (want[0] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,heads,r", [([70, 0, 3], 4, 64), ([3000, 0, 200], 20, 256)])
def test_attend_without_the_logarithm(lens, heads, r, dtype):
    """A NULL lse: the same outputs, split and empty sequences included."""
    cfg = M.make_qpool_config(n_heads=heads, latent_rank=r, rope_dim=32, n_pages=3)
    pages = M.make_qpool(cfg)
    g = torch.Generator(device="cuda").manual_seed(1)
    M.mtla_qpool_write(cfg, pages, torch.randn(192, r + 32, device="cuda", generator=g), torch.arange(192, device="cuda"))
    table = (torch.arange(3 * 50, **I32) % 3).view(3, 50)
    slots = torch.tensor(lens, **I32)
    q = torch.randn(3, heads, r + 32, device="cuda", generator=g).to(dtype)
    ws = torch.empty(M.mtla_qpool_workspace_bytes(cfg, 3), dtype=torch.uint8, device="cuda")
    want, _ = M.mtla_qpool_attend(cfg, pages, table, slots, q, scale=0.1, workspace=ws)
    out = torch.full_like(want, 3.0)
    status = M.load_library().mtla_qpool_attend(
        ctypes.byref(cfg), pages.data_ptr(), table.data_ptr(), 50, slots.data_ptr(), 3, q.data_ptr(),
        1 if dtype is torch.bfloat16 else 0, 0.1, out.data_ptr(), None, ws.data_ptr(), ws.numel(),
        torch.cuda.current_stream().cuda_stream)
    assert status == 0 and torch.equal(out, want)


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("odd", [0, 1])
def test_rope_of_four_tensors_some_in_place(odd, layout, inverse):
    """Four tensors of different heads, widths and places of the rotated part, two of them in place, in 16-byte
    accesses and (odd) in single elements."""
    g = torch.Generator().manual_seed(4)
    n, dim = 37, 32
    shapes = [(8, 96 + odd, 64 + odd), (1, 32, 0), (3, 48, 8), (2, 40 + odd, 0)]      # heads, width, first
    x = [torch.randn(n, h, w, generator=g) for h, w, _ in shapes]
    pos = torch.randint(0, 100000, (n,), generator=g, dtype=torch.int32)
    dev = [v.cuda() for v in x]
    out = [dev[0], torch.full_like(dev[1], 9.0), torch.full_like(dev[2], 9.0), dev[3]]
    cfg = M.make_rope_config(rope_dim=dim, layout=layout)
    got = M.mtla_rope(cfg, dev, pos.cuda(), first=[f for _, _, f in shapes], out=out, inverse=inverse)
    freq = Q.rope_frequencies(dim)
    for v, y, (_, w, first) in zip(x, got, shapes):
        want = Q.rope(host(v), pos.tolist(), freq, layout, first, inverse=inverse)
        assert (np.abs(host(y) - want) <= rope_bound(v, want, first, dim, layout, 1.0, "fp32")).all()
        outside = [i for i in range(w) if i < first or i >= first + dim]
        assert torch.equal(y.cpu()[..., outside], v[..., outside])

"""Operators around the 4-bit pool: calls at the edges of what their documentation allows."""
import time

import pytest
import torch

from paper_2505_13544_b200 import binding as M

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

"""Operators around the 4-bit pool on the GPU against their 64-bit oracle.

Tolerances are sums of the roundings that the kernels make (half a step each, `finfo.eps / 2`):
see bound() for the attention; the pool and the slot maps have to agree exactly.
"""
import math

import numpy as np
import pytest
import torch

from oracle import qpool_oracle as Q
from paper_2505_13544_b200 import binding as M

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def host(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------ slot maps

def run_map(held, fresh, stride, width, pad=0, spare=3, seed=0, out=None):
    rng = np.random.default_rng(seed)
    have = [-(-(-(-h // stride)) // 64) for h in held]
    ids = rng.permutation(sum(have) + spare + sum(-(-(-(-(h + f) // stride)) // 64) for h, f in zip(held, fresh)))
    table, at = [], 0
    for n in have:
        table.append([int(v) for v in ids[at:at + n]] + [-7] * (width - n))
        at += n
    free = [int(v) for v in ids[at:]]
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    t = dev(table)
    m = M.mtla_slot_map(dev(held), dev(fresh), dev(free), t, stride=stride, n_tokens=sum(fresh) + pad, out=out)
    return m, t, table, free


def check_map(m, t, want, table, n, pad):
    assert m.starts.tolist() == want["starts"] and m.slots.tolist() == want["slots"]
    assert m.taken.tolist() == [want["taken"]]
    assert t.tolist() == table
    assert m.seq.tolist() == want["seq"] + [-1] * pad
    assert m.position.tolist() == want["position"] + [0] * pad
    assert m.slot.tolist() == want["slot"] + [-1] * pad
    assert m.store.tolist() == want["store"] + [-1] * pad


@pytest.mark.parametrize("stride", [1, 2, 3, 5])
@pytest.mark.parametrize("batch,held_max,fresh_max,pad", [
    (1, 0, 1, 0), (1, 700, 300, 3), (7, 129, 1, 0), (33, 400, 40, 1), (300, 100, 9, 77), (1100, 5, 2, 2)])
def test_slot_map(stride, batch, held_max, fresh_max, pad):
    rng = np.random.default_rng(batch * 10 + stride)
    held = [int(v) for v in rng.integers(0, held_max + 1, batch)]
    fresh = [int(v) for v in rng.integers(0, fresh_max + 1, batch)]
    fresh[0] = max(fresh[0], 1)
    m, t, table, free = run_map(held, fresh, stride, (held_max + fresh_max) // (64 * stride) + 2, pad)
    want = Q.slot_map(held, fresh, stride, table, free)
    check_map(m, t, want, table, sum(fresh), pad)


def test_slot_map_of_the_largest_batch():
    rng = np.random.default_rng(1)
    held = [int(v) for v in rng.integers(0, 300, 16384)]
    fresh = [int(v) for v in rng.integers(0, 3, 16384)]
    m, t, table, free = run_map(held, fresh, 2, 4, 5)
    want = Q.slot_map(held, fresh, 2, table, free)
    check_map(m, t, want, table, sum(fresh), 5)


def test_slot_map_of_positions_near_the_integer_limit():
    """One request with almost 2^31 tokens at a stride that leaves few slots."""
    held, fresh, stride = [2 ** 31 - 5], [4], 1 << 26
    m, t, table, free = run_map(held, fresh, stride, 2)
    want = Q.slot_map(held, fresh, stride, table, free)
    check_map(m, t, want, table, 4, 0)


def test_slot_map_without_tokens_and_misaligned_outputs():
    m, t, table, free = run_map([5, 0, 64], [0, 0, 0], 1, 2)
    want = Q.slot_map([5, 0, 64], [0, 0, 0], 1, table, free)
    check_map(m, t, want, table, 0, 0)
    # Token arrays that start off a 16-byte boundary.
    big = M.make_slot_map(3, 12)
    out = M.SlotMap(big.starts, big.seq[1:], big.position[1:], big.slot[1:], big.store[1:], big.slots, big.taken)
    m, t, table, free = run_map([5, 0, 64], [2, 3, 5], 2, 2, pad=1, out=out)
    want = Q.slot_map([5, 0, 64], [2, 3, 5], 2, table, free)
    check_map(m, t, want, table, 10, 1)


@pytest.mark.parametrize("what", ["pages", "width", "tokens", "negative", "overflow"])
def test_slot_map_refuses_a_batch_that_does_not_fit(what):
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    held, fresh, width, free, n = [100, 64], [70, 1], 3, [5, 6, 7], 71
    if what == "pages":
        free = [5]
    elif what == "width":
        width = 2
    elif what == "tokens":
        n = 70
    elif what == "negative":
        held = [100, -64]
    else:
        held = [100, (1 << 31) - 1]
    table = dev([[1, 2, -9][:width], [3, -9, -9][:width]])
    before = table.clone()
    m = M.mtla_slot_map(dev(held), dev(fresh), dev(free), table, stride=1, n_tokens=n)
    assert m.taken.item() == -1 and torch.equal(table, before)
    assert m.starts.tolist() == [0, 0, 0] and m.slots.tolist() == [100, max(held[1], 0)]
    assert (m.seq == -1).all() and (m.slot == -1).all() and (m.store == -1).all() and (m.position == 0).all()


# ------------------------------------------------------------------------------ rotary positions

ROPE_CASES = [
    # dtype, tokens, heads, width, first, dim, layout, scaling
    ("bf16", 5, 3, 96, 64, 32, "interleaved", "none"),
    ("bf16", 9, 1, 64, 0, 64, "half", "linear"),
    ("fp32", 17, 2, 40, 5, 30, "half", "ramp"),
    ("fp32", 1, 32, 192, 128, 64, "interleaved", "ramp"),
    ("bf16", 33, 5, 11, 3, 2, "interleaved", "none"),
    ("bf16", 2100, 2, 48, 8, 32, "half", "ramp"),
    ("fp32", 7, 3, 260, 4, 256, "interleaved", "none"),
    ("bf16", 3, 4, 80, 16, 48, "half", "none"),
]


def rope_setup(case, seed=0):
    dtype, n, heads, width, first, dim, layout, scaling = case
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, heads, width, generator=g).to(DT[dtype])
    pos = torch.randint(0, 1 << 20, (n,), generator=g, dtype=torch.int32)
    pos[0] = 0
    kw = dict(scaling=scaling, factor=4.0, ramp_low=1.0, ramp_high=16.0, train_tokens=2048)
    mag = 1.25 if scaling == "ramp" else 1.0
    cfg = M.make_rope_config(rope_dim=dim, layout=layout, magnitude=mag, **kw)
    f = Q.rope_frequencies(dim, scaling=scaling, factor=4.0, low=1.0, high=16.0, train_tokens=2048)
    return x, pos, cfg, f, mag


def rope_bound(x, want, first, dim, layout, mag, dtype):
    """Half a step of the result, and of the pair's two members four roundings of 2^-23 each: the
    fraction of a turn (2^-25 of a turn is 2 pi 2^-25 of angle), cosine / sine (about an ulp), the
    magnitude's product, and the sum."""
    a = np.abs(host(x))
    pair = np.zeros_like(a)
    half = dim // 2
    for k in range(half):
        i, j = (first + k, first + half + k) if layout == "half" else (first + 2 * k, first + 2 * k + 1)
        pair[..., i] = pair[..., j] = a[..., i] + a[..., j]
    return half_step(DT[dtype]) * np.abs(want) + pair * mag * 4 * 2.0 ** -23


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("case", ROPE_CASES)
def test_rope(case, inverse):
    dtype, n, heads, width, first, dim, layout, scaling = case
    x, pos, cfg, f, mag = rope_setup(case)
    want = Q.rope(host(x), pos.tolist(), f, layout, first, mag, inverse)
    tol = rope_bound(x, want, first, dim, layout, mag, dtype)
    xd, pd = x.cuda(), pos.cuda()
    (y,) = M.mtla_rope(cfg, [xd], pd, first=first, inverse=inverse)
    assert (np.abs(host(y) - want) <= tol).all()
    outside = [i for i in range(width) if i < first or i >= first + dim]
    assert torch.equal(y.cpu()[..., outside], x[..., outside])
    # In place, the same bits.
    z = xd.clone()
    M.mtla_rope(cfg, [z], pd, first=first, out=[z], inverse=inverse)
    assert torch.equal(z, y)
    # A wider row around it, heads outermost in the result; nothing outside is touched.
    wide = torch.randn(n, heads * width + 24, device="cuda").to(DT[dtype])
    view = wide[:, 8:8 + heads * width].unflatten(1, (heads, width))
    view.copy_(xd)
    out = torch.full((heads, n, width), 7.0, dtype=DT[dtype], device="cuda")
    M.mtla_rope(cfg, [view], pd, first=first, out=[out.transpose(0, 1)], inverse=inverse)
    assert torch.equal(out.transpose(0, 1), y)
    edges = wide.clone()
    M.mtla_rope(cfg, [view], pd, first=first, out=[view], inverse=inverse)
    assert torch.equal(view, y)
    assert torch.equal(wide[:, :8], edges[:, :8]) and torch.equal(wide[:, 8 + heads * width:], edges[:, 8 + heads * width:])


def test_rope_of_queries_and_shared_key_in_one_launch():
    g = torch.Generator().manual_seed(3)
    q, k = torch.randn(50, 8, 96, generator=g), torch.randn(50, 1, 32, generator=g)
    pos = torch.randint(0, 4000, (50,), generator=g, dtype=torch.int32)
    cfg = M.make_rope_config(rope_dim=32)
    f = Q.rope_frequencies(32)
    got = M.mtla_rope(cfg, [q.cuda(), k.cuda()], pos.cuda(), first=[64, 0])
    for x, y, first in ((q, got[0], 64), (k, got[1], 0)):
        want = Q.rope(host(x), pos.tolist(), f, "interleaved", first)
        assert (np.abs(host(y) - want) <= rope_bound(x, want, first, 32, "interleaved", 1.0, "fp32")).all()


@pytest.mark.parametrize("n,heads,width,first,dim", [(1, 600, 80, 16, 64), (40000, 1, 16, 0, 16), (700, 33, 8, 0, 8)])
def test_rope_shapes_of_work(n, heads, width, first, dim):
    """One token of many heads (several rounds of a CTA's threads), many short tokens side by side."""
    case = ("bf16", n, heads, width, first, dim, "half" if n == 1 else "interleaved", "linear")
    x, pos, cfg, f, mag = rope_setup(case, 2)
    rows = np.unique(np.linspace(0, n - 1, 60).astype(int))
    (y,) = M.mtla_rope(cfg, [x.cuda()], pos.cuda(), first=first)
    y = y.cpu()
    want = Q.rope(host(x[rows]), pos[rows].tolist(), f, case[6], first, mag)
    assert (np.abs(host(y[rows]) - want) <= rope_bound(x[rows], want, first, dim, case[6], mag, "bf16")).all()
    # Rows that were not computed by the oracle keep their length, pair by pair.
    norm = lambda v: v.double().square().sum(-1).sqrt()
    assert (torch.abs(norm(y) - norm(x)) <= norm(x) * 2 * half_step(torch.bfloat16) + 1e-6).all()


def test_rope_gradient_is_the_formula_and_the_difference_quotient():
    """For L = <w, rope(x)> the gradient is the inverse applied to w; L is linear, so a difference
    quotient of the forward call has no truncation error, only the roundings of two sums of 32-bit
    outputs (relative 2^-23 each) divided by the step."""
    case = ("fp32", 4, 2, 24, 4, 16, "half", "ramp")
    x, pos, cfg, f, mag = rope_setup(case, 1)
    w = torch.randn(x.shape, generator=torch.Generator().manual_seed(9))
    (grad,) = M.mtla_rope(cfg, [w.cuda()], pos.cuda(), first=4, inverse=True)
    want = Q.rope(host(w), pos.tolist(), f, "half", 4, mag, True)
    assert (np.abs(host(grad) - want) <= rope_bound(w, want, 4, 16, "half", mag, "fp32")).all()

    def loss(v):
        return float((host(M.mtla_rope(cfg, [v.cuda()], pos.cuda(), first=4)[0]) * host(w)).sum())

    step = 0.5
    for at in [(0, 0, 4), (1, 1, 11), (2, 0, 12), (3, 1, 19), (3, 0, 0)]:
        up, down = x.clone(), x.clone()
        up[at] += step
        down[at] -= step
        # Two elements of each output change; their magnitudes are at most |x| + step, times mag.
        slack = 2 * 4 * 2.0 ** -21 * float((x.abs().max() + step) * mag * w.abs().max()) / (2 * step)
        assert abs((loss(up) - loss(down)) / (2 * step) - host(grad)[at]) <= slack


# ------------------------------------------------------------------------------ the pool

def pool(r, dr, n_pages, heads=1, fill=0xA5):
    cfg = M.make_qpool_config(n_heads=heads, latent_rank=r, rope_dim=dr, n_pages=n_pages)
    pages = M.make_qpool(cfg)
    pages.fill_(fill)
    return cfg, pages


def latent_rows(n, r, dr, dtype, seed):
    """Rows of very different sizes, with zeros, ties, saturating and non-finite groups."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, r + dr, generator=g) * torch.exp(torch.randn(n, 1, generator=g) * 3)
    x[0, :32] = 0
    x[0, 32:40] = torch.tensor([6.0, 0.25, 0.75, 1.25, -1.75, 2.5, -3.5, 5.0]) * 0.5
    x[0, 40:64] = 0
    if n > 3:
        x[1, :32] *= 1e6
        x[2, 3] = math.inf
        x[3, 40] = math.nan
        x[1, 32:64] *= 2.0 ** -30 / x[1, 32:64].abs().max()
        x[2, 32:64] *= 3.0e-5 / x[2, 32:64].abs().max()
    if n > 4:      # exact ties and near ties at scales of every mantissa
        for k in range(8):
            s = (8 + k) / 8.0
            b = torch.tensor([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]) * s
            x[4, 32 * (k % (r // 32)):32 * (k % (r // 32)) + 8] = b
            x[4, 32 * (k % (r // 32)) + 8:32 * (k % (r // 32)) + 15] = b[1:] * (1 + 2.0 ** -23)
            x[4, 32 * (k % (r // 32)) + 15:32 * (k % (r // 32)) + 22] = b[1:] * (1 - 2.0 ** -24)
            x[4, 32 * (k % (r // 32)) + 22:32 * (k % (r // 32)) + 32] = 0
    if n > 5:      # the largest magnitude next to six steps of every scale
        for k in range(r // 32):
            s = Q.SCALES[30 + 11 * (k % 16)] * 6
            x[5, 32 * k:32 * k + 32] = 0
            x[5, 32 * k] = float(np.float32(s) if k % 3 == 0 else np.nextafter(np.float32(s), np.float32(0 if k % 3 == 1 else 1e9)))
    return x.to(DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("r,dr,n", [(64, 32, 1), (64, 64, 70), (128, 32, 9), (192, 64, 33), (256, 32, 40), (320, 32, 7),
                                    (448, 64, 12), (512, 64, 50)])
def test_pool_write_and_read(dtype, r, dr, n):
    n_pages = n // 64 + 3
    cfg, pages = pool(r, dr, n_pages)
    before = pages.cpu().numpy().copy()
    x = latent_rows(n, r, dr, dtype, r + n)
    rng = np.random.default_rng(n)
    index = rng.permutation(n_pages * 64)[:n].astype(np.int64)
    if n > 6:
        index[[6, -1]] = [-1, n_pages * 64]                  # skipped
    wide = torch.full((n, r + dr + 16), 3.0, dtype=DT[dtype], device="cuda")
    wide[:, 8:8 + r + dr] = x.cuda()
    M.mtla_qpool_write(cfg, pages, wide[:, 8:8 + r + dr], torch.from_numpy(index).cuda())
    want = before.copy()
    byte, code = Q.quantise(host(x)[:, :r])
    keys = x[:, r:].bfloat16().view(torch.int16).numpy().view(np.uint16)
    per_page = {}
    for i, at in enumerate(index):
        if 0 <= at < n_pages * 64:
            per_page.setdefault(at // 64, []).append((at % 64, i))
    for p, rows in per_page.items():
        b, c, k = [np.array(v) for v in Q.unpack_page(want[p], r, dr)]
        for place, i in rows:
            b[place], c[place], k[place] = byte[i], code[i], keys[i]
        want[p] = Q.pack_page(b, c, k)
    assert np.array_equal(pages.cpu().numpy(), want)          # every other byte is as it was
    for out_type in ("bf16", "fp32"):
        got = M.mtla_qpool_read(cfg, pages, torch.from_numpy(index).cuda(), dtype=DT[out_type])
        value = np.concatenate([Q.dequantise(byte, code), host(x[:, r:].bfloat16())], 1)
        value[(index < 0) | (index >= n_pages * 64)] = 0
        assert np.array_equal(host(got), value, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pool_rows_of_a_long_prompt(dtype):
    """More rows than one round of CTAs holds at once, most of them skipped."""
    r, dr, n = 128, 32, 70000
    cfg, pages = pool(r, dr, 300)
    x = torch.randn(n, r + dr, generator=torch.Generator().manual_seed(4)).to(DT[dtype])
    index = torch.full((n,), -1, dtype=torch.int64)
    kept = torch.arange(3, n, 5)
    index[kept] = torch.randperm(300 * 64, generator=torch.Generator().manual_seed(5))[:len(kept)]
    M.mtla_qpool_write(cfg, pages, x.cuda(), index.cuda())
    got = M.mtla_qpool_read(cfg, pages, index.cuda(), dtype=torch.float32).cpu()
    skipped = torch.ones(n, dtype=torch.bool)
    skipped[kept] = False
    assert (got[skipped] == 0).all()
    some = kept[::37]
    byte, code = Q.quantise(host(x[some])[:, :r])
    assert np.array_equal(host(got[some])[:, :r], Q.dequantise(byte, code))
    assert torch.equal(got[kept][:, r:], x[kept][:, r:].bfloat16().float())


def test_pool_read_into_strided_rows_leaves_the_rest():
    cfg, pages = pool(64, 32, 2)
    x = latent_rows(5, 64, 32, "fp32", 3)
    index = torch.arange(60, 65, device="cuda")
    M.mtla_qpool_write(cfg, pages, x.cuda(), index)
    wide = torch.full((5, 112), 9.0, device="cuda")
    got = M.mtla_qpool_read(cfg, pages, index, out=wide[:, 8:104])
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(M.mtla_qpool_read(cfg, pages, index, dtype=torch.float32)))
    assert (wide[:, :8] == 9).all() and (wide[:, 104:] == 9).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_row_needs_no_row_stride(dtype):
    cfg, pages = pool(64, 32, 2)
    x = latent_rows(1, 64, 32, dtype, 6).cuda()
    index = torch.tensor([77], device="cuda")
    M.mtla_qpool_write(cfg, pages, x, index)
    want, stored = M.mtla_qpool_read(cfg, pages, index, dtype=DT[dtype]), pages.clone()
    for stride in (0, 1, 97):
        one = x.as_strided((1, 96), (stride, 1))
        pages.fill_(0xA5)
        M.mtla_qpool_write(cfg, pages, one, index)
        assert torch.equal(pages, stored)
        out = torch.empty_like(want).as_strided((1, 96), (stride, 1))
        M.mtla_qpool_read(cfg, pages, index, out=out)
        assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))


def test_calls_without_rows_or_tokens():
    cfg, pages = pool(64, 32, 2)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    before = pages.clone()
    M.mtla_qpool_write(cfg, pages, torch.empty(0, 96, device="cuda"), none)
    assert M.mtla_qpool_read(cfg, pages, none).shape == (0, 96) and torch.equal(pages, before)
    x = torch.empty(0, 3, 48, device="cuda")
    (y,) = M.mtla_rope(M.make_rope_config(rope_dim=16), [x], none.int())
    assert y.shape == x.shape


# ------------------------------------------------------------------------------ attention

def attend_setup(lens, heads, r, dr, dtype, seed, junk=0xFF, size=1.0):
    """Pages of the sequences in shuffled order; every byte that no slot owns is `junk` (0xff reads as
    NaN in scales and keys)."""
    rng = np.random.default_rng(seed)
    held = [-(-n // 64) for n in lens]
    n_pages = sum(held) + 2
    cfg, pages = pool(r, dr, n_pages, heads, junk)
    order = rng.permutation(n_pages)
    width = max(1, max(held)) + 1
    table = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    rows, index = [], []
    for b, n in enumerate(lens):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
        rows.append(rng.standard_normal((n, r + dr)).astype(np.float32) * size)
        index += [int(table[b, j // 64]) * 64 + j % 64 for j in range(n)]
    if index:
        flat = torch.from_numpy(np.concatenate(rows)).cuda()
        idx = torch.tensor(index, dtype=torch.int64, device="cuda")
        M.mtla_qpool_write(cfg, pages, flat, idx)
        stored = host(M.mtla_qpool_read(cfg, pages, idx, dtype=torch.float32))
    else:
        stored = np.zeros((0, r + dr))
    cuts = np.cumsum([0] + list(lens))
    seqs = [stored[cuts[b]:cuts[b + 1]] for b in range(len(lens))]
    q = torch.from_numpy(rng.standard_normal((len(lens), heads, r + dr)).astype(np.float32)).to(DT[dtype])
    return cfg, pages, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), q, seqs


def bound(q, seq, scale, mean_abs, out, dtype, r):
    """Errors of one sequence's output and logarithm.

    A score is a sum of r + d_R products in 32 bits: each of the partial sums is off by at most 2^-24
    of the sum of magnitudes, the query's terms by 2^-22 of it (fp32: two half-precision terms), the
    scaling by 2^-23, and the base-2 exponential by 2^-22; a probability's relative error is the
    score's absolute one.  Its rounding to half precision is 2^-11 (bf16; two terms, 2^-22, for
    fp32), below 2^-14 an absolute 2^-25.  Relative errors of probabilities act twice, on the sum
    of values and on the denominator; the 32-bit sums over the slots add n 2^-24."""
    n = len(seq)
    size = (np.abs(q) @ np.abs(seq).T).max(-1, keepdims=True) * abs(scale)
    score = size * ((q.shape[1] + 2) * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -22
    p = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
    rel = score + p + n * 2.0 ** -24
    tiny = n * 2.0 ** -25 * (1.0 if dtype == "bf16" else 2.0 ** -11)
    top = np.abs(seq[:, :r]).max()
    tol_out = half_step(DT[dtype]) * np.abs(out) + 2 * rel * mean_abs + 2 * tiny * top
    return tol_out, (rel + tiny)[:, 0]


def check_attend(cfg, pages, table, slots, q, seqs, scale, dtype, lens, **kw):
    r = cfg.latent_rank
    out, lse = M.mtla_qpool_attend(cfg, pages, table, slots, q.cuda(), scale=scale, **kw)
    got, got_lse = host(out), host(lse)
    for b, n in enumerate(lens):
        seq = seqs[b][:n]
        want, want_lse, mean_abs = Q.attend(host(q[b]), seq[:, :r], seq[:, r:], scale)
        if n <= 0:
            assert (got[b] == 0).all() and np.isneginf(got_lse[b]).all()
            continue
        tol, tol_lse = bound(host(q[b]), seq, scale, mean_abs, want, dtype, r)
        assert np.isfinite(got[b]).all(), b
        worst = (np.abs(got[b] - want) / tol).max()
        assert worst <= 1, (b, n, worst)
        assert (np.abs(got_lse[b] - want_lse) <= tol_lse + 2.0 ** -23 * np.abs(want_lse)).all(), (b, n)
    return out, lse


ATTEND_CASES = [
    # lens, heads, r, d_R
    ([1], 1, 64, 32), ([64], 4, 64, 64), ([65], 8, 256, 32), ([63, 0, 129], 16, 512, 64),
    ([0, 0], 3, 128, 32), ([5, 700, 1, 0, 64, 128], 17, 192, 32), ([1000], 32, 512, 64),
    ([300] * 5, 31, 448, 32), ([2, 3, 4], 9, 320, 64), ([1, 0, 2000, 17], 24, 384, 64), ([40] * 70, 5, 128, 64),
    ([4500], 16, 256, 64), ([1], 32, 512, 64), ([127, 128, 129, 191, 192, 193], 12, 256, 32),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(ATTEND_CASES)))
def test_attend(case, dtype):
    lens, heads, r, dr = ATTEND_CASES[case]
    s = attend_setup(lens, heads, r, dr, dtype, case)
    check_attend(*s, 1 / math.sqrt(64), dtype, lens)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attend_more_tiles_than_one_share(dtype):
    """Many sequences per CTA and sequences over several CTAs in one batch."""
    rng = np.random.default_rng(4)
    lens = [int(v) for v in rng.integers(0, 130, 500)] + [9000, 0, 3000]
    s = attend_setup(lens, 6, 64, 32, dtype, 8)
    check_attend(*s, 0.2, dtype, lens)


@pytest.mark.parametrize("extra", [0, 200])
@pytest.mark.parametrize("lens,heads,r,dr", [([1, 64, 65, 130, 0, 7], 8, 64, 64), ([257], 32, 256, 32), ([90, 33], 20, 192, 64)])
def test_attend_both_kernels_on_one_batch(lens, heads, r, dr, extra):
    """A wide table sends the same bf16 batch to the tensor-core kernel, a narrow one to the other."""
    cfg, pages, table, slots, q, seqs = attend_setup(lens, heads, r, dr, "bf16", 40)
    wide = torch.full((len(lens), table.shape[1] + extra), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    check_attend(cfg, pages, wide, slots, q, seqs, 0.125, "bf16", lens)


def test_attend_batch_beyond_the_tensor_core_kernels_lists():
    rng = np.random.default_rng(7)
    lens = [int(v) for v in rng.integers(0, 90, 1100)]
    s = attend_setup(lens, 3, 64, 32, "bf16", 41)
    check_attend(*s, 0.2, "bf16", lens)


@pytest.mark.parametrize("r,dr,heads", [(64, 32, 8), (128, 64, 32), (256, 32, 16), (320, 64, 17), (384, 64, 32), (448, 32, 4),
                                        (512, 64, 32), (512, 64, 9)])
def test_attend_many_tiles_and_segments_per_cta(r, dr, heads):
    """Every CTA walks several tiles of several sequences: rings and phases wrap around more than once."""
    rng = np.random.default_rng(r)
    lens = [int(v) for v in rng.integers(0, 1500, 300)] + [0, 1, 128, 129, 5000]
    s = attend_setup(lens, heads, r, dr, "bf16", 42)
    cfg, pages, table, slots, q, seqs = s
    out, lse = M.mtla_qpool_attend(cfg, pages, table, slots, q.cuda(), scale=0.125)
    assert torch.isfinite(out.float()).all()
    again, _ = M.mtla_qpool_attend(cfg, pages, table, slots, q.cuda(), scale=0.125)
    assert torch.equal(out, again)
    got, got_lse = host(out), host(lse)
    for b in list(range(0, 305, 17)) + [300, 301, 302, 303, 304]:
        want, want_lse, mean_abs = Q.attend(host(q[b]), seqs[b][:, :r], seqs[b][:, r:], 0.125)
        if lens[b] == 0:
            assert (got[b] == 0).all() and np.isneginf(got_lse[b]).all()
            continue
        tol, tol_lse = bound(host(q[b]), seqs[b], 0.125, mean_abs, want, "bf16", r)
        assert (np.abs(got[b] - want) <= tol).all(), (b, lens[b])
        assert (np.abs(got_lse[b] - want_lse) <= tol_lse + 2.0 ** -23 * np.abs(want_lse)).all(), b


@pytest.mark.parametrize("heads", [16, 31, 32])
@pytest.mark.parametrize("r", [448, 512])
@pytest.mark.parametrize("lens", [[300] * 5, [128, 127, 1, 0, 256, 129] * 4])
def test_attend_shares_of_a_tile_on_fresh_data(lens, r, heads):
    """The first call on new pages: what a share's only tile needs comes late and unevenly."""
    for seed in range(3):
        check_attend(*attend_setup(lens, heads, r, 64, "bf16", 50 + seed), 0.125, "bf16", lens)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale,size", [(0.0, 1.0), (-0.3, 1.0), (4.0, 1.0), (0.125, 1e-4), (0.125, 300.0), (1e-9, 1e4)])
def test_attend_scales(dtype, scale, size):
    """Flat, negative, very peaked distributions, and latents far from one."""
    lens = [200, 64]
    s = attend_setup(lens, 10, 128, 32, dtype, 2, size=size)
    check_attend(*s, scale, dtype, lens)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("factor", [1e-30, 1e-6, 1e5, 1e28])
def test_attend_query_sizes(dtype, factor):
    """Queries that half precision could not hold: the scores are the ordinary ones, by the scale."""
    lens = [90, 7]
    cfg, pages, table, slots, q, seqs = attend_setup(lens, 4, 192, 64, dtype, 6)
    q = (q.float() * factor).to(DT[dtype])
    check_attend(cfg, pages, table, slots, q, seqs, 0.1 / factor, dtype, lens)


def test_attend_growing_scores_raise_the_reference():
    """Scores that rise by tens from tile to tile, so that every tile rescales what came before."""
    heads, r, dr, n = 20, 128, 32, 640
    cfg, pages, table, slots, q, seqs = attend_setup([n], heads, r, dr, "bf16", 1)
    keys = torch.zeros(n, r + dr, device="cuda")
    keys[:, :r] = torch.from_numpy(seqs[0][:, :r]).cuda()
    keys[:, r] = torch.arange(n, device="cuda") // 64 * 30.0
    idx = (table[0].long()[torch.arange(n, device="cuda") // 64] * 64 + torch.arange(n, device="cuda") % 64)
    M.mtla_qpool_write(cfg, pages, keys, idx)
    q[..., :] = 0.01 * q
    q[..., r] = 1.0
    q[:, ::2, r] = -1.0                        # half of the heads see them fall
    seqs = [host(M.mtla_qpool_read(cfg, pages, idx, dtype=torch.float32))]
    check_attend(cfg, pages, table, slots, q, seqs, 1.0, "bf16", [n])


def test_attend_bad_lengths_and_pages():
    lens = [130, 200, 64, 70]
    cfg, pages, table, slots, q, seqs = attend_setup(lens, 8, 128, 32, "bf16", 11)
    slots[0] = -3                               # no slot
    slots[1] = 10 ** 9                          # cut to the table's width, whose rest is outside the pool
    table[2, 0] = cfg.n_pages                   # its only page is outside the pool
    table[3, 0] = -5                            # the first of two
    out, lse = M.mtla_qpool_attend(cfg, pages, table, slots, q.cuda(), scale=0.125)
    assert (out[0] == 0).all() and torch.isneginf(lse[0]).all()
    assert torch.isnan(out[2]).all()
    want, _, mean_abs = Q.attend(host(q[3]), seqs[3][64:, :128], seqs[3][64:, 128:], 0.125)
    tol, _ = bound(host(q[3]), seqs[3][64:], 0.125, mean_abs, want, "bf16", 128)
    assert (np.abs(host(out[3]) - want) <= tol).all()


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_attend_special_keys(value):
    """A visible infinity or NaN in a key does what the formula says, for its sequence alone."""
    lens = [100, 100]
    cfg, pages, table, slots, q, seqs = attend_setup(lens, 4, 64, 32, "bf16", 12)
    row = torch.from_numpy(seqs[0][70:71].astype(np.float32)).cuda()
    row[0, 64] = value
    M.mtla_qpool_write(cfg, pages, row, (table[0, 1].long() * 64 + 6).view(1))
    q[0, :, 64] = 1.0
    out, lse = M.mtla_qpool_attend(cfg, pages, table, slots, q.cuda(), scale=0.125)
    keep = [i for i in range(100) if i != 70]
    if value == -math.inf:                      # weight zero
        want, _, mean_abs = Q.attend(host(q[0]), seqs[0][keep, :64], seqs[0][keep, 64:], 0.125)
        tol, _ = bound(host(q[0]), seqs[0][keep], 0.125, mean_abs, want, "bf16", 64)
        assert (np.abs(host(out[0]) - want) <= tol).all()
    else:
        assert torch.isnan(out[0]).all()
    assert torch.isfinite(out[1].float()).all()


def test_attend_leaves_other_rows_and_needs_no_clean_workspace():
    lens = [700, 3]
    cfg, pages, table, slots, q, seqs = attend_setup(lens, 16, 256, 32, "bf16", 13)
    big = torch.full((4, 16, 256), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(M.mtla_qpool_workspace_bytes(cfg, 2), dtype=torch.uint8, device="cuda")
    first = None
    for fill in (0, 0xFF, 0x55):
        ws.fill_(fill)
        out, lse = check_attend(cfg, pages, table, slots, q, seqs, 0.125, "bf16", lens, out=big[1:3], workspace=ws)
        first = out.clone() if first is None else first
        assert torch.equal(out, first)
    assert (big[0] == 5).all() and (big[3] == 5).all()


def test_attend_is_reproducible():
    lens = [2000, 1, 900, 64 * 31]
    cfg, pages, table, slots, q, seqs = attend_setup(lens, 32, 512, 64, "bf16", 14)
    runs = [M.mtla_qpool_attend(cfg, pages, table, slots, q.cuda(), scale=0.125) for _ in range(5)]
    for out, lse in runs[1:]:
        assert torch.equal(out, runs[0][0]) and torch.equal(lse, runs[0][1])


# ------------------------------------------------------------------------------ together

def serving_state(heads=8, r=128, dr=32, stride=2, batch=3, n_pages=40, width=6):
    cfg = M.make_qpool_config(n_heads=heads, latent_rank=r, rope_dim=dr, n_pages=n_pages)
    pages = M.make_qpool(cfg)
    pages.fill_(0xFF)
    return cfg, pages, M.make_rope_config(rope_dim=dr)


def test_a_run_of_the_operators_together():
    """Prompts of different lengths, then single-token steps: pages from the map, keys rotated, running
    states stored, attention over the pool; the oracle keeps its own pages and rows."""
    heads, r, dr, stride, scale = 8, 128, 32, 2, 0.125
    cfg, pages, rope = serving_state(heads, r, dr, stride)
    rng = np.random.default_rng(21)
    batch, width = 3, 6
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    free = [int(v) for v in rng.permutation(cfg.n_pages)]
    f = Q.rope_frequencies(dr)
    held = [0] * batch
    cache = [{} for _ in range(batch)]          # slot -> stored row, by the oracle
    o_table = [[-1] * width for _ in range(batch)]
    for fresh in ([126, 33, 0], [1, 1, 1], [1, 0, 1], [64, 1, 130], [1, 1, 1]):
        dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        n = sum(fresh)
        m = M.mtla_slot_map(dev(held), dev(fresh), dev(free), table, stride=stride, n_tokens=n + 5)
        want = Q.slot_map(held, fresh, stride, o_table, free)
        check_map(m, table, want, o_table, n, 5)
        rows = torch.from_numpy(rng.standard_normal((n + 5, r + dr)).astype(np.float32)).bfloat16()
        dev_rows = rows.cuda()
        key = dev_rows[:, None, r:]
        M.mtla_rope(rope, [key], m.position, out=[key])              # the keys, in place in the rows
        M.mtla_qpool_write(cfg, pages, dev_rows, m.store)
        exact_keys = Q.rope(host(rows[:, None, r:]), want["position"] + [0] * 5, f, "interleaved", 0)[:, 0]
        assert (np.abs(host(dev_rows[:, r:]) - exact_keys) <=
                rope_bound(rows[:, None, r:], exact_keys[:, None], 0, dr, "interleaved", 1.0, "bf16")[:, 0]).all()
        byte, code = Q.quantise(host(rows)[:n, :r])
        value = np.concatenate([Q.dequantise(byte, code), host(dev_rows[:n, r:])], 1)
        for t in range(n):
            if want["store"][t] >= 0:
                cache[want["seq"][t]][want["position"][t] // stride] = value[t]
        held = [h + g for h, g in zip(held, fresh)]
        free = free[want["taken"]:]
        q = torch.from_numpy(rng.standard_normal((batch, heads, r + dr)).astype(np.float32)).bfloat16()
        seqs = [np.array([cache[b][j] for j in range(want["slots"][b])]).reshape(-1, r + dr) for b in range(batch)]
        check_attend(cfg, pages, table, m.slots, q, seqs, scale, "bf16", want["slots"])


def test_a_layers_cache_in_four_bits():
    """A handle's exported cache through the pool: attention over it is the layer's attention up to
    the codes' rounding, and exactly the oracle's over the codes."""
    from paper_2505_13544_b200 import synth
    from tests import helpers as H
    w = synth.WORKLOADS["paper"].scaled(batch=2, prefill_tokens=131, decode_steps=1)
    h = H.gpu_handle(w, synth.make_weights(w))
    M.mtla_prefill(h, synth.prompt(w).cuda(), want_output=False)
    rows = M.mtla_cache_export(h)
    M.mtla_destroy(h)
    n = rows.shape[1]
    cfg, pages = pool(w.latent_rank, w.rope_dim, 4, w.n_heads, 0xFF)
    table = torch.tensor([[3, 1], [0, 2]], dtype=torch.int32, device="cuda")
    j = torch.arange(n, device="cuda")
    index = torch.cat([table[b].long()[j // 64] * 64 + j % 64 for b in range(2)])
    M.mtla_qpool_write(cfg, pages, rows.reshape(2 * n, -1), index)
    stored = host(M.mtla_qpool_read(cfg, pages, index)).reshape(2, n, -1)
    # Against the bf16 rows: a code is within one scale (half of the widest step), a scale at most
    # 9 / 8 of a sixth of its group's largest magnitude.
    lat = host(rows)[..., :w.latent_rank].reshape(2, n, -1, 32)
    assert (np.abs(stored[..., :w.latent_rank].reshape(lat.shape) - lat) <=
            np.abs(lat).max(-1, keepdims=True) * 9 / 48 + 2.0 ** -17).all()
    q = torch.randn(2, w.n_heads, w.latent_rank + w.rope_dim, generator=torch.Generator().manual_seed(1)).bfloat16()
    slots = torch.tensor([n, n], dtype=torch.int32, device="cuda")
    check_attend(cfg, pages, table, slots, q, list(stored), 0.125, "bf16", [n, n])


def test_captured_step_replays_with_new_lengths():
    """One graph of all four calls, captured once and replayed while requests grow on the device."""
    heads, r, dr, stride = 16, 64, 32, 2
    cfg, pages, rope = serving_state(heads, r, dr, stride)
    batch, width = 2, 5
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.full((batch, width), -1, **i32)
    held, fresh = torch.zeros(batch, **i32), torch.ones(batch, **i32)
    free = torch.arange(20, **i32)
    out_map = M.make_slot_map(batch, batch)
    rows = torch.randn(batch, r + dr, device="cuda").bfloat16()
    q = torch.randn(batch, heads, r + dr, device="cuda").bfloat16()
    rot, out = torch.empty_like(rows[:, None, r:].contiguous()), torch.empty(batch, heads, r, dtype=q.dtype, device="cuda")
    lse = torch.empty(batch, heads, device="cuda")
    ws = torch.empty(M.mtla_qpool_workspace_bytes(cfg, batch), dtype=torch.uint8, device="cuda")

    def step():
        m = M.mtla_slot_map(held, fresh, free, table, stride=stride, out=out_map)
        M.mtla_rope(rope, [rows[:, None, r:]], m.position, out=[rot])
        M.mtla_qpool_write(cfg, pages, torch.cat([rows[:, :r], rot[:, 0]], 1), m.store)
        M.mtla_qpool_attend(cfg, pages, table, m.slots, q, scale=0.125, out=out, lse=lse, workspace=ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()                                  # on another stream than the default
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for h in (0, 1, 5, 126, 127, 128, 129, 300):
        table.fill_(-1)
        for b in range(batch):                  # the pages that h tokens already hold
            for p in range(-(-(-(-h // stride)) // 64)):
                table[b, p] = 39 - p - 8 * b
        held.fill_(h)
        keep = table.clone()
        pages_before = pages.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = (out.clone(), lse.clone(), table.clone(), pages.clone())
        table.copy_(keep)
        pages.copy_(pages_before)
        step()
        torch.cuda.synchronize()
        assert torch.equal(table, got[2]) and torch.equal(pages, got[3])
        if h == 0:
            assert torch.isfinite(got[0].float()).all()
        assert torch.equal(torch.nan_to_num(out.float()), torch.nan_to_num(got[0].float()))
        assert torch.equal(torch.nan_to_num(lse), torch.nan_to_num(got[1]))


def test_two_streams_with_a_workspace_each():
    lens = [3000, 40]
    cfg, pages, table, slots, q, seqs = attend_setup(lens, 8, 256, 32, "bf16", 30)
    want = M.mtla_qpool_attend(cfg, pages, table, slots, q.cuda(), scale=0.125)[0]
    torch.cuda.synchronize()
    qd = q.cuda()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for i in range(6):
        outs.append(M.mtla_qpool_attend(cfg, pages, table, slots, qd, scale=0.125, stream=streams[i % 2],
                                        workspace=torch.empty(M.mtla_qpool_workspace_bytes(cfg, 2), dtype=torch.uint8,
                                                              device="cuda"))[0])
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, want)


def test_buffers_of_a_call_come_from_its_stream(monkeypatch):
    """Memory that a call allocates is the given stream's: freed at once (the workspace), it must not go to
    work that another stream has queued."""
    cfg, pages, table, slots, q, seqs = attend_setup([70, 3], 8, 64, 32, "bf16", 31)
    qd, index = q.cuda(), torch.arange(4, device="cuda")
    lens = torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    stream, made, empty = torch.cuda.Stream(), [], torch.empty
    monkeypatch.setattr(M.torch, "empty", lambda *s, **kw: made.append(torch.cuda.current_stream()) or empty(*s, **kw))
    M.mtla_qpool_attend(cfg, pages, table, slots, qd, scale=0.125, stream=stream)
    assert len(made) == 3
    M.mtla_qpool_read(cfg, pages, index, stream=stream)
    M.mtla_rope(M.make_rope_config(rope_dim=16), [qd], lens, stream=stream)
    M.mtla_slot_map(lens * 0, lens, lens, table.clone(), stride=1, n_tokens=3, stream=stream)
    torch.cuda.synchronize()
    assert len(made) == 12 and all(s == stream for s in made)
    made.clear()
    M.mtla_qpool_attend(cfg, pages, table, slots, qd, scale=0.125)
    assert len(made) == 3 and all(s == torch.cuda.current_stream() for s in made)


def test_page_numbers_past_32_bit_offsets():
    """A pool larger than 4 GiB: the last pages hold the slots."""
    r, dr = 512, 64
    n_pages = (1 << 32) // (34 * r + 128 * dr) + 300
    if torch.cuda.mem_get_info()[0] < 6 << 30:
        pytest.skip("less than 6 GiB free")
    cfg = M.make_qpool_config(n_heads=4, latent_rank=r, rope_dim=dr, n_pages=n_pages)
    pages = M.make_qpool(cfg)
    x = torch.randn(130, r + dr, generator=torch.Generator().manual_seed(2))
    table = torch.tensor([[n_pages - 1, n_pages - 200, n_pages - 7]], dtype=torch.int32, device="cuda")
    j = torch.arange(130, device="cuda")
    index = table[0].long()[j // 64] * 64 + j % 64
    M.mtla_qpool_write(cfg, pages, x.cuda(), index)
    stored = host(M.mtla_qpool_read(cfg, pages, index, dtype=torch.float32))
    byte, code = Q.quantise(host(x)[:, :r])
    assert np.array_equal(stored[:, :r], Q.dequantise(byte, code))
    q = torch.randn(1, 4, r + dr, generator=torch.Generator().manual_seed(3)).bfloat16()
    check_attend(cfg, pages, table, torch.tensor([130], dtype=torch.int32, device="cuda"), q, [stored], 0.1, "bf16", [130])

"""Attention over long sequences of the 4-bit pool, whose pages repeat so that the pool stays small: the
weight of a stored row is the number of times that the sequence reads it."""
import math

import numpy as np
import pytest
import torch

from paper_2505_13544_b200 import binding as M

pytestmark = pytest.mark.gpu
PAGES = 12


def stored_pool(heads, r, dr, seed, lift=0.0):
    """PAGES pages of latents of one sign, so that their sums grow; `lift`: what the first key element of
    page p rises by with p."""
    cfg = M.make_qpool_config(n_heads=heads, latent_rank=r, rope_dim=dr, n_pages=PAGES)
    pages = M.make_qpool(cfg)
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(PAGES * 64, r + dr, generator=g)
    x[:, :r] = x[:, :r].abs() + 0.5
    x[:, r] = (torch.arange(PAGES * 64) // 64) * lift
    index = torch.arange(PAGES * 64, device="cuda")
    M.mtla_qpool_write(cfg, pages, x.cuda(), index)
    return cfg, pages, M.mtla_qpool_read(cfg, pages, index, dtype=torch.float32).double().cpu().numpy()


def attend_exact(q, rows, counts, r, scale):
    """Softmax over rows that occur counts[j] times, 64-bit: output, logarithm, largest score magnitude, and
    how many slots' probabilities lie more than 21 binary orders below their head's largest."""
    seen = counts > 0
    rows, counts = rows[seen], counts[seen]
    score = (q @ rows.T) * scale
    top = score.max(-1, keepdims=True)
    p = counts * np.exp(score - top)
    total = p.sum(-1, keepdims=True)
    size = (np.abs(q) @ np.abs(rows).T).max() * abs(scale)
    small = (counts * (top - score > 21 * math.log(2))).sum(-1).max()
    return p @ rows[:, :r] / total, (top + np.log(total))[:, 0], size, small


def row_counts(page_list, n):
    counts = np.zeros((PAGES, 64))
    full = n // 64
    np.add.at(counts, page_list[:full], 1.0)
    counts[page_list[full] if n % 64 else 0, :n % 64] += 1.0
    return counts.reshape(-1)


def bounds(n, size, width, cut, added, small, spread):
    """Relative to the mean magnitude (all latents are positive: to the output itself).

    Output: half a step of bf16; the probabilities' half step of half precision, 2^-11, and the scores' error
    (see the ordinary tests), each in the sum of values and in the denominator; what the matrix
    instructions cut off from sums of `cut` slots, where every 16 slots each of the 16 products and the sum may
    lose a unit, 2^-23; and `added` sums of such pieces rounded outside, 2^-24 each.  The denominator is
    summed outside altogether, n / 64 rounded additions at most in a row, and the combine's few.  Below 2^-14
    half precision keeps a probability to 2^-25 only; as the largest ones are kept as 2^7 at least, that
    is the case of the `small` ones 21 binary orders below them, and each is then off by 2^-32 of the largest,
    which a latent `spread` times the output's size at most multiplies."""
    score = size * ((width + 2) * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -22
    total = score + (n / 64 + 600) * 2.0 ** -24
    out = torch.finfo(torch.bfloat16).eps / 2 + 2 * 2.0 ** -11 + score + total
    return out + cut / 16 * 17 * 2.0 ** -23 + added * 2.0 ** -24 + small * 2.0 ** -32 * spread, 2 * 2.0 ** -11 + total


def check(lens, lists, heads, r, dr, scale, seed, cut, added, lift=0.0, look=None):
    cfg, pages, rows = stored_pool(heads, r, dr, seed, lift)
    width = max(-(-n // 64) for n in lens)
    kinds = sorted(set(zip(lens, lists)))
    table = np.zeros((len(lens), width), dtype=np.int32)
    for b, (n, k) in enumerate(zip(lens, lists)):
        table[b] = PAGE_LISTS[k](width)
    q = torch.randn(1, heads, r + dr, generator=torch.Generator().manual_seed(seed + 1))
    if lift:
        q *= 0.01
        q[..., r] = 1.0
        q[:, ::2, r] = -1.0                     # half of the heads see the lifted keys fall
    q = q.bfloat16()
    out, lse = M.mtla_qpool_attend(cfg, pages, torch.from_numpy(table).cuda(),
                                   torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                   q.cuda().expand(len(lens), -1, -1).contiguous(), scale=scale)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    qd = q[0].double().numpy()
    for n, k in kinds:
        same = [b for b in range(len(lens)) if (lens[b], lists[b]) == (n, k)]
        if n == 0:
            assert (out[same] == 0).all() and np.isneginf(lse[same]).all()
            continue
        want, want_lse, size, small = attend_exact(qd, rows, row_counts(PAGE_LISTS[k](width), n), r, scale)
        tol, tol_lse = bounds(n, size, r + dr, min(n, cut), added(n), small,
                              rows[:, :r].max() / rows[:, :r].min())
        worst = (np.abs(out[same] - want) / want).max()
        assert worst <= tol, (n, k, worst, tol)
        assert (np.abs(lse[same] - want_lse) <= tol_lse + 2.0 ** -23 * np.abs(want_lse)).all(), (n, k)


PAGE_LISTS = [
    lambda w: np.arange(w) % PAGES,
    lambda w: np.minimum(np.arange(w) * PAGES // w, PAGES - 1),           # page by page: a lift rises slowly
    lambda w: PAGES - 1 - np.minimum(np.arange(w) * PAGES // w, PAGES - 1),
    lambda w: (np.arange(w) // 300) % PAGES,
]
TC = dict(cut=16384, added=lambda n: n / 16384 + 600)        # sums in tensor memory over 128 tiles of 128 slots


@pytest.mark.parametrize("r,dr,heads", [(64, 32, 4), (192, 64, 20), (512, 64, 16)])
def test_long_sequences_keep_their_sums(r, dr, heads):
    """2^20 slots of every sequence, each in one CTA: sums that the matrix unit alone would leave 6.6e-3 short."""
    check([1 << 20] * 148, [0] * 148, heads, r, dr, 0.03, r, **TC)


@pytest.mark.parametrize("r,dr,heads,lift", [(64, 32, 8, 0.0), (64, 64, 32, 4.0), (128, 32, 17, 30.0), (256, 32, 16, 4.0),
                                             (320, 64, 9, 2.0), (384, 64, 32, 30.0), (448, 32, 32, 0.0), (512, 64, 9, 4.0),
                                             (512, 64, 32, 30.0)])
def test_sums_are_set_down_at_any_place_of_a_sequence(r, dr, heads, lift):
    """Sequences around the 16384 slots after which sums leave tensor memory, several to a CTA and cut by the
    CTAs' borders, with references that rise before, at and behind that place."""
    kinds = [(16384, 1), (16385, 1), (16512, 2), (16513, 1), (32768, 2), (32769, 1), (50001, 3), (100003, 1), (1, 0), (0, 0),
             (40000, 3), (129, 0)]
    lens, lists = zip(*[kinds[i % len(kinds)] for i in range(180)])
    check(list(lens), list(lists), heads, r, dr, 0.125, r + heads, lift=lift, **TC)


# The warp-level kernel, for batches beyond the other one's lists (1022), adds products of 32 slots outside.
WARP = dict(cut=32, added=lambda n: n / 32 + 600)


@pytest.mark.parametrize("r,dr,heads", [(64, 32, 4), (128, 64, 20)])
def test_long_sequences_of_a_large_batch(r, dr, heads):
    """2^20 slots of 1030 sequences, which take about half a second."""
    check([1 << 20] * 1030, [0] * 1030, heads, r, dr, 0.03, r + 7, **WARP)


@pytest.mark.parametrize("r,dr,heads,lift", [(64, 32, 8, 4.0), (320, 64, 9, 30.0), (512, 64, 32, 4.0), (448, 32, 20, 30.0)])
def test_sums_of_a_large_batch_of_ragged_lengths(r, dr, heads, lift):
    kinds = [(16384, 1), (16385, 1), (16448, 2), (33, 1), (32768, 2), (32769, 1), (50001, 3), (0, 0), (1, 0), (700, 1)]
    lens, lists = zip(*[kinds[i % len(kinds)] for i in range(1030)])
    check(list(lens), list(lists), heads, r, dr, 0.125, r + heads, lift=lift, **WARP)

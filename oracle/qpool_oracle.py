"""64-bit statements of the operators around the 4-bit latent pool (numpy, no CUDA, no shared code).

Every function follows its definition word by word and slowly: a code is the nearest of the sixteen
by distance, a scale the first grid value that reaches, a slot map a loop over tokens.
"""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# Every scale: zero, then numbers of four significant bits, the smallest 2^-17 apart, up to 10240.
SCALES = np.array([k * 2.0 ** -17 for k in range(8)]
                  + [(8 + k) * 2.0 ** (e - 3) for e in range(-14, 14) for k in range(8)
                     if (8 + k) * 2.0 ** (e - 3) <= 10240.0])
PAGE, GROUP = 64, 32


def quantise(x: np.ndarray):
    """(scale bytes [n][r/32], codes [n][r]) of latents x [n][r]; byte i is SCALES[i], 255 is NaN."""
    n, r = x.shape
    x = np.asarray(x, dtype=np.float64).reshape(n, r // GROUP, GROUP)
    byte = np.zeros((n, r // GROUP), dtype=np.uint8)
    code = np.zeros(x.shape, dtype=np.uint8)
    for i in range(n):
        for g in range(r // GROUP):
            v = x[i, g]
            if not np.isfinite(v).all():
                byte[i, g] = 255
                continue
            reach = np.nonzero(6 * SCALES >= np.abs(v).max())[0]
            byte[i, g] = reach[0] if len(reach) else len(SCALES) - 1
            s = SCALES[byte[i, g]]
            dist = np.abs(np.abs(v)[:, None] - MAGNITUDES[None, :] * s)
            near = dist.min(-1, keepdims=True)
            for j in range(GROUP):
                hits = np.nonzero(dist[j] == near[j])[0]
                c = min(hits, key=lambda h: (h & 1, h))        # the even one on a tie
                code[i, g, j] = c | (8 if v[j] < 0 else 0)
    return byte, code.reshape(n, r)


def dequantise(byte: np.ndarray, code: np.ndarray) -> np.ndarray:
    n, r = code.shape
    scale = np.where(byte == 255, np.nan, SCALES[np.minimum(byte, len(SCALES) - 1)])
    sign = np.where(code & 8, -1.0, 1.0)
    return (sign * MAGNITUDES[code & 7]).reshape(n, r // GROUP, GROUP).__mul__(scale[..., None]).reshape(n, r)


def _code_chunk(row: int, chunk: int, r: int) -> int:
    n = r // 32
    m = 1
    while m < 8 and n % (2 * m) == 0:
        m *= 2
    return chunk ^ (row & (m - 1))


def _key_chunk(row: int, chunk: int, dr: int) -> int:
    return chunk ^ ((row & 7) if dr == 64 else ((row >> 1) & 3))


def unpack_page(page: np.ndarray, r: int, dr: int):
    """(scale bytes [64][r/32], codes [64][r], key bits [64][d_R] uint16) of one page's bytes."""
    codes = np.zeros((PAGE, r), dtype=np.uint8)
    keys = np.zeros((PAGE, dr), dtype=np.uint16)
    for i in range(PAGE):
        for c in range(r // 32):
            at = i * (r // 2) + 16 * _code_chunk(i, c, r)
            b = page[at:at + 16]
            codes[i, 32 * c:32 * c + 32:2] = b & 15
            codes[i, 32 * c + 1:32 * c + 32:2] = b >> 4
        for c in range(dr // 8):
            at = 34 * r + i * 2 * dr + 16 * _key_chunk(i, c, dr)
            keys[i, 8 * c:8 * c + 8] = page[at:at + 16].view(np.uint16)
    return page[32 * r:34 * r].reshape(PAGE, r // 32), codes, keys


def pack_page(byte: np.ndarray, codes: np.ndarray, keys: np.ndarray) -> np.ndarray:
    """The inverse of unpack_page."""
    r, dr = codes.shape[1], keys.shape[1]
    page = np.zeros(34 * r + 128 * dr, dtype=np.uint8)
    page[32 * r:34 * r] = byte.reshape(-1)
    for i in range(PAGE):
        for c in range(r // 32):
            at = i * (r // 2) + 16 * _code_chunk(i, c, r)
            part = codes[i, 32 * c:32 * c + 32]
            page[at:at + 16] = part[0::2] | (part[1::2] << 4)
        for c in range(dr // 8):
            at = 34 * r + i * 2 * dr + 16 * _key_chunk(i, c, dr)
            page[at:at + 16] = keys[i, 8 * c:8 * c + 8].view(np.uint8)
    return page


def slot_map(held, fresh, stride, table, free):
    """Loop over requests and tokens; table: list of lists (changed in place)."""
    starts, seq, position, slot, store, slots, taken = [0], [], [], [], [], [], 0
    for b, (h, f) in enumerate(zip(held, fresh)):
        slots.append(-(-(h + f) // stride))
        for p in range(-(-(-(-h // stride)) // PAGE), -(-slots[b] // PAGE)):
            table[b][p] = free[taken]
            taken += 1
        for i in range(h, h + f):
            j = i // stride
            seq.append(b)
            position.append(i)
            slot.append(table[b][j // PAGE] * PAGE + j % PAGE)
            closes = i % stride == stride - 1 or i == h + f - 1
            store.append(slot[-1] if closes else -1)
        starts.append(len(seq))
    return dict(starts=starts, seq=seq, position=position, slot=slot, store=store, slots=slots, taken=taken)


def rope_frequencies(dim, theta=10000.0, scaling="none", factor=1.0, low=1.0, high=32.0, train_tokens=0):
    out = []
    for k in range(dim // 2):
        f = float(theta) ** (-2.0 * k / dim)
        if scaling == "linear":
            f /= factor
        elif scaling == "ramp":
            turns = train_tokens * f / (2 * np.pi)
            g = min(1.0, max(0.0, (turns - low) / (high - low)))
            f = g * f + (1 - g) * f / factor
        out.append(f)
    return np.array(out)


def rope(x, positions, freq, layout, first, magnitude=1.0, inverse=False):
    """x [n][heads][width] with the rotated part at `first`."""
    y = np.array(x, dtype=np.float64)
    half = len(freq)
    for t, p in enumerate(positions):
        for k in range(half):
            i, j = (first + k, first + half + k) if layout == "half" else (first + 2 * k, first + 2 * k + 1)
            ang = float(p) * freq[k] * (-1 if inverse else 1)
            c, s = np.cos(ang) * magnitude, np.sin(ang) * magnitude
            a, b = y[t, :, i].copy(), y[t, :, j].copy()
            y[t, :, i], y[t, :, j] = a * c - b * s, b * c + a * s
    return y


def attend(q, latents, keys, scale):
    """One sequence: q [heads][r + d_R], latents [n][r], keys [n][d_R] -> (out, lse, |out| bound):
    the last is the probability-weighted mean magnitude, the size that relative errors act on."""
    heads, r = q.shape[0], latents.shape[1]
    if latents.shape[0] == 0:
        return np.zeros((heads, r)), np.full(heads, -np.inf), np.zeros((heads, r))
    score = (q[:, :r] @ latents.T + q[:, r:] @ keys.T) * scale
    top = score.max(-1, keepdims=True)
    p = np.exp(score - top)
    total = p.sum(-1, keepdims=True)
    return p @ latents / total, (top + np.log(total))[:, 0], p @ np.abs(latents) / total

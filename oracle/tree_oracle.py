"""64-bit statements of the operators of a verification step over drafted trees (numpy, no CUDA, no shared code):
what nodes see follows their path token by token, a weight is found byte by byte in its block."""
from __future__ import annotations

import numpy as np

from oracle import qpool_oracle as Q

MAX_NODES = 64


def tree_map(held, starts, parents, stride, n_nodes):
    """Loop over requests, nodes and their paths; masks as sets of bits."""
    seq, position, seen = [-1] * n_nodes, [0] * n_nodes, [0] * n_nodes
    slots = [max(h, 0) // stride for h in held]
    ends = [0] + list(starts)
    if any(a > b for a, b in zip(ends, ends[1:])) or starts[-1] > n_nodes:
        return dict(seq=seq, position=position, seen=seen, slots=slots)
    for b, h in enumerate(held):
        lo, hi = starts[b], starts[b + 1]
        paths, fine = [], h >= 0 and hi - lo <= MAX_NODES
        for i in range(hi - lo):
            p = parents[lo + i]
            fine = fine and -1 <= p < i
            if not fine:
                break
            paths.append([i] if p < 0 else paths[p] + [i])
        fine = fine and all(h + len(path) - 1 < 2 ** 31 for path in paths)
        if not fine:
            continue
        for i, path in enumerate(paths):
            seq[lo + i], position[lo + i] = b, h + len(path) - 1
            for d, node in enumerate(path):
                if node == i or (h + d + 1) % stride == 0:
                    seen[lo + i] |= 1 << node
    return dict(seq=seq, position=position, seen=[s - (1 << 64) if s >> 63 else s for s in seen], slots=slots)


def attend_node(q, context, rows, seen, scale, r):
    """One node: q [heads][r + d_R] over context [n][r + d_R] and the rows whose bits are set -> (out, lse, mean
    magnitude); rows that are not seen are not touched."""
    picked = [rows[j] for j in range(min(len(rows), MAX_NODES)) if seen >> j & 1]
    both = np.concatenate([context, np.array(picked).reshape(-1, context.shape[1])])
    return Q.attend(q, both[:, :r], both[:, r:], scale)


SIGN_AT, MAG_AT = (15, 12, 14, 13), (6, 3, 0, 9)


def pack_weight(w):
    """Packed bytes of w [in][out]."""
    n_in, n_out = w.shape
    kb, ob = -(-n_in // 128), -(-n_out // 16)
    full = np.zeros((kb * 128, ob * 16))
    full[:n_in, :n_out] = w
    scale, code = Q.quantise(full.T)
    out = np.zeros((ob, kb, 1088), dtype=np.uint8)
    for o in range(ob * 16):
        i = o % 16
        for k in range(kb * 128):
            group, pair, half, word = k // 32 % 4, k // 2 % 4, k % 2, k // 8 % 4
            at = 64 * i + 16 * (group ^ (i >> 1 & 3)) + 4 * word
            c = int(code[o, k])
            bits = (c >> 3) << (SIGN_AT[pair] + 16 * half) | (c & 7) << (MAG_AT[pair] + 16 * half)
            for n in range(4):
                out[o // 16, k // 128, at + n] |= bits >> (8 * n) & 255
            if k % 32 == 0:
                out[o // 16, k // 128, 1024 + 2 * (4 * (i & 7) + group) + (i >> 3)] = scale[o, k // 32]
    return out.reshape(-1)


def unpack_weight(packed, n_in, n_out):
    """The weights [in][out] in 64 bits."""
    kb = -(-n_in // 128)
    blocks = packed.reshape(-1, kb, 1088)
    k, o = np.arange(n_in)[:, None], np.arange(n_out)[None, :]
    group, pair, half, word, i = k // 32 % 4, k // 2 % 4, k % 2, k // 8 % 4, o % 16
    at = 64 * i + 16 * (group ^ (i >> 1 & 3)) + 4 * word + 2 * half
    bits = blocks[o // 16, k // 128, at].astype(int) | blocks[o // 16, k // 128, at + 1].astype(int) << 8
    mag = Q.MAGNITUDES[bits >> np.array(MAG_AT)[pair] & 7]
    sign = 1.0 - 2.0 * (bits >> np.array(SIGN_AT)[pair] & 1)
    byte = blocks[o // 16, k // 128, 1024 + 2 * (4 * (i & 7) + group) + (i >> 3)]
    scale = np.where(byte == 255, np.nan, Q.SCALES[np.minimum(byte, len(Q.SCALES) - 1)])
    return sign * mag * scale

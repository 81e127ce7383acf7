"""Operators around a paged latent cache held in 4 bits: plain forms, inputs and 64-bit answers.

A serving loop over compressed latent slots runs these next to each other:

  map      block tables and slot maps from request lengths            (mtla_slot_map)
  rope     rotation of the RoPE part of query heads and shared keys   (mtla_rope; inverse = gradient)
  store    latent rows into the 4-bit pool, and read back             (mtla_qpool_write / mtla_qpool_read)
  attend   one query per sequence over its 4-bit slots                (mtla_qpool_attend)

A pool page holds 64 slots: [64][r/2] bytes of 4-bit codes (e2m1: sign, two exponent bits, one
fraction bit; latent 2k in the low half of byte k), [64][r/32] bytes of group scales (the upper
bits of a positive half-precision number: 5 exponent bits, 3 fraction bits), [64][d_R] bf16 RoPE
keys.  The 16-byte chunk c of row i sits at chunk position c ^ (i & m) of its row: in the code block
m + 1 is the largest power of two, 8 at most, that divides the number of chunks; in the key block
the place is c ^ (i & 7) for d_R = 64 and c ^ ((i >> 1) & 3) for d_R = 32.
"""
from __future__ import annotations

import math
import random

import torch

own = False

PAGE = 64
GROUP = 32
SCALE_MAX = 10240.0          # six steps of it still fit half precision
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------ cases

def listed():
    return [
        # One decode step of a large batch: every request gets one token.
        dict(name="map_step", op="map", batch=128, stride=2, held_max=32768, fresh_max=1, all_fresh=True, pad=0),
        # A batch of prompts entering at once, ragged, some requests idle.
        dict(name="map_prompts", op="map", batch=64, stride=4, held_max=2048, fresh_max=16384, all_fresh=False,
             pad=37),
        # Decode step: the RoPE part behind 128 plain elements of 32 query heads, and the shared key.
        dict(name="rope_step", op="rope", dtype="bf16", tokens=128, heads=32, plain=128, rope=64,
             layout="interleaved", scaling="none", inverse=False, pos_max=32768),
        # A long prompt in the half layout with positions past the trained length.
        dict(name="rope_prompt", op="rope", dtype="bf16", tokens=65536, heads=16, plain=64, rope=64,
             layout="half", scaling="ramp", inverse=False, pos_max=131072),
        # The gradient of the rotation on a training batch, an odd number of rows.
        dict(name="rope_grad", op="rope", dtype="fp32", tokens=4095, heads=8, plain=64, rope=32,
             layout="interleaved", scaling="linear", inverse=True, pos_max=2048),
        # One decode step's newest slots of a large batch.
        dict(name="store_step", op="store", dtype="bf16", rows=128, rank=512, rope=64, stride=1),
        # A prompt's running states, of which every second one closes a slot.
        dict(name="store_prompt", op="store", dtype="bf16", rows=131071, rank=512, rope=64, stride=2),
        # A few short fp32 sequences, one without any slot.
        dict(name="attend_tiny", op="attend", dtype="fp32", batch=3, heads=4, rank=64, rope=32, slots=200,
             spread="empty", head_dim=64),
        # The paper's decoder layer, ragged.
        dict(name="attend_paper", op="attend", dtype="bf16", batch=32, heads=8, rank=256, rope=32, slots=1024,
             spread="ragged", head_dim=64),
        # Long context, 16 heads: 16384 tokens at stride 4.
        dict(name="attend_long", op="attend", dtype="bf16", batch=8, heads=16, rank=512, rope=64, slots=4112,
             spread="even", head_dim=64),
        # A single stream whose one query reads a very long cache.
        dict(name="attend_one", op="attend", dtype="bf16", batch=1, heads=16, rank=512, rope=64, slots=32773,
             spread="even", head_dim=64),
        # The largest decode batch: 16384 slots of each of 128 sequences.
        dict(name="attend_large", op="attend", dtype="bf16", batch=128, heads=32, rank=512, rope=64, slots=16384,
             spread="even", head_dim=128),
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    op = rng.choice(["map", "rope", "store", "attend", "attend"])
    if op == "map":
        batch = _log_int(rng, 1, 1024)
        step = rng.random() < 0.5
        return dict(op="map", batch=batch, stride=rng.randint(1, 5), held_max=_log_int(rng, 1, 65536),
                    fresh_max=1 if step else _log_int(rng, 2, max(2, min(32768, (1 << 20) // batch))),
                    all_fresh=rng.random() < 0.5, pad=rng.choice([0, rng.randint(1, 500)]))
    if op == "rope":
        heads = rng.randint(1, 32)
        plain = rng.choice([0, 32, 64, 128, 8 * rng.randint(1, 20), rng.randint(1, 96)])
        rope = rng.choice([32, 64, 128, 2 * rng.randint(1, 64)])
        most = max(2, (65536 * 16 * 128) // (heads * (plain + rope)))
        return dict(op="rope", dtype=rng.choice(["bf16", "fp32"]), tokens=_log_int(rng, 1, min(65536, most)),
                    heads=heads, plain=plain, rope=rope, layout=rng.choice(["interleaved", "half"]),
                    scaling=rng.choice(["none", "linear", "ramp"]), inverse=rng.random() < 0.4,
                    pos_max=_log_int(rng, 16, 1 << 20))
    if op == "store":
        return dict(op="store", dtype=rng.choice(["bf16", "fp32"]), rows=_log_int(rng, 1, 65536),
                    rank=64 * rng.randint(1, 8), rope=rng.choice([32, 64]), stride=rng.randint(1, 4))
    batch = _log_int(rng, 1, 256)
    return dict(op="attend", dtype=rng.choice(["bf16", "bf16", "fp32"]), batch=batch, heads=rng.randint(1, 32),
                rank=64 * rng.randint(1, 8), rope=rng.choice([32, 64]),
                slots=_log_int(rng, 1, min(65536, (1 << 20) // batch)),
                spread=rng.choice(["even", "ragged", "empty"]), head_dim=rng.choice([64, 128]))


# ------------------------------------------------------------------------------ inputs

def _gen(seed: int):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _slot_counts(case):
    """Slots of every sequence: the case fixes the set, a seed their order."""
    rng = random.Random(11)
    n, b = case["slots"], case["batch"]
    if case["spread"] == "even":
        return [n] * b
    lens = [rng.randint(max(1, n // 2), n) for _ in range(b)]
    if case["spread"] == "empty":
        lens = [rng.choice([0, 1, v, v]) for v in lens]
        lens[-1] = 0
    lens[0] = n
    return lens


def _token_counts(case):
    """Tokens held and new tokens of every request: the case fixes the sets, a seed their order."""
    rng = random.Random(3)
    b = case["batch"]
    held = [rng.randint(0, case["held_max"]) for _ in range(b)]
    fresh = [rng.randint(1, case["fresh_max"]) for _ in range(b)]
    if not case["all_fresh"]:
        fresh = [f if rng.random() < 0.8 else 0 for f in fresh]
    return held, fresh


def _shuffled(values, seed: int):
    values = list(values)
    random.Random(seed).shuffle(values)
    return values


def _latent_rows(n: int, rank: int, rope: int, g):
    """Rows of a merged cache: latents like a two-fold merge of unit normals, unit-normal keys."""
    rows = torch.randn(n, rank + rope, device="cuda", generator=g)
    rows[:, :rank] *= 0.75
    return rows


def _place(n_chunks: int, key_block: bool):
    """place[i][c]: chunk position of chunk c in row i of a page."""
    i, c = torch.arange(PAGE, device="cuda")[:, None], torch.arange(n_chunks, device="cuda")[None, :]
    if key_block:
        return c ^ ((i & 7) if n_chunks == 8 else ((i >> 1) & 3))
    m = min(8, n_chunks & -n_chunks) - 1
    return c ^ (i & m)


def _pages(rows, n_pages: int, rank: int, rope: int):
    """A pool of n_pages pages from n_pages * 64 rows."""
    size = 34 * rank + 128 * rope
    pages = torch.empty(n_pages, size, dtype=torch.uint8, device="cuda")
    step = 256
    for p0 in range(0, n_pages, step):
        p1 = min(n_pages, p0 + step)
        scale, codes = _encode(rows(p0 * PAGE, p1 * PAGE)[:, :rank])
        keys = rows(p0 * PAGE, p1 * PAGE)[:, rank:].bfloat16()
        n = p1 - p0
        byte = (codes[:, 0::2] | (codes[:, 1::2] << 4)).to(torch.uint8).view(n, PAGE, rank // 32, 16)
        at = _place(rank // 32, False)[None, :, :, None].expand(n, PAGE, rank // 32, 16)
        pages[p0:p1, :32 * rank] = torch.empty_like(byte).scatter_(2, at, byte).view(n, -1)
        pages[p0:p1, 32 * rank:34 * rank] = (scale.half().view(torch.int16) >> 7).to(torch.uint8).view(n, -1)
        kb = keys.contiguous().view(torch.uint8).view(n, PAGE, rope // 8, 16)
        at = _place(rope // 8, True)[None, :, :, None].expand(n, PAGE, rope // 8, 16)
        pages[p0:p1, 34 * rank:] = torch.empty_like(kb).scatter_(2, at, kb).view(n, -1)
    return pages


def prepare(case, seed: int):
    g = _gen(seed)
    op = case["op"]
    if op == "map":
        b, s = case["batch"], case["stride"]
        held, fresh = _token_counts(case)
        held, fresh = _shuffled(held, 2 * seed), _shuffled(fresh, 2 * seed + 1)
        after = [-(-(h + f) // s) for h, f in zip(held, fresh)]
        width = -(-(-(-(case["held_max"] + case["fresh_max"]) // s)) // PAGE)
        have = [-(-(-(-h // s)) // PAGE) for h in held]
        need = sum(-(-a // PAGE) - h for a, h in zip(after, have))
        total = sum(have) + need + 16
        ids = torch.randperm(total, device="cuda", generator=g).int()
        at = sum(have)
        col = torch.arange(width, device="cuda")[None, :]
        first = torch.tensor([sum(have[:i]) for i in range(b)], device="cuda")[:, None]
        table = torch.where(col < torch.tensor(have, device="cuda")[:, None],
                            ids[(first + col).clamp(max=total - 1)], torch.full_like(ids[:1], -1))
        n = sum(fresh) + case["pad"]
        i32 = dict(dtype=torch.int32, device="cuda")
        buf = dict(starts=torch.empty(b + 1, **i32), seq=torch.empty(n, **i32), position=torch.empty(n, **i32),
                   slot=torch.empty(n, dtype=torch.int64, device="cuda"),
                   store=torch.empty(n, dtype=torch.int64, device="cuda"), slots=torch.empty(b, **i32),
                   taken=torch.empty(1, **i32))
        return dict(case=case, held=torch.tensor(held, **i32), fresh=torch.tensor(fresh, **i32),
                    free=ids[at:].contiguous(), table=table.contiguous(), n=n, buf=buf)
    if op == "rope":
        t, h, d = case["tokens"], case["heads"], case["plain"] + case["rope"]
        dt = DTYPES[case["dtype"]]
        q = torch.randn(t, h, d, device="cuda", generator=g).to(dt)
        k = torch.randn(t, 1, case["rope"], device="cuda", generator=g).to(dt)
        pos = torch.randint(0, case["pos_max"], (t,), device="cuda", generator=g).int()
        return dict(case=case, q=q, k=k, pos=pos, out=[torch.empty_like(q), torch.empty_like(k)])
    if op == "store":
        n, r, dr, s = case["rows"], case["rank"], case["rope"], case["stride"]
        rows = _latent_rows(n, r, dr, g).to(DTYPES[case["dtype"]])
        kept = n // s
        n_pages = -(-max(kept, 1) // PAGE) + 3
        order = torch.randperm(n_pages, device="cuda", generator=g)
        j = torch.arange(max(kept, 1), device="cuda")
        place = order[j // PAGE] * PAGE + j % PAGE
        index = torch.full((n,), -1, dtype=torch.int64, device="cuda")
        index[s - 1::s] = place[:kept]
        return dict(case=case, rows=rows, index=index, out=torch.empty_like(rows),
                    pages=torch.zeros(n_pages, 34 * r + 128 * dr, dtype=torch.uint8, device="cuda"),
                    n_pages=n_pages)
    r, dr, b = case["rank"], case["rope"], case["batch"]
    lens = _shuffled(_slot_counts(case), seed)
    held = [-(-v // PAGE) for v in lens]
    n_pages = sum(held) + 2
    order = torch.randperm(n_pages, device="cuda", generator=g).int()
    width = max(1, max(held))
    first = torch.tensor([sum(held[:i]) for i in range(b)], device="cuda")[:, None]
    col = torch.arange(width, device="cuda")[None, :]
    table = torch.where(col < torch.tensor(held, device="cuda")[:, None],
                        order[(first + col).clamp(max=n_pages - 1)], torch.full_like(col, -1, dtype=torch.int32))
    cache = {}

    def rows(lo, hi):
        if cache.get("at") != (lo, hi):
            cache.update(at=(lo, hi), rows=_latent_rows(hi - lo, r, dr, g))
        return cache["rows"]

    pages = _pages(rows, n_pages, r, dr)
    q = torch.randn(b, case["heads"], r + dr, device="cuda", generator=g).to(DTYPES[case["dtype"]])
    state = dict(case=case, pages=pages, n_pages=n_pages, table=table.int().contiguous(), lens=lens,
                 slots=torch.tensor(lens, dtype=torch.int32, device="cuda"), q=q,
                 scale=1.0 / math.sqrt(case["head_dim"]),
                 out=torch.empty(b, case["heads"], r, dtype=q.dtype, device="cuda"),
                 lse=torch.empty(b, case["heads"], dtype=torch.float32, device="cuda"))
    if own:
        from paper_2505_13544_b200 import binding as M
        cfg = M.make_qpool_config(n_heads=case["heads"], latent_rank=r, rope_dim=dr, n_pages=n_pages)
        # The workspace that a serving loop keeps for its batch.
        state["workspace"] = torch.empty(M.mtla_qpool_workspace_bytes(cfg, b), dtype=torch.uint8, device="cuda")
    return state


# ------------------------------------------------------------------------------ the plain forms

def _encode(x):
    """Scales [n][r/32] and codes [n][r] of latent rows, by comparisons with the code borders."""
    n, r = x.shape
    x = x.float().view(n, r // GROUP, GROUP)
    a = x.abs()
    top = a.amax(-1).double() / 6
    finite = torch.isfinite(top)
    _, e = torch.frexp(torch.where(finite, top, torch.zeros_like(top)))
    quantum = torch.ldexp(torch.ones_like(top), e.clamp(min=-13) - 4)
    scale = (torch.ceil(top / quantum) * quantum).clamp(max=SCALE_MAX)
    scale = torch.where(finite, scale, torch.full_like(scale, math.nan)).float()
    s = scale[..., None]
    code = ((a > 0.25 * s).int() + (a >= 0.75 * s).int() + (a > 1.25 * s).int() + (a >= 1.75 * s).int()
            + (a > 2.5 * s).int() + (a >= 3.5 * s).int() + (a > 5 * s).int())
    code = torch.where(s > 0, code, torch.zeros_like(code)) | ((x < 0).int() << 3)
    return scale, code.view(n, r)


def _e2m1(code):
    """The value of a 4-bit code: magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6."""
    m = (code & 7).float()
    mag = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2, 2 * m - 8))
    return torch.where(code & 8 > 0, -mag, mag)


def _page_rows(pages, rank: int, rope: int):
    """Latents [n][64][r] and keys [n][64][d_R] of pages, 32-bit."""
    n = pages.shape[0]
    at = _place(rank // 32, False)[None, :, :, None].expand(n, PAGE, rank // 32, 16)
    byte = pages[:, :32 * rank].view(n, PAGE, rank // 32, 16).gather(2, at).int()
    code = torch.stack([byte & 15, byte >> 4], -1).view(n, PAGE, rank // 32, 32)
    scale = (pages[:, 32 * rank:34 * rank].to(torch.int16) << 7).view(torch.float16).float()
    latent = _e2m1(code) * scale.view(n, PAGE, rank // 32, 1)
    at = _place(rope // 8, True)[None, :, :, None].expand(n, PAGE, rope // 8, 16)
    keys = pages[:, 34 * rank:].view(n, PAGE, rope // 8, 16).gather(2, at).contiguous().view(n, PAGE, rope * 2)
    return latent.view(n, PAGE, rank), keys.contiguous().view(torch.bfloat16).float()


def _plain_map(st):
    s = st["case"]["stride"]
    held, fresh, table, n = st["held"], st["fresh"], st["table"], st["n"]
    b, width = table.shape
    cut = lambda v, d: torch.div(v + d - 1, d, rounding_mode="floor")
    have = cut(cut(held, s), PAGE)
    slots = cut(held + fresh, s)
    need = cut(slots, PAGE) - have
    before = torch.cumsum(need, 0) - need
    col = torch.arange(width, device="cuda")[None, :]
    pick = before[:, None] + col - have[:, None]
    grown = torch.where((col >= have[:, None]) & (col < (have + need)[:, None]),
                        st["free"][pick.clamp(0, max(st["free"].numel() - 1, 0))] if st["free"].numel() else table,
                        table)
    starts = torch.zeros(b + 1, dtype=torch.int64, device="cuda")
    starts[1:] = torch.cumsum(fresh, 0)
    t = torch.arange(n, device="cuda")
    seq = torch.searchsorted(starts[1:], t, right=True)
    real = seq < b
    i = seq.clamp(max=b - 1)
    pos = held[i] + (t - starts[i])
    j = torch.div(pos, s, rounding_mode="floor")
    page = grown[i, torch.div(j, PAGE, rounding_mode="floor").clamp(max=width - 1)].long()
    slot = torch.where(real, page * PAGE + j % PAGE, torch.full_like(t, -1))
    last = ((pos + 1) % s == 0) | (t + 1 == starts[i + 1])
    return dict(table=grown, starts=starts.int(), seq=torch.where(real, seq, -torch.ones_like(seq)).int(),
                position=torch.where(real, pos, torch.zeros_like(pos)).int(), slot=slot,
                store=torch.where(last, slot, torch.full_like(t, -1)), slots=slots.int(),
                taken=need.sum().int().view(1))


ROPE = dict(theta=10000.0, factor=4.0, ramp_low=1.0, ramp_high=32.0, train_tokens=4096, magnitude=1.125)


def _frequencies(case):
    """Angle per position of every pair, 64-bit, after the scaling for long contexts."""
    d = case["rope"]
    f = ROPE["theta"] ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    if case["scaling"] == "linear":
        return f / ROPE["factor"]
    if case["scaling"] == "ramp":
        turns = ROPE["train_tokens"] * f / (2 * math.pi)
        keep = ((turns - ROPE["ramp_low"]) / (ROPE["ramp_high"] - ROPE["ramp_low"])).clamp(0, 1)
        return f * keep + f / ROPE["factor"] * (1 - keep)
    return f


def _plain_rope(st):
    case = st["case"]
    d = case["rope"]
    ang = st["pos"].double()[:, None] * _frequencies(case)          # far positions lose their angle in 32 bits
    mag = ROPE["magnitude"] if case["scaling"] == "ramp" else 1.0
    cos, sin = (torch.cos(ang) * mag).float()[:, None], (torch.sin(ang) * mag).float()[:, None]
    if case["inverse"]:
        sin = -sin
    outs = []
    for x, first in ((st["q"], case["plain"]), (st["k"], 0)):
        v = x[..., first:].float()
        y = torch.empty_like(v)
        if case["layout"] == "half":
            a, b = v[..., :d // 2], v[..., d // 2:]
            y[..., :d // 2], y[..., d // 2:] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = v[..., 0::2], v[..., 1::2]
            y[..., 0::2], y[..., 1::2] = a * cos - b * sin, b * cos + a * sin
        outs.append(torch.cat([x[..., :first], y.to(x.dtype)], -1))
    return outs


def _plain_store(st):
    case = st["case"]
    r = case["rank"]
    scale, code = _encode(st["rows"][:, :r])
    latent = (_e2m1(code).view(-1, r // GROUP, GROUP) * scale[..., None]).view(-1, r)
    row = torch.cat([latent, st["rows"][:, r:].bfloat16().float()], 1)
    return torch.where((st["index"] >= 0)[:, None], row, torch.zeros_like(row)).to(st["rows"].dtype)


def _plain_attend(st):
    case = st["case"]
    r = case["rank"]
    out, lse = torch.zeros_like(st["out"]), torch.full_like(st["lse"], -math.inf)
    for b, n in enumerate(st["lens"]):
        if n == 0:
            continue
        pages = st["pages"][st["table"][b, :-(-n // PAGE)].long()]
        latent, keys = _page_rows(pages, r, case["rope"])
        latent, keys = latent.reshape(-1, r)[:n], keys.reshape(-1, case["rope"])[:n]
        q = st["q"][b].float()
        score = (q[:, :r] @ latent.T + q[:, r:] @ keys.T) * st["scale"]
        top = score.amax(-1, keepdim=True)
        p = torch.exp(score - top)
        total = p.sum(-1, keepdim=True)
        out[b] = ((p @ latent) / total).to(out.dtype)
        lse[b] = (top + torch.log(total))[:, 0]
    return [out, lse]


# ------------------------------------------------------------------------------ a pass

def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        return dict(map=_plain_map, rope=_plain_rope, store=_plain_store, attend=_plain_attend)[op](state)
    from paper_2505_13544_b200 import binding as M
    if op == "map":
        m = M.mtla_slot_map(state["held"], state["fresh"], state["free"], state["table"], stride=case["stride"],
                            out=M.SlotMap(**state["buf"]))
        return dict(table=state["table"], starts=m.starts, seq=m.seq, position=m.position, slot=m.slot,
                    store=m.store, slots=m.slots, taken=m.taken)
    if op == "rope":
        scaled = case["scaling"] != "none"
        ramp = case["scaling"] == "ramp"
        cfg = M.make_rope_config(rope_dim=case["rope"], layout=case["layout"], theta=ROPE["theta"],
                                 scaling=case["scaling"], factor=ROPE["factor"] if scaled else 1.0,
                                 ramp_low=ROPE["ramp_low"], ramp_high=ROPE["ramp_high"],
                                 train_tokens=ROPE["train_tokens"], magnitude=ROPE["magnitude"] if ramp else 1.0)
        return M.mtla_rope(cfg, [state["q"], state["k"]], state["pos"], first=[case["plain"], 0],
                           out=state["out"], inverse=case["inverse"])
    if op == "store":
        cfg = M.make_qpool_config(n_heads=1, latent_rank=case["rank"], rope_dim=case["rope"],
                                  n_pages=state["n_pages"])
        M.mtla_qpool_write(cfg, state["pages"], state["rows"], state["index"])
        return M.mtla_qpool_read(cfg, state["pages"], state["index"], out=state["out"])
    cfg = M.make_qpool_config(n_heads=case["heads"], latent_rank=case["rank"], rope_dim=case["rope"],
                              n_pages=state["n_pages"])
    return list(M.mtla_qpool_attend(cfg, state["pages"], state["table"], state["slots"], state["q"],
                                    scale=state["scale"], out=state["out"], lse=state["lse"],
                                    workspace=state["workspace"]))


def work(case):
    op = case["op"]
    if op == "map":
        n = sum(_token_counts(case)[1]) + case["pad"]
        # Lengths in, two 32-bit and two 64-bit entries per token out, the new table entries.
        return dict(bytes=16 * case["batch"] + 24 * n + 8 * (n // (PAGE * case["stride"]) + 1), flops=8 * n)
    size = 2 if case.get("dtype") == "bf16" else 4
    if op == "rope":
        n = case["tokens"] * (case["heads"] * (case["plain"] + case["rope"]) + case["rope"])
        return dict(bytes=2 * size * n + 4 * case["tokens"],
                    flops=3 * case["tokens"] * (case["heads"] + 1) * case["rope"])
    r, dr = case["rank"], case["rope"]
    row = r // 2 + r // 32 + 2 * dr
    if op == "store":
        kept = case["rows"] // case["stride"]
        # Kept rows in and out, their 4-bit rows written and read, zeros for the rest.
        return dict(bytes=kept * ((r + dr) * size + 2 * row) + case["rows"] * ((r + dr) * size + 8),
                    flops=12 * kept * r)
    n = sum(_slot_counts(case))
    return dict(bytes=n * row + case["batch"] * case["heads"] * ((2 * r + dr) * size + 4),
                flops=n * case["heads"] * (4 * r + 2 * dr))


# ------------------------------------------------------------------------------ 64-bit answers

def exact(case, seed: int):
    st = prepare(case, seed)
    op = case["op"]
    if op == "map":
        s, n = case["stride"], st["n"]
        held, fresh = st["held"].tolist(), st["fresh"].tolist()
        table, free = st["table"].cpu(), st["free"].tolist()
        if n > 200000:
            return None
        starts, seq, position, slot, store, slots, taken = [0], [], [], [], [], [], 0
        for b, (h, f) in enumerate(zip(held, fresh)):
            have = -(-(-(-h // s)) // PAGE)
            slots.append(-(-(h + f) // s))
            for p in range(have, -(-slots[-1] // PAGE)):
                table[b, p] = free[taken]
                taken += 1
            row = table[b].tolist()
            for i in range(h, h + f):
                seq.append(b)
                position.append(i)
                slot.append(row[i // s // PAGE] * PAGE + i // s % PAGE)
                store.append(slot[-1] if (i % s == s - 1 or i == h + f - 1) else -1)
            starts.append(len(seq))
        pad = n - len(seq)
        i32, i64 = torch.int32, torch.int64
        return dict(table=table, starts=torch.tensor(starts, dtype=i32),
                    seq=torch.tensor(seq + [-1] * pad, dtype=i32),
                    position=torch.tensor(position + [0] * pad, dtype=i32),
                    slot=torch.tensor(slot + [-1] * pad, dtype=i64),
                    store=torch.tensor(store + [-1] * pad, dtype=i64), slots=torch.tensor(slots, dtype=i32),
                    taken=torch.tensor([taken], dtype=i32))
    if op == "rope":
        d = case["rope"]
        freq = []
        for k in range(d // 2):
            f = math.exp(-2.0 * k / d * math.log(ROPE["theta"]))
            if case["scaling"] == "linear":
                f = f / ROPE["factor"]
            elif case["scaling"] == "ramp":
                turns = f * ROPE["train_tokens"] / math.tau
                keep = min(1.0, max(0.0, (turns - ROPE["ramp_low"]) / (ROPE["ramp_high"] - ROPE["ramp_low"])))
                f = f / ROPE["factor"] + keep * (f - f / ROPE["factor"])
            freq.append(f)
        turn = torch.polar(torch.full((case["tokens"], d // 2), ROPE["magnitude"] if case["scaling"] == "ramp" else 1.0,
                                      dtype=torch.float64, device="cuda"),
                           torch.outer(st["pos"].double(), torch.tensor(freq, dtype=torch.float64, device="cuda")))
        if case["inverse"]:
            turn = turn.conj()
        outs = []
        for x, first in ((st["q"], case["plain"]), (st["k"], 0)):
            out = x.double()
            v = out[..., first:]
            half = case["layout"] == "half"
            pair = v.unflatten(-1, (2, d // 2)).transpose(-1, -2) if half else v.unflatten(-1, (d // 2, 2))
            y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[:, None])
            out[..., first:] = (y.transpose(-1, -2) if half else y).flatten(-2)
            outs.append(out)
        return outs
    r, dr = case["rank"], case["rope"]
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64,
                         device="cuda")
    if op == "store":
        # The grid of all scales, and the nearest code (an even one on a tie) by its distance.
        grid = (torch.arange(227, device="cuda", dtype=torch.int16) << 7).view(torch.float16).double()
        out = torch.zeros(case["rows"], r + dr, dtype=torch.float64, device="cuda")
        for i in range(0, case["rows"], 8192):
            x = st["rows"][i:i + 8192].double()
            lat = x[:, :r].view(-1, r // GROUP, GROUP)
            at = torch.searchsorted(6 * grid, lat.abs().amax(-1)).clamp(max=226)
            s = grid[at][..., None]
            best = torch.zeros_like(lat)
            gap = lat.abs()
            for m in (2, 4, 6, 1, 3, 5, 7):                     # even codes first: an odd one has to be nearer
                far = (lat.abs() - value[m] * s).abs()
                better = far < gap
                best, gap = torch.where(better, value[m] * s, best), torch.where(better, far, gap)
            row = torch.cat([(best * lat.sign()).view(-1, r), x[:, r:].bfloat16().double()], 1)
            out[i:i + 8192] = torch.where((st["index"][i:i + 8192] >= 0)[:, None], row, torch.zeros_like(row))
        return out
    out = torch.zeros(case["batch"], case["heads"], r, dtype=torch.float64, device="cuda")
    lse = torch.full((case["batch"], case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    chunk = r // 32
    mask = (chunk & -chunk if (chunk & -chunk) < 8 else 8) - 1
    for b, n in enumerate(st["lens"]):
        if n == 0:
            continue
        page = st["pages"].index_select(0, st["table"][b, :-(-n // PAGE)])
        row = torch.arange(n, device="cuda")
        p, i = row // PAGE, row % PAGE
        col = torch.arange(r, device="cuda")
        at = i[:, None] * (r // 2) + (((col // 32)[None] ^ (i & mask)[:, None]) * 16 + (col % 32 // 2)[None])
        nib = (page[p[:, None], at] >> (4 * (col % 2)).to(torch.uint8)) & 15
        bits = page[p[:, None], 32 * r + i[:, None] * chunk + (col // 32)[None]].short() * 128
        latent = value[nib.long()] * bits.view(torch.float16).double()
        col = torch.arange(dr, device="cuda")
        twist = (i & 7) if dr == 64 else (i // 2 & 3)
        at = 34 * r + i[:, None] * 2 * dr + ((col // 8)[None] ^ twist[:, None]) * 16 + (col % 8 * 2)[None]
        low, high = page[p[:, None], at].int(), page[p[:, None], at + 1].int()
        key = ((low << 16) | (high << 24)).view(torch.float32).double()
        q = st["q"][b].double()
        score = (torch.cat([latent, key], 1) @ q.T) * st["scale"]
        lse[b] = torch.logsumexp(score, 0)
        out[b] = torch.softmax(score, 0).T @ latent
    return [out, lse]

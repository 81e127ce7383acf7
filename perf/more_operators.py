"""Operators of a verification step over drafted trees: plain forms, inputs and 64-bit answers.

A serving loop that lets a small model draft a tree of tokens for every request verifies all of its nodes in
one step.  Next to the 4-bit latent pool it then runs

  tree     positions of the nodes, and what each of them sees        (mtla_tree_map)
  attend   every node's query over its request's 4-bit slots and the drafted rows it sees
                                                                     (mtla_qpool_attend_tree)
  w4       products of the step's few rows with 4-bit weights        (mtla_qweight_product)

Trees: node i of a request has a parent among the nodes before it, or -1: it follows the last token held.
With `held` tokens it stands at position held + depth.  With stride s a node's row is the running state of its
chunk, so it sees the closed slots of the context, held // s of them (an open one is continued by every path),
those of its ancestors that close a chunk, and itself: bit j of its mask is node j of the request.

Pool pages: [64][r/2] bytes of 4-bit codes (e2m1: sign, two exponent bits, one fraction bit; latent 2k in the
low half of byte k), [64][r/32] bytes of group scales (the upper bits of a positive half-precision number: 5
exponent bits, 3 fraction bits), [64][d_R] bf16 RoPE keys.  The 16-byte chunk c of row i sits at chunk position
c ^ (i & m) of its row: in the code block m + 1 is the largest power of two, 8 at most, that divides the number of
chunks; in the key block the place is c ^ (i & 7) for d_R = 64 and c ^ ((i >> 1) & 3) for d_R = 32.

4-bit weights [in][out]: the same codes and scales, a scale per 32 inputs of one output.  Blocks of 16 outputs by
128 inputs, the blocks of 16 outputs one after the other, both sizes filled up with zeros; a block is 1024 bytes
of codes, output i at 64 i, its four groups of 32 inputs at 16-byte chunk c ^ ((i >> 1) & 3), and then 64 scales,
that of output i and group c at 2 (4 (i & 7) + c) + (i >> 3).  A 32-bit word holds eight codes, inputs 2k in its lower
and 2k + 1 in its upper half: signs at bits 15, 12, 14, 13 of the half for k = 0 .. 3, magnitudes at 6, 3, 0, 9.
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
SIGN_AT, MAG_AT = (15, 12, 14, 13), (6, 3, 0, 9)


# ------------------------------------------------------------------------------ cases

def listed():
    return [
        # A step of a few requests with small trees.
        dict(name="tree_step", op="tree", batch=16, nodes=16, stride=2, shape="wide", spread="even", held_max=32768,
             pad=0),
        # A large ragged batch in buffers that are longer than its nodes.
        dict(name="tree_batch", op="tree", batch=1024, nodes=64, stride=3, shape="wide", spread="empty",
             held_max=65536, pad=301),
        # A few short fp32 requests, one without any slot, one without nodes.
        dict(name="attend_tiny", op="attend", dtype="fp32", batch=3, heads=4, rank=64, rope=32, slots=200, nodes=5,
             stride=2, shape="chain", spread="empty", head_dim=64),
        # The paper's decoder layer, ragged contexts, small trees.
        dict(name="attend_paper", op="attend", dtype="bf16", batch=32, heads=8, rank=256, rope=32, slots=1024,
             nodes=12, stride=2, shape="wide", spread="ragged", head_dim=64),
        # One request whose drafted chain reads a very long cache.
        dict(name="attend_one", op="attend", dtype="bf16", batch=1, heads=16, rank=512, rope=64, slots=32773, nodes=7,
             stride=1, shape="chain", spread="even", head_dim=64),
        # Long context, 16 heads, bushy trees.
        dict(name="attend_long", op="attend", dtype="bf16", batch=8, heads=16, rank=512, rope=64, slots=4112, nodes=26,
             stride=4, shape="wide", spread="ragged", head_dim=64),
        # fp32, an odd number of heads and a rank that is no multiple of 128.
        dict(name="attend_fp32", op="attend", dtype="fp32", batch=4, heads=5, rank=192, rope=64, slots=1500, nodes=9,
             stride=2, shape="wide", spread="ragged", head_dim=128),
        # The largest step: full trees of 64 nodes, 32 heads.
        dict(name="attend_large", op="attend", dtype="bf16", batch=8, heads=32, rank=512, rope=64, slots=4096,
             nodes=64, stride=2, shape="wide", spread="even", head_dim=128),
        # One token through the output projection of a layer of 32 heads of 128 and width 4096.
        dict(name="w4_token", op="w4", dtype="bf16", rows=1, n_in=4096, n_out=4096),
        # A few fp32 rows, an odd number of outputs, inputs that do not fill their last block.
        dict(name="w4_fp32", op="w4", dtype="fp32", rows=7, n_in=1000, n_out=777),
        # A step's rows through the paper's second feed-forward product.
        dict(name="w4_paper", op="w4", dtype="bf16", rows=24, n_in=2048, n_out=512),
        # 512 rows (8 trees of 64) through the fused input projection of a width-4096 layer of 32 heads.
        dict(name="w4_tree", op="w4", dtype="bf16", rows=512, n_in=4096, n_out=6720),
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    op = rng.choice(["tree", "attend", "attend", "w4", "w4"])
    spread = rng.choice(["even", "ragged", "empty"])
    shape = rng.choice(["chain", "wide", "wide"])
    if op == "tree":
        return dict(op="tree", batch=_log_int(rng, 1, 1024), nodes=_log_int(rng, 1, 64), stride=rng.randint(1, 5),
                    shape=shape, spread=spread, held_max=_log_int(rng, 1, 1 << 20),
                    pad=rng.choice([0, rng.randint(1, 500)]))
    if op == "w4":
        n_in, n_out = 8 * _log_int(rng, 4, 1024), _log_int(rng, 1, 8192)
        rows = _log_int(rng, 1, max(1, min(512, (512 * 4096 * 6720) // (n_in * n_out))))
        return dict(op="w4", dtype=rng.choice(["bf16", "bf16", "fp32"]), rows=rows, n_in=n_in, n_out=n_out)
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    heads, nodes, batch = rng.randint(1, 32), _log_int(rng, 1, 64), _log_int(rng, 1, 64)
    pairs = 1 << (26 if dtype == "bf16" else 23)              # columns (nodes x heads) times slots
    batch = max(1, min(batch, pairs // (heads * nodes * 16)))
    return dict(op="attend", dtype=dtype, batch=batch, heads=heads, rank=64 * rng.randint(1, 8),
                rope=rng.choice([32, 64]), slots=_log_int(rng, 1, min(32768, pairs // (heads * nodes * batch))),
                nodes=nodes, stride=rng.randint(1, 4), shape=shape, spread=spread, head_dim=rng.choice([64, 128]))


# ------------------------------------------------------------------------------ inputs

def _gen(seed: int):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _spread(n: int, count: int, kind: str, salt: int):
    """`count` numbers up to n: all n, between half of it and n, or some of them 0 and 1; the case fixes the set."""
    rng = random.Random(salt)
    if kind == "even":
        return [n] * count
    out = [rng.randint(max(1, n // 2), n) for _ in range(count)]
    if kind == "empty":
        out = [rng.choice([0, 1, v, v]) for v in out]
        out[-1] = 0
    out[0] = n
    return out


def _node_counts(case):
    return _spread(case["nodes"], case["batch"], case["spread"], 5)


def _slot_counts(case):
    return _spread(case["slots"], case["batch"], case["spread"], 11)


def _parents(count: int, shape: str, rng: random.Random):
    """A chain, or a tree whose nodes follow one of the few nodes before them."""
    if shape == "chain":
        return [i - 1 for i in range(count)]
    return [rng.randint(max(-1, i - 6), i - 1) for i in range(count)]


def _shuffled(values, seed: int):
    values = list(values)
    random.Random(seed).shuffle(values)
    return values


def _sees(parents, held: int, stride: int):
    """Masks of one request's nodes."""
    depth, masks, closing = [], [], []
    for i, p in enumerate(parents):
        depth.append(0 if p < 0 else depth[p] + 1)
        above = 0 if p < 0 else closing[p]
        masks.append(above | (1 << i))
        closing.append(above | ((1 << i) if (held + depth[i] + 1) % stride == 0 else 0))
    return depth, masks


def _signed(mask: int) -> int:
    return mask - (1 << 64) if mask >> 63 else mask


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


def _pages(n_pages: int, rank: int, rope: int, g):
    """A pool of filled pages."""
    pages = torch.empty(n_pages, 34 * rank + 128 * rope, dtype=torch.uint8, device="cuda")
    for p0 in range(0, n_pages, 256):
        n = min(n_pages, p0 + 256) - p0
        rows = _latent_rows(n * PAGE, rank, rope, g)
        scale, codes = _encode(rows[:, :rank])
        byte = (codes[:, 0::2] | (codes[:, 1::2] << 4)).to(torch.uint8).view(n, PAGE, rank // 32, 16)
        at = _place(rank // 32, False)[None, :, :, None].expand(n, PAGE, rank // 32, 16)
        pages[p0:p0 + n, :32 * rank] = torch.empty_like(byte).scatter_(2, at, byte).view(n, -1)
        pages[p0:p0 + n, 32 * rank:34 * rank] = (scale.half().view(torch.int16) >> 7).to(torch.uint8).view(n, -1)
        kb = rows[:, rank:].bfloat16().contiguous().view(torch.uint8).view(n, PAGE, rope // 8, 16)
        at = _place(rope // 8, True)[None, :, :, None].expand(n, PAGE, rope // 8, 16)
        pages[p0:p0 + n, 34 * rank:] = torch.empty_like(kb).scatter_(2, at, kb).view(n, -1)
    return pages


def _block_places():
    """place[i][c]: chunk position of group c of output i in a weight block."""
    i, c = torch.arange(16, device="cuda")[:, None], torch.arange(4, device="cuda")[None, :]
    return c ^ ((i >> 1) & 3)


def _pack_weights(scale, code):
    """Packed bytes from scales [out][in / 32] and codes [out][in] (sizes filled up already)."""
    rb, kb = code.shape[0] // 16, code.shape[1] // 128
    c = code.view(rb, 16, kb, 4, 4, 4, 2).int()                       # ..., group, word, pair, half
    sign = torch.tensor(SIGN_AT, device="cuda")[:, None]
    mag = torch.tensor(MAG_AT, device="cuda")[:, None]
    half = (((c >> 3) << sign) | ((c & 7) << mag)).sum(-2)            # ..., group, word, half
    byte = torch.stack([half & 255, half >> 8], -1).to(torch.uint8).reshape(rb, 16, kb, 4, 16)
    byte = byte.transpose(1, 2).contiguous()
    at = _block_places()[None, None, :, :, None].expand(rb, kb, 16, 4, 16)
    out = torch.empty(rb, kb, 1088, dtype=torch.uint8, device="cuda")
    out[..., :1024] = torch.empty_like(byte).scatter_(3, at, byte).view(rb, kb, 1024)
    sb = (scale.half().view(torch.int16) >> 7).to(torch.uint8).view(rb, 2, 8, kb, 4)
    out[..., 1024:] = sb.permute(0, 3, 2, 4, 1).reshape(rb, kb, 64)
    return out.view(-1)


def _fill_up(n: int, to: int) -> int:
    return -(-n // to) * to


def prepare(case, seed: int):
    g = _gen(seed)
    op = case["op"]
    if op == "w4":
        k, o = case["n_in"], case["n_out"]
        kp, opad = _fill_up(k, 128), _fill_up(o, 16)
        w = torch.zeros(opad, kp, device="cuda")
        w[:o, :k] = torch.randn(o, k, device="cuda", generator=g) / math.sqrt(k)
        scale, code = _encode(w)
        x = torch.randn(case["rows"], k, device="cuda", generator=g).to(DTYPES[case["dtype"]])
        return dict(case=case, packed=_pack_weights(scale, code), x=x,
                    y=torch.empty(case["rows"], o, dtype=x.dtype, device="cuda"))
    counts = _shuffled(_node_counts(case), 2 * seed)
    rng = random.Random(seed)
    b = case["batch"]
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    parents = [_parents(c, case["shape"], rng) for c in counts]
    i32 = dict(dtype=torch.int32, device="cuda")
    if op == "tree":
        n = starts[-1] + case["pad"]
        held = [rng.randint(0, case["held_max"]) for _ in range(b)]
        flat = [p for row in parents for p in row] + [0] * case["pad"]
        buf = dict(seq=torch.empty(n, **i32), position=torch.empty(n, **i32),
                   seen=torch.empty(n, dtype=torch.int64, device="cuda"), slots=torch.empty(b, **i32))
        return dict(case=case, held=torch.tensor(held, **i32), starts=torch.tensor(starts, **i32),
                    parents=torch.tensor(flat, **i32), n=n, buf=buf)
    r, dr, n = case["rank"], case["rope"], starts[-1]
    lens = _shuffled(_slot_counts(case), seed)
    pages_of = [-(-v // PAGE) for v in lens]
    n_pages = sum(pages_of) + 2
    order = torch.randperm(n_pages, device="cuda", generator=g).int()
    first = torch.tensor([sum(pages_of[:i]) for i in range(b)], device="cuda")[:, None]
    col = torch.arange(max(1, max(pages_of)), device="cuda")[None, :]
    table = torch.where(col < torch.tensor(pages_of, device="cuda")[:, None],
                        order[(first + col).clamp(max=n_pages - 1)], torch.full_like(col, -1, dtype=torch.int32))
    dt = DTYPES[case["dtype"]]
    seen = [_signed(m) for v, p in zip(lens, parents)
            for m in _sees(p, v * case["stride"] + rng.randrange(case["stride"]), case["stride"])[1]]
    state = dict(case=case, pages=_pages(n_pages, r, dr, g), n_pages=n_pages, table=table.int().contiguous(),
                 lens=lens, counts=counts, slots=torch.tensor(lens, **i32), starts=torch.tensor(starts, **i32),
                 rows=_latent_rows(n, r, dr, g).to(dt), seen=torch.tensor(seen, dtype=torch.int64, device="cuda"),
                 q=torch.randn(n, case["heads"], r + dr, device="cuda", generator=g).to(dt),
                 scale=1.0 / math.sqrt(case["head_dim"]),
                 out=torch.empty(n, case["heads"], r, dtype=dt, device="cuda"),
                 lse=torch.empty(n, case["heads"], dtype=torch.float32, device="cuda"))
    if own:
        from paper_2505_13544_b200 import binding as M
        cfg = M.make_qpool_config(n_heads=case["heads"], latent_rank=r, rope_dim=dr, n_pages=n_pages)
        # The workspace that a serving loop keeps for its batch.
        state["workspace"] = torch.empty(M.mtla_qpool_tree_workspace_bytes(cfg, b, n), dtype=torch.uint8,
                                         device="cuda")
    return state


# ------------------------------------------------------------------------------ the plain forms

def _encode(x):
    """Scales [n][r/32] and codes [n][r] of rows, by comparisons with the code borders."""
    n, r = x.shape
    x = x.float().view(n, r // GROUP, GROUP)
    a = x.abs()
    top = a.amax(-1).double() / 6
    _, e = torch.frexp(top)
    quantum = torch.ldexp(torch.ones_like(top), e.clamp(min=-13) - 4)
    scale = (torch.ceil(top / quantum) * quantum).clamp(max=SCALE_MAX).float()
    s = scale[..., None]
    code = (a > 0.25 * s).to(torch.uint8)
    for border in (0.75, 1.75, 3.5):
        code += a >= border * s
    for border in (1.25, 2.5, 5.0):
        code += a > border * s
    code = torch.where(s > 0, code, torch.zeros_like(code)) | ((x < 0).to(torch.uint8) << 3)
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


def _plain_tree(st):
    s, n, b = st["case"]["stride"], st["n"], st["case"]["batch"]
    t = torch.arange(n, device="cuda")
    seq = torch.searchsorted(st["starts"][1:].contiguous(), t, right=True)
    real = seq < b
    i = seq.clamp(max=b - 1)
    first, held = st["starts"][i].long(), st["held"][i]
    parent = torch.where(real & (st["parents"] >= 0), first + st["parents"], torch.full_like(t, -1))
    depth, up = torch.zeros_like(held), parent
    for _ in range(st["case"]["nodes"] - 1):                # depths first: a mask asks for ancestors' positions
        depth += (up >= 0).int()
        up = torch.where(up >= 0, parent[up.clamp(min=0)], up)
    pos = held + depth
    bit = torch.where(real, torch.ones_like(t) << (t - first).clamp(0, 63), torch.zeros_like(t))
    closes = torch.where((pos + 1) % s == 0, bit, torch.zeros_like(bit))
    seen, up = bit, parent
    for _ in range(st["case"]["nodes"] - 1):
        seen = seen | torch.where(up >= 0, closes[up.clamp(min=0)], torch.zeros_like(bit))
        up = torch.where(up >= 0, parent[up.clamp(min=0)], up)
    return dict(seq=torch.where(real, seq, torch.full_like(seq, -1)).int(),
                position=torch.where(real, pos, torch.zeros_like(pos)), seen=seen,
                slots=torch.div(st["held"], s, rounding_mode="floor"))


def _plain_attend(st):
    case = st["case"]
    r, dr, heads = case["rank"], case["rope"], case["heads"]
    out, lse = torch.empty_like(st["out"]), torch.empty_like(st["lse"])
    at = 0
    for b, (n, m) in enumerate(zip(st["lens"], st["counts"])):
        if m == 0:
            continue
        latent, keys = _page_rows(st["pages"][st["table"][b, :-(-n // PAGE)].long()], r, dr)
        rows = st["rows"][at:at + m].float()
        latent = torch.cat([latent.reshape(-1, r)[:n], rows[:, :r]])
        keys = torch.cat([keys.reshape(-1, dr)[:n], rows[:, r:]])
        q = st["q"][at:at + m].float().view(m * heads, r + dr)
        score = ((q[:, :r] @ latent.T + q[:, r:] @ keys.T) * st["scale"]).view(m, heads, n + m)
        hidden = (st["seen"][at:at + m, None] >> torch.arange(m, device="cuda")) & 1 == 0
        score[:, :, n:].masked_fill_(hidden[:, None], -math.inf)
        top = score.amax(-1, keepdim=True)
        p = torch.exp(score - top)
        total = p.sum(-1, keepdim=True)
        out[at:at + m] = ((p.view(m * heads, n + m) @ latent).view(m, heads, r) / total).to(out.dtype)
        lse[at:at + m] = (top + torch.log(total))[..., 0]
        at += m
    return [out, lse]


def _plain_w4(st):
    k, o = st["case"]["n_in"], st["case"]["n_out"]
    rb, kb = -(-o // 16), -(-k // 128)
    blocks = st["packed"].view(rb, kb, 1088)
    at = _block_places()[None, None, :, :, None].expand(rb, kb, 16, 4, 16)
    byte = blocks[..., :1024].view(rb, kb, 16, 4, 16).gather(3, at).view(rb, kb, 16, 4, 4, 1, 2, 2).int()
    half = byte[..., 0] | (byte[..., 1] << 8)
    sign = torch.tensor(SIGN_AT, device="cuda")[:, None]
    mag = torch.tensor(MAG_AT, device="cuda")[:, None]
    code = ((half >> sign & 1) << 3) | (half >> mag & 7)               # block, ..., group, word, pair, half
    scale = (blocks[..., 1024:].to(torch.int16) << 7).view(torch.float16).float()
    scale = scale.view(rb, kb, 8, 4, 2).permute(0, 1, 4, 2, 3).reshape(rb, kb, 16, 4, 1)
    w = (_e2m1(code).view(rb, kb, 16, 4, 32) * scale).transpose(1, 2).reshape(rb * 16, kb * 128)[:o, :k]
    return (st["x"].float() @ w.T).to(st["x"].dtype)


# ------------------------------------------------------------------------------ a pass

def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        return dict(tree=_plain_tree, attend=_plain_attend, w4=_plain_w4)[op](state)
    from paper_2505_13544_b200 import binding as M
    if op == "tree":
        m = M.mtla_tree_map(state["held"], state["starts"], state["parents"], stride=case["stride"],
                            out=M.TreeMap(**state["buf"]))
        return dict(seq=m.seq, position=m.position, seen=m.seen, slots=m.slots)
    if op == "w4":
        return M.mtla_qweight_product(state["packed"], state["x"], case["n_out"], out=state["y"])
    cfg = M.make_qpool_config(n_heads=case["heads"], latent_rank=case["rank"], rope_dim=case["rope"],
                              n_pages=state["n_pages"])
    return list(M.mtla_qpool_attend_tree(cfg, state["pages"], state["table"], state["slots"], state["starts"],
                                         state["rows"], state["seen"], state["q"], scale=state["scale"],
                                         out=state["out"], lse=state["lse"], workspace=state["workspace"]))


def work(case):
    op = case["op"]
    if op == "tree":
        n = sum(_node_counts(case))
        # Parents in; request, position and mask out; a request's length, place and slots.
        return dict(bytes=4 * n + 16 * (n + case["pad"]) + 12 * case["batch"], flops=4 * n)
    size = 2 if case["dtype"] == "bf16" else 4
    if op == "w4":
        m, k, o = case["rows"], case["n_in"], case["n_out"]
        return dict(bytes=k * o // 2 + -(-k // GROUP) * o + size * m * (k + o), flops=2 * m * k * o)
    r, dr, heads = case["rank"], case["rope"], case["heads"]
    counts, lens = _node_counts(case), _slot_counts(case)
    n = sum(counts)
    slots = sum(lens)
    # Every request's slots once, whatever its tree; nodes see themselves at least.
    pairs = heads * (sum(c * sum(lens) / len(lens) for c in counts) + n)
    return dict(bytes=slots * (r // 2 + r // 32 + 2 * dr) + n * (heads * ((2 * r + dr) * size + 4) + (r + dr) * size + 8),
                flops=int(pairs * (4 * r + 2 * dr)))


# ------------------------------------------------------------------------------ 64-bit answers

def exact(case, seed: int):
    st = prepare(case, seed)
    op = case["op"]
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64,
                         device="cuda")
    if op == "tree":
        held, starts, parents = st["held"].tolist(), st["starts"].tolist(), st["parents"].tolist()
        seq, position, seen = [-1] * st["n"], [0] * st["n"], [0] * st["n"]
        for b, h in enumerate(held):
            for i in range(starts[b], starts[b + 1]):
                path, up = [], parents[i]
                while up >= 0:
                    path.append(up)
                    up = parents[starts[b] + up]
                seq[i], position[i] = b, h + len(path)
                mask = 1 << (i - starts[b])
                for far, a in enumerate(path):
                    if (position[i] - far) % case["stride"] == 0:        # an ancestor `far` + 1 above
                        mask |= 1 << a
                seen[i] = _signed(mask)
        return dict(seq=torch.tensor(seq, dtype=torch.int32), position=torch.tensor(position, dtype=torch.int32),
                    seen=torch.tensor(seen, dtype=torch.int64),
                    slots=torch.tensor([h // case["stride"] for h in held], dtype=torch.int32))
    if op == "w4":
        k, o = case["n_in"], case["n_out"]
        y = torch.empty(case["rows"], o, dtype=torch.float64, device="cuda")
        x = st["x"].double()
        col = torch.arange(k, device="cuda")
        block, c, word, pair, half = col // 128, col // 32 % 4, col // 8 % 4, col // 2 % 4, col % 2
        sign, mag = torch.tensor(SIGN_AT, device="cuda")[pair], torch.tensor(MAG_AT, device="cuda")[pair]
        blocks = st["packed"].view(-1, -(-k // 128), 1088)
        for o0 in range(0, o, 1024):
            row = torch.arange(o0, min(o, o0 + 1024), device="cuda")[:, None]
            i = row % 16
            at = 64 * i + 16 * (c ^ (i // 2 & 3)) + 4 * word + 2 * half
            bits = blocks[row // 16, block, at].int() + 256 * blocks[row // 16, block, at + 1].int()
            code = (bits >> mag) % 8 + 8 * ((bits >> sign) % 2)
            scale = blocks[row // 16, block, 1024 + 2 * (4 * (i % 8) + c) + i // 8].short() * 128
            w = value[code.long()] * scale.view(torch.float16).double()
            y[:, o0:o0 + 1024] = torch.einsum("nk,ok->no", x, w)
        return y
    r, dr, heads = case["rank"], case["rope"], case["heads"]
    out = torch.empty(st["q"].shape[0], heads, r, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["q"].shape[0], heads, dtype=torch.float64, device="cuda")
    chunk = r // 32
    mask = (chunk & -chunk if (chunk & -chunk) < 8 else 8) - 1
    first = st["starts"].tolist()
    for b, n in enumerate(st["lens"]):
        lo, hi = first[b], first[b + 1]
        if lo == hi:
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
        shared = torch.cat([latent, key], 1)
        for j in range(lo, hi):                             # node by node, only the rows that it sees
            m = st["seen"][j].item()
            rows = st["rows"][[lo + a for a in range(hi - lo) if m >> a & 1]].double()
            both = torch.cat([shared, rows])
            score = (st["q"][j].double() @ both.T) * st["scale"]
            lse[j] = torch.logsumexp(score, 1)
            out[j] = torch.softmax(score, 1) @ both[:, :r]
    return [out, lse]

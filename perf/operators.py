"""The paged 8-bit cache: the calls that fill it and the attention that reads it, over the sizes that programs make them at.

One case is one pass of one kind of work:

  rotate  q and k of a layer turned by their positions (one axis, or time, height and width)
  append  the kept tokens of a prompt, keys rotated on the way, into the cache
  decode  a few generation steps of one layer: attention of the new token over the cache, and its append
  turn    many new tokens at once (the next turn of a conversation, or a first prompt): attention over the cache as it stands
          and over themselves, and their append

Where `own` is false, everything is computed in its plain form, with elementary torch operations in 32 bits.

The cache.  A unit is one (sequence, KV head); its rows are counted in order of arrival, 64 of them are a block.  A full block is
held in 8 bits (e4m3) with a power of two as its scale, in the page that the unit's row of the page table names; the last,
incomplete one is held in bf16, in the unit's tail.  Pages and tails keep their rows in the order in which matrix instructions
take them (_pack_k, _pack_v).
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 64
AXES = {1: None, 3: (0.25, 0.375, 0.375)}   # shares of the pairs that turn by time, height and width
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------------- the cases
def _rotate(name, **kw):
    return {"name": name, "kind": "rotate", "dtype": "bf16", "B": 1, "L": 4096, "Hq": 32, "Hkv": 32, "D": 128, "axes": 1, **kw}


def _append(name, **kw):
    return {"name": name, "kind": "append", "dtype": "bf16", "B": 1, "L": 4096, "Hq": 32, "Hkv": 32, "D": 128, "axes": 1, "max_len": 0,
            "keep_lo": 0.2, "keep_hi": 0.9, **kw}


def _decode(name, **kw):
    return {"name": name, "kind": "decode", "dtype": "bf16", "B": 1, "L": 1, "Hq": 32, "Hkv": 8, "D": 128, "axes": 1, "max_len": 777,
            "keep_new": 0.5, "steps": 8, **kw}


def _turn(name, **kw):
    return {"name": name, "kind": "turn", "dtype": "bf16", "B": 1, "L": 1501, "Hq": 32, "Hkv": 8, "D": 128, "axes": 1, "max_len": 0,
            "keep_lo": 0.2, "keep_hi": 0.9, **kw}


def listed():
    return [
        # the new tokens of a batch of 32 sequences before a decode step of the bf16 cache: latency is all there is
        _rotate("rotate_step", B=32, L=1, Hkv=8),
        # the 7B-shaped layer the benchmark runs, q and k of all its heads
        _rotate("rotate_prompt", L=4096),
        # frames of a video and the text around them: three axes, head dimension 64, fp32 (where a layer is checked)
        _rotate("rotate_frames", dtype="f32", B=2, L=2900, D=64, Hkv=8, axes=3),
        # a chat turn that is only cached (its attention ran elsewhere): a few hundred tokens behind a partly filled block
        _append("append_short", L=333, Hkv=8, max_len=777),
        # a batch of prompts in a middle layer of the 32-layer stack, half of the tokens kept, into empty caches
        _append("append_batch", B=16, L=2048, keep_lo=0.46, keep_hi=0.52),
        # one user's chat: one sequence, grouped heads, a few hundred kept tokens; latency and launches are all there is
        _decode("decode_chat"),
        # serving: 32 sequences of a 7B-shaped model with all their heads, caches of 400 to 4096 rows
        _decode("decode_batch", B=32, Hkv=32, max_len=4096, steps=4),
        # a few long documents (32k tokens, 30 % kept) under generation with grouped heads, every new token kept
        _decode("decode_long", B=4, max_len=13000, keep_new=1.0),
        # a question of a few dozen tokens to a chat of some hundreds
        _turn("turn_short", L=37, max_len=777),
        # a long turn over a long document, two sequences, head dimension 64
        _turn("turn_d64", B=2, L=900, Hq=16, D=64, max_len=5000),
        # the first prompt: the 7B-shaped layer over an empty cache
        _turn("turn_first", L=4096, Hkv=32),
        # another document of 4096 tokens behind one of which 13000 rows are held
        _turn("turn_long", L=4096, max_len=13000, keep_lo=0.3, keep_hi=0.3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(["rotate"] * 2 + ["append"] * 2 + ["decode"] * 4 + ["turn"] * 4)
    Hq, Hkv = rng.choice([(32, 32), (32, 8), (32, 8), (32, 8), (16, 8), (16, 16), (8, 8), (32, 4)])
    c = {"Hq": Hq, "Hkv": Hkv, "D": rng.choice([128, 128, 128, 64]), "axes": rng.choice([1, 1, 3])}
    lo, hi = sorted((rng.uniform(0.05, 1.0), rng.uniform(0.05, 1.0)))
    keep = {"keep_lo": round(lo, 3), "keep_hi": round(hi, 3)}
    if kind == "rotate":
        return _rotate("", B=_log_int(rng, 1, 48), L=_log_int(rng, 1, 8192), dtype=rng.choice(["bf16", "bf16", "f32"]), **c)
    if kind == "append":
        return _append("", B=_log_int(rng, 1, 16), L=_log_int(rng, 1, 16384), max_len=rng.choice([0, _log_int(rng, 1, 8000)]), **c, **keep)
    if kind == "decode":
        return _decode("", B=_log_int(rng, 1, 48), max_len=_log_int(rng, 1, 16000), keep_new=rng.choice([0.5, 1.0]), steps=rng.choice([4, 6, 8]), **c)
    return _turn("", B=rng.choice([1, 1, 1, 2, 3, 4]), L=_log_int(rng, 2, 4096), max_len=rng.choice([0, _log_int(rng, 1, 13000), _log_int(rng, 1, 13000)]),
                 **c, **keep)


def _least(case):  # seconds at generous rates: only to compare sizes
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 8e14


def _held(case):  # bytes that the plain form holds at once, roughly
    c = case
    if c["kind"] == "turn":
        return 16.0 * c["B"] * c["Hq"] * c["L"] * (c["max_len"] + c["L"])
    if c["kind"] == "decode":
        return 20.0 * c["B"] * c["Hkv"] * c["max_len"] * c["D"]
    return 0.0


def draw(rng):
    """One more case; those that would outgrow the largest listed ones are drawn again."""
    most, held = max(_least(c) for c in listed()), max(_held(c) for c in listed())
    while True:
        c = _draw_once(rng)
        if _least(c) <= 0.8 * most and _held(c) <= held:
            del c["name"]
            return c


# ------------------------------------------------------------------------------------------------- inputs of one case
class State:
    pass


def _normal(g, shape, dtype):
    """N(0, 1) in slices, so that no fp32 copy of a large tensor is held."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 27):
        n = min(1 << 27, flat.numel() - a)
        flat[a:a + n] = torch.randn(n, generator=g, device=DEV)
    return out


def _sections(case):
    """Pairs that turn by each axis."""
    pairs = case["D"] // 2
    if case["axes"] == 1:
        return [pairs]
    n = [int(s * pairs) for s in AXES[case["axes"]]]
    return n[:-1] + [pairs - sum(n[:-1])]


def _positions(case, g, first, L):
    """[axes, B, L]: text counts on; frames have a time, and a place in a grid 24 patches wide."""
    t = torch.arange(L, device=DEV)[None] + first[:, None]
    if case["axes"] == 1:
        return t[None].int().contiguous()
    return torch.stack([t // 384, t % 384 // 24, t % 24]).int().contiguous()


def _table(rows, D):
    """[rows, D]: the cosines, then the sines, of a row's angles."""
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)[None]
    return torch.cat([angle.cos(), angle.sin()], dim=1).float().to(DEV)


def prepare(case, seed):
    c, g, s = case, torch.Generator(device=DEV), State()
    g.manual_seed(int(seed))
    B, L, Hq, Hkv, D, dt = c["B"], c["L"], c["Hq"], c["Hkv"], c["D"], TORCH[c["dtype"]]
    U, s.case, s.scale, n = B * Hkv, dict(c), 1.0 / math.sqrt(D), c.get("steps", 1)
    most = c.get("max_len", 0)
    # a sequence has seen about twice the rows that are held of it
    first = torch.full((B,), 2 * most, device=DEV) - torch.randint(0, 10, (B,), generator=g, device=DEV).clamp(max=2 * most)
    s.table = _table(2 * most + L + n, D)
    s.sections = _sections(c)
    s.pos = [_positions(c, g, first + i, L) for i in range(n)]
    lead = (n, B) if c["kind"] == "decode" else (B,)
    if c["kind"] != "append":
        s.q = _normal(g, lead + (Hq, L, D), dt)
    s.k = _normal(g, lead + (Hkv, L, D), dt)
    if c["kind"] == "rotate":
        s.q_out, s.k_out = torch.empty_like(s.q), torch.empty_like(s.k)
        return s
    s.v = _normal(g, lead + (Hkv, L, D), dt)
    if c["kind"] == "decode":
        s.q, s.k, s.v = (x.squeeze(3).contiguous() for x in (s.q, s.k, s.v))
        keep = torch.full((n, B, Hkv), c["keep_new"], device=DEV)
        s.all_kept = c["keep_new"] >= 1.0
    else:
        keep = (c["keep_lo"] + (c["keep_hi"] - c["keep_lo"]) * torch.rand(B, Hkv, 1, generator=g, device=DEV)).expand(B, Hkv, L)
        s.all_kept = c["keep_lo"] >= 1.0
    s.flags = (torch.rand(keep.shape, generator=g, device=DEV) < keep).to(torch.uint8)
    # the rows that are held: 10 % to 100 % of the most, and one unit in twenty that has evicted nearly everything
    rows = (most * (0.1 + 0.9 * torch.rand(U, generator=g, device=DEV))).round().int()
    rows[torch.rand(U, generator=g, device=DEV) < 0.05] = min(1, most)
    s.max_blocks = max(1, -(-(most + n * L) // BLOCK))
    s.n_pages = U * s.max_blocks
    # (one page more than there are: the plain form writes there what has no page)
    s.pages_k, s.pages_v = (torch.empty(s.n_pages + 1, BLOCK * D, dtype=torch.uint8, device=DEV) for _ in range(2))
    s.scales_k, s.scales_v = (torch.empty(s.n_pages + 1, device=DEV) for _ in range(2))
    for codes, scales in ((s.pages_k, s.scales_k), (s.pages_v, s.scales_v)):
        for a in range(0, s.n_pages + 1, 1 << 14):
            m = min(1 << 14, s.n_pages + 1 - a)
            codes[a:a + m], scales[a:a + m] = _eight_bits(_normal(g, (m, BLOCK * D), dt).float()) if most else (0, 1.0)
    s.page = torch.randperm(s.n_pages, generator=g, device=DEV).int().view(U, s.max_blocks)
    # tails and lengths in one piece of memory, and how they stand when the pass begins (a program that keeps a conversation's state
    # to answer from it again restores these)
    tail = U * BLOCK * D
    s.kept_state = torch.cat([_normal(g, (2 * tail,), torch.bfloat16) if most else torch.zeros(2 * tail, dtype=torch.bfloat16, device=DEV),
                              rows.view(torch.bfloat16)])
    s.live = s.kept_state.clone()
    s.tail_k, s.tail_v = s.live[:tail].view(U, BLOCK * D), s.live[tail:2 * tail].view(U, BLOCK * D)
    s.len = s.live[2 * tail:].view(torch.int32)
    if c["kind"] in ("decode", "turn"):
        s.out = torch.empty_like(s.q)
    return s


# ------------------------------------------------------------------------------------------------------ the plain form
def _turned(x, table, pos, sections):
    """x [B, H, L, D] turned by pos [axes, B, L], in 32 bits."""
    half = x.shape[-1] // 2
    axis = torch.repeat_interleave(torch.arange(len(sections), device=x.device), torch.tensor(sections, device=x.device), output_size=half)
    row = pos.long()[axis].permute(1, 2, 0)                                  # [B, L, D/2]
    pair = torch.arange(half, device=x.device).expand_as(row)
    c, s = table[row, pair][:, None], table[row, pair + half][:, None]
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _eight_bits(x):
    """x fp32 [n, values of a block] -> codes (uint8), scales: the least power of two that brings all finite values to at most 448."""
    top = torch.where(x.isfinite(), x.abs(), 0.0).amax(1)
    m, e = torch.frexp(top)
    e = (e - torch.where(m <= 0.875, 9, 8)).clamp(min=-100)
    e = torch.where(top > 0, e, -100)
    codes = torch.ldexp(x, -e[:, None]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), torch.ldexp(torch.ones_like(top), e)


def _pack_k(rows):
    """[n, 64, D] -> [n, 64 D]: 16 rows, 64 columns a piece; in it 16 columns of a row lie together."""
    n, _, D = rows.shape
    return rows.reshape(n, 4, 16, D // 64, 4, 16).permute(0, 1, 3, 4, 2, 5).reshape(n, BLOCK * D)


def _unpack_k(x):
    n, D = x.shape[0], x.shape[1] // BLOCK
    return x.view(n, 4, D // 64, 4, 16, 16).permute(0, 1, 4, 2, 3, 5).reshape(n, BLOCK, D)


def _pack_v(rows):
    """[n, 64, D] -> [n, 64 D]: 16 columns a piece; in it rows 16 i + 4 j + 0..3, i = 0..3, of a column lie together."""
    n, _, D = rows.shape
    return rows.reshape(n, 4, 4, 4, D // 16, 16).permute(0, 4, 2, 5, 1, 3).reshape(n, BLOCK * D)


def _unpack_v(x):
    n, D = x.shape[0], x.shape[1] // BLOCK
    return x.view(n, D // 16, 4, 16, 4, 4).permute(0, 4, 2, 5, 1, 3).reshape(n, BLOCK, D)


def _held_rows(s, codes, scales, tail, unpack, blocks):
    """The rows of all units, in 32 bits: [U, 64 blocks + 64, D], those of the pages and then the tail's."""
    U, D = s.page.shape[0], s.case["D"]
    ids = s.page[:, :blocks].long().reshape(-1)
    full = unpack(codes[ids].view(torch.float8_e4m3fn).float() * scales[ids][:, None]).view(U, blocks * BLOCK, D)
    return torch.cat([full, unpack(tail.float())], dim=1)


def _plain_append(s, k, v, flags):
    """k (turned), v fp32 [U, L, D], flags [U, L]: the kept rows join the cache."""
    U, L, D = k.shape
    held, kept = s.len.long() % BLOCK, flags != 0
    room = -(-(BLOCK - 1 + L) // BLOCK)                            # blocks that tail and new rows can fill, and begin
    at = torch.where(kept, held[:, None] + kept.cumsum(1) - 1, room * BLOCK)   # (the last place is for what is not kept)
    total = held + kept.sum(1)
    done = total // BLOCK
    block = torch.arange(room, device=k.device)[None]
    ids = s.page.long().gather(1, (s.len.long()[:, None] // BLOCK + block).clamp(max=s.max_blocks - 1))
    ids = torch.where(block < done[:, None], ids, s.n_pages).reshape(-1)
    left = (total - done * BLOCK)[:, None, None]
    row = torch.arange(BLOCK, device=k.device)[None, :, None]
    for rows, tail, pack, unpack, codes, scales in ((k, s.tail_k, _pack_k, _unpack_k, s.pages_k, s.scales_k),
                                                    (v, s.tail_v, _pack_v, _unpack_v, s.pages_v, s.scales_v)):
        all_rows = torch.zeros(U, room * BLOCK + 1, D, device=k.device)
        old = unpack(tail.float())
        all_rows[:, :BLOCK] = torch.where(row < held[:, None, None], old, 0.0)
        all_rows.scatter_(1, at[..., None].expand(U, L, D), rows.to(torch.bfloat16).float())
        all_rows = all_rows[:, :-1].reshape(U, room, BLOCK, D)
        eight = _eight_bits(pack(all_rows.reshape(-1, BLOCK, D)))
        codes[ids], scales[ids] = eight
        last = all_rows.gather(1, done.clamp(max=room - 1)[:, None, None, None].expand(U, 1, BLOCK, D)).squeeze(1)
        tail.copy_(pack(torch.where(row < left, last, old)).to(torch.bfloat16))
    s.len.add_(kept.sum(1).int())


def _plain_attend(s, q, k, v, flags, blocks):
    """q [U, G, L, D], k, v [U, L, D] (turned) fp32, flags [U, L] -> [U, G, L, D]: over the rows held, then over the call's own."""
    U, G, L, D = q.shape
    K = torch.cat([_held_rows(s, s.pages_k, s.scales_k, s.tail_k, _unpack_k, blocks), k], dim=1)
    V = torch.cat([_held_rows(s, s.pages_v, s.scales_v, s.tail_v, _unpack_v, blocks), v], dim=1)
    n = s.len.long()[:, None]
    i = torch.arange(blocks * BLOCK, device=q.device)[None]
    seen = torch.cat([i < n // BLOCK * BLOCK, torch.arange(BLOCK, device=q.device)[None] < n % BLOCK], dim=1)   # [U, rows held]
    j = torch.arange(L, device=q.device)
    mine = ((flags != 0)[:, None, :] & (j[None] < j[:, None])[None]) | torch.eye(L, dtype=torch.bool, device=q.device)[None]
    see = torch.cat([seen[:, None, :].expand(U, L, seen.shape[1]), mine], dim=2)[:, None]                   # [U, 1, L, rows]
    score = torch.matmul(q.reshape(U, G * L, D), K.transpose(1, 2).contiguous()).view(U, G, L, -1).mul_(s.scale)
    score.masked_fill_(~see, -math.inf)
    score.sub_(score.amax(-1, keepdim=True)).exp_()
    total = score.sum(-1, keepdim=True)
    V = torch.where(see.any(2).view(U, -1, 1), V, 0.0)   # rows that nobody sees hold whatever was there
    return torch.matmul(score.view(U, G * L, -1), V).view(U, G, L, D).div_(total)


def _flat(x):
    """[B, H, L, D] -> [B H, L, D]"""
    return x.reshape(-1, *x.shape[2:])


def _plain(s):
    c = s.case
    B, L, Hq, Hkv, D = c["B"], c["L"], c["Hq"], c["Hkv"], c["D"]
    U, G = B * Hkv, Hq // Hkv
    if c["kind"] == "rotate":
        s.q_out.copy_(_turned(s.q, s.table, s.pos[0], s.sections))
        s.k_out.copy_(_turned(s.k, s.table, s.pos[0], s.sections))
    elif c["kind"] == "append":
        k = _turned(s.k, s.table, s.pos[0], s.sections)
        _plain_append(s, _flat(k), _flat(s.v).float(), _flat(s.flags))
    elif c["kind"] == "turn":
        q, k, v = _turned(s.q, s.table, s.pos[0], s.sections), _flat(_turned(s.k, s.table, s.pos[0], s.sections)), _flat(s.v).float()
        s.out.copy_(_plain_attend(s, q.view(U, G, L, D), k, v, _flat(s.flags), -(-c["max_len"] // BLOCK)).view(B, Hq, L, D))
        _plain_append(s, k, v, _flat(s.flags))
    else:
        for i in range(c["steps"]):  # (a step needs the one before it)
            q = _turned(s.q[i].unsqueeze(2), s.table, s.pos[i], s.sections)
            k = _flat(_turned(s.k[i].unsqueeze(2), s.table, s.pos[i], s.sections))
            v, f = _flat(s.v[i].unsqueeze(2)).float(), s.flags[i].view(U, 1)
            s.out[i] = _plain_attend(s, q.reshape(U, G, 1, D), k, v, f, s.max_blocks).view(B, Hq, D)
            _plain_append(s, k, v, f)


# ------------------------------------------------------------------------------------------- the framework's operators
def _handles(s):
    """What a program makes once and keeps: the context, the cache's and the positions' descriptions."""
    import paper_2410_12876_amd as ag
    c = s.case
    s.ag = ag
    s.ropes = [ag.Rope(s.table, p, s.sections) for p in s.pos]
    if c["kind"] == "rotate":
        s.ctx = ag.Context(0)
        return
    s.cache = ag.Q8Cache(s.pages_k[:s.n_pages], s.pages_v[:s.n_pages], s.scales_k[:s.n_pages], s.scales_v[:s.n_pages], s.tail_k, s.tail_v, s.page, s.len,
                         c["B"], c["Hkv"], c["D"])
    s.ctx = ag.Context(0, ag.q8_workspace_bytes(c["B"], c["L"], c["Hq"], c["Hkv"], c["D"], s.max_blocks))


def _own(s):
    if not hasattr(s, "ag"):
        _handles(s)
    ag, c = s.ag, s.case
    flags = None if c["kind"] == "rotate" or s.all_kept else s.flags
    if c["kind"] == "rotate":
        ag.ag_rotate(s.ctx, s.q, s.k, s.ropes[0], s.q_out, s.k_out)
    elif c["kind"] == "append":
        ag.ag_q8_append(s.ctx, s.k, s.v, flags, s.ropes[0], s.cache)
    elif c["kind"] == "turn":
        ag.ag_q8_prefill_attn(s.ctx, s.q, s.k, s.v, flags, s.ropes[0], s.scale, s.cache, s.out)
    else:
        for i in range(c["steps"]):
            ag.ag_q8_decode_attn(s.ctx, s.q[i], s.k[i], s.v[i], None if flags is None else flags[i], s.ropes[i], s.scale, s.cache, s.out[i])


def run(state):
    s = state
    if s.case["kind"] != "rotate":
        if s.case["max_len"] or s.case["kind"] == "decode":
            s.live.copy_(s.kept_state)
        else:
            s.len.zero_()  # an empty cache: nothing else of it is read
    (_own if own else _plain)(s)
    if s.case["kind"] == "rotate":
        return {"q": s.q_out, "k": s.k_out}
    got = {"k": s.pages_k[:s.n_pages].view(torch.float8_e4m3fn), "v": s.pages_v[:s.n_pages].view(torch.float8_e4m3fn),
           "k_scale": s.scales_k[:s.n_pages], "v_scale": s.scales_v[:s.n_pages], "k_tail": s.tail_k, "v_tail": s.tail_v, "len": s.len}
    if s.case["kind"] != "append":
        got["out"] = s.out
    return got


# ----------------------------------------------------------------------------------------------- what a pass must cost
def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    B, L, Hq, Hkv, D = c["B"], c["L"], c["Hq"], c["Hkv"], c["D"]
    angles = B * L * (D * 4 + c["axes"] * 4)
    if c["kind"] == "rotate":
        n = B * L * (Hq + Hkv) * D
        return {"bytes": 2.0 * n * e + angles, "flops": 3.0 * n}
    U, n = B * Hkv, c.get("steps", 1)
    held = U * (0.95 * 0.55 * c["max_len"] + 0.05)                 # rows at the start
    tails = U * min(31.5, 0.55 * c["max_len"])                     # ... of which these are in bf16
    if c["kind"] == "decode":
        rows = held + U * (n - 1) / 2 * c["keep_new"]
        small = B * (2 * Hq + 2 * Hkv) * D * e + angles + U * (c["keep_new"] * 2 * D * 2 + 8 + rows / U / BLOCK * 12)
        return {"bytes": n * (rows * 2 * D + tails * 2 * D + small), "flops": n * 4.0 * D * (rows + U) * Hq / Hkv}
    keep = 0.5 * (c["keep_lo"] + c["keep_hi"])
    kept = keep * U * L
    nbytes = kept * 2 * D * (e + 1) + U * L + angles + 2 * tails * 2 * D * 2
    if c["kind"] == "append":
        return {"bytes": float(nbytes), "flops": 3.0 * kept * D}
    nbytes += 2 * B * Hq * L * D * e + (1 - keep) * U * L * 2 * D * e + held * 2 * D
    pairs = Hq / Hkv * (held * L + U * L * (keep * (L - 1) / 2 + 1))
    return {"bytes": float(nbytes), "flops": 4.0 * D * pairs}


# --------------------------------------------------------------------------------------- the definition, in 64 bits
def _exact_turn(x, s, pos):
    """x [B, H, L, D] in 64 bits, pair by pair."""
    y, half, first = x.double().clone(), x.shape[-1] // 2, 0
    for a, n in enumerate(s.sections):
        lo, hi = slice(first, first + n), slice(half + first, half + first + n)
        angle = s.table[pos[a].long()].double()[:, None]                      # [B, 1, L, D]
        c, sn = angle[..., lo], angle[..., hi]
        y[..., lo] = x[..., lo].double() * c - x[..., hi].double() * sn
        y[..., hi] = x[..., hi].double() * c + x[..., lo].double() * sn
        first += n
    return y


def _places(D, values):
    """Where value (row, column) of a block lies in its page: [64, D]."""
    t, d = torch.arange(BLOCK, device=DEV)[:, None], torch.arange(D, device=DEV)[None]
    if values:
        return (d // 16) * 1024 + (t // 4 % 4) * 256 + (d % 16) * 16 + (t // 16) * 4 + t % 4
    return ((t // 16) * (D // 64) + d // 64) * 1024 + (d // 16 % 4) * 256 + (t % 16) * 16 + d % 16


def _exact_codes(x):
    """x (64 bits, any shape) -> the 8-bit numbers and the scale of one block."""
    top = float(x.abs().max())
    e = -100 if top == 0.0 else max(-100, math.ceil(math.log2(top / 448.0)))
    while top > math.ldexp(448.0, e):
        e += 1
    while e > -100 and top <= math.ldexp(448.0, e - 1):
        e -= 1
    y = x * 2.0 ** -e
    step = torch.exp2((torch.frexp(y).exponent.double() - 4).clamp(min=-9))    # 4 bits of a number, the least exponent -6
    return torch.round(y / step) * step, 2.0 ** e


class _Unit:
    """One unit's rows: the full blocks' values, the tail's, and where they are held."""

    def __init__(self, s, u, codes, scales, tail, values):
        self.s, self.u, self.codes, self.scales, self.place = s, u, codes, scales, _places(s.case["D"], values)
        n = int(s.exact_len[u])
        ids = s.page[u, :n // BLOCK].long()
        self.full = [(codes[ids] * scales[ids][:, None])[:, self.place.reshape(-1)].view(-1, s.case["D"])]
        self.tail = tail[u]
        self.last = self.tail[self.place[:n % BLOCK].reshape(-1)].view(-1, s.case["D"])

    def rows(self):
        return torch.cat(self.full + [self.last])

    def append(self, rows):
        rows = torch.cat([self.last, rows.float().to(torch.bfloat16).double()])
        while rows.shape[0] >= BLOCK:
            page = int(self.s.page[self.u, sum(f.shape[0] for f in self.full) // BLOCK])
            y, scale = _exact_codes(rows[:BLOCK])
            self.codes[page, self.place.reshape(-1)], self.scales[page] = y.reshape(-1), scale
            self.full.append(y * scale)
            rows = rows[BLOCK:]
        self.last = rows
        self.tail[self.place[:rows.shape[0]].reshape(-1)] = rows.reshape(-1)


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    B, L, Hq, Hkv, D = c["B"], c["L"], c["Hq"], c["Hkv"], c["D"]
    if c["kind"] == "rotate":
        return {"q": _exact_turn(s.q, s, s.pos[0]), "k": _exact_turn(s.k, s, s.pos[0])}
    n, U, G = c.get("steps", 1), B * Hkv, Hq // Hkv
    if n * U * (1 + 0.02 * c["max_len"] / 100 + L / BLOCK) > 60000:
        return None
    codes = [x[:s.n_pages].view(torch.float8_e4m3fn).double() for x in (s.pages_k, s.pages_v)]
    scales = [x[:s.n_pages].double() for x in (s.scales_k, s.scales_v)]
    tails = [s.tail_k.double(), s.tail_v.double()]
    s.exact_len = s.len.tolist()
    if c["kind"] == "decode":
        ks = [_exact_turn(s.k[i].unsqueeze(2), s, s.pos[i]) for i in range(n)]
        qs = [_exact_turn(s.q[i].unsqueeze(2), s, s.pos[i]) for i in range(n)]
        vs, flags = [s.v[i].unsqueeze(2).double() for i in range(n)], [s.flags[i].unsqueeze(2) for i in range(n)]
    else:
        ks, vs, flags = [_exact_turn(s.k, s, s.pos[0])], [s.v.double()], [s.flags]
        qs = None if c["kind"] == "append" else [_exact_turn(s.q, s, s.pos[0])]
    out = [torch.empty(B, Hq, L, D, dtype=torch.float64, device=DEV) for _ in range(n)]
    flags_host = torch.stack(flags).bool().cpu()
    for u in range(U):
        b, h = divmod(u, Hkv)
        K, V = _Unit(s, u, codes[0], scales[0], tails[0], False), _Unit(s, u, codes[1], scales[1], tails[1], True)
        for i in range(n):
            k, v = ks[i][b, h], vs[i][b, h]
            kept = torch.nonzero(flags_host[i, b, h]).view(-1).to(DEV)
            if qs is not None:
                rows_k, rows_v = torch.cat([K.rows(), k[kept]]), torch.cat([V.rows(), v[kept]])
                old = rows_k.shape[0] - kept.numel()
                for a in range(0, L, 512):       # some queries at a time
                    j = torch.arange(a, min(L, a + 512), device=DEV)
                    see = torch.cat([torch.ones(j.numel(), old, dtype=torch.bool, device=DEV), kept[None] < j[:, None]], dim=1)
                    for x in range(h * G, h * G + G):
                        q = qs[i][b, x, j]
                        score = torch.cat([torch.where(see, q @ rows_k.T * s.scale, -math.inf), (q * k[j]).sum(1, keepdim=True) * s.scale], dim=1)
                        p = torch.softmax(score, dim=1)
                        out[i][b, x, j] = p[:, :-1] @ rows_v + p[:, -1:] * v[j]
            K.append(k[kept])
            V.append(v[kept])
            s.exact_len[u] += kept.numel()
    got = {"k": codes[0], "v": codes[1], "k_scale": scales[0], "v_scale": scales[1], "k_tail": tails[0], "v_tail": tails[1],
           "len": torch.tensor(s.exact_len, dtype=torch.int32)}
    if c["kind"] == "decode":
        got["out"] = torch.stack(out).squeeze(3)
    elif c["kind"] == "turn":
        got["out"] = out[0]
    return got

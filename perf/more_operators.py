"""Several continuations of one conversation over the paged 8-bit cache, over the sizes that programs make them at.

One case is one pass of one kind of work:

  norm     q and k of a layer, each head's vector normalised and turned by its position, in one pass
  tree     a tree of drafted tokens, verified at once: every node attends to the cache, to its ancestors and to itself
  accept   the path that was accepted joins the cache
  fork     a step of beam search: every sequence takes over a beam's state, full blocks shared, and gets pages for what it will add
  compact  sequences end, their pages are given back, and the pages still in use move together at the front of the pool

Where `own` is false, everything is computed in its plain form, with elementary torch operations in 32 bits.

The cache.  A unit is one (sequence, KV head); its rows are counted in order of arrival, 64 of them are a block.  A full block is
held in 8 bits (e4m3) with a power of two as its scale, in the page that the unit's row of the page table names; the last,
incomplete one is held in bf16, in the unit's tail.  Pages and tails keep their rows in the order in which matrix instructions
take them (_pack_k, _pack_v).  ref counts, for each page, the entries of all tables that name it; 0 is a free page.
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 64
EPS = 1e-6
AXES = {1: None, 3: (0.25, 0.375, 0.375)}   # shares of the pairs that turn by time, height and width
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------------- the cases
def _norm(name, **kw):
    return {"name": name, "kind": "norm", "dtype": "bf16", "B": 1, "L": 4096, "Hq": 32, "Hkv": 32, "D": 128, "axes": 1, **kw}


def _tree(name, **kw):
    return {"name": name, "kind": "tree", "dtype": "bf16", "B": 1, "L": 12, "Hq": 32, "Hkv": 8, "D": 128, "axes": 1, "max_len": 777,
            "keep_new": 1.0, **kw}


def _accept(name, **kw):
    return {"name": name, "kind": "accept", "dtype": "bf16", "B": 1, "L": 12, "Hq": 32, "Hkv": 8, "D": 128, "axes": 1, "max_len": 777,
            "keep_new": 0.5, **kw}


def _fork(name, **kw):
    return {"name": name, "kind": "fork", "groups": 1, "beams": 4, "Hkv": 8, "D": 128, "max_len": 777, "generated": 150, "rows": 64, **kw}


def _compact(name, **kw):
    return {"name": name, "kind": "compact", "B": 4, "Hkv": 8, "D": 128, "max_len": 777, "ended": 0.4, **kw}


def listed():
    return [
        # the new tokens of a batch of 32 sequences before a decode step: latency is all there is
        _norm("norm_step", B=32, L=1, Hkv=8),
        # the 7B-shaped layer the benchmark runs, q and k of all its heads
        _norm("norm_prompt"),
        # frames of a video and the text around them: three axes, head dimension 64, fp32 (where a layer is checked)
        _norm("norm_frames", dtype="f32", B=2, L=2900, D=64, Hkv=8, axes=3),
        # one user's chat, a dozen drafted tokens: latency and launches are all there is
        _tree("tree_chat"),
        # serving: 16 sequences with caches of 400 to 4096 rows, 31 drafted tokens each, of which the gate keeps half
        _tree("tree_batch", B=16, L=31, max_len=4096, keep_new=0.5),
        # a few long documents (32k tokens, 30 % kept), wide trees
        _tree("tree_long", B=4, L=64, max_len=13000),
        # the chat's accepted tokens
        _accept("accept_chat"),
        # the accepted tokens of 48 sequences
        _accept("accept_batch", B=48, L=31, max_len=1501),
        # one conversation, four beams
        _fork("fork_chat"),
        # 16 prompts with eight beams each
        _fork("fork_batch", groups=16, beams=8, max_len=4096, generated=333),
        # four chats, of which one or two end
        _compact("compact_chat"),
        # a server's pool after a third of its sequences has ended
        _compact("compact_batch", B=48, max_len=4096, ended=0.33),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(["norm"] * 3 + ["tree"] * 5 + ["accept"] * 2 + ["fork"] * 2 + ["compact"] * 2)
    Hq, Hkv = rng.choice([(32, 32), (32, 8), (32, 8), (32, 8), (16, 8), (16, 16), (8, 8), (32, 4)])
    D, axes = rng.choice([128, 128, 128, 64]), rng.choice([1, 1, 3])
    c = {"Hq": Hq, "Hkv": Hkv, "D": D, "axes": axes}
    if kind == "norm":
        return _norm("", B=_log_int(rng, 1, 48), L=_log_int(rng, 1, 8192), dtype=rng.choice(["bf16", "bf16", "f32"]), **c)
    if kind == "tree":
        return _tree("", B=_log_int(rng, 1, 32), L=_log_int(rng, 1, 160), max_len=rng.choice([0] + [_log_int(rng, 1, 13000)] * 7),
                     keep_new=rng.choice([0.5, 1.0]), **c)
    if kind == "accept":
        return _accept("", B=_log_int(rng, 1, 48), L=_log_int(rng, 1, 160), max_len=_log_int(rng, 1, 2000), keep_new=rng.choice([0.5, 1.0]), **c)
    if kind == "fork":
        return _fork("", groups=_log_int(rng, 1, 16), beams=rng.choice([2, 3, 4, 5, 8]), Hkv=Hkv, D=D, max_len=_log_int(rng, 1, 8000),
                     generated=_log_int(rng, 1, 1000), rows=rng.choice([1, 64, 200]))
    return _compact("", B=_log_int(rng, 1, 48), Hkv=Hkv, D=D, max_len=_log_int(rng, 1, 8000), ended=round(rng.uniform(0.0, 1.0), 2))


def _least(case):  # seconds at generous rates: only to compare sizes
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 8e14


def _held(case):  # bytes that a pass's state and the plain form hold at once, roughly
    c = case
    if c["kind"] == "norm":
        return 0.0
    if c["kind"] == "fork":
        return 2.0 * BLOCK * c["D"] * _fork_pages(c) + 16.0 * c["groups"] * c["beams"] * c["Hkv"] * BLOCK * c["D"]
    n = c["B"] * c["Hkv"] * (c["max_len"] + BLOCK)
    if c["kind"] == "tree":
        return 24.0 * n * c["D"] + 16.0 * n * c["L"] * c["Hq"] / c["Hkv"]
    return (2.0 if c["kind"] == "accept" else 6.0) * n * c["D"]


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


def _by_axis(case, t):
    """[axes, B, L] of the places t [B, L]: text counts on; frames have a time, and a place in a grid 24 patches wide."""
    return (t[None] if case["axes"] == 1 else torch.stack([t // 384, t % 384 // 24, t % 24])).int().contiguous()


def _table(rows, D):
    """[rows, D]: the cosines, then the sines, of a row's angles."""
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)[None]
    return torch.cat([angle.cos(), angle.sin()], dim=1).float().to(DEV)


def _trees(cpu, B, L):
    """parent [B, L] (-1: none) of trees as drafting grows them -- a node continues the one before it or a late one --, and depth."""
    parent = torch.full((B, L), -1, dtype=torch.long)
    depth = torch.zeros(B, L, dtype=torch.long)
    r, pick = torch.rand(B, L, generator=cpu), torch.rand(B, L, generator=cpu)
    at = torch.arange(B)
    for t in range(1, L):
        late = max(0, t - 8) + (pick[:, t] * (t - max(0, t - 8))).long()
        p = torch.where(r[:, t] < 0.4, torch.full_like(late, t - 1), late)
        p = torch.where(r[:, t] > 0.93, -1, p)
        parent[:, t] = p
        depth[:, t] = torch.where(p >= 0, depth[at, p.clamp(min=0)] + 1, 0)
    return parent, depth


def _pages(s, g, n, D, dt=torch.bfloat16, fill=True):
    """A pool of n pages and one more (the plain form writes there what has no page)."""
    s.n_pages = n
    s.pages_k, s.pages_v = (torch.zeros(n + 1, BLOCK * D, dtype=torch.uint8, device=DEV) for _ in range(2))
    s.scales_k, s.scales_v = (torch.ones(n + 1, device=DEV) for _ in range(2))
    for codes, scales in ((s.pages_k, s.scales_k), (s.pages_v, s.scales_v)):
        for a in range(0, n + 1 if fill else 0, 1 << 14):
            m = min(1 << 14, n + 1 - a)
            codes[a:a + m], scales[a:a + m] = _eight_bits(_normal(g, (m, BLOCK * D), dt).float())


def _whole(parts):
    """Tensors of 2 or 4 bytes an element in one piece of memory: (it, how it stands now, views of it)."""
    flat = torch.cat([p.contiguous().view(torch.bfloat16).reshape(-1) for p in parts])
    live, views, at = flat.clone(), [], 0
    for p in parts:
        n = p.numel() * p.element_size() // 2
        views.append(live[at:at + n].view(p.dtype).view(p.shape))
        at += n
    return flat, live, views


def _some_rows(g, U, most):
    """10 % to 100 % of the most, and one unit in twenty that has evicted nearly everything."""
    rows = (most * (0.1 + 0.9 * torch.rand(U, generator=g, device=DEV))).round().int()
    rows[torch.rand(U, generator=g, device=DEV) < 0.05] = min(1, most)
    return rows


def _prepare_norm(s, c, g):
    B, L, Hq, Hkv, D, dt = c["B"], c["L"], c["Hq"], c["Hkv"], c["D"], TORCH[c["dtype"]]
    first = torch.randint(0, 2000, (B,), generator=g, device=DEV)
    s.table, s.sections = _table(2000 + L, D), _sections(c)
    s.pos = _by_axis(c, torch.arange(L, device=DEV)[None] + first[:, None])
    s.q, s.k = _normal(g, (B, Hq, L, D), dt), _normal(g, (B, Hkv, L, D), dt)
    s.wq, s.wk = ((1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dt) for _ in range(2))
    s.q_out, s.k_out = torch.empty_like(s.q), torch.empty_like(s.k)


def _prepare_tokens(s, c, g, cpu):
    B, L, Hq, Hkv, D, dt = c["B"], c["L"], c["Hq"], c["Hkv"], c["D"], TORCH[c["dtype"]]
    U, most = B * Hkv, c["max_len"]
    s.scale, s.sections = 1.0 / math.sqrt(D), _sections(c)
    parent, depth = _trees(cpu, B, L)
    # a sequence has seen about twice the rows that are held of it; nodes of one depth share a position
    first = torch.randint(max(0, 2 * most - 10), 2 * most + 1, (B, 1), generator=cpu)
    s.pos = _by_axis(c, (first + depth).to(DEV))
    s.table = _table(2 * most + L + 1, D)
    s.parent = parent.int().to(DEV)
    if c["kind"] == "tree":
        s.q = _normal(g, (B, Hq, L, D), dt)
        s.out = torch.empty_like(s.q)
    s.k, s.v = _normal(g, (B, Hkv, L, D), dt), _normal(g, (B, Hkv, L, D), dt)
    s.all_kept = c["keep_new"] >= 1.0
    s.flags = (torch.rand(B, Hkv, L, generator=g, device=DEV) < c["keep_new"]).to(torch.uint8)
    # a few drafted tokens are accepted; sometimes none
    near = torch.where(depth < 8, torch.rand(B, L, generator=cpu), -1.0).argmax(1)
    s.last = torch.where(torch.rand(B, generator=cpu) < 0.15, -1, near).int().to(DEV)
    rows = _some_rows(g, U, most)
    s.max_blocks = max(1, -(-(most + L) // BLOCK))
    _pages(s, g, U * s.max_blocks, D, dt, fill=most > 0)
    s.page = torch.randperm(s.n_pages, generator=g, device=DEV).int().view(U, s.max_blocks)
    # how tails and lengths stand when a pass begins (a program that keeps a conversation's state to answer from it again restores these)
    s.kept_state, s.live, (s.tail_k, s.tail_v, s.len) = _whole([_normal(g, (U, BLOCK * D), dt), _normal(g, (U, BLOCK * D), dt), rows])


def _fork_blocks(c):  # table entries of a sequence: its prompt's, what it has generated, and what it is given room for
    return (c["max_len"] + c["generated"] + c["rows"] + BLOCK) // BLOCK + 1


def _fork_pages(c):  # prompts' blocks, two generations of beams' own blocks, new room
    own_blocks = c["generated"] // BLOCK + 2
    return c["groups"] * c["Hkv"] * (c["max_len"] // BLOCK + 1 + c["beams"] * (2 * own_blocks + c["rows"] // BLOCK + 1))


def _prepare_fork(s, c, g, cpu):
    """Beams that have come from one prompt each: full blocks of the prompt shared by all, later ones by those with a common past."""
    N, W, H, D = c["groups"], c["beams"], c["Hkv"], c["D"]
    B, U = N * W, N * W * H
    s.max_blocks, n_pages = _fork_blocks(c), _fork_pages(c)
    _pages(s, g, n_pages, D, fill=False)
    prompt = _some_rows(g, N * H, c["max_len"]).cpu().view(N, 1, H).expand(N, W, H)
    made = torch.randint(c["generated"] // 2, c["generated"] + 1, (N, 1, H), generator=cpu).expand(N, W, H)
    rows = (prompt + made).reshape(U)
    shared = (prompt // BLOCK).reshape(U)
    blocks = rows // BLOCK
    j = torch.arange(s.max_blocks)[None]
    # one entry in three of the later blocks is another beam's: they share a past
    beam = torch.arange(B).view(N, W, 1).expand(N, W, H).reshape(U)
    head = torch.arange(H).view(1, 1, H).expand(N, W, H).reshape(U)
    group = beam // W
    other = group * W + torch.randint(0, W, (U,), generator=cpu)
    whose = torch.where(torch.rand(U, generator=cpu) < 0.33, torch.minimum(other, beam), beam)
    own_key = (whose * H + head)[:, None] * s.max_blocks + j
    key = torch.where(j < shared[:, None], -1 - ((group * H + head)[:, None] * s.max_blocks + j), own_key)
    names, index = torch.unique(key[j < blocks[:, None]], return_inverse=True)
    number = torch.randperm(n_pages, generator=cpu)[:names.numel()]
    page = torch.full((U, s.max_blocks), -1, dtype=torch.long)
    page[j < blocks[:, None]] = number[index]
    # the generation before: other beams of the same past, a row less each
    order = group * W + torch.randint(0, W, (U,), generator=cpu)
    old = (order.view(N, W, H)[:, :, :1].expand(N, W, H).reshape(U) * H + head)
    old_len = (rows[old] - 1).clamp(min=0)
    old_page = torch.where(j < (old_len // BLOCK)[:, None], page[old], -1)
    ref = torch.bincount(page[page >= 0], minlength=n_pages) + torch.bincount(old_page[old_page >= 0], minlength=n_pages)
    s.src_page, s.src_len = page.int().to(DEV), rows.int().to(DEV)
    s.src_k, s.src_v = _normal(g, (U, BLOCK * D), torch.bfloat16), _normal(g, (U, BLOCK * D), torch.bfloat16)
    s.dst_k, s.dst_v = torch.empty_like(s.src_k), torch.empty_like(s.src_v)
    s.parent = (torch.arange(N)[:, None] * W + torch.randint(0, W, (N, W), generator=cpu)).reshape(B).int().to(DEV)
    s.kept_state, s.live, (s.ref, s.page, s.len) = _whole([ref.int().to(DEV), old_page.int().to(DEV), old_len.int().to(DEV)])


def _prepare_compact(s, c, g, cpu):
    B, H, D = c["B"], c["Hkv"], c["D"]
    U = B * H
    rows = _some_rows(g, U, c["max_len"]).cpu().long()
    s.max_blocks = max(1, -(-c["max_len"] // BLOCK))
    _pages(s, g, U * s.max_blocks, D)
    page = torch.randperm(s.n_pages, generator=cpu).view(U, s.max_blocks)
    page = torch.where(torch.arange(s.max_blocks)[None] < (rows // BLOCK)[:, None], page, -1)
    # a prompt that several sequences began with: the first two blocks of one unit in four are the ones of the unit before
    twin = (torch.rand(U, generator=cpu) < 0.25) & (torch.arange(U) >= H)
    for u in torch.nonzero(twin).view(-1).tolist():
        n = min(2, int(rows[u]) // BLOCK, int(rows[u - H]) // BLOCK)
        page[u, :n] = page[u - H, :n]
    ref = torch.bincount(page[page >= 0], minlength=s.n_pages)
    s.which = (torch.rand(B, generator=cpu) < c["ended"]).to(torch.uint8).to(DEV)
    s.tail_k, s.tail_v = (torch.zeros(U, BLOCK * D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    s.moved = torch.empty(s.n_pages, dtype=torch.int32, device=DEV)
    s.used = torch.empty(1, dtype=torch.int32, device=DEV)
    s.kept_state, s.live, (s.ref, s.page, s.len, s.scales) = _whole(
        [ref.int().to(DEV), page.int().to(DEV), rows.int().to(DEV), torch.stack([s.scales_k[:-1], s.scales_v[:-1]])])


def prepare(case, seed):
    c, g, cpu, s = case, torch.Generator(device=DEV), torch.Generator(), State()
    g.manual_seed(int(seed))
    cpu.manual_seed(int(seed))
    s.case = dict(c)
    if c["kind"] == "norm":
        _prepare_norm(s, c, g)
    elif c["kind"] == "fork":
        _prepare_fork(s, c, g, cpu)
    elif c["kind"] == "compact":
        _prepare_compact(s, c, g, cpu)
    else:
        _prepare_tokens(s, c, g, cpu)
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


def _normed(x, w):
    x = x.float()
    return x * (1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)) * w.float()


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


def _plain_append(s, k, v, kept):
    """k (turned), v fp32 [U, L, D], kept [U, L]: the kept rows join the cache."""
    U, L, D = k.shape
    held = s.len.long() % BLOCK
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


def _ancestors(parent):
    """parent [B, L] -> [B, L, L]: node j is t or above it."""
    B, L = parent.shape
    j = torch.arange(L, device=parent.device)
    above = torch.eye(L, dtype=torch.bool, device=parent.device).expand(B, L, L)
    up = torch.where(parent >= 0, parent, torch.arange(L, device=parent.device)[None]).long()   # (a root's is itself)
    for _ in range(max(1, (L - 1).bit_length())):   # everything up to 2^i steps above
        above = above | above.gather(1, up[:, :, None].expand(B, L, L))
        up = up.gather(1, up)
    return above & (j[None] <= j[:, None])[None]


def _plain_tree(s, q, k, v, flags, blocks):
    """q [U, G, L, D], k, v [U, L, D] (turned) fp32, flags [U, L] -> [U, G, L, D]: over the rows held, kept ancestors and itself."""
    U, G, L, D = q.shape
    H = s.case["Hkv"]
    K = torch.cat([_held_rows(s, s.pages_k, s.scales_k, s.tail_k, _unpack_k, blocks), k], dim=1)
    V = torch.cat([_held_rows(s, s.pages_v, s.scales_v, s.tail_v, _unpack_v, blocks), v], dim=1)
    n = s.len.long()[:, None]
    i = torch.arange(blocks * BLOCK, device=q.device)[None]
    seen = torch.cat([i < n // BLOCK * BLOCK, torch.arange(BLOCK, device=q.device)[None] < n % BLOCK], dim=1)   # [U, rows held]
    above = _ancestors(s.parent).repeat_interleave(H, 0)
    mine = (above & (flags != 0)[:, None, :]) | torch.eye(L, dtype=torch.bool, device=q.device)[None]
    see = torch.cat([seen[:, None, :].expand(U, L, seen.shape[1]), mine], dim=2)[:, None]                   # [U, 1, L, rows]
    score = torch.matmul(q.reshape(U, G * L, D), K.transpose(1, 2).contiguous()).view(U, G, L, -1).mul_(s.scale)
    score.masked_fill_(~see, -math.inf)
    score.sub_(score.amax(-1, keepdim=True)).exp_()
    total = score.sum(-1, keepdim=True)
    V = torch.where(see.any(2).view(U, -1, 1), V, 0.0)   # rows that nobody sees hold whatever was there
    return torch.matmul(score.view(U, G * L, -1), V).view(U, G, L, D).div_(total)


def _plain_path(s):
    """[B, L]: the accepted node and those above it."""
    at = s.last.long()
    above = _ancestors(s.parent)
    path = above.gather(1, at.clamp(min=0)[:, None, None].expand(-1, 1, above.shape[2])).squeeze(1)
    return path & (at >= 0)[:, None]


def _named(page, n):
    """How many entries of a table name each of n pages."""
    return torch.zeros(n + 1, dtype=torch.int32, device=page.device).index_add_(
        0, torch.where(page >= 0, page, n).reshape(-1).long(), torch.ones(page.numel(), dtype=torch.int32, device=page.device))[:n]


def _plain_fork(s):
    c = s.case
    B, H, n = c["groups"] * c["beams"], c["Hkv"], s.n_pages
    U, j = B * H, torch.arange(s.max_blocks, device=DEV)[None]
    src = (s.parent.long()[:, None] * H + torch.arange(H, device=DEV)[None]).reshape(U)
    s.ref.sub_(_named(s.page, n))
    s.len.copy_(s.src_len[src])
    blocks = (s.len // BLOCK)[:, None]
    s.page.copy_(torch.where(j < blocks, s.src_page[src], -1))
    s.ref.add_(_named(s.page, n))
    s.dst_k.copy_(s.src_k[src])
    s.dst_v.copy_(s.src_v[src])
    # room for `rows` more: the free pages in order, to units and blocks in order
    want = (j >= blocks) & (j < ((s.len + c["rows"]) // BLOCK)[:, None]) & (s.page < 0)
    free = s.ref == 0
    rank = want.reshape(-1).long().cumsum(0).view(want.shape) - 1
    order = torch.argsort(torch.where(free, 0, 1), stable=True)
    got = want & (rank < free.sum())
    s.page.copy_(torch.where(got, order[rank.clamp(min=0, max=n - 1)].int(), s.page))
    s.ref.add_(_named(torch.where(got, s.page, -1), n))


def _plain_compact(s):
    c, n = s.case, s.n_pages
    gone = s.which.bool().repeat_interleave(c["Hkv"])
    s.ref.sub_(_named(torch.where(gone[:, None], s.page, -1), n))
    s.page.masked_fill_(gone[:, None], -1)
    s.len.masked_fill_(gone, 0)
    used = s.ref != 0
    count = used.sum()
    p = torch.arange(n, device=DEV)
    high, low = used & (p >= count), ~used & (p < count)     # as many of these as of those
    room = torch.argsort(torch.where(low, 0, 1), stable=True)
    to = torch.where(high, room[(high.long().cumsum(0) - 1).clamp(min=0)], p)
    s.moved.copy_(torch.where(used, to, -1))
    s.used.copy_(count)
    target = torch.where(high, to, n)                         # (the page past the last takes what does not move)
    for codes in (s.pages_k, s.pages_v):
        codes[target] = codes[:n].clone()
    for x in (s.scales[0], s.scales[1]):
        x.copy_(torch.cat([x, x[:1]]).scatter(0, target, x)[:n])
    s.ref.copy_(torch.zeros(n + 1, dtype=torch.int32, device=DEV).scatter(0, torch.where(used, to, n), s.ref)[:n])
    s.page.copy_(torch.where(s.page >= 0, s.moved[s.page.long().clamp(min=0)], -1))


def _flat(x):
    """[B, H, L, D] -> [B H, L, D]"""
    return x.reshape(-1, *x.shape[2:])


def _plain(s):
    c = s.case
    if c["kind"] == "fork":
        return _plain_fork(s)
    if c["kind"] == "compact":
        return _plain_compact(s)
    B, L, Hq, Hkv, D = c["B"], c["L"], c["Hq"], c["Hkv"], c["D"]
    U, G = B * Hkv, Hq // Hkv
    if c["kind"] == "norm":
        s.q_out.copy_(_turned(_normed(s.q, s.wq), s.table, s.pos, s.sections))
        s.k_out.copy_(_turned(_normed(s.k, s.wk), s.table, s.pos, s.sections))
        return
    k, v = _flat(_turned(s.k, s.table, s.pos, s.sections)), _flat(s.v).float()
    if c["kind"] == "tree":
        q = _turned(s.q, s.table, s.pos, s.sections)
        s.out.copy_(_plain_tree(s, q.view(U, G, L, D), k, v, _flat(s.flags), -(-c["max_len"] // BLOCK)).view(B, Hq, L, D))
    else:
        _plain_append(s, k, v, (_plain_path(s)[:, None] & (s.flags != 0)).view(U, L))


# ------------------------------------------------------------------------------------------- the framework's operators
def _handles(s):
    """What a program makes once and keeps: the context, the caches' and the positions' descriptions."""
    import paper_2410_12876_amd as ag
    c = s.case
    s.ag = ag
    if c["kind"] == "norm":
        s.rope, s.ctx = ag.Rope(s.table, s.pos, s.sections), ag.Context(0)
        return
    n = s.n_pages
    pool = (s.pages_k[:n], s.pages_v[:n], s.scales_k[:n], s.scales_v[:n])
    if c["kind"] == "fork":
        B = c["groups"] * c["beams"]
        s.src = ag.Q8Cache(*pool, s.src_k, s.src_v, s.src_page, s.src_len, B, c["Hkv"], c["D"])
        s.dst = ag.Q8Cache(*pool, s.dst_k, s.dst_v, s.page, s.len, B, c["Hkv"], c["D"])
        s.ctx = ag.Context(0, ag.q8_pool_workspace_bytes(B, c["Hkv"], n))
    elif c["kind"] == "compact":
        s.cache = ag.Q8Cache(*pool[:2], s.scales[0], s.scales[1], s.tail_k, s.tail_v, s.page, s.len, c["B"], c["Hkv"], c["D"])
        s.ctx = ag.Context(0, ag.q8_pool_workspace_bytes(c["B"], c["Hkv"], n))
    else:
        s.rope = ag.Rope(s.table, s.pos, s.sections)
        s.cache = ag.Q8Cache(*pool, s.tail_k, s.tail_v, s.page, s.len, c["B"], c["Hkv"], c["D"])
        s.ctx = ag.Context(0, ag.q8_tree_workspace_bytes(c["B"], c["L"], c["Hq"], c["Hkv"], c["D"], s.max_blocks))


def _own(s):
    if not hasattr(s, "ag"):
        _handles(s)
    ag, c = s.ag, s.case
    if c["kind"] == "norm":
        ag.ag_norm_rotate(s.ctx, s.q, s.k, s.wq, s.wk, EPS, s.rope, s.q_out, s.k_out)
    elif c["kind"] == "tree":
        ag.ag_q8_tree_attn(s.ctx, s.q, s.k, s.v, None if s.all_kept else s.flags, s.parent, s.rope, s.scale, s.cache, s.out)
    elif c["kind"] == "accept":
        ag.ag_q8_tree_append(s.ctx, s.k, s.v, None if s.all_kept else s.flags, s.parent, s.last, s.rope, s.cache)
    elif c["kind"] == "fork":
        ag.ag_q8_fork(s.ctx, s.src, s.parent, s.dst, s.ref)
        ag.ag_q8_reserve(s.ctx, s.dst, s.ref, c["rows"])
    else:
        ag.ag_q8_release(s.ctx, s.cache, s.ref, s.which)
        ag.ag_q8_compact_pages(s.ctx, s.cache, s.ref, s.moved, s.used)
        ag.ag_q8_remap(s.ctx, s.cache, s.moved)


def run(state):
    s, c = state, state.case
    if c["kind"] in ("accept", "fork", "compact"):
        s.live.copy_(s.kept_state)
    (_own if own else _plain)(s)
    if c["kind"] == "norm":
        return {"q": s.q_out, "k": s.k_out}
    if c["kind"] == "tree":
        return {"out": s.out}
    if c["kind"] == "fork":
        return {"ref": s.ref, "page": s.page, "len": s.len, "k_tail": s.dst_k, "v_tail": s.dst_v}
    got = {"k": s.pages_k[:s.n_pages].view(torch.float8_e4m3fn), "v": s.pages_v[:s.n_pages].view(torch.float8_e4m3fn), "len": s.len}
    if c["kind"] == "accept":
        return {**got, "k_scale": s.scales_k[:s.n_pages], "v_scale": s.scales_v[:s.n_pages], "k_tail": s.tail_k, "v_tail": s.tail_v}
    return {**got, "k_scale": s.scales[0], "v_scale": s.scales[1], "page": s.page, "ref": s.ref, "moved": s.moved, "used": s.used}


# ----------------------------------------------------------------------------------------------- what a pass must cost
def work(case):
    c = case
    if c["kind"] == "fork":  # tails in and out, both tables, lengths and counts
        U, e = c["groups"] * c["beams"] * c["Hkv"], _fork_blocks(c)
        return {"bytes": U * (2.0 * 2 * BLOCK * c["D"] * 2 + 12.0 * e + 8) + 8.0 * _fork_pages(c), "flops": 1.0 * U * e}
    if c["kind"] == "compact":  # pages that move in and out, the table, counts and the map
        U, e = c["B"] * c["Hkv"], max(1, -(-c["max_len"] // BLOCK))
        share = (1.0 - c["ended"]) * 0.95 * 0.55
        return {"bytes": U * e * (share * (1.0 - share) * 4.0 * BLOCK * c["D"] + 24.0), "flops": 1.0 * U * e}
    e = 2 if c["dtype"] == "bf16" else 4
    B, L, Hq, Hkv, D = c["B"], c["L"], c["Hq"], c["Hkv"], c["D"]
    angles = B * L * (D * 4 + c["axes"] * 4)
    if c["kind"] == "norm":
        n = B * L * (Hq + Hkv) * D
        return {"bytes": 2.0 * n * e + angles, "flops": 7.0 * n}
    U = B * Hkv
    if c["kind"] == "accept":  # a path of a few tokens, and the blocks that it completes
        rows = U * min(4.0, 0.5 * L + 0.5) * c["keep_new"]
        return {"bytes": rows * 2 * D * (2 * e + 1) + U * (L + 8) + B * 4.0 * (L + 1) + rows / BLOCK * 2 * BLOCK * D * 3, "flops": 3.0 * rows * D}
    held = U * (0.95 * 0.55 * c["max_len"] + 0.05)                 # rows at the start
    tails = U * min(31.5, 0.55 * c["max_len"])                     # ... of which these are in bf16
    nbytes = held * 2 * D + tails * 2 * D + B * L * (2 * Hq + 2 * Hkv) * D * e + angles + U * L
    return {"bytes": float(nbytes), "flops": 4.0 * D * Hq / Hkv * L * (held + U * min(6.0, L / 2))}


# --------------------------------------------------------------------------------------- the definition, in 64 bits
def _exact_turn(x, s):
    """x [B, H, L, D] in 64 bits, pair by pair."""
    y, half, first = x.double().clone(), x.shape[-1] // 2, 0
    for a, n in enumerate(s.sections):
        lo, hi = slice(first, first + n), slice(half + first, half + first + n)
        angle = s.table[s.pos[a].long()].double()[:, None]                    # [B, 1, L, D]
        c, sn = angle[..., lo], angle[..., hi]
        y[..., lo] = x[..., lo].double() * c - x[..., hi].double() * sn
        y[..., hi] = x[..., hi].double() * c + x[..., lo].double() * sn
        first += n
    return y


def _exact_norm(x, w):
    x = x.double()
    return x * torch.rsqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / x.shape[-1] + EPS) * w.double()


def _places(D, values):
    """Where value (row, column) of a block lies in its page: [64 D]."""
    t, d = torch.arange(BLOCK, device=DEV)[:, None], torch.arange(D, device=DEV)[None]
    if values:
        return ((d // 16) * 1024 + (t // 4 % 4) * 256 + (d % 16) * 16 + (t // 16) * 4 + t % 4).reshape(-1)
    return ((t // 16) * (D // 64) * 1024 + d // 64 * 1024 + (d // 16 % 4) * 256 + (t % 16) * 16 + d % 16).reshape(-1)


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


def _chains(parent):
    """For every node the list of itself and those above it, in order."""
    out = []
    for t, p in enumerate(parent):
        out.append((out[p] if p >= 0 else []) + [t])
    return out


def _exact_tree(s, c):
    B, L, Hq, H, D = c["B"], c["L"], c["Hq"], c["Hkv"], c["D"]
    G, q, k, v = Hq // H, _exact_turn(s.q, s), _exact_turn(s.k, s), s.v.double()
    places, lens, parents = [_places(D, False), _places(D, True)], s.len.tolist(), s.parent.tolist()
    out = torch.empty(B, Hq, L, D, dtype=torch.float64, device=DEV)
    for b in range(B):
        see = torch.zeros(L, L, dtype=torch.bool)
        for t, chain in enumerate(_chains(parents[b])):
            see[t, chain] = True
        see = see.to(DEV)
        for h in range(H):
            u = b * H + h
            n, ids = lens[u], s.page[u, :lens[u] // BLOCK].long()
            rows = []
            for codes, scales, tail, at in ((s.pages_k, s.scales_k, s.tail_k, places[0]), (s.pages_v, s.scales_v, s.tail_v, places[1])):
                full = (codes[ids].view(torch.float8_e4m3fn).double() * scales[ids].double()[:, None])[:, at].view(-1, D)
                rows.append(torch.cat([full, tail[u].double()[at].view(BLOCK, D)[:n % BLOCK]]))
            mine = see & (s.flags[b, h] != 0)[None]
            mine = mine | torch.eye(L, dtype=torch.bool, device=DEV)
            K, V = torch.cat([rows[0], k[b, h]]), torch.cat([rows[1], v[b, h]])
            for x in range(h * G, h * G + G):
                score = q[b, x] @ K.T * s.scale
                score[:, n:] = torch.where(mine, score[:, n:], -math.inf)
                out[b, x] = torch.softmax(score, dim=1) @ V
    return {"out": out}


def _exact_accept(s, c):
    B, L, H, D, n = c["B"], c["L"], c["Hkv"], c["D"], s.n_pages
    k, v = _exact_turn(s.k, s).float().to(torch.bfloat16).double(), s.v.double()
    codes = [x[:n].view(torch.float8_e4m3fn).double() for x in (s.pages_k, s.pages_v)]
    scales = [x[:n].double() for x in (s.scales_k, s.scales_v)]
    tails, places = [s.tail_k.double(), s.tail_v.double()], [_places(D, False), _places(D, True)]
    lens, parents, last, flags = s.len.tolist(), s.parent.tolist(), s.last.tolist(), s.flags.tolist()
    for b in range(B):
        path = _chains(parents[b])[last[b]] if last[b] >= 0 else []
        for h in range(H):
            u = b * H + h
            keep = [t for t in path if flags[b][h][t]]
            if not keep:
                continue
            held, block = lens[u] % BLOCK, lens[u] // BLOCK
            for x, new in enumerate((k[b, h, keep], v[b, h, keep])):
                rows = torch.cat([tails[x][u][places[x][:held * D]].view(-1, D), new])
                j = block
                while rows.shape[0] >= BLOCK:
                    page = int(s.page[u, j])
                    y, scales[x][page] = _exact_codes(rows[:BLOCK])
                    codes[x][page, places[x]] = y.reshape(-1)
                    rows, j = rows[BLOCK:], j + 1
                tails[x][u][places[x][:rows.shape[0] * D]] = rows.reshape(-1)
            lens[u] += len(keep)
    return {"k": codes[0], "v": codes[1], "len": torch.tensor(lens, dtype=torch.int32), "k_scale": scales[0], "v_scale": scales[1],
            "k_tail": tails[0], "v_tail": tails[1]}


def _exact_fork(s, c):
    H, W = c["Hkv"], c["groups"] * c["beams"]
    ref, page, lens = s.ref.tolist(), s.page.tolist(), []
    src_page, src_len, parent = s.src_page.tolist(), s.src_len.tolist(), s.parent.tolist()
    for row in page:
        for p in row:
            if p >= 0:
                ref[p] -= 1
    new, tails = [], []
    for b in range(W):
        for h in range(H):
            u = parent[b] * H + h
            tails.append(u)
            lens.append(src_len[u])
            done = src_len[u] // BLOCK
            new.append(src_page[u][:done] + [-1] * (s.max_blocks - done))
            for p in new[-1][:done]:
                ref[p] += 1
    free = iter([p for p, r in enumerate(ref) if r == 0])
    for u, row in enumerate(new):
        for j in range(lens[u] // BLOCK, min(s.max_blocks, (lens[u] + c["rows"]) // BLOCK)):
            row[j] = next(free, -1)
            if row[j] >= 0:
                ref[row[j]] = 1
    return {"ref": torch.tensor(ref, dtype=torch.int32), "page": torch.tensor(new, dtype=torch.int32), "len": torch.tensor(lens, dtype=torch.int32),
            "k_tail": torch.stack([s.src_k[u] for u in tails]).double(), "v_tail": torch.stack([s.src_v[u] for u in tails]).double()}


def _exact_compact(s, c):
    H, n = c["Hkv"], s.n_pages
    ref, page, lens, which = s.ref.tolist(), s.page.tolist(), s.len.tolist(), s.which.tolist()
    for u, row in enumerate(page):
        if which[u // H]:
            for j, p in enumerate(row):
                if p >= 0:
                    ref[p] -= 1
                row[j] = -1
            lens[u] = 0
    used = sum(r != 0 for r in ref)
    holes = [p for p in range(used) if ref[p] == 0]
    moved, count = [p if r else -1 for p, r in enumerate(ref)], [r if p < used else 0 for p, r in enumerate(ref)]
    source, target = [], []
    for p in range(used, n):
        if ref[p]:
            moved[p] = holes[len(source)]
            count[moved[p]] = ref[p]
            source.append(p)
            target.append(moved[p])
    got = {}
    at, to = torch.tensor(source, dtype=torch.long, device=DEV), torch.tensor(target, dtype=torch.long, device=DEV)
    for name, x in (("k", s.pages_k[:n].view(torch.float8_e4m3fn)), ("v", s.pages_v[:n].view(torch.float8_e4m3fn)), ("k_scale", s.scales[0]),
                    ("v_scale", s.scales[1])):
        y = x.double()
        y[to] = y[at]
        got[name] = y
    as_int = lambda x: torch.tensor(x, dtype=torch.int32)
    page = [[moved[p] if p >= 0 else -1 for p in row] for row in page]
    return {"k": got["k"], "v": got["v"], "len": as_int(lens), "k_scale": got["k_scale"], "v_scale": got["v_scale"], "page": as_int(page),
            "ref": as_int(count), "moved": as_int(moved), "used": as_int([used])}


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["kind"] == "norm":
        return {"q": _exact_turn(_exact_norm(s.q, s.wq), s), "k": _exact_turn(_exact_norm(s.k, s.wk), s)}
    return {"tree": _exact_tree, "accept": _exact_accept, "fork": _exact_fork, "compact": _exact_compact}[c["kind"]](s, c)

"""Pools of counted pages: reserve, fork, release, compact, remap, entry by entry against plain loops on the CPU (tree_reference)."""
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
import tree_reference as T
from gpu_util import DEV, ensure_built
from test_q8_gpu import BF, flags_of, gen, rope_of, some

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


class Pool:
    def __init__(self, g, n_pages, D):
        self.n, self.D = n_pages, D
        self.k, self.v = (torch.randint(0, 120, (n_pages, 64 * D), generator=g).to(torch.uint8).to(DEV) for _ in range(2))
        self.ks, self.vs = (torch.exp2(torch.randint(-9, 9, (n_pages,), generator=g).float()).to(DEV) for _ in range(2))
        self.ref = torch.zeros(n_pages, dtype=torch.int32, device=DEV)

    def cache(self, g, B, H, blocks, lens=None):
        U = B * H
        tails = [some(g, U, 64 * self.D).to(DEV) for _ in range(2)]
        length = torch.zeros(U, dtype=torch.int32) if lens is None else torch.tensor(lens, dtype=torch.int32)
        return ag.Q8Cache(self.k, self.v, self.ks, self.vs, *tails, torch.full((U, blocks), -1, dtype=torch.int32, device=DEV), length.to(DEV), B, H, self.D)

    def ctx(self, U):
        return ag.Context(0, ag.q8_pool_workspace_bytes(1, U, self.n))


def expect_capacity(ctx):
    with pytest.raises(ag.AgError) as e:
        ctx.poll_error()
    assert e.value.status == ag.AG_ECAPACITY
    ctx.poll_error()


@pytest.mark.parametrize("U,n_pages,blocks,rows", [(1, 1, 1, 64), (4, 9, 3, 64), (6, 5000, 40, 200), (1030, 9000, 5, 130), (3, 12289, 2100, 64 * 2000), (5, 20, 3, 0),
                                                      (1024, 8192, 30, 64 * 3 + 63), (1024, 8193, 30, 64 * 3 + 63), (1025, 3000, 4, 100), (7, 900, 40, 64 * 4), (1024, 700, 3, 64)])
def test_reserve(U, n_pages, blocks, rows):
    g = gen(U + n_pages)
    pool = Pool(g, n_pages, 64)
    c, ctx = pool.cache(g, U, 1, blocks, torch.randint(0, 64 * min(blocks, 3), (U,), generator=g).tolist()), pool.ctx(U)
    ref = (torch.rand(n_pages, generator=g) < 0.3).int() * 2          # pages that others hold
    page = torch.full((U, blocks), -1, dtype=torch.int32)
    page[0, 0] = n_pages + 5                                           # (no page either)
    pool.ref.copy_(ref)
    c.page.copy_(page)
    for _ in range(3):
        ag.ag_q8_reserve(ctx, c, pool.ref, rows)
        enough = T.reserve(page, c.len.cpu(), ref, rows)
        assert torch.equal(c.page.cpu(), page) and torch.equal(pool.ref.cpu(), ref)
        if enough:
            ctx.poll_error()
        else:
            expect_capacity(ctx)
        n = c.len.cpu() + torch.randint(0, 100, (U,), generator=g).int()
        c.len.copy_(n.clamp(max=64 * blocks))


def test_reserve_when_pages_run_out():
    """The last units and blocks stay without; a later call gives them what has become free."""
    g = gen(1)
    pool = Pool(g, 7, 64)
    c, ctx = pool.cache(g, 4, 1, 4, [0, 10, 64, 5]), pool.ctx(4)
    ag.ag_q8_reserve(ctx, c, pool.ref, 128)
    page, ref = torch.full((4, 4), -1, dtype=torch.int32), torch.zeros(7, dtype=torch.int32)
    assert not T.reserve(page, c.len.cpu(), ref, 128)
    assert torch.equal(c.page.cpu(), page) and torch.equal(pool.ref.cpu(), ref) and int((ref == 1).sum()) == 7
    expect_capacity(ctx)
    ag.ag_q8_release(ctx, c, pool.ref, torch.tensor([1, 0, 0, 0], dtype=torch.uint8, device=DEV))
    ag.ag_q8_reserve(ctx, c, pool.ref, 64)
    ref[page[0][page[0] >= 0].long()] = 0
    page[0] = -1
    assert T.reserve(page, c.len.cpu(), ref, 64)
    assert torch.equal(c.page.cpu(), page) and torch.equal(pool.ref.cpu(), ref)
    ctx.poll_error()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,B2,H,blocks,more", [(1, 1, 1, 1, 0), (2, 5, 3, 6, 2), (4, 4, 8, 20, 0), (3, 2, 1, 700, 1), (40, 60, 4, 3, 0)])
def test_fork(D, B, B2, H, blocks, more):
    """Two generations of beams, forth and back; parents that are not there; tables of different lengths."""
    g = gen(B + B2 + blocks + D)
    U, U2 = B * H, B2 * H
    pool = Pool(g, U * blocks + 9, D)
    a = pool.cache(g, B, H, blocks, torch.randint(0, 64 * blocks + 64, (U,), generator=g).tolist())
    b = pool.cache(g, B2, H, blocks + more)
    ctx = pool.ctx(max(U, U2))
    order = torch.randperm(pool.n, generator=g)[:U * blocks].int().view(U, blocks)
    order[0, 0] = pool.n + 3                                          # a full block without a page: rows that are not there
    a.page.copy_(order)
    pool.ref.copy_(T.count([order], pool.n))
    ref, page, length = pool.ref.cpu(), b.page.cpu(), b.len.cpu()
    for turn in range(3):
        parent = torch.randint(-1 if turn else 0, B + (1 if turn else 0), (B2,), generator=g).int()
        old = [b.k_tail.cpu(), b.v_tail.cpu()]
        ag.ag_q8_fork(ctx, a, parent.to(DEV), b, pool.ref)
        tails = T.fork((a.page.cpu(), a.len.cpu()), parent, page, length, ref, H)
        assert torch.equal(b.page.cpu(), page) and torch.equal(b.len.cpu(), length) and torch.equal(pool.ref.cpu(), ref)
        for x, (got, src) in enumerate(((b.k_tail, a.k_tail), (b.v_tail, a.v_tail))):
            got, src = got.cpu(), src.cpu()
            for u, v in enumerate(tails):
                assert torch.equal(got[u].view(torch.int16), (old[x][u] if v is None else src[v]).view(torch.int16))
        assert torch.equal(pool.ref.cpu(), T.count([a.page.cpu(), b.page.cpu()], pool.n))
    ag.ag_q8_release(ctx, b, pool.ref)
    assert torch.equal(pool.ref.cpu(), T.count([a.page.cpu()], pool.n)) and int(b.len.abs().sum()) == 0 and int(b.page.max()) == -1
    ctx.poll_error()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_pages,used", [(1, 0.0), (1, 1.0), (70, 0.5), (4096, 0.3), (4097, 0.97), (9000, 0.02), (13000, 0.6), (500, 0.0), (500, 1.0),
                                          (2, 0.5), (3, 0.4), (255, 0.9), (257, 0.1), (600, 0.5), (2047, 0.95), (2048, 0.5), (2049, 0.4)])
def test_compact(D, n_pages, used):
    g = gen(n_pages + D)
    pool = Pool(g, n_pages, D)
    ref = (torch.rand(n_pages, generator=g) < used).int() * torch.randint(1, 5, (n_pages,), generator=g).int()
    pool.ref.copy_(ref)
    B, blocks = 3, 50
    c = pool.cache(g, B, 1, blocks)
    table = torch.randint(-1, n_pages + 1, (B, blocks), generator=g).int()
    c.page.copy_(table)
    before = [x.clone() for x in (pool.k, pool.v, pool.ks, pool.vs)]
    moved, count, ctx = torch.full((n_pages,), 77, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV), pool.ctx(B)
    ag.ag_q8_compact_pages(ctx, c, pool.ref, moved, count)
    ag.ag_q8_remap(ctx, c, moved)
    want, new, n = T.compact(ref)
    assert int(count) == n and torch.equal(moved.cpu(), want) and torch.equal(pool.ref.cpu(), new)
    is_used = torch.nonzero(ref).view(-1)
    for x, y in zip((pool.k, pool.v, pool.ks, pool.vs), before):
        assert torch.equal(x.cpu()[want[is_used].long()], y.cpu()[is_used])
    inside = (table >= 0) & (table < n_pages)
    assert torch.equal(c.page.cpu(), torch.where(inside, want[table.clamp(0, n_pages - 1).long()], table))
    count.fill_(-1)
    ag.ag_q8_compact_pages(ctx, c, pool.ref, moved, count)  # now they are together
    at = torch.arange(n_pages)
    assert int(count) == n and torch.equal(moved.cpu().long(), torch.where(at < n, at, -1)) and torch.equal(pool.ref.cpu(), new)
    ctx.poll_error()


def test_beams_speculation_and_eviction_together():
    """A conversation as a program would have it: a prompt, three beams from it, trees verified and accepted over shared pages, a reorder, a
    sequence that ends, the pool moved together, decode steps; every unit's rows are those of a cache of its own that saw the same."""
    g, H, Hq, D, L, blocks, n_pages = gen(12), 2, 4, 64, 150, 8, 60
    B = 3
    pool = Pool(g, n_pages, D)
    one, a, b = pool.cache(g, 1, H, blocks), pool.cache(g, B, H, blocks), pool.cache(g, B, H, blocks)
    ctx = ag.Context(0, max(ag.q8_pool_workspace_bytes(B, H, n_pages), ag.q8_workspace_bytes(B, L, Hq, H, D, blocks), ag.q8_tree_workspace_bytes(B, 20, Hq, H, D, blocks)))
    host = lambda n: [[[torch.empty(0, D), torch.empty(0, D)] for _ in range(H)] for _ in range(n)]  # noqa: E731  rows of (sequence, head)

    # a reference cache per unit: appended rows in order
    def grown(rows, u, k, v):
        return [torch.cat([rows[0], k.bfloat16().float()]), torch.cat([rows[1], v.bfloat16().float()])]

    def check(cache, rows):
        for u in range(cache.B * H):
            r = R.Cache(1, 1, D, blocks, blocks, gen(0), [0], page=torch.arange(blocks).int().view(1, blocks))
            r.append(0, *rows[u // H][u % H])
            n = int(cache.len[u])
            assert n == int(r.len[0])
            for x, (codes, scale, tail) in enumerate(((cache.k, cache.k_scale, cache.k_tail), (cache.v, cache.v_scale, cache.v_tail))):
                at = R.places(D)[x].reshape(-1)
                for j in range(n // 64):
                    p = int(cache.page[u, j])
                    assert 0 <= p < n_pages and int(pool.ref[p]) > 0
                    got = codes[p].cpu().view(torch.float8_e4m3fn).float()
                    assert float(scale[p]) == float(r.scales[x][j]) and torch.equal(got, r.codes[x][j])
                assert torch.equal(tail[u].cpu().float()[at[:n % 64 * D]], r.tails[x][0][at[:n % 64 * D]])
        assert torch.equal(pool.ref.cpu(), T.count([one.page.cpu(), a.page.cpu(), b.page.cpu()], n_pages))

    # the prompt
    ag.ag_q8_reserve(ctx, one, pool.ref, L)
    q, k, v, f = some(g, 1, Hq, L, D), some(g, 1, H, L, D), some(g, 1, H, L, D), flags_of(g, "rand", 1, H, L)
    args, rope = rope_of(g, D, 1, L, 1, first=0)
    ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), f.to(DEV), rope, 0.1, one, torch.empty(q.shape, dtype=BF, device=DEV))
    kt = R.turned(k.float(), *args)
    first = host(1)
    for h in range(H):
        keep = f[0, h] != 0
        first[0][h] = grown(first[0][h], h, kt[0, h][keep], v[0, h].float()[keep])
    check(one, first)
    # three beams from it; what the prompt reserved and did not fill stays with it
    ag.ag_q8_fork(ctx, one, torch.zeros(B, dtype=torch.int32, device=DEV), a, pool.ref)
    beams = [[list(x) for x in first[0]] for _ in range(B)]
    check(a, beams)
    ag.ag_q8_release(ctx, one, pool.ref)
    cur, other = a, b
    for turn in range(4):
        n = 20
        ag.ag_q8_reserve(ctx, cur, pool.ref, n)
        q, k, v, f = some(g, B, Hq, n, D), some(g, B, H, n, D), some(g, B, H, n, D), flags_of(g, "rand", B, H, n)
        parent, last = T.random_tree(g, B, n), torch.randint(-1, n, (B,), generator=g).int()
        args, rope = rope_of(g, D, B, n, 1)
        out = torch.empty(q.shape, dtype=BF, device=DEV)
        turned = [torch.empty(x.shape, dtype=BF, device=DEV) for x in (q, k)]
        w = (1 + 0.1 * torch.randn(2, D, generator=g)).to(BF).to(DEV)
        ag.ag_norm_rotate(ctx, q.to(DEV), k.to(DEV), w[0], w[1], 1e-6, rope, *turned)
        ag.ag_q8_tree_attn(ctx, turned[0], turned[1], v.to(DEV), f.to(DEV), parent.to(DEV), None, 0.1, cur, out)
        ag.ag_q8_tree_append(ctx, turned[1], v.to(DEV), f.to(DEV), parent.to(DEV), last.to(DEV), None, cur)
        kt, qt = turned[1].cpu().float(), turned[0].cpu().float()
        for i in range(B):
            for h in range(H):
                r = R.Cache(1, 1, D, blocks, blocks, gen(0), [0], page=torch.arange(blocks).int().view(1, blocks))
                r.append(0, *beams[i][h])
                want = T.attend(r, qt[i:i + 1, 2 * h:2 * h + 2], kt[i:i + 1, h:h + 1], v[i:i + 1, h:h + 1], f[i:i + 1, h:h + 1] != 0, parent[i:i + 1], 0.1)
                got = out[i, 2 * h:2 * h + 2].double().cpu()
                assert ((got - want[0]).pow(2).mean(-1) / want[0].pow(2).mean(-1)).sqrt().max() <= 2.0 ** -9 + 1.2e-3
                keep = [t for t in T.path(parent[i], last[i]) if f[i, h, t]]
                beams[i][h] = grown(beams[i][h], h, kt[i, h][keep], v[i, h].float()[keep])
        check(cur, beams)
        order = torch.randint(0, B, (B,), generator=g)
        ag.ag_q8_fork(ctx, cur, order.int().to(DEV), other, pool.ref)
        beams = [[list(x) for x in beams[int(o)]] for o in order]
        check(other, beams)
        ag.ag_q8_release(ctx, cur, pool.ref)
        cur, other = other, cur
        if turn == 2:
            ag.ag_q8_release(ctx, cur, pool.ref, torch.tensor([0, 1, 0], dtype=torch.uint8, device=DEV))
            beams[1] = host(1)[0]
            moved, used = torch.empty(n_pages, dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)
            ag.ag_q8_compact_pages(ctx, cur, pool.ref, moved, used)
            for c in (one, a, b):
                ag.ag_q8_remap(ctx, c, moved)
            assert int((pool.ref[:int(used)] > 0).sum()) == int(used) == int((pool.ref > 0).sum())
            check(cur, beams)
    # decode steps go on over the shared pages
    for _ in range(70):
        ag.ag_q8_reserve(ctx, cur, pool.ref, 1)
        q, k, v = some(g, B, Hq, D), some(g, B, H, D), some(g, B, H, D)
        ag.ag_q8_decode_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), None, None, 0.1, cur, torch.empty(q.shape, dtype=BF, device=DEV))
        for i in range(B):
            for h in range(H):
                beams[i][h] = grown(beams[i][h], h, k[i, h:h + 1].float(), v[i, h:h + 1].float())
    check(cur, beams)
    ctx.poll_error()


def test_captured_and_replayed():
    """A beam step (fork, reserve) and a clean-up (release, compact, remap) as graphs, replayed with eager work in between."""
    g, B, H, D, blocks = gen(4), 4, 2, 64, 6
    pools = [Pool(gen(9), 80, D) for _ in range(2)]
    caches = [[p.cache(gen(8), B, H, blocks, [130, 64, 5, 200, 63, 128, 90, 191]), p.cache(gen(7), B, H, blocks)] for p in pools]
    ctxs = [p.ctx(B * H) for p in pools]
    for p, (a, b), c in zip(pools, caches, ctxs):
        ag.ag_q8_reserve(c, a, p.ref, 0)
        n = torch.arange(B * H * blocks, dtype=torch.int32, device=DEV).view(B * H, blocks)
        a.page.copy_(torch.where(torch.arange(blocks, device=DEV)[None] < (a.len // 64)[:, None], n, -1))
        p.ref.copy_(T.count([a.page.cpu()], p.n))
    parent, which = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.uint8, device=DEV)
    moved, used = [torch.zeros(80, dtype=torch.int32, device=DEV) for _ in range(2)], [torch.zeros(1, dtype=torch.int32, device=DEV) for _ in range(2)]

    def step(i):
        p, (a, b), c = pools[i], caches[i], ctxs[i]
        ag.ag_q8_fork(c, a, parent, b, p.ref)
        ag.ag_q8_reserve(c, b, p.ref, 70)
        ag.ag_q8_release(c, b, p.ref, which)
        ag.ag_q8_compact_pages(c, a, p.ref, moved[i], used[i])
        ag.ag_q8_remap(c, a, moved[i])
        ag.ag_q8_remap(c, b, moved[i])

    step(0)
    step(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for _ in range(6):
        parent.copy_(torch.randint(0, B, (B,), generator=g).int())
        which.copy_((torch.rand(B, generator=g) < 0.4).to(torch.uint8))
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        for x, y in zip(caches[0], caches[1]):
            assert torch.equal(x.page, y.page) and torch.equal(x.len, y.len) and torch.equal(x.k_tail, y.k_tail)
        assert torch.equal(pools[0].ref, pools[1].ref) and torch.equal(moved[0], moved[1]) and torch.equal(used[0], used[1])
        n = int(used[0])
        assert torch.equal(pools[0].k[:n], pools[1].k[:n])
        assert torch.equal(pools[0].ref.cpu(), T.count([x.page.cpu() for x in caches[0]], 80))
    ctxs[0].poll_error()

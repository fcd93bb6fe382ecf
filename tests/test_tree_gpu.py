"""Trees of drafted tokens over the paged 8-bit cache against plain loops on the CPU (tree_reference), output row by output row.

The bar of a row is on RMS(error) / RMS(row).  The store rounds to bf16: at most 2^-9 of the row in RMS (half a step, 2^-8, at the worst
element).  Before it queries are rounded to f16 (2^-12 / sqrt 3 = 1.4e-4 RMS of themselves), the nodes' keys to 16 bits (nothing beside it), weights
to f16 or 16 bits: scores of unit size times `spread` are off by 2e-4 spread, weights relatively by as much and by 1.4e-4.  A row that one or
two keys make up shows a single draw of that: five times its RMS, 1.2e-3 max(1, spread).  What a unit's cache holds is compared to the bit."""
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
import tree_reference as T
from gpu_util import DEV, ensure_built
from test_q8_gpu import BF, flags_of, gen, on_device, rope_of, same_cache, some

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def bar(spread=1.0):
    return 2.0 ** -9 + 1.2e-3 * max(1.0, spread)


def row_errors(got, want):
    got, want = got.double().cpu(), want.double()
    return ((got - want).pow(2).mean(-1) / want.pow(2).mean(-1).clamp(min=1e-300)).sqrt()


def tree_ctx(c, L, Hq):
    return ag.Context(0, ag.q8_tree_workspace_bytes(c.B, L, Hq, c.Hkv, c.D, c.max_blocks))


def cache_of(B, H, D, lens, room, g, values=0, width=0):
    """width: the table has so many columns, those behind the pages empty (a call chooses its tiles by the table, not by the lengths)."""
    blocks = (max(lens) + room) // 64 + 1
    c = R.Cache(B, H, D, B * H * blocks + 2, blocks, g, lens)
    if width > blocks:
        c.page, c.max_blocks = torch.cat([c.page, torch.full((B * H, width - blocks), -1, dtype=torch.int32)], 1), width
    c.scales[1] *= 2.0 ** values
    c.tails[1] *= 2.0 ** values
    return c


def tree_out(dev, ctx, q, k, v, f, parent, rope, scale):
    out = torch.full(q.shape, 7.0, dtype=BF, device=DEV)
    ag.ag_q8_tree_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), None if f is None else f.to(DEV), parent.to(DEV), rope, scale, dev, out)
    return out


def tree_both(ref, g, Hq, L, axes, kind, tree, scale=None, size=1.0, touch=None):
    """(device output, reference output)"""
    B, H, D = ref.B, ref.Hkv, ref.D
    scale = D ** -0.5 if scale is None else scale
    q, k, v = some(g, B, Hq, L, D), some(g, B, H, L, D), (some(g, B, H, L, D).float() * size).to(BF)
    f = None if kind is None else flags_of(g, kind, B, H, L)
    parent = T.random_tree(g, B, L, tree)
    if touch:
        touch(q, k, v, f, parent)
    args, rope = rope_of(g, D, B, L, axes) if axes else (None, None)
    dev, ctx = on_device(ref), tree_ctx(ref, L, Hq)
    out = tree_out(dev, ctx, q, k, v, f, parent, rope, scale)
    ctx.poll_error()
    again = tree_out(dev, ctx, q, k, v, f, parent, rope, scale)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)), "the same call twice"
    q64, k64 = (R.turned64(q.float(), *args), R.turned64(k.float(), *args)) if axes else (q, k)
    keep = torch.ones(B, H, L, dtype=torch.bool) if f is None else f != 0
    same_cache(dev, ref)
    return out, T.attend(ref, q64, k64, v, keep, parent, scale)


@pytest.mark.parametrize("B,Hq,H,D,L,lens,axes,kind,tree", [
    (1, 1, 1, 128, 1, [0], 1, None, "mixed"), (1, 2, 2, 64, 1, [5, 64], 0, "none", "mixed"), (1, 4, 4, 128, 2, [0, 1, 63, 64], 1, "rand", "mixed"),
    (2, 4, 2, 128, 12, [0, 3, 62, 200], 3, "rand", "mixed"), (1, 8, 1, 128, 33, [700], 1, None, "chain"), (1, 16, 2, 64, 64, [64, 129], 3, "rand", "mixed"),
    (1, 2, 2, 128, 65, [0, 63], 1, "rand", "chain"), (1, 2, 2, 64, 130, [31, 0], 1, "rand", "mixed"), (1, 4, 2, 128, 17, [3000, 100], 1, "rand", "star"),
    (3, 4, 4, 64, 31, [0, 64, 65, 128, 1, 2, 3, 4, 5, 6, 7, 191], 1, "all", "mixed"), (1, 16, 2, 128, 100, [63, 1000], 1, "rand", "roots"),
    (1, 4, 1, 128, 256, [77], 1, "rand", "mixed"), (1, 8, 8, 64, 256, [0, 1, 63, 64, 65, 127, 128, 300], 0, "rand", "mixed"),
    (1, 32, 4, 128, 16, [1500, 3, 777, 64], 1, None, "mixed"), (1, 8, 2, 64, 255, [1, 62], 1, "none", "chain"), (1, 1, 1, 64, 32, [62 + 64 * 31], 1, "rand", "mixed")])
def test_tree(B, Hq, H, D, L, lens, axes, kind, tree):
    g = gen(L + sum(lens) + D)
    print("tree", B, Hq, H, D, L, lens, kind, tree, flush=True)
    ref = cache_of(B, H, D, lens, 0, g)
    got, want = tree_both(ref, g, Hq, L, axes, kind, tree)
    e = row_errors(got, want)
    print("row errors: mean %.2e, worst %.2e" % (e.mean().item(), e.max().item()), flush=True)
    assert e.max() <= bar()


@pytest.mark.parametrize("U,Hq,H,D,L,longest", [(250, 10, 5, 64, 9, 700), (300, 4, 4, 128, 3, 400), (520, 8, 4, 64, 20, 100), (1100, 10, 10, 64, 2, 64), (40, 8, 8, 64, 5, 3000),
                                                (96, 64, 8, 64, 24, 1500)])
def test_tree_over_many_units(U, Hq, H, D, L, longest):
    """Ranges that cover several units, units that several ranges cover, several tiles of query rows a unit."""
    g = gen(U + D)
    lens = torch.randint(0, longest + 1, (U,), generator=g).tolist()
    lens[7], lens[U - 1], lens[0] = longest, 0, 63
    page = torch.randint(0, 9, (U, longest // 64 + 1), generator=g).int()
    ref = R.Cache(U // H, H, D, 9, longest // 64 + 1, g, lens, page=page)
    print("tree", U, Hq, H, D, L, longest, flush=True)
    got, want = tree_both(ref, g, Hq, L, 0, "rand", "mixed")
    e = row_errors(got, want)
    assert e.max() <= bar(), (e.max(), e.mean())


def test_a_chain_is_a_turn():
    """parent[t] = t - 1: the rows that ag_q8_prefill_attn and, node by node, ag_q8_decode_attn give."""
    g, B, Hq, H, D, L = gen(4), 2, 8, 2, 128, 40
    ref = cache_of(B, H, D, [100, 0, 63, 640], L, g)
    q, k, v, f = some(g, B, Hq, L, D), some(g, B, H, L, D), some(g, B, H, L, D), flags_of(g, "rand", B, H, L)
    _, rope = rope_of(g, D, B, L, 1)
    ctx = ag.Context(0, max(ag.q8_tree_workspace_bytes(B, L, Hq, H, D, ref.max_blocks), ag.q8_workspace_bytes(B, L, Hq, H, D, ref.max_blocks)))
    tree = tree_out(on_device(ref), ctx, q, k, v, f, T.random_tree(g, B, L, "chain"), rope, 0.1)
    turn = torch.empty_like(tree)
    ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), f.to(DEV), rope, 0.1, on_device(ref), turn)
    assert row_errors(tree, turn.cpu()).max() <= 2 * bar()
    ctx.poll_error()


@pytest.mark.parametrize("values", [-100, -60, -20, -6, 20, 60, 100])
@pytest.mark.parametrize("D,lens", [(128, [0, 700, 30, 64]), (64, [130, 64, 63, 0])])
def test_values_of_any_size(D, lens, values):
    """The cache's values 2^values as large as the usual, the nodes' of unit size, and the other way round."""
    g = gen(values + 200 + D)
    for cached, own in ((values, 0), (0, values), (values, values)):
        ref = cache_of(1, 4, D, lens, 0, g, values=cached)
        got, want = tree_both(ref, g, 8, 20, 1, "rand", "mixed", size=2.0 ** own)
        e = row_errors(got, want)
        print("values", values, cached, own, "%.2e" % e.max().item(), flush=True)
        assert e.max() <= bar()


# Widths of a table with which a tile has one, two and four groups of 32 rows, where the rows are that many.
WIDTHS = [0, 1000, 5000]


@pytest.mark.parametrize("a_cu", [60, 120])
@pytest.mark.parametrize("B,Hq,H,D,L,lens,axes,kind,tree", [
    (1, 16, 2, 64, 64, [64, 1500], 3, "rand", "mixed"), (1, 4, 2, 128, 33, [3000, 100], 1, "rand", "star"), (1, 4, 4, 128, 200, [0, 65, 128, 777], 1, "none", "chain"),
    (2, 16, 2, 128, 12, [0, 3, 62, 2000], 3, "rand", "mixed"), (1, 8, 1, 128, 256, [700], 1, "rand", "mixed"), (1, 2, 2, 64, 97, [63, 64 * 70], 0, None, "roots")])
def test_tree_in_larger_tiles(B, Hq, H, D, L, lens, axes, kind, tree, a_cu):
    g, tiles = gen(L + D + a_cu), (L * Hq // H + 31) // 32
    ref = cache_of(B, H, D, lens, 0, g, width=a_cu * 256 // (B * H * tiles) + 1)
    got, want = tree_both(ref, g, Hq, L, axes, kind, tree)
    e = row_errors(got, want)
    print("tree", B, Hq, H, D, L, lens, a_cu, "%.2e" % e.max().item(), flush=True)
    assert e.max() <= bar()


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("D,lens", [(128, [64 * 9 + 5, 64 * 20]), (64, [64 * 5, 64 * 40 + 63])])
def test_pages_of_different_sizes(D, lens, width):
    """Blocks of zeros (their rows count in the row sum), blocks 2^-60 to 2^60 as large as others, keys of different sizes."""
    g = gen(D + 7)
    for kind in ("zeros", "small", "large", "mixed", "keys"):
        ref = cache_of(1, 2, D, lens, 0, g, width=width)
        n = ref.n_pages
        if kind == "zeros":
            some_pages = torch.rand(n, generator=g) < 0.5
            ref.codes[1][some_pages] = 0.0
            ref.scales[1][some_pages] = 2.0 ** -100
        elif kind == "keys":
            size = torch.exp2(torch.randint(-8, 1, (n,), generator=g).float())
            ref.scales[0] *= size
        else:
            lo, hi = {"small": (-60, 1), "large": (0, 61), "mixed": (-60, 61)}[kind]
            ref.scales[1] *= torch.exp2(torch.randint(lo, hi, (n,), generator=g).float())
        got, want = tree_both(ref, g, 8, 20, 1, "rand", "mixed")
        e = row_errors(got, want)
        print("pages", kind, "%.2e" % e.max().item(), flush=True)
        assert e.max() <= bar()


@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** -20, 2.0 ** 20, 2.0 ** 60])
def test_queries_of_any_size(size):
    """The scores are the usual ones: the scale makes up for it."""
    g, D = gen(31), 128

    def touch(q, k, v, f, parent):
        q *= size

    got, want = tree_both(cache_of(1, 2, D, [100, 300], 0, g), g, 4, 12, 1, "rand", "mixed", scale=D ** -0.5 / size, touch=touch)
    assert row_errors(got, want).max() <= bar()


@pytest.mark.parametrize("L,width", [(10, 0)] + [(70, w) for w in WIDTHS])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_the_cache_that_are_not_finite(D, L, width):
    """In the tail (taken one by one) and in pages: columns of a value that is not finite are not finite, everything else is as it should be."""
    g, H = gen(D + 3), 4
    ref = cache_of(1, H, D, [64 + 20, 64 + 20, 64 * 2 + 5, 64 * 2 + 5], 0, g, width=width)
    at = R.places(D)
    ref.tails[1][0][at[1][7, 3]], ref.tails[1][0][at[1][19, 9]] = float("inf"), float("nan")
    ref.tails[0][1][at[0][11, 2]] = float("nan")                      # a key: every row of the unit
    ref.codes[1][ref.page[2, 1]][at[1][40, 5]] = float("nan")
    ref.codes[0][ref.page[3, 0]][at[0][1, 1]] = float("nan")
    got, want = tree_both(ref, g, H, L, 0, "rand", "mixed")
    got = got.cpu()
    for u in range(H):
        for t in range(L):
            a, b = got[0, u, t].double(), want[0, u, t]
            assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a[torch.isinf(b)], b[torch.isinf(b)])
            fine = torch.isfinite(b)
            if fine.any():
                assert (a[fine] - b[fine]).pow(2).mean().sqrt() <= bar() * b[fine].pow(2).mean().sqrt()
    assert torch.isnan(want[0, 1]).all() and torch.isnan(want[0, 3]).all() and torch.isinf(want[0, 0, 0, 3]) and torch.isnan(want[0, 2, 0, 5])


@pytest.mark.parametrize("spread", [3.0, 7.0, 30.0])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("D,lens", [(128, [0, 700]), (64, [130, 64])])
def test_sharp_scores(D, lens, spread, width):
    g = gen(int(spread) + D)
    got, want = tree_both(cache_of(1, 2, D, lens, 0, g, width=width), g, 8, 50, 1, "rand", "mixed", scale=spread * D ** -0.5)
    e = row_errors(got, want)
    print("spread", spread, "%.2e mean %.2e" % (e.max().item(), e.mean().item()), flush=True)
    assert e.max() <= bar(spread)


def test_many_small_weights():
    """A row that one key dominates by 2^17 to 2^25 beside thousands of others: their sum counts."""
    g, D, n = gen(9), 64, 6000
    for gap in (9.0, 13.0, 17.0):
        ref = cache_of(1, 1, D, [n], 0, g)
        ref.codes[0].zero_()
        ref.tails[0].zero_()
        ref.scales[0].fill_(1.0)
        q, k = torch.zeros(1, 1, 2, D, dtype=BF), torch.zeros(1, 1, 2, D, dtype=BF)
        q[..., 0], k[..., 0] = 1.0, gap
        v = some(g, 1, 1, 2, D)
        ref.codes[1], ref.tails[1] = ref.codes[1].abs(), ref.tails[1].abs()
        dev, ctx, parent = on_device(ref), tree_ctx(ref, 2, 1), torch.tensor([[-1, -1]], dtype=torch.int32)
        got = tree_out(dev, ctx, q, k, v, None, parent, None, 1.0)
        want = T.attend(ref, q, k, v, torch.ones(1, 1, 2, dtype=torch.bool), parent, 1.0)
        e = row_errors(got, want)
        print("gap", gap, e.view(-1).tolist(), flush=True)
        assert e.max() <= bar()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("length,width", [(0, 0), (30, 0), (100, 0), (30, 1000), (100, 5000)])
def test_what_a_node_does_not_see_does_not_reach_it(D, length, width):
    """Infinities and NaN in keys and values of nodes, and in rows of the tail that are not there: only those below them see them, and the rest
    has the bits of a clean run."""
    g, L, H, Hq = gen(D + length), 70, 2, 4
    ref = cache_of(1, H, D, [length] * H, 0, g, width=width)
    parent = T.random_tree(g, 1, L)
    q, k, v, f = some(g, 1, Hq, L, D), some(g, 1, H, L, D), some(g, 1, H, L, D), flags_of(g, "rand", 1, H, L)
    ctx = tree_ctx(ref, L, Hq)
    clean = tree_out(on_device(ref), ctx, q, k, v, f, parent, None, 0.1).cpu()
    at = R.places(D)
    for x in range(2):
        ref.tails[x][:, at[x][length % 64:].reshape(-1)] = float("nan")
    bad = {5: ("k", float("nan")), 11: ("v", float("inf")), 23: ("v", float("nan")), 40: ("k", float("inf")), 66: ("v", float("-inf"))}
    for t, (which, value) in bad.items():
        (k if which == "k" else v)[0, :, t, 3] = value
    got = tree_out(on_device(ref), ctx, q, k, v, f, parent, None, 0.1).cpu()
    want = T.attend(ref, q, k, v, f != 0, parent, 0.1)
    touched = 0
    for h in range(Hq):
        for t, chain in enumerate(T.chains(parent[0])):
            seen = [x for x in chain[:-1] if f[0, h // 2, x]] + [t]
            row, ref_row = got[0, h, t], want[0, h, t]
            if any(x in bad for x in seen):
                touched += 1
                assert torch.equal(torch.isnan(row), torch.isnan(ref_row)), (h, t)
                fine = torch.isfinite(ref_row)
                assert torch.equal(row[~fine & ~torch.isnan(row)].double(), ref_row[~fine & ~torch.isnan(ref_row)])
                if fine.any():
                    assert (row[fine].double() - ref_row[fine]).pow(2).mean().sqrt() <= bar() * ref_row[fine].pow(2).mean().sqrt()
            else:
                assert torch.equal(row.view(torch.int16), clean[0, h, t].view(torch.int16)), (h, t)
    assert touched > 20
    ctx.poll_error()


def test_scores_that_overflow():
    """A node that sees nothing else gets its value whatever its score is; a score of -infinity of its own counts as the least number."""
    g, D, L, H = gen(3), 64, 6, 2
    ref = cache_of(1, H, D, [0, 0], 0, g)
    q, k, v = some(g, 1, H, L, D), some(g, 1, H, L, D), some(g, 1, H, L, D)
    q[:], k[:] = 3e38, -3e38
    f = torch.zeros(1, H, L, dtype=torch.uint8)
    parent = T.random_tree(g, 1, L, "chain")
    ctx = tree_ctx(ref, L, H)
    got = tree_out(on_device(ref), ctx, q, k, v, f, parent, None, 1.0)
    assert torch.equal(got.cpu(), v)
    k[:, :, 0] = float("nan")
    got = tree_out(on_device(ref), ctx, q, k, v, f, parent, None, 1.0)
    assert torch.equal(got.cpu(), v)
    # node 0 is kept, its score 0: the others' own ones overflow
    k[:, :, 0], f[:, :, 0] = 0.0, 1
    got = tree_out(on_device(ref), ctx, q, k, v, f, parent, None, 1.0)
    assert torch.equal(got.cpu(), v[:, :, :1].expand_as(v))
    ctx.poll_error()


def test_pages_outside_the_pool_are_rows_that_are_not_there():
    g, D, H = gen(8), 128, 4
    ref = cache_of(1, H, D, [400, 64, 128, 1000], 0, g)
    ref.page[0, 1], ref.page[0, 5], ref.page[1, 0], ref.page[3, 2] = -1, ref.n_pages, -7, 1 << 30
    got, want = tree_both(ref, g, 8, 9, 1, "rand", "mixed")
    assert row_errors(got, want).max() <= bar()


def test_a_parent_that_is_not_before_its_node_is_reported():
    g, D, L = gen(2), 64, 10
    ref = cache_of(1, 2, D, [70, 5], L, g)
    ctx, dev = tree_ctx(ref, L, 2), on_device(ref)
    q, k, v = some(g, 1, 2, L, D), some(g, 1, 2, L, D), some(g, 1, 2, L, D)
    parent = T.random_tree(g, 1, L)
    parent[0, 4], parent[0, 6] = 4, 2000000000
    got = tree_out(dev, ctx, q, k, v, None, parent, None, 0.1)
    with pytest.raises(ag.AgError) as e:
        ctx.poll_error()
    assert e.value.status == ag.AG_EINVAL
    ctx.poll_error()
    assert row_errors(got, T.attend(ref, q, k, v, torch.ones(1, 2, L, dtype=torch.bool), parent, 0.1)).max() <= bar()
    for last in (L, 2000000000, 6, 4):
        before = dev.len.clone()
        ag.ag_q8_tree_append(ctx, k.to(DEV), v.to(DEV), None, parent.to(DEV), torch.tensor([last], dtype=torch.int32, device=DEV), None, dev)
        with pytest.raises(ag.AgError) as e:
            ctx.poll_error()
        assert e.value.status == ag.AG_EINVAL
        assert torch.equal(dev.len - before, torch.full_like(before, len(T.path(parent[0], last))))


# ------------------------------------------------------------------------------------------------------------------ the accepted path
@pytest.mark.parametrize("B,H,D,L,lens,kind,axes,tree", [
    (1, 1, 128, 1, [0], None, 1, "mixed"), (2, 3, 64, 12, [0, 1, 63, 64, 65, 100], "rand", 1, "mixed"), (1, 4, 128, 64, [5, 60, 128, 191], "rand", 3, "chain"),
    (3, 2, 128, 31, [62, 63, 0, 127, 60, 61], None, 0, "mixed"), (1, 2, 64, 256, [3, 63], "rand", 1, "chain"), (1, 2, 128, 256, [0, 64], None, 1, "mixed"),
    (5, 1, 64, 7, [63, 62, 61, 60, 59], "all", 1, "star"), (2, 1, 64, 200, [10, 20], "none", 1, "chain")])
def test_the_accepted_path_joins_the_cache(B, H, D, L, lens, kind, axes, tree):
    g = gen(L + D + B)
    for last in ("deep", "some", "none"):
        ref = cache_of(B, H, D, lens, L, g)
        dev, ctx = on_device(ref), ag.Context(0)
        k, v, parent = some(g, B, H, L, D), some(g, B, H, L, D), T.random_tree(g, B, L, tree)
        f = None if kind is None else flags_of(g, kind, B, H, L)
        at = torch.full((B,), -3) if last == "none" else torch.randint(-1, L, (B,), generator=g) if last == "some" else torch.full((B,), L - 1)
        args, rope = rope_of(g, D, B, L, axes) if axes else (None, None)
        print("accept", B, H, D, L, lens, kind, last, flush=True)
        ag.ag_q8_tree_append(ctx, k.to(DEV), v.to(DEV), None if f is None else f.to(DEV), parent.to(DEV), at.int().to(DEV), rope, dev)
        kt = R.turned(k.float(), *args) if axes else k.float()
        for u in range(B * H):
            b, h = divmod(u, H)
            keep = [t for t in T.path(parent[b], at[b]) if f is None or f[b, h, t]]
            ref.append(u, kt[b, h][keep], v[b, h].float()[keep])
        same_cache(dev, ref)
        ctx.poll_error()


def test_an_accepted_path_without_room_is_reported():
    g, D, L = gen(1), 64, 100
    ref = R.Cache(1, 2, D, 2, 1, g, [10, 60])
    dev, ctx = on_device(ref), ag.Context(0)
    k, v, parent = some(g, 1, 2, L, D), some(g, 1, 2, L, D), T.random_tree(g, 1, L, "chain")
    ag.ag_q8_tree_append(ctx, k.to(DEV), v.to(DEV), None, parent.to(DEV), torch.tensor([L - 1], dtype=torch.int32, device=DEV), None, dev)
    with pytest.raises(ag.AgError) as e:
        ctx.poll_error()
    assert e.value.status == ag.AG_ECAPACITY
    for u in range(2):
        ref.append(u, k[0, u].float(), v[0, u].float())
    same_cache(dev, ref)


# ---------------------------------------------------------------------------------------------------------------- streams, graphs, order
def test_captured_and_replayed():
    """Verification and acceptance as one graph, replayed over changing inputs with eager work in between: bit for bit the eager result."""
    g, B, Hq, H, D, L = gen(6), 2, 8, 2, 128, 20
    ref = cache_of(B, H, D, [100, 0, 63, 640], 12 * L, g)
    dev, twin = on_device(ref), on_device(ref)
    one = lambda: (some(g, B, Hq, L, D).to(DEV), some(g, B, H, L, D).to(DEV), some(g, B, H, L, D).to(DEV), flags_of(g, "rand", B, H, L).to(DEV),  # noqa: E731
                   T.random_tree(g, B, L).to(DEV), torch.randint(-1, L, (B,), generator=g).int().to(DEV))
    static, out = one(), torch.empty(B, Hq, L, D, dtype=BF, device=DEV)
    (_, rope), ctx, eager = rope_of(g, D, B, L, 1), tree_ctx(ref, L, Hq), tree_ctx(ref, L, Hq)

    def step(c, cache, q, k, v, f, parent, last, o):
        ag.ag_q8_tree_attn(c, q, k, v, f, parent, rope, 0.1, cache, o)
        ag.ag_q8_tree_append(c, k, v, f, parent, last, rope, cache)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(ctx, dev, *static, out)
        step(eager, twin, *static, torch.empty_like(out))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ctx, dev, *static, out)
    for _ in range(6):
        new = one()
        for a, b in zip(static, new):
            a.copy_(b)
        graph.replay()
        want = torch.empty_like(out)
        step(eager, twin, *new, want)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        for name in ("k", "v", "k_scale", "v_scale", "len"):
            assert torch.equal(getattr(dev, name), getattr(twin, name)), name
    ctx.poll_error()


def test_two_contexts_at_once():
    g, B, Hq, H, D, L = gen(7), 4, 8, 2, 128, 30
    refs = [cache_of(B, H, D, torch.randint(0, 2000, (B * H,), generator=g).tolist(), 0, g) for _ in range(2)]
    devs, ins = [on_device(r) for r in refs], []
    for _ in range(2):
        ins.append((some(g, B, Hq, L, D).to(DEV), some(g, B, H, L, D).to(DEV), some(g, B, H, L, D).to(DEV), T.random_tree(g, B, L).to(DEV)))
    ctxs, streams = [tree_ctx(r, L, Hq) for r in refs], [torch.cuda.Stream() for _ in range(2)]
    want = []
    for i in range(2):
        o = torch.empty(B, Hq, L, D, dtype=BF, device=DEV)
        ag.ag_q8_tree_attn(ctxs[i], *ins[i][:3], None, ins[i][3], None, 0.1, devs[i], o)
        want.append(o)
    torch.cuda.synchronize()
    got = [[torch.empty_like(want[0]) for _ in range(10)] for _ in range(2)]
    for n in range(10):
        for i in range(2):
            ag.ag_q8_tree_attn(ctxs[i], *ins[i][:3], None, ins[i][3], None, 0.1, devs[i], got[i][n], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for o in got[i]:
            assert torch.equal(o.view(torch.int16), want[i].view(torch.int16))

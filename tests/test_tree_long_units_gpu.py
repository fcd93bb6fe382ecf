"""Trees over units of more pages than a wave looks up at a time (64), in tiles of one, two and four groups of rows, against plain loops.

255 units on 256 CUs: each is one workgroup's, but the longest, which two share.  The bar of a row is on RMS(error) / RMS(row): at most 2^-9 from the
store; queries, the nodes' keys and weights are f16, 2^-12 / sqrt 3 = 1.4e-4 RMS of themselves each, so a score of unit size is off by 2e-4 and a weight by
2.5e-4; five times that for a row that one or two keys make up."""
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
import tree_reference as T
from gpu_util import DEV, ensure_built
from test_q8_gpu import BF, flags_of, gen, on_device, some

pytestmark = pytest.mark.gpu
BAR = 2.0 ** -9 + 1.2e-3
B, H, POOL = 51, 5, 48


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def of_unit(c, u):
    """Unit u of a reference cache as a cache of its own."""
    one = R.Cache.__new__(R.Cache)
    one.B = one.Hkv = 1
    one.D, one.n_pages, one.max_blocks, one.codes, one.scales = c.D, c.n_pages, c.max_blocks, c.codes, c.scales
    one.page, one.len, one.tails = c.page[u:u + 1], c.len[u:u + 1], [x[u:u + 1] for x in c.tails]
    return one


@pytest.mark.parametrize("D,L,G,waves", [(64, 17, 4, 2), (128, 17, 4, 2), (64, 9, 4, 4), (64, 3, 2, 8), (128, 3, 2, 8)])
def test_more_pages_than_are_looked_up_at_a_time(D, L, G, waves):
    """waves: those that share a group's pages, so 64 times as many are a wave's first part."""
    g, first = gen(D + waves), 64 * waves
    n = first + 6
    blocks = 2 * n + 6
    lens = (torch.randint(0, 64, (B * H,), generator=g) + 64 * n).tolist()
    # pages [0, 16): usual, [16, 32): values 2^20 as large, [32, 48): zeros
    page = torch.randint(0, 16, (B * H, blocks), generator=g).int()
    none, large, zeros = torch.full((blocks,), POOL + 3).int(), page[0] + 16, page[0] + 32
    lens[0], lens[1], lens[8] = 64 * first + 5, 64 * (first + 1), 64 * blocks + 63
    page[2, :first] = none[:first]                                  # nothing in the first part
    page[3] = torch.where(torch.rand(blocks, generator=g) < 0.5, page[3], -1)
    page[4, first:] = large[first:]                                 # larger values in the second part, in the first, zeros in either
    page[5, :first] = large[:first]
    page[6, :first] = zeros[:first]
    page[7, first:] = none[first:]
    page[9, first:] = zeros[first:]
    ref = R.Cache(B, H, D, POOL, blocks, g, lens, page=page)
    ref.scales[1][16:32] *= 2.0 ** 20
    ref.codes[1][32:], ref.scales[1][32:] = 0.0, 2.0 ** -100
    q, k, v, f, parent = some(g, B, H * G, L, D), some(g, B, H, L, D), some(g, B, H, L, D), flags_of(g, "rand", B, H, L), T.random_tree(g, B, L)
    ctx = ag.Context(0, ag.q8_tree_workspace_bytes(B, L, H * G, H, D, blocks))
    dev, out = on_device(ref), torch.full(q.shape, 7.0, dtype=BF, device=DEV)
    print("tree", D, L, G, waves, blocks, flush=True)
    for _ in range(2):
        ag.ag_q8_tree_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), f.to(DEV), parent.to(DEV), None, D ** -0.5, dev, out)
    got = out.double().cpu()
    assert bool(torch.isfinite(got).all())
    for u in [*range(10), 100, 254]:
        b, h = divmod(u, H)
        heads = slice(h * G, h * G + G)
        want = T.attend(of_unit(ref, u), q[b:b + 1, heads], k[b:b + 1, h:h + 1], v[b:b + 1, h:h + 1], f[b:b + 1, h:h + 1] != 0, parent[b:b + 1], D ** -0.5)[0]
        e = ((got[b, heads] - want).pow(2).mean(-1) / want.pow(2).mean(-1)).sqrt().max().item()
        print("unit", u, int(ref.len[u]), "%.2e" % e, flush=True)
        assert e <= BAR, (u, e)
    ctx.poll_error()

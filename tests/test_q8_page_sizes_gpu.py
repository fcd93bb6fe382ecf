"""Attention over units whose pages hold values of very different sizes (blocks of zeros have the least scale there is, 2^-100), row by row.

The bar of a row is on RMS(error) / RMS(row).  The store rounds an element by at most 2^-9 of itself, so at most 2^-9 of the row.  Before it queries,
the call's own keys, and weights are rounded to f16, each to within 2^-12 / sqrt 3 = 1.4e-4 RMS of itself: a score of unit size is off by 1.4e-4
sqrt 2 = 2e-4, a weight relatively by as much and by its own 1.4e-4, together 2.5e-4; a row that one or two keys make up shows a single draw, so five
times that, 1.2e-3.  What some pages are preferred by is a product of powers of two (8 in the query, 64 in the key) and so exact."""
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
import tree_reference as T
from gpu_util import DEV, ensure_built
from test_q8_gpu import BF, flags_of, gen, on_device, some

pytestmark = pytest.mark.gpu
BAR = 2.0 ** -9 + 1.2e-3


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def cache(g, B, H, D, longest, kind, bits, room=0):
    """Units of 0 to `longest` rows over few pages that they share (the blocks that `room` more rows can fill have pages of their own).  Half of the pages are
    zeros: beside others 2^bits as large as usual; tiny: of the least scale, beside such;
    small: 2^-bits as large as usual, and preferred (a score higher by 512 / sqrt D); preferred: of zeros, and preferred."""
    U = B * H
    lens = torch.randint(0, longest + 1, (U,), generator=g).tolist()
    lens[U // 2] = longest
    own = (room + 63) // 64 + 1
    blocks, shared = longest // 64 + own, U * own
    page = torch.randint(shared, shared + 16, (U, blocks), generator=g).int()
    for u in range(U):
        page[u, lens[u] // 64:lens[u] // 64 + own] = torch.arange(u * own, u * own + own)
    c = R.Cache(B, H, D, shared + 16, blocks, g, lens, page=page)
    at = R.places(D)
    for x in c.tails:
        x[:, at[0][:, 0]] = 0.0
    half = torch.zeros(c.n_pages, dtype=torch.bool)
    half[shared:][torch.randperm(16, generator=g)[:8]] = True
    for p in range(shared, c.n_pages):
        keys = (c.codes[0][p] * c.scales[0][p]).clone()
        keys[at[0][:, 0]] = 64.0 if half[p] and kind in ("small", "preferred") else 0.0
        codes, c.scales[0][p] = R.eight_bits(keys)
        c.codes[0][p] = codes.float()
    if kind in ("zeros", "preferred"):
        c.codes[1][half] = 0.0
    if kind == "small":
        c.scales[1][half] *= 2.0 ** -bits
    else:
        c.scales[1][half] = 2.0 ** -100
        c.scales[1][~half] *= 2.0 ** bits
    return c


def worst(got, want, what):
    got, want = got.double().cpu(), want.double()
    off = ((got - want).abs() - 2.0 ** -126).clamp(min=0.0)  # smaller numbers are subnormal in bf16 (and in fp32): they have fewer bits, or are 0
    e = (off.pow(2).mean(-1) / want.pow(2).mean(-1)).sqrt()
    print(*what, "row errors: mean %.2e, worst %.2e" % (e.mean().item(), e.max().item()), flush=True)
    return e.max().item() if bool(torch.isfinite(got).all()) else float("inf")


def inputs(g, B, Hq, H, L, D, own):
    q, k, v = some(g, B, Hq, L, D), some(g, B, H, L, D), (some(g, B, H, L, D).float() * 2.0 ** own).to(BF)
    q[..., 0], k[..., 0] = 8.0, 0.0
    return q, k, v


SIZES = [("zeros", 0), ("zeros", 20), ("zeros", 46), ("zeros", 47), ("zeros", 60), ("zeros", 100), ("zeros", -60), ("tiny", 0), ("tiny", 60), ("tiny", 100),
         ("small", 10), ("small", 24), ("small", 40), ("small", 80), ("preferred", 0), ("preferred", 50), ("preferred", 100)]


@pytest.mark.parametrize("kind,bits", SIZES)
@pytest.mark.parametrize("B,H,G,D,L,longest", [(1, 4, 2, 128, 20, 2500), (130, 2, 1, 64, 3, 1300), (65, 4, 4, 128, 20, 700), (1, 2, 4, 64, 80, 4000)])
def test_trees(B, H, G, D, L, longest, kind, bits):
    g = gen(D + L + bits)
    ref = cache(g, B, H, D, longest, kind, bits)
    q, k, v = inputs(g, B, H * G, H, L, D, 0)
    f, parent = flags_of(g, "rand", B, H, L), T.random_tree(g, B, L)
    ctx = ag.Context(0, ag.q8_tree_workspace_bytes(B, L, H * G, H, D, ref.max_blocks))
    out = torch.empty(q.shape, dtype=BF, device=DEV)
    ag.ag_q8_tree_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), f.to(DEV), parent.to(DEV), None, D ** -0.5, on_device(ref), out)
    ctx.poll_error()
    assert worst(out, T.attend(ref, q, k, v, f != 0, parent, D ** -0.5), ("tree", B, H, G, D, L, kind, bits)) <= BAR


@pytest.mark.parametrize("own", [0, -40, 40])
@pytest.mark.parametrize("kind,bits", SIZES)
@pytest.mark.parametrize("B,H,G,D,L,longest", [(1, 4, 2, 128, 60, 2500), (130, 4, 1, 64, 2, 500), (1, 2, 4, 64, 80, 4000)])
def test_turns(B, H, G, D, L, longest, kind, bits, own):
    """own: the call's values are 2^own as large as usual, those of evicted tokens among them."""
    g = gen(D + L + bits)
    ref = cache(g, B, H, D, longest, kind, bits, L)
    q, k, v = inputs(g, B, H * G, H, L, D, own)
    f = flags_of(g, "rand", B, H, L)
    ctx = ag.Context(0, ag.q8_workspace_bytes(B, L, H * G, H, D, ref.max_blocks))
    out = torch.empty(q.shape, dtype=BF, device=DEV)
    ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), f.to(DEV), None, D ** -0.5, on_device(ref), out)
    assert worst(out, R.attend(ref, q, k, v, f != 0, D ** -0.5), ("turn", B, H, G, D, L, kind, bits, own)) <= BAR


@pytest.mark.parametrize("own", [0, -40, 40])
@pytest.mark.parametrize("kind,bits", SIZES)
@pytest.mark.parametrize("B,H,G,D,longest", [(1, 4, 2, 128, 6000), (40, 8, 1, 64, 300), (40, 8, 4, 128, 900), (2, 2, 8, 64, 9000)])
def test_steps(B, H, G, D, longest, kind, bits, own):
    """own: the tails' values and the new token's are 2^own as large as usual."""
    g = gen(D + longest + bits)
    ref = cache(g, B, H, D, longest, kind, bits)
    ref.tails[1] *= 2.0 ** own
    q, k, v = inputs(g, B, H * G, H, 1, D, own)
    ctx = ag.Context(0, ag.q8_workspace_bytes(B, 1, H * G, H, D, ref.max_blocks))
    out = torch.empty(B, H * G, D, dtype=BF, device=DEV)
    one = lambda x: x[:, :, 0].contiguous().to(DEV)  # noqa: E731
    ag.ag_q8_decode_attn(ctx, one(q), one(k), one(v), torch.zeros(B, H, dtype=torch.uint8, device=DEV), None, D ** -0.5, on_device(ref), out)
    ctx.poll_error()
    want = R.attend(ref, q, k, v, torch.zeros(B, H, 1, dtype=torch.bool), D ** -0.5)[:, :, 0]
    assert worst(out, want, ("step", B, H, G, D, kind, bits, own)) <= BAR


@pytest.mark.parametrize("bits", [-40, -76, -90, -100])
@pytest.mark.parametrize("D,lens", [(128, [0, 0]), (64, [0, 30])])
def test_turns_of_small_values(D, lens, bits):
    """Nothing but the call's own values (and a tail's), 2^bits as large as usual."""
    g, L, H = gen(D - bits), 90, 2
    ref = R.Cache(1, H, D, H * 3, 3, g, lens)
    ref.tails[1] *= 2.0 ** bits
    q, k, v, f = some(g, 1, 2 * H, L, D), some(g, 1, H, L, D), (some(g, 1, H, L, D).float() * 2.0 ** bits).to(BF), flags_of(g, "rand", 1, H, L)
    ctx = ag.Context(0, ag.q8_workspace_bytes(1, L, 2 * H, H, D, ref.max_blocks))
    out = torch.empty(q.shape, dtype=BF, device=DEV)
    ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), f.to(DEV), None, D ** -0.5, on_device(ref), out)
    assert worst(out, R.attend(ref, q, k, v, f != 0, D ** -0.5), ("turn", D, lens, bits)) <= BAR

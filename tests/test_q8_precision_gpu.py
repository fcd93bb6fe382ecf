"""How exactly the attention over the paged 8-bit cache computes, output row by output row, where sizes are far from 1.

The bar of a row is on RMS(error) / RMS(row).  The store's rounding to bf16 (8 significant bits) moves an element by at most 2^-9 of
itself, so it gives at most 2^-9 of the row.  Before it: queries, the call's own keys and values, and the weights are rounded to f16, each to within
2^-12 / sqrt 3 = 1.4e-4 RMS of itself; a score of queries and keys of unit size times `spread` is then off by 2e-4 spread, a weight relatively by
as much and by its own 1.4e-4.  A row that one or two keys make up shows a single draw of that: with five times its RMS, 1.2e-3
max(1, spread) holds everything.  (bf16 operands would be 8 times that, weights below f16's normal range more.)"""
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
from gpu_util import DEV, ensure_built
from test_q8_gpu import BF, ctx_of, flags_of, gen, on_device, rope_of, some

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def bar(spread=1.0):
    return 2.0 ** -9 + 1.2e-3 * max(1.0, spread)


def row_errors(got, want):
    """RMS(error) / RMS(row) of every row of [..., D]"""
    got, want = got.double().cpu(), want.double()
    return ((got - want).pow(2).mean(-1) / want.pow(2).mean(-1)).sqrt()


def cache_of(B, H, D, lens, room, g, values=0):
    """A reference cache whose values are N(0, 1) times 2^values"""
    blocks = (max(lens) + room) // 64 + 1
    c = R.Cache(B, H, D, B * H * blocks, blocks, g, lens)
    c.scales[1] *= 2.0 ** values
    c.tails[1] *= 2.0 ** values
    return c


def turn_error(ref, g, q, k, v, f, scale, axes=0):
    """The largest row error of a turn, and the rows' errors"""
    B, Hq, L, D = q.shape
    args, rope = rope_of(g, D, B, L, axes) if axes else (None, None)
    dev, ctx, out = on_device(ref), ctx_of(ref, L, Hq), torch.empty(q.shape, dtype=BF, device=DEV)
    ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), f.to(DEV), rope, scale, dev, out)
    ctx.poll_error()
    q64, k64 = (R.turned64(q.float(), *args), R.turned64(k.float(), *args)) if axes else (q, k)
    e = row_errors(out, R.attend(ref, q64, k64, v, f != 0, scale))
    print("turn", tuple(q.shape), "row errors: mean %.2e, worst %.2e" % (e.mean().item(), e.max().item()), flush=True)
    return e


# ------------------------------------------------------------------------------------- sizes of values, tokens that are evicted
@pytest.mark.parametrize("values", [0, -6, -10, -20, 20])
@pytest.mark.parametrize("D,lens,axes", [(128, [0, 700], 1), (64, [130, 64], 0)])
def test_turns_over_values_of_any_size(D, lens, axes, values):
    g, L = gen(values + 100 + D), 300
    ref = cache_of(1, 2, D, lens, L, g, values)
    q, k, v, f = some(g, 1, 4, L, D), some(g, 1, 2, L, D), some(g, 1, 2, L, D) * 2.0 ** values, flags_of(g, "runs", 1, 2, L)
    assert turn_error(ref, g, q, k, v, f, D ** -0.5, axes).max() <= bar()


@pytest.mark.parametrize("D", [64, 128])
def test_turns_whose_evicted_tokens_see_mostly_themselves(D):
    """Scores of a token with itself up to 11, those with others of unit size; its own value up to 2^-12 of theirs."""
    g, L = gen(D + 5), 260
    ref = cache_of(1, 2, D, [90, 400], L, g)
    q, v, f = some(g, 1, 2, L, D), some(g, 1, 2, L, D), flags_of(g, "runs", 1, 2, L)
    own = torch.rand(1, 2, L, 1, generator=g)
    k = torch.where(f[..., None] != 0, some(g, 1, 2, L, D), (q * own).to(BF))
    v = torch.where(f[..., None] != 0, v, v * 2.0 ** -torch.randint(0, 13, (1, 2, L, 1), generator=g)).to(BF)
    assert turn_error(ref, g, q, k, v, f, D ** -0.5).max() <= bar()


def test_a_turn_that_is_cut_into_pieces_over_small_values():
    g, L, D = gen(8), 40, 128
    ref = cache_of(1, 2, D, [2500, 1400], L, g, -9)
    q, k, v, f = some(g, 1, 8, L, D), some(g, 1, 2, L, D), some(g, 1, 2, L, D) * 2.0 ** -9, flags_of(g, "rand", 1, 2, L)
    assert turn_error(ref, g, q, k, v, f, D ** -0.5, 1).max() <= bar()


# ----------------------------------------------------------------------------------------------------------------- one new token
def many_units(B, H, D, longest, g, values=0):
    """A reference cache of units of 0 to `longest` rows (one of them the longest) on a few pages that they share; each unit's last block has
    a page of its own."""
    U = B * H
    lens = torch.randint(0, longest + 1, (U,), generator=g).tolist()
    lens[U // 2] = longest
    page = torch.randint(U, U + 9, (U, longest // 64 + 1), generator=g).int()
    for u in range(U):
        page[u, lens[u] // 64] = u
    c = R.Cache(B, H, D, U + 9, longest // 64 + 1, g, lens, page=page)
    c.scales[1] *= 2.0 ** values
    c.tails[1] *= 2.0 ** values
    return c


def step_error(ref, g, q, k, v, f, scale, axes=0):
    """The row errors of a step"""
    B, Hq, D = q.shape
    args, rope = rope_of(g, D, B, 1, axes) if axes else (None, None)
    dev, ctx, out = on_device(ref), ctx_of(ref, 1, Hq), torch.empty(q.shape, dtype=BF, device=DEV)
    ag.ag_q8_decode_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), f.to(DEV), rope, scale, dev, out)
    ctx.poll_error()
    q, k, v = q.unsqueeze(2), k.unsqueeze(2), v.unsqueeze(2)
    q64, k64 = (R.turned64(q.float(), *args), R.turned64(k.float(), *args)) if axes else (q, k)
    e = row_errors(out, R.attend(ref, q64, k64, v, torch.ones(v.shape[:3], dtype=torch.bool), scale)[:, :, 0])
    print("step", tuple(q.shape), "row errors: mean %.2e, worst %.2e" % (e.mean().item(), e.max().item()), flush=True)
    return e


@pytest.mark.parametrize("B,H,G,D,longest", [(20, 8, 1, 128, 500), (20, 8, 1, 64, 500), (4, 4, 4, 128, 900), (70, 4, 2, 64, 300)])
def test_steps_whose_new_token_has_half_of_the_weight_at_large_scores(B, H, G, D, longest):
    """Scores of seven times the usual size; the new token's is about the logarithm of the others' sum, for one head of a group."""
    g, spread = gen(B + D + longest), 7.0
    scale = spread * D ** -0.5
    ref = many_units(B, H, D, longest, g)
    q, k, v = some(g, B, H * G, D), some(g, B, H, D), some(g, B, H, D)
    args, _ = rope_of(gen(5), D, B, 1, 1)
    q64 = R.turned64(q.unsqueeze(2).float(), *args)
    for u in range(B * H):
        b, h = divmod(u, H)
        K, one = ref.rows(u, 0), q[b, h * G].double()
        others = torch.logsumexp(K @ q64[b, h * G, 0] * scale, 0) if K.shape[0] else torch.tensor(0.0)
        k[b, h] = (k[b, h].double() + one * (others / scale - one @ k[b, h].double()) / (one @ one)).to(BF)
    assert step_error(ref, gen(5), q, k, v, torch.ones(B, H, dtype=torch.uint8), scale, 1).max() <= bar(spread)


@pytest.mark.parametrize("values", [0, -6, -10, -20, 20])
@pytest.mark.parametrize("B,H,G,D,longest", [(1, 8, 4, 128, 3000), (2, 3, 1, 64, 800), (130, 10, 1, 64, 320), (65, 4, 2, 64, 900)])
def test_steps_over_values_of_any_size(B, H, G, D, longest, values):
    """Eight waves a unit, one wave a unit, units in equal ranges: a wave has the tail and pages behind it."""
    g = gen(values + D + longest)
    ref = many_units(B, H, D, longest, g, values)
    q, k, v, f = some(g, B, H * G, D), some(g, B, H, D), some(g, B, H, D) * 2.0 ** values, flags_of(g, "rand", B, H, 1)[:, :, 0].contiguous()
    assert step_error(ref, g, q, k, v, f, D ** -0.5, 1).max() <= bar()


@pytest.mark.parametrize("D", [64, 128])
def test_steps_whose_tail_and_pages_hold_values_of_different_sizes(D):
    g, H = gen(D + 9), 8
    for pages, tail in ((-12, 0), (0, -12), (30, 0), (0, 30), (90, -20), (-20, 90), (40, 90)):
        ref = many_units(1, H, D, 500, g)
        ref.scales[1] *= 2.0 ** pages
        ref.tails[1] *= 2.0 ** tail
        q, k, v = some(g, 1, H, D), some(g, 1, H, D), some(g, 1, H, D) * 2.0 ** tail
        assert step_error(ref, g, q, k, v, torch.zeros(1, H, dtype=torch.uint8), D ** -0.5).max() <= bar()


# ------------------------------------------------------------------------------------------------------------ many small weights
@pytest.mark.parametrize("rows,bits", [(300000, 25.5), (400000, 24.5), (64 * 3000, 22.3)])
def test_many_small_weights_are_not_lost(rows, bits):
    """One row that every query sees with a score of bits ln 2, and so many with a score of 0 that they make 0.6 to 4 % of the sum: in closed
    form, as all of these are alike."""
    g, H, G, D, L = gen(rows), 8, 8, 128, 512       # (so many query rows that no row's keys are cut into pieces)
    blocks, scale, low = rows // 64, D ** -0.5, 2.0
    sign = torch.randint(0, 2, (D,), generator=g).float() * 2 - 1
    value = torch.randn(D, generator=g).to(torch.float8_e4m3fn).float()
    keys, values = torch.zeros(2, 64 * D), torch.full((2, 64 * D), low)
    keys[0, R.places(D)[0][7]], values[0, R.places(D)[1][7]] = sign, value           # row 7 of page 0, which is every unit's first one
    page = torch.ones(H, blocks + L // 64 + 1, dtype=torch.int32)
    page[:, 0] = 0
    pools = [x.to(torch.float8_e4m3fn).view(torch.uint8).to(DEV) for x in (keys, values)]
    tails = [torch.zeros(H, 64 * D, dtype=BF, device=DEV) for _ in range(2)]
    cache = ag.Q8Cache(*pools, torch.ones(2, device=DEV), torch.ones(2, device=DEV), *tails, page.to(DEV),
                       torch.full((H,), blocks * 64, dtype=torch.int32, device=DEV), 1, H, D)
    q = (sign * (bits * 0.6931471805599453 / scale / D) + 0.02 * torch.randn(1, H * G, L, D, generator=g)).to(BF)
    k, v = (-sign).expand(1, H, L, D).to(BF).contiguous(), some(g, 1, H, L, D)        # evicted, and their own scores are the least
    ctx, out = ag.Context(0, ag.q8_workspace_bytes(1, L, H * G, H, D, blocks + L // 64 + 1)), torch.empty_like(q, device=DEV)
    print("turn", rows, bits, flush=True)
    ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), torch.zeros(1, H, L, dtype=torch.uint8, device=DEV), None, scale, cache, out)
    ctx.poll_error()
    own = (q.double() * k.double().repeat_interleave(G, dim=1)).sum(-1, keepdim=True) * scale
    score = (q.double() @ sign.double())[..., None] * scale
    w, w_own = torch.exp(-score) * (blocks * 64 - 1), torch.exp(own - score)
    e = row_errors(out, (value.double() + w * low + w_own * v.double().repeat_interleave(G, dim=1)) / (1 + w + w_own))
    print("turn", rows, bits, "row errors: mean %.2e, worst %.2e" % (e.mean().item(), e.max().item()), flush=True)
    assert e.max() <= bar()


# ------------------------------------------------------------------------------------------------------------------ large scores
@pytest.mark.parametrize("Hq,H,D,lens,kind", [(4, 2, 128, [0, 700], "runs"), (8, 2, 64, [130, 64], "rand"), (2, 2, 128, [1500, 90], "none")])
def test_turns_at_large_scores(Hq, H, D, lens, kind):
    g, L, spread = gen(sum(lens) + D), 260, 7.0
    ref = cache_of(1, H, D, lens, L, g)
    q, k, v, f = some(g, 1, Hq, L, D), some(g, 1, H, L, D), some(g, 1, H, L, D), flags_of(g, kind, 1, H, L)
    assert turn_error(ref, g, q, k, v, f, spread * D ** -0.5, 1).max() <= bar(spread)


@pytest.mark.parametrize("B,H,G,D,longest", [(1, 8, 4, 128, 3000), (130, 10, 1, 64, 320), (65, 4, 2, 64, 900)])
def test_steps_at_large_scores(B, H, G, D, longest):
    g, spread = gen(D + longest + 1), 7.0
    ref = many_units(B, H, D, longest, g)
    q, k, v, f = some(g, B, H * G, D), some(g, B, H, D), some(g, B, H, D), flags_of(g, "rand", B, H, 1)[:, :, 0].contiguous()
    assert step_error(ref, g, q, k, v, f, spread * D ** -0.5, 1).max() <= bar(spread)

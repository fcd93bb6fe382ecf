"""The paged 8-bit cache where a call is long or has many units: several blocks a workgroup, flags counted in several pieces or by a
scan, pages looked up in several portions.  Caches to the bit; the attention's bars are those of test_q8_gpu."""
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
from gpu_util import DEV, ensure_built
from test_q8_gpu import BF, append_both, check_out, ctx_of, flags_of, gen, on_device, prefill_both, rope_of, same_cache, some

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


@pytest.mark.parametrize("D,L,kind", [(128, 8191, "rand"), (128, 8193, "rand"), (64, 4097, "rand"), (64, 16384, "runs"), (128, 16385, "rand"), (64, 16400, None)])
def test_long_calls(D, L, kind):
    g = gen(L)
    blocks = L // 64 + 2
    ref = R.Cache(1, 2, D, 2 * blocks, blocks, g, [41, 0])
    dev, ctx = on_device(ref), ctx_of(ref, L, 2)
    print("append", D, L, kind, flush=True)
    assert append_both(ctx, ref, dev, g, L, None if kind is None else flags_of(g, kind, 1, 2, L), 1)
    same_cache(dev, ref)
    ctx.poll_error()


@pytest.mark.parametrize("B,H,D,L,kind,axes", [(130, 4, 64, 260, "rand", 1), (130, 4, 128, 200, None, 0), (20, 10, 128, 600, "rand", 3)])
def test_many_units_with_several_blocks_a_workgroup(B, H, D, L, kind, axes):
    """Blocks with infinities and NaN among them, and units whose room ends within the call."""
    g = gen(B + L)
    lens, blocks = torch.randint(0, 130, (B * H,), generator=g).tolist(), L // 64 + 4
    ref = R.Cache(B, H, D, B * H * blocks, blocks, g, lens)
    k, v = some(g, B, H, L, D), some(g, B, H, L, D)
    k[3, 1, 70, 5], v[3, 1, 5, 9], v[5, 2, 150, 0], k[B - 1, 0, L - 1, D - 1] = float("inf"), float("nan"), -float("inf"), float("nan")
    k[7], v[8] = k[7] * 2.0 ** 60, v[8] * 2.0 ** -60
    if axes:
        k[3, 1, 70, 5] = 1.0      # (a turned infinity is a matter of the pair's signs)
    ref.page[9, lens[9] // 64 + 1] = -1
    ref.page[10, lens[10] // 64:] = ref.n_pages
    dev, ctx = on_device(ref), ctx_of(ref, L, H)
    print("append", B, H, D, L, kind, flush=True)
    full = append_both(ctx, ref, dev, g, L, None if kind is None else flags_of(g, kind, B, H, L), axes, k, v)
    same_cache(dev, ref)
    assert not full
    with pytest.raises(ag.AgError) as e:
        ctx.poll_error()
    assert e.value.status == ag.AG_ECAPACITY


@pytest.mark.parametrize("B,H,G,D,L", [(65, 4, 1, 64, 140), (65, 4, 2, 128, 70)])
def test_prompts_of_many_units(B, H, G, D, L):
    g = gen(D + L)
    lens, blocks = torch.randint(0, 100, (B * H,), generator=g).tolist(), 5
    ref = R.Cache(B, H, D, B * H * blocks, blocks, g, lens)
    ctx = ctx_of(ref, L, H * G)
    print("prefill", B, H, G, D, L, flush=True)

    def touch(q, k, v, f):      # rows of too different sizes, and a value that is not finite, in tiles of one workgroup's
        k[1, 0, 9] *= 2.0 ** -30
        v[2, 1, 80 % L] *= 2.0 ** 20
    prefill_both(ref, on_device(ref), ctx, g, H * G, L, 1, "rand", touch)
    ctx.poll_error()


@pytest.mark.parametrize("D", [64, 128])
def test_items_of_many_tiles(D):
    """A query tile over more pages than are looked up at once, some of them outside the pool, uncut.  Checked at some of the tokens."""
    g, H, G, L = gen(D), 8, 8, 1040 if D == 64 else 520
    lens = [64 * 70 + 5, 64 * 130, 64 * 64, 64 * 63 + 63, 0, 64 * 65 + 1, 64 * 128 + 63, 64 * 129]
    blocks = max(lens) // 64 + L // 64 + 2
    page = torch.randint(0, 24, (H, blocks), generator=g).int()
    page[0, 66], page[1, 63], page[1, 64], page[6, 127] = -1, 24 + H * (L // 64 + 2), 1 << 30, -5
    for u in range(H):      # blocks that the call fills have their own
        n = L // 64 + 2
        page[u, lens[u] // 64:lens[u] // 64 + n] = torch.arange(n).int() + 24 + u * n
    ref = R.Cache(1, H, D, 24 + H * (L // 64 + 2), blocks, g, lens, page=page)
    dev, ctx = on_device(ref), ctx_of(ref, L, H * G)
    q, k, v, f = some(g, 1, H * G, L, D), some(g, 1, H, L, D), some(g, 1, H, L, D), flags_of(g, "rand", 1, H, L)
    args, rope = rope_of(g, D, 1, L, 1, rows=2000, first=700)
    out = torch.empty(1, H * G, L, D, dtype=BF, device=DEV)
    print("prefill", D, L, flush=True)
    ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), f.to(DEV), rope, D ** -0.5, dev, out)
    q64, k64, kt = R.turned64(q.float(), *args), R.turned64(k.float(), *args), R.turned(k.float(), *args)
    at = [0, 1, 15, 16, 17, 63, 64, 129, 300, L - 2, L - 1]
    want = torch.empty(1, H * G, len(at), D, dtype=torch.float64)
    for u in range(H):
        K, V = ref.rows(u, 0), ref.rows(u, 1)
        kept = torch.nonzero(f[0, u]).view(-1)
        for x, j in enumerate(at):
            mine = torch.cat([kept[kept < j], torch.tensor([j])])
            s = q64[0, u * G:(u + 1) * G, j] @ torch.cat([K, k64[0, u, mine]]).T * D ** -0.5
            want[0, u * G:(u + 1) * G, x] = torch.softmax(s, dim=1) @ torch.cat([V, v[0, u, mine].double()])
    check_out(out[:, :, at], want)
    for u in range(H):
        ref.append(u, kt[0, u][f[0, u] != 0], v[0, u].float()[f[0, u] != 0])
    same_cache(dev, ref)
    ctx.poll_error()

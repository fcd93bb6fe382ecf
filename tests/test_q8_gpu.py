"""Rotation, the paged 8-bit cache and the attention over it, against plain loops on the CPU (q8_reference).

What the cache holds is defined to the bit, so codes, scales, tails and lengths are compared as such.  The attention's bars are those
of the bf16 prefill: per output row, the largest error beyond what the store's own rounding adds within 2e-2 of the row's RMS, and the RMS
of the error within 5e-3.  Where they come from, for rows of unit size: the turned query and key are rounded to bf16 (relative 2^-9 / sqrt 3 =
1.1e-3 RMS each, so the scores, of unit size, are off by 1.6e-3 and the weights relatively as much), a prompt's weights once more, and the
output's store by 1.1e-3: together 2.3e-3 RMS, and 4.5 times that at the worst of 10^6 values, 1e-2."""
import numpy as np
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
from gpu_util import DEV, attn_error, attn_rms_error, attn_tolerance, bf16_half_spacing, ensure_built

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def sections(D, axes, odd=False):
    if axes == 1:
        return [D // 2]
    if axes == 2:
        return [D // 4, D // 4]
    a = D // 8 + (3 if odd else 0)
    b = (D // 2 - a) // 2 // (1 if odd else 4) * (1 if odd else 4)
    return [a, b, D // 2 - a - b]


def rope_of(g, D, B, L, axes, rows=500, odd=False, first=None):
    """(reference arguments, ag.Rope)"""
    tab, sec = R.table(rows, D), sections(D, axes, odd)
    pos = torch.randint(0, rows, (axes, B, L), generator=g).int() if first is None else (torch.arange(L).int() + first).expand(axes, B, L).contiguous()
    return (tab, pos, sec), ag.Rope(tab.to(DEV), pos.to(DEV), sec)


def on_device(c):
    """ag.Q8Cache with the contents of a reference cache"""
    codes = [x.to(torch.float8_e4m3fn).view(torch.uint8).to(DEV) for x in c.codes]
    scales = [x.clone().to(DEV) for x in c.scales]
    tails = [x.to(BF).to(DEV) for x in c.tails]
    return ag.Q8Cache(codes[0], codes[1], scales[0], scales[1], tails[0], tails[1], c.page.to(DEV), c.len.clone().to(DEV), c.B, c.Hkv, c.D)


def same_cache(dev, ref):
    assert torch.equal(dev.len.cpu(), ref.len)
    for x, (codes, scale, tail) in enumerate(((dev.k, dev.k_scale, dev.k_tail), (dev.v, dev.v_scale, dev.v_tail))):
        assert torch.equal(scale.cpu(), ref.scales[x]), "scales"
        got = codes.cpu().view(torch.float8_e4m3fn).float()
        assert torch.equal(torch.isnan(got), torch.isnan(ref.codes[x])) and torch.equal(got.nan_to_num(), ref.codes[x].nan_to_num()), "codes"
        got = tail.cpu().float()
        assert torch.equal(torch.isnan(got), torch.isnan(ref.tails[x])) and torch.equal(got.nan_to_num(), ref.tails[x].nan_to_num()), "tails"


def some(g, *shape):
    return torch.randn(*shape, generator=g).to(BF)


def flags_of(g, kind, B, H, L):
    if kind == "all":
        return torch.ones(B, H, L, dtype=torch.uint8)
    if kind == "none":
        return torch.zeros(B, H, L, dtype=torch.uint8)
    if kind == "runs":
        return (torch.arange(L)[None, None] // 37 + torch.arange(H)[None, :, None]).expand(B, H, L).remainder(2).to(torch.uint8)
    keep = torch.rand(B, H, 1, generator=g)
    return (torch.rand(B, H, L, generator=g) < keep).to(torch.uint8) * torch.randint(1, 256, (B, H, L), generator=g).to(torch.uint8)


def ctx_of(c, L, Hq):
    return ag.Context(0, ag.q8_workspace_bytes(c.B, L, Hq, c.Hkv, c.D, c.max_blocks))


def check_out(got, ref):
    got, ref = got.double().cpu().numpy(), ref.double().numpy()
    fine = np.isfinite(ref)
    assert np.array_equal(got[~fine], ref[~fine], equal_nan=True) and np.isfinite(got[fine]).all()
    got, ref = np.where(fine, got, 0.0), np.where(fine, ref, 0.0)
    err = attn_error("bf16", got, ref)
    assert err <= attn_tolerance("bf16"), err
    assert attn_rms_error(got, ref) <= 5e-3


# ------------------------------------------------------------------------------------------------------------ rotation
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("B,Hq,Hkv,L,D,axes,odd", [
    (1, 1, 1, 1, 16, 1, False), (3, 5, 2, 1, 128, 1, False), (2, 4, 4, 77, 64, 3, False), (2, 4, 1, 33, 128, 3, True), (1, 3, 0, 50, 256, 2, False),
    (2, 9, 3, 19, 48, 3, True), (1, 40, 8, 300, 128, 1, False), (1, 2, 2, 5, 512, 1, False)])
def test_rotate(dtype, B, Hq, Hkv, L, D, axes, odd):
    g = gen(B * 1000 + L + D)
    (tab, pos, sec), rope = rope_of(g, D, B, L, axes, odd=odd)
    q, k = torch.randn(B, Hq, L, D, generator=g).to(dtype), torch.randn(B, Hkv, L, D, generator=g).to(dtype) if Hkv else None
    print("rotate", dtype, B, Hq, Hkv, L, D, axes, flush=True)
    ctx = ag.Context(0)
    dq, dk = q.to(DEV), k.to(DEV) if Hkv else None
    oq, ok = torch.full_like(dq, 7.0), torch.full_like(dk, 7.0) if Hkv else None
    ag.ag_rotate(ctx, dq, dk, rope, oq, ok)
    for x, out in ((q, oq),) + (((k, ok),) if Hkv else ()):
        ref = R.turned64(x.float(), tab, pos, sec).numpy()
        # two products and a sum, each within 2^-24 of itself, then the store
        size = R.turned64(x.float().abs(), tab.abs(), pos, sec).abs().numpy() + 2 * np.abs(R.turned64(x.float(), tab, pos, sec).numpy()) + 8.0
        bar = 2.0 ** -23 * size + (bf16_half_spacing(ref) * (1 + 2.0 ** -7) if dtype == BF else 0.0)
        assert (np.abs(out.double().cpu().numpy() - ref) <= bar).all()
        assert torch.equal(out.cpu(), R.turned(x.float(), tab, pos, sec).to(dtype))
    ag.ag_rotate(ctx, dq, dk, rope, dq, dk)     # in place
    assert torch.equal(dq, oq) and (not Hkv or torch.equal(dk, ok))
    ctx.poll_error()


def test_a_position_outside_the_table_is_reported_and_reads_the_nearest_row():
    g, B, L, D = gen(3), 2, 9, 64
    (tab, pos, sec), _ = rope_of(g, D, B, L, 1, rows=50)
    pos[0, 0, 3], pos[0, 1, 7] = 50, -4
    q = some(g, B, 2, L, D)
    ctx, out = ag.Context(0), torch.empty(B, 2, L, D, dtype=BF, device=DEV)
    ag.ag_rotate(ctx, q.to(DEV), None, ag.Rope(tab.to(DEV), pos.to(DEV)), out, None)
    with pytest.raises(ag.AgError) as e:
        ctx.poll_error()
    assert e.value.status == ag.AG_EINVAL
    assert torch.equal(out.cpu(), R.turned(q.float(), tab, pos, sec).to(BF))
    ctx.poll_error()


# -------------------------------------------------------------------------------------------------------------- append
def append_both(ctx, ref, dev, g, L, flags, axes, k=None, v=None):
    B, H, D = ref.B, ref.Hkv, ref.D
    k, v = (some(g, B, H, L, D) if k is None else k), (some(g, B, H, L, D) if v is None else v)
    args, rope = rope_of(g, D, B, L, axes) if axes else (None, None)
    ag.ag_q8_append(ctx, k.to(DEV), v.to(DEV), None if flags is None else flags.to(DEV), rope, dev)
    kt = R.turned(k.float(), *args) if axes else k.float()
    full = True
    for u in range(B * H):
        b, h = divmod(u, H)
        keep = torch.ones(L, dtype=torch.bool) if flags is None else flags[b, h] != 0
        full &= ref.append(u, kt[b, h][keep], v[b, h].float()[keep]) == int(keep.sum())
    return full


@pytest.mark.parametrize("B,H,D,L,lens,flags,axes", [
    (1, 1, 128, 1, [0], "all", 1), (1, 2, 64, 1, [63, 127], "all", 0), (2, 3, 128, 70, [0, 1, 63, 64, 65, 100], "rand", 1),
    (1, 4, 128, 333, [5, 60, 128, 191], "rand", 3), (2, 2, 64, 257, [3, 0, 64, 90], "runs", 3), (1, 2, 128, 64, [0, 1], None, 1),
    (1, 2, 64, 63, [1, 0], None, 0), (1, 3, 128, 200, [17, 64, 0], "none", 1), (1, 1, 128, 2100, [77], "rand", 1),
    (5, 3, 64, 5, [63, 62, 61, 60, 59, 0, 1, 2, 3, 4, 126, 127, 128, 129, 130], "rand", 1)])
def test_append(B, H, D, L, lens, flags, axes):
    g = gen(L + D + len(lens))
    blocks = (max(lens) + L) // 64 + 1
    ref = R.Cache(B, H, D, B * H * blocks + 3, blocks, g, lens)
    dev, ctx = on_device(ref), ctx_of(ref, L, H)
    print("append", B, H, D, L, lens, flags, flush=True)
    assert append_both(ctx, ref, dev, g, L, None if flags is None else flags_of(g, flags, B, H, L), axes)
    same_cache(dev, ref)
    ctx.poll_error()


def test_the_cache_does_not_depend_on_how_its_rows_were_cut_into_calls():
    g, B, H, D, L = gen(11), 1, 3, 128, 230
    whole = R.Cache(B, H, D, 40, 6, g, [10, 0, 63])
    a, b, c = on_device(whole), on_device(whole), on_device(whole)
    k, v, f = some(g, B, H, L, D).to(DEV), some(g, B, H, L, D).to(DEV), flags_of(g, "rand", B, H, L).to(DEV)
    q = some(g, B, H, L, D).to(DEV)
    tab, pos = R.table(400, D).to(DEV), torch.arange(L).int().view(1, 1, L).to(DEV)
    ctx = ctx_of(whole, L, H)
    ag.ag_q8_append(ctx, k, v, f, ag.Rope(tab, pos), a)
    for lo, hi in ((0, 1), (1, 64), (64, 150), (150, 150 + 63), (213, L)):
        sl = lambda x: x[:, :, lo:hi].contiguous()  # noqa: E731
        ag.ag_q8_prefill_attn(ctx, sl(q), sl(k), sl(v), sl(f), ag.Rope(tab, pos[:, :, lo:hi].contiguous()), 0.1, b, torch.empty_like(sl(q)))
    for t in range(L):
        one = lambda x: x[:, :, t].contiguous()  # noqa: E731
        ag.ag_q8_decode_attn(ctx, one(q), one(k), one(v), one(f), ag.Rope(tab, pos[:, :, t:t + 1].contiguous()), 0.1, c, torch.empty_like(one(q)))
    for other in (b, c):
        for name in ("k", "v", "k_scale", "v_scale", "len"):
            assert torch.equal(getattr(a, name), getattr(other, name)), name
        for u in range(B * H):      # (rows of a tail past the unit's end hold anything)
            n = int(a.len[u]) % 64
            for x, tails in enumerate(((a.k_tail, other.k_tail), (a.v_tail, other.v_tail))):
                at = R.places(D)[x][:n].reshape(-1).to(DEV)
                assert torch.equal(tails[0][u][at], tails[1][u][at])
    ctx.poll_error()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("call", ["append", "prefill", "decode"])
def test_rows_without_room_are_dropped_and_reported(call, D):
    g, B, H, L = gen(5 + D), 1, 4, 200
    page = torch.arange(16).int().view(4, 4).clone()
    page[0, 1], page[1, 0], page[2, 3] = -1, 99, 16          # 16 pages; the last unit's table simply ends
    ref = R.Cache(B, H, D, 16, 4, g, [64 + 62, 3, 250, 4 * 64 + 50] if call != "decode" else [127, 63, 255, 319], page=page)
    ref.len[1] = 3 if call != "decode" else 63
    dev, ctx = on_device(ref), ctx_of(ref, L, H)
    if call == "append":
        assert not append_both(ctx, ref, dev, g, L, None, 1)
    else:
        n = L if call == "prefill" else 1
        q, k, v = some(g, B, H, n, D), some(g, B, H, n, D), some(g, B, H, n, D)
        out = torch.empty(q.shape, dtype=BF, device=DEV)
        want = R.attend(ref, q.float(), k.float(), v.float(), torch.ones(B, H, n, dtype=torch.bool), 0.1)
        if call == "prefill":
            ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), None, None, 0.1, dev, out)
        else:
            ag.ag_q8_decode_attn(ctx, q[:, :, 0].contiguous().to(DEV), k[:, :, 0].contiguous().to(DEV), v[:, :, 0].contiguous().to(DEV), None, None, 0.1,
                                 dev, out[:, :, 0])
        check_out(out, want)
        for u in range(H):
            ref.append(u, k[0, u].float(), v[0, u].float())
    same_cache(dev, ref)
    with pytest.raises(ag.AgError) as e:
        ctx.poll_error()
    assert e.value.status == ag.AG_ECAPACITY
    ctx.poll_error()


@pytest.mark.parametrize("D", [64, 128])
def test_blocks_of_extreme_values(D):
    """Zeros, one value, tiny and huge blocks, values that are not finite among kept rows, and among evicted ones (never seen)."""
    g, H, L = gen(D), 8, 64
    ref = R.Cache(1, H, D, 20, 2, g, [0] * H)
    dev, ctx = on_device(ref), ctx_of(ref, L + 5, H)
    k, v, f = some(g, 1, H, L + 5, D), some(g, 1, H, L + 5, D), torch.zeros(1, H, L + 5, dtype=torch.uint8)
    f[:, :, 5:] = 1
    k[:, :, :5], v[:, :, 2] = float("nan"), float("-inf")
    k[0, 0, 5:] = 0.0
    v[0, 1, 5:], v[0, 1, 9, 3] = 0.0, 1e-38
    k[0, 2] *= 2.0 ** -110
    v[0, 3] *= 2.0 ** 125
    k[0, 4, 20, 7], k[0, 4, 30, 8] = float("inf"), float("nan")
    v[0, 5, 68], v[0, 5, 5, 0] = float("-inf"), 448.0
    k[0, 6, 5:], v[0, 6, 5:] = 449.0, 447.0
    k[0, 7, 5:] = torch.linspace(-300, 300, L * D).view(L, D).to(BF)
    assert append_both(ctx, ref, dev, g, L + 5, f, 0, k=k, v=v)
    same_cache(dev, ref)
    ctx.poll_error()


# ----------------------------------------------------------------------------------------------------------- attention
def decode_both(ref, dev, ctx, g, Hq, steps, axes, kind, scale=None):
    B, H, D = ref.B, ref.Hkv, ref.D
    scale = D ** -0.5 if scale is None else scale
    for i in range(steps):
        q, k, v = some(g, B, Hq, D), some(g, B, H, D), some(g, B, H, D)
        f = None if kind is None else flags_of(g, kind, B, H, 1)
        args, rope = rope_of(g, D, B, 1, axes) if axes else (None, None)
        out = torch.empty(B, Hq, D, dtype=BF, device=DEV)
        ag.ag_q8_decode_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), None if f is None else f[:, :, 0].contiguous().to(DEV), rope, scale, dev, out)
        qt, kt = q.float().unsqueeze(2), k.float().unsqueeze(2)
        if axes:
            q64, k64, kt = R.turned64(qt, *args), R.turned64(kt, *args), R.turned(kt, *args)
        else:
            q64, k64 = qt, kt
        want = R.attend(ref, q64, k64, v.unsqueeze(2), torch.ones(B, H, 1, dtype=torch.bool), scale)
        check_out(out, want[:, :, 0])
        for u in range(B * H):
            b, h = divmod(u, H)
            if f is None or f[b, h, 0]:
                ref.append(u, kt[b, h], v[b, h].float().unsqueeze(0))
    same_cache(dev, ref)


@pytest.mark.parametrize("B,Hq,H,D,lens,axes,kind", [
    (1, 1, 1, 128, [0], 1, "all"), (1, 4, 4, 128, [0, 1, 62, 63], 1, None), (1, 8, 8, 64, [0, 1, 63, 64, 65, 127, 128, 500], 3, "rand"),
    (2, 8, 2, 128, [700, 63, 130, 0], 3, "rand"), (1, 16, 2, 128, [2000, 640], 1, None), (1, 32, 4, 64, [1500, 3, 777, 64], 0, "rand"),
    (3, 4, 2, 128, [64 * 8 - 1, 64 * 8, 64 * 9, 64 * 16 - 1, 64 * 16, 5], 1, "none")])
def test_decode(B, Hq, H, D, lens, axes, kind):
    g = gen(sum(lens) + D)
    blocks = max(lens) // 64 + 2
    ref = R.Cache(B, H, D, B * H * blocks + 2, blocks, g, lens)
    print("decode", B, Hq, H, D, lens, flush=True)
    ctx = ctx_of(ref, 1, Hq)
    decode_both(ref, on_device(ref), ctx, g, Hq, 3, axes, kind)
    ctx.poll_error()


@pytest.mark.parametrize("U,Hq,H,D,longest", [
    (250, 10, 5, 64, 700), (300, 4, 4, 64, 150), (300, 4, 4, 128, 700), (520, 4, 4, 64, 100), (1100, 10, 10, 64, 64), (260, 16, 4, 64, 900), (40, 8, 8, 64, 3000)])
def test_decode_of_many_units(U, Hq, H, D, longest):
    """More units than workgroups, all short (teams of waves), or one long (equal ranges); units that are cut."""
    g = gen(U + D)
    lens = torch.randint(0, longest + 1, (U,), generator=g).tolist()
    lens[7], lens[U - 1] = longest, 0
    blocks = longest // 64 + 1
    # (few pages, shared by all units; every unit's last block, which a step may fill, has its own)
    page = torch.randint(U, U + 9, (U, blocks), generator=g).int()
    for u in range(U):
        page[u, lens[u] // 64] = u
    ref = R.Cache(U // H, H, D, U + 9, blocks, g, lens, page=page)
    print("decode", U, Hq, H, D, longest, flush=True)
    ctx = ctx_of(ref, 1, Hq)
    decode_both(ref, on_device(ref), ctx, g, Hq, 1, 1, "rand")
    ctx.poll_error()


def prefill_both(ref, dev, ctx, g, Hq, L, axes, kind, touch=None, scale=None):
    B, H, D = ref.B, ref.Hkv, ref.D
    scale = D ** -0.5 if scale is None else scale
    q, k, v = some(g, B, Hq, L, D), some(g, B, H, L, D), some(g, B, H, L, D)
    f = None if kind is None else flags_of(g, kind, B, H, L)
    if touch:
        touch(q, k, v, f)
    args, rope = rope_of(g, D, B, L, axes) if axes else (None, None)
    out = torch.empty(B, Hq, L, D, dtype=BF, device=DEV)
    ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), None if f is None else f.to(DEV), rope, scale, dev, out)
    q64, k64, kt = (R.turned64(q.float(), *args), R.turned64(k.float(), *args), R.turned(k.float(), *args)) if axes else (q, k, k.float())
    keep = torch.ones(B, H, L, dtype=torch.bool) if f is None else f != 0
    check_out(out, R.attend(ref, q64, k64, v, keep, scale))
    for u in range(B * H):
        b, h = divmod(u, H)
        ref.append(u, kt[b, h][keep[b, h]], v[b, h].float()[keep[b, h]])
    same_cache(dev, ref)
    return out


@pytest.mark.parametrize("B,Hq,H,D,L,lens,axes,kind", [
    (1, 1, 1, 128, 1, [0], 1, "none"), (1, 2, 2, 64, 1, [5, 64], 0, "rand"), (1, 4, 4, 128, 2, [0, 1, 63, 64], 1, "rand"), (2, 4, 2, 128, 65, [0, 3, 62, 200], 3, "rand"),
    (1, 8, 1, 128, 33, [700], 1, None), (1, 16, 2, 64, 130, [64, 129], 3, "rand"), (1, 2, 2, 128, 300, [0, 0], 1, "runs"), (1, 2, 2, 64, 257, [31, 0], 1, "none"),
    (1, 4, 2, 128, 17, [3000, 100], 1, "rand"), (3, 4, 4, 64, 129, [0, 64, 65, 128, 1, 2, 3, 4, 5, 6, 7, 191], 1, "all"), (1, 8, 2, 128, 100, [63, 64], 1, "rand")])
def test_prefill(B, Hq, H, D, L, lens, axes, kind):
    g = gen(L + sum(lens) + D)
    blocks = (max(lens) + L) // 64 + 1
    ref = R.Cache(B, H, D, B * H * blocks + 2, blocks, g, lens)
    print("prefill", B, Hq, H, D, L, lens, kind, flush=True)
    ctx = ctx_of(ref, L, Hq)
    prefill_both(ref, on_device(ref), ctx, g, Hq, L, axes, kind)
    ctx.poll_error()


def test_turns_and_steps_one_after_the_other():
    g = gen(77)
    ref = R.Cache(2, 2, 128, 40, 8, g, [0, 0, 0, 0])
    dev, ctx = on_device(ref), ctx_of(ref, 150, 8)
    prefill_both(ref, dev, ctx, g, 8, 150, 1, "rand")
    decode_both(ref, dev, ctx, g, 8, 5, 1, "rand")
    prefill_both(ref, dev, ctx, g, 8, 40, 1, "rand")
    decode_both(ref, dev, ctx, g, 8, 2, 1, None)
    ctx.poll_error()


@pytest.mark.parametrize("D", [64, 128])
def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(D):
    g, L, bad = gen(D + 1), 150, 70

    def touch(q, k, v, f):
        f[0, 0, bad], f[0, 1, bad], f[0, 2, bad] = 1, 1, 0
        v[0, 0, bad, 3], v[0, 0, bad + 1, 5] = float("nan"), float("inf")
        f[0, 0, bad + 1] = 1
        v[0, 1, bad] = float("-inf")
        v[0, 2, bad], k[0, 2, bad + 1], f[0, 2, bad + 1] = float("nan"), float("nan"), 0   # evicted: seen by themselves alone
    ref = R.Cache(1, 3, D, 12, 4, g, [0, 70, 3])
    ctx = ctx_of(ref, L, 6)
    out = prefill_both(ref, on_device(ref), ctx, g, 6, L, 0, "rand", touch=touch).float()
    assert torch.isfinite(out[0, 0, :bad]).all() and torch.isnan(out[0, 0, bad + 1:, 3]).all() and torch.isinf(out[0, 0, bad + 1:, 5]).all()
    assert not torch.isfinite(out[0, 4, bad]).any() and not torch.isfinite(out[0, 4, bad + 1]).any() and torch.isfinite(out[0, 4, bad + 2:]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_a_token_that_sees_nothing_else_gets_its_own_value(D):
    g = gen(D)
    big = 3e38
    ref = R.Cache(1, 2, D, 4, 1, g, [0, 0])
    dev, ctx = on_device(ref), ctx_of(ref, 9, 4)
    q, k, v = some(g, 1, 4, 9, D), some(g, 1, 2, 9, D), some(g, 1, 2, 9, D)
    k[0, 0, 3], q[0, :, 3] = big, -big           # a score of -infinity
    out = torch.empty(1, 4, 9, D, dtype=BF, device=DEV)
    ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), torch.zeros(1, 2, 9, dtype=torch.uint8, device=DEV), None, 1.0, dev, out)
    assert torch.equal(out.cpu(), v.repeat_interleave(2, dim=1))
    one = lambda x: x[:, :, 3].contiguous().to(DEV)  # noqa: E731
    step = torch.empty(1, 4, D, dtype=BF, device=DEV)
    ag.ag_q8_decode_attn(ctx, one(q), one(k), one(v), torch.zeros(1, 2, dtype=torch.uint8, device=DEV), None, 1.0, dev, step)
    assert torch.equal(step.cpu(), v[:, :, 3].repeat_interleave(2, dim=1))
    assert dev.len.tolist() == [0, 0]


def test_large_scores_and_large_scales():
    """One row far above the others wins; weights that underflow leave nothing behind."""
    g = gen(9)
    ref = R.Cache(1, 2, 128, 12, 4, g, [150, 64], magnitude=30.0)
    dev, ctx = on_device(ref), ctx_of(ref, 70, 2)
    prefill_both(ref, dev, ctx, g, 2, 70, 1, "rand", scale=0.02)
    decode_both(ref, dev, ctx, g, 2, 2, 0, None, scale=0.02)


def test_a_page_number_outside_the_pool_counts_as_evicted_rows():
    g = gen(21)
    ref = R.Cache(1, 2, 128, 30, 10, g, [600, 200])
    ref.page[0, 3], ref.page[0, 7], ref.page[1, 0] = -1, 30, 1 << 30
    dev, ctx = on_device(ref), ctx_of(ref, 5, 4)
    decode_both(ref, dev, ctx, g, 4, 2, 1, "rand")
    prefill_both(ref, dev, ctx, g, 4, 5, 1, "rand")


def test_pages_beyond_four_gigabytes():
    g, B, H, D = gen(31), 1, 2, 128
    n = (1 << 32) // (64 * D) + 5000
    ref = R.Cache(B, H, D, 12, 4, g, [150, 64 + 60])
    dev = on_device(ref)
    big = [torch.empty(n, 64 * D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.empty(n, device=DEV) for _ in range(2)]
    at = torch.arange(12, device=DEV) * 5 + n - 60
    for x, (codes, sc) in enumerate(((dev.k, dev.k_scale), (dev.v, dev.v_scale))):
        big[x][at], scales[x][at] = codes, sc
    far = ag.Q8Cache(big[0], big[1], scales[0], scales[1], dev.k_tail, dev.v_tail, (ref.page.to(DEV) * 5 + n - 60).int().contiguous(), dev.len, B, H, D)
    ctx = ctx_of(ref, 70, 4)

    class Near:        # the pages that matter, for the comparison
        pass
    q, k, v = some(g, B, 4, 70, D), some(g, B, H, 70, D), some(g, B, H, 70, D)
    out = torch.empty(B, 4, 70, D, dtype=BF, device=DEV)
    ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), None, None, D ** -0.5, far, out)
    check_out(out, R.attend(ref, q, k, v, torch.ones(B, H, 70, dtype=torch.bool), D ** -0.5))
    for u in range(H):
        ref.append(u, k[0, u].float(), v[0, u].float())
    step = torch.empty(B, 4, D, dtype=BF, device=DEV)
    one = lambda x: x[:, :, 0].contiguous()  # noqa: E731
    want = R.attend(ref, q[:, :, :1], k[:, :, :1], v[:, :, :1], torch.ones(B, H, 1, dtype=torch.bool), D ** -0.5)
    ag.ag_q8_decode_attn(ctx, one(q).to(DEV), one(k).to(DEV), one(v).to(DEV), None, None, D ** -0.5, far, step)
    check_out(step, want[:, :, 0])
    for u in range(H):
        ref.append(u, k[0, u, :1].float(), v[0, u, :1].float())
    near = Near()
    near.k, near.v, near.k_scale, near.v_scale = big[0][at], big[1][at], scales[0][at], scales[1][at]
    near.k_tail, near.v_tail, near.len = far.k_tail, far.v_tail, far.len
    same_cache(near, ref)
    ctx.poll_error()


def test_a_captured_step_gives_the_eager_step_again_and_again():
    g, B, Hq, H, D = gen(41), 2, 8, 4, 128
    ref = R.Cache(B, H, D, 80, 8, g, [60, 300, 0, 64, 127, 400, 1, 63])
    eager, graphed = on_device(ref), on_device(ref)
    q, k, v = some(g, B, Hq, D).to(DEV), some(g, B, H, D).to(DEV), some(g, B, H, D).to(DEV)
    tab, pos = R.table(600, D).to(DEV), torch.full((1, B, 1), 450, dtype=torch.int32, device=DEV)
    ctx, other = ctx_of(ref, 1, Hq), ctx_of(ref, 1, Hq)
    a, b = torch.empty(B, Hq, D, dtype=BF, device=DEV), torch.empty(B, Hq, D, dtype=BF, device=DEV)
    before = [x.clone() for x in (graphed.k, graphed.v, graphed.k_scale, graphed.v_scale, graphed.k_tail, graphed.v_tail, graphed.len)]
    stream = torch.cuda.Stream()
    rope = ag.Rope(tab, pos)
    with torch.cuda.stream(stream):
        ag.ag_q8_decode_attn(other, q, k, v, None, rope, 0.1, graphed, b)      # (first use outside the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        ag.ag_q8_decode_attn(other, q, k, v, None, rope, 0.1, graphed, b)
        pos.add_(1)
    for x, y in zip((graphed.k, graphed.v, graphed.k_scale, graphed.v_scale, graphed.k_tail, graphed.v_tail, graphed.len), before):
        x.copy_(y)
    pos.fill_(450)
    eager_pos = pos.clone()
    for i in range(6):
        ag.ag_q8_decode_attn(ctx, q, k, v, None, ag.Rope(tab, eager_pos), 0.1, eager, a)
        eager_pos.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, b), i
        for name in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "len"):
            assert torch.equal(getattr(eager, name), getattr(graphed, name)), (i, name)
        q.mul_(0.9)
        k.add_(v * 0.1)


def test_the_order_of_workgroups_does_not_change_results():
    """Two steps over units that are cut, alternating under memory traffic of another stream: the same bits every time."""
    g = gen(51)
    refs = [R.Cache(1, 2, 128, 150, 60, g, [3800, 2500]), R.Cache(1, 4, 128, 150, 30, g, [1900, 64, 1200, 700])]
    devs, ctx = [on_device(r) for r in refs], ctx_of(refs[1], 40, 8)
    ins = [[some(g, 1, 8, D).to(DEV) if D else None for D in (128,)] + [some(g, 1, r.Hkv, 128).to(DEV) for _ in range(2)] for r in refs]
    turn = [(some(g, 1, 8, 40, 128).to(DEV), some(g, 1, r.Hkv, 40, 128).to(DEV), some(g, 1, r.Hkv, 40, 128).to(DEV)) for r in refs]
    none = [torch.zeros(1, r.Hkv, 40, dtype=torch.uint8, device=DEV) for r in refs]
    ctx = ag.Context(0, max(ag.q8_workspace_bytes(1, 40, 8, r.Hkv, 128, r.max_blocks) for r in refs))
    noise, side, first = torch.zeros(1 << 26, device=DEV), torch.cuda.Stream(), [None, None]
    for i in range(40):
        with torch.cuda.stream(side):
            noise.add_(1.0)
        x = i % 2
        q, k, v = ins[x]
        out, many = torch.empty_like(q), torch.empty_like(turn[x][0])
        ag.ag_q8_decode_attn(ctx, q, k, v, none[x][:, :, 0].contiguous(), None, 0.1, devs[x], out)
        ag.ag_q8_prefill_attn(ctx, *turn[x], none[x], None, 0.1, devs[x], many)
        if first[x] is None:
            first[x] = (out.clone(), many.clone())
        assert torch.equal(out, first[x][0]) and torch.equal(many, first[x][1]), i
    torch.cuda.synchronize()


def test_calls_on_a_stream_of_their_own():
    g = gen(61)
    ref = R.Cache(1, 2, 64, 20, 6, g, [100, 3])
    dev, ctx, stream = on_device(ref), ctx_of(ref, 60, 4), torch.cuda.Stream()
    torch.cuda.synchronize()
    k, v, q = some(g, 1, 2, 60, 64).to(DEV), some(g, 1, 2, 60, 64).to(DEV), some(g, 1, 4, 60, 64).to(DEV)
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    ag.ag_q8_prefill_attn(ctx, q, k, v, None, None, 0.125, dev, out, stream=stream)
    stream.synchronize()
    check_out(out, R.attend(ref, q.cpu(), k.cpu(), v.cpu(), torch.ones(1, 2, 60, dtype=torch.bool), 0.125))
    for u in range(2):
        ref.append(u, k[0, u].float().cpu(), v[0, u].float().cpu())
    same_cache(dev, ref)

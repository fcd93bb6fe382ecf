"""The rotation's and the paged 8-bit cache's boundary without a GPU: refusals, sizes, and the reference that the GPU tests use."""
import math

import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
from test_boundary import expect, lib  # noqa: F401

BF = torch.bfloat16


def cache(B=1, Hkv=2, D=64, n_pages=6, blocks=3):
    U = B * Hkv
    return ag.Q8Cache(torch.zeros(n_pages, 64 * D, dtype=torch.uint8), torch.zeros(n_pages, 64 * D, dtype=torch.uint8), torch.ones(n_pages),
                      torch.ones(n_pages), torch.zeros(U, 64 * D, dtype=BF), torch.zeros(U, 64 * D, dtype=BF),
                      torch.arange(U * blocks, dtype=torch.int32).view(U, blocks), torch.zeros(U, dtype=torch.int32), B, Hkv, D)


def rope(D=64, B=1, L=8, axes=1, rows=20):
    sec = [D // 2] if axes == 1 else [D // 4] * 2 if axes == 2 else [D // 8, D // 8, D // 4]
    return ag.Rope(torch.zeros(rows, D), torch.zeros(axes, B, L, dtype=torch.int32), sec)


def test_refusals(lib):  # noqa: F811
    ctx = ag.Context(device=-1, workspace=ag.q8_workspace_bytes(1, 8, 4, 2, 64, 3))
    q, k, f = torch.zeros(1, 4, 8, 64, dtype=BF), torch.zeros(1, 2, 8, 64, dtype=BF), torch.zeros(1, 2, 8, dtype=torch.uint8)
    r, c, o = rope(), cache(), torch.zeros(1, 4, 8, 64, dtype=BF)
    # well-formed calls pass validation and report that the context has no device
    expect(ag.AG_EHIP, ag.ag_rotate, ctx, q, k, r, q, k, stream=0)
    expect(ag.AG_EHIP, ag.ag_rotate, ctx, q.float(), None, r, q.float(), None, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_append, ctx, k, k, f, r, c, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_append, ctx, k, k, None, None, c, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_prefill_attn, ctx, q, k, k, f, rope(axes=3), 0.1, c, o, stream=0)
    one = lambda x: x[:, :, 0].contiguous()  # noqa: E731
    expect(ag.AG_EHIP, ag.ag_q8_decode_attn, ctx, one(q), one(k), one(k), None, rope(L=1), 0.1, c, one(o), stream=0)
    # rotation
    expect(ag.AG_EINVAL, ag.ag_rotate, ctx, q, k, r, q, None, stream=0)
    expect(ag.AG_EUNSUPPORTED, ag.ag_rotate, ctx, torch.zeros(1, 4, 8, 40), None, rope(D=40), torch.zeros(1, 4, 8, 40), None, stream=0)
    bad = rope()
    bad.c.section[0] = 31
    expect(ag.AG_EINVAL, ag.ag_rotate, ctx, q, k, bad, q, k, stream=0)
    bad = rope(axes=2)
    bad.c.section[0], bad.c.section[1] = 40, -8
    expect(ag.AG_EINVAL, ag.ag_q8_append, ctx, k, k, f, bad, c, stream=0)
    uneven = rope(axes=3)
    uneven.c.section[0], uneven.c.section[1] = 9, 7
    expect(ag.AG_EHIP, ag.ag_rotate, ctx, q, k, uneven, q, k, stream=0)                     # any sections ...
    expect(ag.AG_EUNSUPPORTED, ag.ag_q8_append, ctx, k, k, f, uneven, c, stream=0)          # ... here multiples of 4 pairs
    bad = rope()
    bad.c.n_axes = 4
    expect(ag.AG_EINVAL, ag.ag_rotate, ctx, q, k, bad, q, k, stream=0)
    with pytest.raises(ValueError):
        ag.ag_rotate(ctx, q, k, rope(L=7), q, k, stream=0)                                  # positions of another length
    with pytest.raises(ValueError):
        ag.ag_rotate(ctx, q, k.float(), r, q, k, stream=0)
    with pytest.raises(ValueError):
        ag.Rope(torch.zeros(20, 64), torch.zeros(1, 8, dtype=torch.int32))                   # no axis
    with pytest.raises(ValueError):
        ag.Rope(torch.zeros(20, 64), torch.zeros(2, 1, 8, dtype=torch.int32))                # two axes, one section
    # alignment
    loose = torch.zeros(q.numel() + 1, dtype=BF)[1:].view(q.shape)
    if loose.data_ptr() % 16:
        expect(ag.AG_EINVAL, ag.ag_rotate, ctx, loose, k, r, q, k, stream=0)
        expect(ag.AG_EINVAL, ag.ag_q8_prefill_attn, ctx, loose, k, k, f, r, 0.1, c, o, stream=0)
    # cache and attention
    for scale in (0.0, -1.0, math.inf, math.nan):
        expect(ag.AG_EINVAL, ag.ag_q8_prefill_attn, ctx, q, k, k, f, r, scale, c, o, stream=0)
        expect(ag.AG_EINVAL, ag.ag_q8_decode_attn, ctx, one(q), one(k), one(k), None, None, scale, c, one(o), stream=0)
    q3, q6, q10 = (torch.zeros(1, n, 8, 64, dtype=BF) for n in (3, 6, 10))
    expect(ag.AG_EINVAL, ag.ag_q8_prefill_attn, ctx, q3, k, k, f, r, 0.1, c, q3, stream=0)        # Hq % Hkv
    expect(ag.AG_EUNSUPPORTED, ag.ag_q8_prefill_attn, ctx, q6, k, k, f, r, 0.1, c, q6, stream=0)  # three heads a group
    expect(ag.AG_EUNSUPPORTED, ag.ag_q8_decode_attn, ctx, one(q10), one(k), one(k), None, None, 0.1, c, one(q10), stream=0)
    for field in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "page", "len"):
        bad = cache()
        setattr(bad.c, field, None)
        expect(ag.AG_EINVAL, ag.ag_q8_append, ctx, k, k, f, r, bad, stream=0)
    for field in ("n_pages", "max_blocks"):
        bad = cache()
        setattr(bad.c, field, 0)
        expect(ag.AG_EINVAL, ag.ag_q8_decode_attn, ctx, one(q), one(k), one(k), None, None, 0.1, bad, one(o), stream=0)
    c32 = cache(D=32)
    k32 = torch.zeros(1, 2, 8, 32, dtype=BF)
    expect(ag.AG_EUNSUPPORTED, ag.ag_q8_append, ctx, k32, k32, f, None, c32, stream=0)
    many = cache(B=4097, Hkv=2, D=64, n_pages=1, blocks=1)
    km = torch.zeros(4097, 2, 1, 64, dtype=BF)
    expect(ag.AG_EUNSUPPORTED, ag.ag_q8_append, ctx, km, km, None, None, many, stream=0)
    for args in ((k.float(), k.float()), (k, k[:, :, :7].contiguous()), (k[:, :1].contiguous(), k[:, :1].contiguous())):
        with pytest.raises(ValueError):
            ag.ag_q8_append(ctx, args[0], args[1], f, None, c, stream=0)
    with pytest.raises(ValueError):
        ag.ag_q8_prefill_attn(ctx, q, k, k, f, r, 0.1, c, o[:, :, :7].contiguous(), stream=0)
    with pytest.raises(ValueError):
        ag.ag_q8_append(ctx, k.transpose(2, 3), k.transpose(2, 3), f, None, c, stream=0)
    with pytest.raises(ValueError):
        ag.Q8Cache(c.k, c.v, c.k_scale, c.v_scale, c.k_tail.float(), c.v_tail, c.page, c.len, 1, 2, 64)
    ctx.close()


def test_workspace(lib):  # noqa: F811
    assert ag.q8_workspace_bytes(1, 8, 4, 3, 64, 3) == ag.q8_workspace_bytes(0, 8, 4, 2, 64, 3) == ag.q8_workspace_bytes(1, 8, 4, 2, 96, 3) == 0
    assert ag.q8_workspace_bytes(1, 4096, 32, 8, 128, 300) > 2 * 8 * 4096 * 128 * 2
    ctx = ag.Context(device=-1, workspace=1024)
    q, k, c, f = torch.zeros(1, 4, 300, 64, dtype=BF), torch.zeros(1, 2, 300, 64, dtype=BF), cache(), torch.zeros(1, 2, 300, dtype=torch.uint8)
    expect(ag.AG_EWORKSPACE, ag.ag_q8_prefill_attn, ctx, q, k, k, f, None, 0.1, c, q.clone(), stream=0)
    expect(ag.AG_EWORKSPACE, ag.ag_q8_decode_attn, ctx, q[:, :, 0].contiguous(), k[:, :, 0].contiguous(), k[:, :, 0].contiguous(), None, None, 0.1, c,
           q[:, :, 0].contiguous(), stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_append, ctx, k, k, None, None, c, stream=0)      # without flags it needs none
    ctx.close()
    ctx = ag.Context(device=-1, workspace=0)
    expect(ag.AG_EWORKSPACE, ag.ag_q8_append, ctx, k, k, f, None, c, stream=0)
    ctx.close()


# ---- the reference ----
@pytest.mark.parametrize("D", [64, 128])
def test_every_value_has_a_place_of_its_own(D):
    for p in R.places(D):
        assert sorted(p.reshape(-1).tolist()) == list(range(64 * D))


def test_codes_are_the_nearest_numbers():
    g = torch.Generator()
    g.manual_seed(1)
    for size in (1.0, 300.0, 2.0 ** -90, 2.0 ** 100, 0.0):
        x = (torch.randn(64, 64, generator=g) * size).bfloat16().float()
        code, scale = R.eight_bits(x)
        assert code.abs().max() <= 448 and (size == 0.0 or scale == 2.0 ** -100 or code.abs().max() > 224 - 8)
        assert math.frexp(scale)[0] == 0.5
        assert torch.equal((x.double() / scale).float().to(torch.float8_e4m3fn).double(), code)


def test_rotation_by_known_angles():
    """Row p of the table turns by p quarter turns: (x, y) -> (-y, x) -> (-x, -y)."""
    D = 4
    tab = torch.tensor([[1., 1., 0., 0.], [0., 0., 1., 1.], [-1., -1., 0., 0.]])
    x = torch.tensor([1., 2., 3., 4.]).view(1, 1, 1, D)
    want = {0: [1., 2., 3., 4.], 1: [-3., -4., 1., 2.], 2: [-1., -2., -3., -4.]}
    for p, y in want.items():
        assert R.turned(x, tab, torch.full((1, 1, 1), p), [2]).view(-1).tolist() == y
    mixed = R.turned(x, tab, torch.tensor([1, 2]).view(2, 1, 1), [1, 1])
    assert mixed.view(-1).tolist() == [-3., -2., 1., -4.]


def test_attention_of_the_reference():
    """All kept, empty cache: causal attention of the library in 64 bits; no flag: a token sees the cache and itself."""
    g = torch.Generator()
    g.manual_seed(2)
    c = R.Cache(1, 2, 64, 6, 3, g, [0, 0])
    q, k, v = (torch.randn(1, n, 12, 64, generator=g) for n in (4, 2, 2))
    got = R.attend(c, q, k, v, torch.ones(1, 2, 12, dtype=torch.bool), 0.125)
    rep = lambda x: x.double().repeat_interleave(2, dim=1)  # noqa: E731
    want = torch.nn.functional.scaled_dot_product_attention(q.double(), rep(k), rep(v), is_causal=True, scale=0.125)
    assert torch.allclose(got, want, atol=1e-12)
    assert torch.equal(R.attend(c, q, k, v, torch.zeros(1, 2, 12, dtype=torch.bool), 0.125), rep(v))
    for u in range(2):
        assert c.append(u, k[0, u], v[0, u]) == 12 and c.rows(u, 0).shape == (12, 64)
        assert torch.equal(c.rows(u, 1), v[0, u].bfloat16().double())
    c.append(0, k[0, 0].repeat(6, 1), v[0, 0].repeat(6, 1))
    assert c.len.tolist() == [84, 12]
    r = c.rows(0, 0)
    assert r.shape == (84, 64) and (r - k[0, 0].repeat(7, 1).double()).abs().max() <= k.abs().max() / 16

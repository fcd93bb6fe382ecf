"""Calls of the paged 8-bit cache that must be taken, and others that must be refused, without a GPU."""
import math

import pytest
import torch

import paper_2410_12876_amd as ag
from test_boundary import expect, lib  # noqa: F401
from test_q8_boundary import BF, cache


@pytest.mark.parametrize("B,Hq,Hkv,D,L,blocks", [(1, 32, 8, 128, 4096, 300), (2, 16, 16, 64, 3000, 90), (4, 8, 8, 128, 1500, 40), (1, 8, 1, 64, 2500, 2000)])
def test_a_workspace_covers_shorter_calls(lib, B, Hq, Hkv, D, L, blocks):  # noqa: F811
    """A context made for a prompt takes every shorter turn and the steps of the same cache (validation goes as far as the missing device)."""
    ctx, c = ag.Context(device=-1, workspace=ag.q8_workspace_bytes(B, L, Hq, Hkv, D, blocks)), cache(B, Hkv, D, 2, blocks)
    assert ag.q8_workspace_bytes(B, L, Hq, Hkv, D, blocks) >= ag.q8_workspace_bytes(B, L // 3, Hq, Hkv, D, blocks)
    many, flags = torch.zeros(B * Hq * L * D, dtype=BF), torch.zeros(B * Hkv * L, dtype=torch.uint8)
    of = lambda *s: many[:math.prod(s)].view(s)  # noqa: E731
    for n in sorted({1, 2, 5, 30, 37, 61, 64, 100, 333, 500, 700, 900, 962, 990, 1000, 1024, L // 2, L - 100, L}):
        f = flags[:B * Hkv * n].view(B, Hkv, n)
        expect(ag.AG_EHIP, ag.ag_q8_prefill_attn, ctx, of(B, Hq, n, D), of(B, Hkv, n, D), of(B, Hkv, n, D), f, None, 0.1, c, of(B, Hq, n, D), stream=0)
        expect(ag.AG_EHIP, ag.ag_q8_append, ctx, of(B, Hkv, n, D), of(B, Hkv, n, D), f, None, c, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_decode_attn, ctx, of(B, Hq, D), of(B, Hkv, D), of(B, Hkv, D), None, None, 0.1, c, of(B, Hq, D), stream=0)
    ctx.close()


def test_flags_and_outputs_of_another_size_or_type_are_refused(lib):  # noqa: F811
    ctx = ag.Context(device=-1, workspace=ag.q8_workspace_bytes(1, 8, 4, 2, 64, 3))
    q, k, c = torch.zeros(1, 4, 8, 64, dtype=BF), torch.zeros(1, 2, 8, 64, dtype=BF), cache()
    r = ag.Rope(torch.zeros(20, 64), torch.zeros(1, 1, 8, dtype=torch.int32))
    one = lambda x: x[:, :, 0].contiguous()  # noqa: E731
    turn = lambda f: ag.ag_q8_prefill_attn(ctx, q, k, k, f, None, 0.1, c, q.clone(), stream=0)  # noqa: E731
    append = lambda f: ag.ag_q8_append(ctx, k, k, f, None, c, stream=0)  # noqa: E731
    step = lambda f: ag.ag_q8_decode_attn(ctx, one(q), one(k), one(k), f, None, 0.1, c, one(q), stream=0)  # noqa: E731
    for call, shape in ((turn, (1, 2, 8)), (append, (1, 2, 8)), (step, (1, 2))):
        for good in (torch.zeros(shape, dtype=torch.uint8), torch.zeros(shape, dtype=torch.bool), None):
            expect(ag.AG_EHIP, call, good)
        for bad in (torch.zeros(shape, dtype=torch.int32), torch.zeros(shape, dtype=BF), torch.zeros(shape[:-1] + (shape[-1] - 1,), dtype=torch.uint8),
                    torch.zeros((2,) + shape[1:], dtype=torch.uint8)):
            with pytest.raises(ValueError):
                call(bad)
    expect(ag.AG_EHIP, ag.ag_rotate, ctx, q, k, r, q, k.clone(), stream=0)
    expect(ag.AG_EHIP, ag.ag_rotate, ctx, q, None, r, q.clone(), None, stream=0)
    for q_out, k_out in ((q[:, :, :7].contiguous(), k), (q.float(), k), (q, k[:, :1].contiguous()), (q, k.float())):
        with pytest.raises(ValueError):
            ag.ag_rotate(ctx, q, k, r, q_out, k_out, stream=0)
    with pytest.raises(ValueError):
        ag.ag_rotate(ctx, q.float(), None, ag.Rope(r.table, r.pos), q, None, stream=0)
    ctx.close()


def test_a_page_table_whose_blocks_the_step_cannot_count_is_refused(lib):  # noqa: F811
    """A step adds up the blocks of all units, and a few more for each, in 32 bits."""
    B, H, D = 16, 8, 64
    ctx, c = ag.Context(device=-1, workspace=ag.q8_workspace_bytes(B, 1, H, H, D, 1)), cache(B, H, D, 2, 1)
    x = torch.zeros(B, H, D, dtype=BF)
    for blocks, status in ((1 << 24, ag.AG_EUNSUPPORTED), ((1 << 24) - 600, ag.AG_EHIP), (1 << 20, ag.AG_EHIP)):
        c.c.max_blocks = blocks
        expect(status, ag.ag_q8_decode_attn, ctx, x, x, x, None, None, 0.1, c, x.clone(), stream=0)
    ctx.close()

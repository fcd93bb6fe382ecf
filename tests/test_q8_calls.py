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

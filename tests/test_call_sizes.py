"""Sizes that calls can have and need, without a GPU: a rotation's threads, the workspaces of trees and pools."""
import ctypes as C

import pytest
import torch

import paper_2410_12876_amd as ag
from test_boundary import expect, lib  # noqa: F401
from test_q8_boundary import BF, cache


def test_rotate_of_more_threads_than_a_launch_has(lib):  # noqa: F811
    """A token of 512 values has 32 threads in bf16 and 64 in fp32; a launch has fewer than 2^32."""
    ctx, x = ag.Context(device=-1), torch.zeros(512)
    pos = torch.zeros(1, dtype=torch.int32)
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731

    def call(B, D, dtype):
        rope = ag.ag_rope(table=x.data_ptr(), pos=pos.data_ptr(), n_rows=1, n_axes=1)
        rope.section[0] = D // 2
        return lib.ag_rotate(C.c_void_p(ctx._addr), None, p(x), None, dtype, B, 1, 0, 1, D, C.byref(rope), p(x), None)

    for D, dtype, threads in ((512, ag.AG_BF16, 32), (512, ag.AG_F32, 64), (272, ag.AG_BF16, 17)):
        most = ((1 << 32) - 256) // threads
        assert call(most, D, dtype) == ag.AG_EHIP and call(most + 1, D, dtype) == ag.AG_EUNSUPPORTED
    assert call((1 << 31) - 1, 16, ag.AG_BF16) == ag.AG_EHIP
    ctx.close()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,lengths", [(1, [1, 32, 33, 64, 65, 256]), (2, [16, 17, 32, 33, 256]), (4, [8, 9, 16, 17, 256]), (8, [1, 4, 5, 8, 9, 255, 256])])
def test_a_tree_workspace_is_what_the_call_takes(lib, D, G, lengths):  # noqa: F811
    """On both sides of where a tile has one, two and four groups of 32 rows; a call takes all but the 4096 bytes of slack (on 256 CUs, as here; a
    context rounds its workspace up to 256)."""
    H = 2
    c, last = cache(D=D), 0
    for L in lengths:
        q, k, p = torch.zeros(1, H * G, L, D, dtype=BF), torch.zeros(1, H, L, D, dtype=BF), torch.full((1, L), -1, dtype=torch.int32)
        n = ag.q8_tree_workspace_bytes(1, L, H * G, H, D, 3)
        assert n > 4096 and n >= last
        last = n
        for size, status in ((n, ag.AG_EHIP), (n - 4096, ag.AG_EHIP), (n - 4096 - 256, ag.AG_EWORKSPACE)):
            ctx = ag.Context(device=-1, workspace=size)
            expect(status, ag.ag_q8_tree_attn, ctx, q, k, k, None, p, None, 0.1, c, q, stream=0)
            ctx.close()


@pytest.mark.parametrize("n_pages", [1, 4096, 4097, 100000])
def test_a_pool_workspace_is_what_the_calls_take(lib, n_pages):  # noqa: F811
    n, ref = ag.q8_pool_workspace_bytes(1, 2, n_pages), torch.zeros(n_pages, dtype=torch.int32)
    c, moved, used = cache(), torch.zeros(n_pages, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    c.c.n_pages = n_pages
    for size, status in ((n, ag.AG_EHIP), (n - 4096, ag.AG_EHIP), (4 * n_pages, ag.AG_EWORKSPACE)):
        ctx = ag.Context(device=-1, workspace=size)
        expect(status, ag.ag_q8_reserve, ctx, c, ref, 1, stream=0)
        expect(status, ag.ag_q8_compact_pages, ctx, c, ref, moved, used, stream=0)
        ctx.close()

"""Sizes that calls can have and need, without a GPU: a rotation's threads."""
import ctypes as C

import torch

import paper_2410_12876_amd as ag
from test_boundary import lib  # noqa: F401


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

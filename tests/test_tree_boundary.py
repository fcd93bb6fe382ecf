"""The boundary of the normalised rotation, of trees and of page pools without a GPU: refusals, sizes, and the reference that the GPU tests use."""
import ctypes as C
import math

import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
import tree_reference as T
from test_boundary import expect, lib  # noqa: F401
from test_q8_boundary import BF, cache, rope


def test_norm_rotate_refusals(lib):  # noqa: F811
    ctx = ag.Context(device=-1)
    q, k, w, r = torch.zeros(1, 4, 8, 64, dtype=BF), torch.zeros(1, 2, 8, 64, dtype=BF), torch.ones(64, dtype=BF), rope()
    call = lambda *a: ag.ag_norm_rotate(ctx, *a, stream=0)  # noqa: E731
    expect(ag.AG_EHIP, call, q, k, w, w, 1e-6, r, q, k)
    expect(ag.AG_EHIP, call, q, None, w, None, 1e-6, None, q, None)
    expect(ag.AG_EHIP, call, q.float(), None, w.float(), None, 1e-6, rope(axes=3), q.float(), None)
    for bad in ((q, k, None, w, 1e-6, r, q, k), (q, k, w, None, 1e-6, r, q, k), (q, k, w, w, 1e-6, r, q, None), (q, None, w, w, 1e-6, r, q, None)):
        expect(ag.AG_EINVAL, call, *bad)
    for eps in (0.0, -1.0, math.inf, math.nan, 2.0 ** -101):
        expect(ag.AG_EINVAL, call, q, k, w, w, eps, r, q, k)
    q40 = torch.zeros(1, 4, 8, 40)
    expect(ag.AG_EUNSUPPORTED, call, q40, None, torch.ones(40), None, 1e-6, None, q40, None)
    q528 = torch.zeros(1, 1, 1, 528)
    expect(ag.AG_EUNSUPPORTED, call, q528, None, torch.ones(528), None, 1e-6, None, q528, None)
    loose = torch.ones(65, dtype=BF)[1:]
    if loose.data_ptr() % 16:
        expect(ag.AG_EINVAL, call, q, k, loose, w, 1e-6, r, q, k)
    for bad in ((q, k, w.float(), w, 1e-6, r, q, k), (q, k, w, w[:32], 1e-6, r, q, k), (q, k.float(), w, w, 1e-6, r, q, k), (q, k, w, w, 1e-6, rope(L=7), q, k),
                (q, k, w, w, 1e-6, r, q.float(), k), (q, k, w, w, 1e-6, r, q, k[:, :1].contiguous())):
        with pytest.raises(ValueError):
            call(*bad)
    ctx.close()


def test_norm_rotate_of_more_threads_than_a_launch_has(lib):  # noqa: F811
    """A token of 512 bf16 values has 32 threads, one of 272 values too; a launch has fewer than 2^32."""
    ctx, x = ag.Context(device=-1), torch.zeros(512, dtype=BF)
    raw = lambda B, D: lib.ag_norm_rotate(C.c_void_p(ctx._addr), None, C.c_void_p(x.data_ptr()), None, ag.AG_BF16, B, 1, 0, 1, D, C.c_void_p(x.data_ptr()), None,  # noqa: E731
                                          C.c_float(1e-6), None, C.c_void_p(x.data_ptr()), None)
    for D in (512, 272):
        assert raw((1 << 27) - 8, D) == ag.AG_EHIP
        assert raw(1 << 27, D) == ag.AG_EUNSUPPORTED
    assert raw((1 << 31) - 1, 16) == ag.AG_EHIP
    ctx.close()


def test_tree_refusals(lib):  # noqa: F811
    ctx = ag.Context(device=-1, workspace=ag.q8_tree_workspace_bytes(1, 8, 4, 2, 64, 3))
    q, k, f = torch.zeros(1, 4, 8, 64, dtype=BF), torch.zeros(1, 2, 8, 64, dtype=BF), torch.zeros(1, 2, 8, dtype=torch.uint8)
    p, last, r, c, o = torch.full((1, 8), -1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), rope(), cache(), torch.zeros(1, 4, 8, 64, dtype=BF)
    attn = lambda q_=q, k_=k, v_=k, f_=f, p_=p, r_=r, s_=0.1, c_=c, o_=o: ag.ag_q8_tree_attn(ctx, q_, k_, v_, f_, p_, r_, s_, c_, o_, stream=0)  # noqa: E731
    append = lambda k_=k, v_=k, f_=f, p_=p, l_=last, r_=r, c_=c: ag.ag_q8_tree_append(ctx, k_, v_, f_, p_, l_, r_, c_, stream=0)  # noqa: E731
    for call in (attn, append):
        expect(ag.AG_EHIP, call)
        expect(ag.AG_EHIP, call, f_=None, r_=None)
        uneven = rope(axes=3)
        uneven.c.section[0], uneven.c.section[1] = 9, 7
        expect(ag.AG_EUNSUPPORTED, call, r_=uneven)
        for field in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "page", "len"):
            bad = cache()
            setattr(bad.c, field, None)
            expect(ag.AG_EINVAL, call, c_=bad)
        for kw in ({"p_": p.long()}, {"p_": p[:, :7].contiguous()}, {"f_": f[:, :, :7].contiguous()}, {"f_": f.int()}, {"k_": k.float(), "v_": k.float()},
                   {"v_": k[:, :, :7].contiguous()}, {"r_": rope(L=7)}):
            with pytest.raises(ValueError):
                call(**kw)
        with pytest.raises(TypeError):
            call(p_=None)
    with pytest.raises(ValueError):
        append(l_=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        attn(o_=o.float())
    for scale in (0.0, -1.0, math.inf, math.nan):
        expect(ag.AG_EINVAL, attn, s_=scale)
    q3, q6 = (torch.zeros(1, n, 8, 64, dtype=BF) for n in (3, 6))
    expect(ag.AG_EINVAL, attn, q_=q3, o_=q3)
    expect(ag.AG_EUNSUPPORTED, attn, q_=q6, o_=q6)
    n = 257
    expect(ag.AG_EUNSUPPORTED, append, k_=torch.zeros(1, 2, n, 64, dtype=BF), v_=torch.zeros(1, 2, n, 64, dtype=BF), f_=None, p_=torch.zeros(1, n, dtype=torch.int32), r_=None)
    qn = torch.zeros(1, 4, n, 64, dtype=BF)
    expect(ag.AG_EUNSUPPORTED, attn, q_=qn, o_=qn, k_=qn[:, :2].contiguous(), v_=qn[:, :2].contiguous(), f_=None, p_=torch.zeros(1, n, dtype=torch.int32), r_=None)
    big = cache(D=64, B=64, Hkv=8, n_pages=1, blocks=1)
    qb, kb = torch.zeros(64, 64, 32, 64, dtype=BF), torch.zeros(64, 8, 32, 64, dtype=BF)
    big.c.max_blocks = 1 << 22
    expect(ag.AG_EUNSUPPORTED, attn, q_=qb, o_=qb, k_=kb, v_=kb, f_=None, p_=torch.zeros(64, 32, dtype=torch.int32), r_=None, c_=big)
    small = ag.Context(device=-1, workspace=1024)
    expect(ag.AG_EWORKSPACE, ag.ag_q8_tree_attn, small, q, k, k, f, p, r, 0.1, c, o, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_tree_append, small, k, k, f, p, last, r, c, stream=0)    # it needs none
    ctx.close()
    small.close()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 1), (8, 2), (32, 8)])
def test_a_tree_workspace_covers_smaller_trees(lib, Hq, Hkv):  # noqa: F811
    assert ag.q8_tree_workspace_bytes(1, 257, 1, 1, 64, 3) == ag.q8_tree_workspace_bytes(1, 0, 1, 1, 64, 3) == ag.q8_tree_workspace_bytes(1, 8, 6, 2, 64, 3) == 0
    last = 0
    for L in range(1, 257):
        n = ag.q8_tree_workspace_bytes(2, L, Hq, Hkv, 128, 30)
        assert n >= last > -1
        last = n


def test_pool_refusals(lib):  # noqa: F811
    n, U = 6, 2
    ctx = ag.Context(device=-1, workspace=ag.q8_pool_workspace_bytes(1, 2, n))
    a, b, ref = cache(), cache(), torch.zeros(n, dtype=torch.int32)
    for field in ("k", "v", "k_scale", "v_scale"):
        setattr(b.c, field, getattr(a.c, field))
    par, which, used = torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.uint8), torch.zeros(1, dtype=torch.int32)
    expect(ag.AG_EHIP, ag.ag_q8_reserve, ctx, a, ref, 64, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_fork, ctx, a, par, b, ref, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_release, ctx, a, ref, which, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_release, ctx, a, ref, None, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_compact_pages, ctx, a, ref, ref.clone(), used, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_remap, ctx, a, ref, stream=0)
    expect(ag.AG_EINVAL, ag.ag_q8_reserve, ctx, a, ref, -1, stream=0)
    moved = ref.clone()
    for bad in ((ref, ref, used), (ref, moved, ref[:1]), (ref, moved, moved[:1])):
        expect(ag.AG_EINVAL, ag.ag_q8_compact_pages, ctx, a, *bad, stream=0)
    for bad in (ref[:5], ref.long()):
        for call in (lambda x: ag.ag_q8_reserve(ctx, a, x, 1, stream=0), lambda x: ag.ag_q8_release(ctx, a, x, which, stream=0),
                     lambda x: ag.ag_q8_fork(ctx, a, par, b, x, stream=0), lambda x: ag.ag_q8_compact_pages(ctx, a, x, ref, used, stream=0),
                     lambda x: ag.ag_q8_compact_pages(ctx, a, ref, x, used, stream=0), lambda x: ag.ag_q8_remap(ctx, a, x, stream=0)):
            with pytest.raises(ValueError):
                call(bad)
    with pytest.raises(ValueError):
        ag.ag_q8_fork(ctx, a, torch.zeros(2, dtype=torch.int32), b, ref, stream=0)
    with pytest.raises(ValueError):
        ag.ag_q8_release(ctx, a, ref, torch.zeros(2, dtype=torch.uint8), stream=0)
    with pytest.raises(ValueError):
        ag.ag_q8_compact_pages(ctx, a, ref, ref, torch.zeros(2, dtype=torch.int32), stream=0)
    with pytest.raises(ValueError):
        ag.ag_q8_reserve(ctx, a, ref, 1 << 31, stream=0)
    # two caches that are one, or over two pools
    expect(ag.AG_EINVAL, ag.ag_q8_fork, ctx, a, par, a, ref, stream=0)
    expect(ag.AG_EINVAL, ag.ag_q8_fork, ctx, a, par, cache(), ref, stream=0)
    short, other = cache(blocks=2), cache(D=128)
    for field in ("k", "v", "k_scale", "v_scale"):
        setattr(short.c, field, getattr(a.c, field))
        setattr(other.c, field, getattr(a.c, field))
    expect(ag.AG_EINVAL, ag.ag_q8_fork, ctx, a, par, short, ref, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_fork, ctx, short, par, a, ref, stream=0)
    expect(ag.AG_EINVAL, ag.ag_q8_fork, ctx, a, par, other, ref, stream=0)
    none = ag.Context(device=-1)
    expect(ag.AG_EWORKSPACE, ag.ag_q8_reserve, none, a, ref, 1, stream=0)
    expect(ag.AG_EWORKSPACE, ag.ag_q8_compact_pages, none, a, ref, ref.clone(), used, stream=0)
    expect(ag.AG_EHIP, ag.ag_q8_fork, none, a, par, b, ref, stream=0)
    assert ag.q8_pool_workspace_bytes(1, 2, 0) == ag.q8_pool_workspace_bytes(0, 2, 5) == ag.q8_pool_workspace_bytes(1, 2, (1 << 25) + 1) == 0
    ctx.close()
    none.close()


# ---- the reference ----
def test_chains_and_paths():
    assert T.chains([-1, 0, 0, 2, -5, 4, 9, 7]) == [[0], [0, 1], [0, 2], [0, 2, 3], [4], [4, 5], [6], [7]]
    p = torch.tensor([-1, 0, 1, 0])
    assert T.path(p, 2) == [0, 1, 2] and T.path(p, 3) == [0, 3] and T.path(p, -1) == T.path(p, 4) == []


def test_a_chain_of_the_reference_is_a_turn():
    g = torch.Generator()
    g.manual_seed(2)
    c = R.Cache(1, 2, 64, 6, 3, g, [70, 0])
    q, k, v = (torch.randn(1, n, 12, 64, generator=g) for n in (4, 2, 2))
    f = torch.rand(1, 2, 12, generator=g) < 0.5
    assert torch.allclose(T.attend(c, q, k, v, f, T.random_tree(g, 1, 12, "chain"), 0.125), R.attend(c, q, k, v, f, 0.125), atol=1e-12)
    alone = T.attend(c, q, k, v, f, T.random_tree(g, 1, 12, "roots"), 0.125)
    for t in range(12):   # roots: every node is a turn of one token
        one = lambda x: x[:, :, t:t + 1]  # noqa: E731
        assert torch.allclose(alone[:, :, t:t + 1], R.attend(c, one(q), one(k), one(v), one(f), 0.125), atol=1e-12)


def test_pools_of_the_reference():
    page, ref = torch.tensor([[3, -1, -1], [-1, -1, -1]], dtype=torch.int32), torch.tensor([0, 2, 0, 1, 0], dtype=torch.int32)
    assert T.reserve(page, [64, 10], ref, 64) and page.tolist() == [[3, 0, -1], [2, -1, -1]] and ref.tolist() == [1, 2, 1, 1, 0]
    assert not T.reserve(page, [64, 64], ref, 128) and page.tolist() == [[3, 0, 4], [2, -1, -1]]
    moved, new, n = T.compact(torch.tensor([0, 2, 0, 0, 5, 1], dtype=torch.int32))
    assert n == 3 and moved.tolist() == [-1, 1, -1, -1, 0, 2] and new.tolist() == [5, 2, 1, 0, 0, 0]
    assert T.count([page], 5).tolist() == [1, 0, 1, 1, 1]

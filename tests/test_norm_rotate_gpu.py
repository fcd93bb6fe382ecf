"""Queries and keys normalised head by head and turned, against 64 bits.

An element's error: r from a sum of at most 512 squares in 32 bits (every rounding 2^-24, at most log2(32) + 16 of them in line, halved by the root:
under 2^-20 of r with the mean, the root and the division), two products (2^-24 each), the turn's two products and sum (2^-24 of |a cos| + |b sin|
each), and the store: half a step."""
import numpy as np
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
import tree_reference as T
from gpu_util import DEV, bf16_half_spacing, ensure_built
from test_q8_gpu import BF, gen, rope_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def bar(n, args, dtype):
    """n: the normalised vectors in 64 bits"""
    turned = lambda x, tab: R.turned64(x, tab, *args[1:]) if args else x  # noqa: E731
    size = turned(n.abs(), args[0].abs()).abs().numpy() if args else n.abs().numpy()
    if args:   # |a cos| + |b sin| whatever the signs: the lower half of a turn by (|cos|, -|sin|)
        tab = args[0].abs().clone()
        low = tab.clone()
        low[:, low.shape[1] // 2:] *= -1
        half = n.shape[-1] // 2
        size = np.concatenate([turned(n.abs(), low).numpy()[..., :half], turned(n.abs(), tab).numpy()[..., half:]], axis=-1)
    ref = (turned(n, args[0]) if args else n).numpy()
    fine = (2.0 ** -20 + 2.0 ** -21) * size + 2.0 ** -140
    return ref, fine + (bf16_half_spacing(ref) * (1 + 2.0 ** -7) + 2.0 ** -130 if dtype == BF else 0.0)


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("B,Hq,Hkv,L,D,axes,odd", [
    (1, 1, 1, 1, 16, 1, False), (3, 5, 2, 1, 128, 1, False), (2, 4, 4, 77, 64, 3, False), (2, 4, 1, 33, 128, 3, True), (1, 3, 0, 50, 256, 2, False),
    (2, 9, 3, 19, 48, 3, True), (1, 40, 8, 300, 128, 1, False), (1, 2, 2, 5, 512, 1, False), (2, 3, 1, 21, 80, 0, False), (1, 5, 5, 13, 496, 1, False),
    (1, 17, 1, 2, 112, 0, False)])
def test_norm_rotate(dtype, B, Hq, Hkv, L, D, axes, odd):
    g = gen(B * 1000 + L + D)
    args, rope = rope_of(g, D, B, L, axes, odd=odd) if axes else (None, None)
    size = torch.exp2(torch.randint(-12, 13, (B, 1, L, 1), generator=g).float())
    q, k = (torch.randn(B, Hq, L, D, generator=g) * size).to(dtype), (torch.randn(B, Hkv, L, D, generator=g) * size).to(dtype) if Hkv else None
    wq, wk = (torch.randn(D, generator=g).to(dtype) for _ in range(2))
    print("norm_rotate", dtype, B, Hq, Hkv, L, D, axes, flush=True)
    for eps in (1e-6, 0.3):
        ctx = ag.Context(0)
        dq, dk = q.to(DEV), k.to(DEV) if Hkv else None
        oq, ok = torch.full_like(dq, 7.0), torch.full_like(dk, 7.0) if Hkv else None
        dwq, dwk = wq.to(DEV), wk.to(DEV) if Hkv else None
        ag.ag_norm_rotate(ctx, dq, dk, dwq, dwk, eps, rope, oq, ok)
        eps32 = float(torch.tensor(eps, dtype=torch.float32))
        for x, w, out in ((q, wq, oq),) + (((k, wk, ok),) if Hkv else ()):
            ref, most = bar(T.normed64(x, w, eps32), args, dtype)
            assert (np.abs(out.double().cpu().numpy() - ref) <= most).all()
        ag.ag_norm_rotate(ctx, dq, dk, dwq, dwk, eps, rope, dq, dk)     # in place
        assert torch.equal(dq, oq) and (not Hkv or torch.equal(dk, ok))
        ctx.poll_error()


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_vectors_of_extreme_size(dtype):
    """Sums of squares beyond 32 bits; zeros; values that are not finite stay with their vector."""
    g, L, D = gen(5), 12, 128
    q = torch.randn(1, 2, L, D, generator=g)
    sizes = [2.0 ** 60, 2.0 ** 70, 2.0 ** 100, 2.0 ** 124, 2.0 ** -30, 2.0 ** -70, 2.0 ** -126, 0.0]
    for t, s in enumerate(sizes):
        q[:, :, t] *= s
    q[0, 0, 1, 5:] = 0.0
    q[0, 0, 8, 3], q[0, 1, 9, 7], q[0, 0, 10, 1] = float("inf"), float("nan"), float("-inf")
    q = q.to(dtype)
    w = torch.randn(D, generator=g).to(dtype)
    ctx, out = ag.Context(0), torch.empty(q.shape, dtype=dtype, device=DEV)
    ag.ag_norm_rotate(ctx, q.to(DEV), None, w.to(DEV), None, 1e-6, None, out, None)
    n = T.normed64(q, w, float(torch.tensor(1e-6)))
    ref, most = bar(n, None, dtype)
    got = out.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    fine = ~np.isnan(ref)
    assert (np.abs(got - ref) <= most)[fine].all()
    ctx.poll_error()


def test_a_position_outside_the_table_is_reported():
    g, B, L, D = gen(3), 2, 9, 64
    (tab, pos, sec), _ = rope_of(g, D, B, L, 1, rows=50)
    pos[0, 0, 3], pos[0, 1, 7] = 50, -4
    q, w = torch.randn(B, 2, L, D, generator=g), torch.ones(D)
    ctx, out = ag.Context(0), torch.empty(B, 2, L, D, device=DEV)
    ag.ag_norm_rotate(ctx, q.to(DEV), None, w.to(DEV), None, 1e-5, ag.Rope(tab.to(DEV), pos.to(DEV)), out, None)
    with pytest.raises(ag.AgError) as e:
        ctx.poll_error()
    assert e.value.status == ag.AG_EINVAL
    ref, most = bar(T.normed64(q, w, float(torch.tensor(1e-5))), (tab, pos, sec), torch.float32)
    assert (np.abs(out.double().cpu().numpy() - ref) <= most).all()
    ctx.poll_error()

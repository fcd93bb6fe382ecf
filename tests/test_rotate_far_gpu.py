"""Rotation and normalised rotation of more than 2^31 vectors: those behind the 2^31-th are found (the smallest such tensor, 64 GiB in place)."""
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
import tree_reference as T
from gpu_util import DEV, ensure_built
from test_q8_gpu import BF, gen

pytestmark = pytest.mark.gpu
B, D = (1 << 30) + 8, 16
MARKED = [0, 1, (1 << 29) - 1, 1 << 29, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, B - 1]  # sequences: of two heads, so the 2^31-th vector is 2^30's


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


@pytest.fixture
def vectors():
    if torch.cuda.get_device_properties(0).total_memory < 90 << 30:
        pytest.skip("needs 70 GiB")
    x = torch.zeros(B, 2, 1, D, dtype=BF, device=DEV)
    yield x
    del x
    torch.cuda.empty_cache()


def marked(x, g):
    new = torch.randn(len(MARKED), 2, 1, D, generator=g).to(BF)
    for i, b in enumerate(MARKED):
        x[b] = new[i].to(DEV)
    return new


def near(x):  # that the vectors beside the marked ones are as they were
    for b in (2, (1 << 30) - 2, B - 2):
        assert int(x[b].count_nonzero()) == 0


def test_more_than_2_31_vectors(vectors):
    g, x = gen(1), vectors
    new, tab = marked(x, g), R.table(40, D)
    pos = torch.zeros(1, B, 1, dtype=torch.int32, device=DEV)
    at = torch.arange(len(MARKED)).int() + 5
    for i, b in enumerate(MARKED):
        pos[0, b, 0] = at[i]
    ctx = ag.Context(0)
    print("rotate", tuple(x.shape), flush=True)
    ag.ag_rotate(ctx, x, None, ag.Rope(tab.to(DEV), pos, [D // 2]), x, None)
    got = torch.stack([x[b] for b in MARKED]).cpu()
    assert torch.equal(got, R.turned(new.float(), tab, at.view(1, -1, 1), [D // 2]).to(BF))
    near(x)
    del pos
    new, w = marked(x, g), torch.randn(D, generator=g).to(BF)
    print("norm_rotate", tuple(x.shape), flush=True)
    ag.ag_norm_rotate(ctx, x, None, w.to(DEV), None, 1e-6, None, x, None)
    got, want = torch.stack([x[b] for b in MARKED]).cpu().double(), T.normed64(new, w, float(torch.tensor(1e-6)))
    assert ((got - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want.abs()).all()  # the store's half step, the rest in 32 bits
    near(x)
    ctx.poll_error()


def test_more_than_2_31_vectors_of_k(vectors):
    """As k, behind one head of q: its place is found from its own number of heads."""
    g, x = gen(2), vectors
    q, w = torch.zeros(B, 1, 1, D, dtype=BF, device=DEV), torch.randn(D, generator=g).to(BF)
    new, dw, ctx = marked(x, g), w.to(DEV), ag.Context(0)
    print("norm_rotate, k", tuple(x.shape), flush=True)
    ag.ag_norm_rotate(ctx, q, x, dw, dw, 1e-6, None, q, x)
    got, want = torch.stack([x[b] for b in MARKED]).cpu().double(), T.normed64(new, w, float(torch.tensor(1e-6)))
    assert ((got - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want.abs()).all()
    near(x)
    assert int(q[-1].count_nonzero()) == 0 and int(q[1 << 30].count_nonzero()) == 0
    ctx.poll_error()

"""Scores that overflow 32 bits, in the attention over the paged 8-bit cache."""
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
from gpu_util import DEV, ensure_built
from test_q8_gpu import BF, check_out, ctx_of, gen, on_device, some

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("D", [64, 128])
def test_a_kept_token_that_sees_nothing_else_gets_its_own_value(D, sign):
    """The first token that is kept, over an empty cache: whatever its score is, its weight is 1."""
    g, L, big = gen(D), 4, 3e38
    ref = R.Cache(1, 2, D, 4, 1, g, [0, 0])
    dev, ctx = on_device(ref), ctx_of(ref, L, 4)
    q, k, v, f = some(g, 1, 4, L, D), some(g, 1, 2, L, D), some(g, 1, 2, L, D), torch.zeros(1, 2, L, dtype=torch.uint8)
    f[:, :, 3] = 1
    k[:, :, 3], q[:, :, 3] = big, sign * big
    out = torch.empty(1, 4, L, D, dtype=BF, device=DEV)
    ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), f.to(DEV), None, 1.0, dev, out)
    assert torch.equal(out.cpu(), v.repeat_interleave(2, dim=1))
    assert dev.len.tolist() == [1, 1]


def huge_cache(D, g):
    """Two units of 150 and 64 rows: keys of 2^100, every third of them 0"""
    ref = R.Cache(1, 2, D, 8, 4, g, [150, 64])
    at = R.places(D)[0]
    for x in [ref.codes[0][p] for p in range(ref.n_pages)] + [ref.tails[0][u] for u in range(2)]:
        x[at[::3].reshape(-1)] = 0.0
    ref.scales[0] *= 2.0 ** 100
    ref.tails[0] *= 2.0 ** 100
    return ref


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("call", ["turn", "step"])
def test_rows_of_zero_beside_scores_of_minus_infinity(D, call):
    """Query and keys so large that their scores pass 32 bits: those of 0 stay 0 and share the weight, those of -infinity have none."""
    g, L = gen(D + 1), 3 if call == "turn" else 1
    ref = huge_cache(D, g)
    sign = torch.randint(0, 2, (D,), generator=g).float() * 2 - 1
    for codes in (ref.codes[0], ref.tails[0]):       # all keys opposite to the queries
        codes.copy_(codes.abs())
    at = R.places(D)[0]
    for x in [ref.codes[0][p] for p in range(ref.n_pages)] + [ref.tails[0][u] for u in range(2)]:
        x[at] = x[at] * sign
    q = (-sign * 2.0 ** 100).expand(1, 4, L, D).to(BF).contiguous()
    k, v, f = torch.zeros(1, 2, L, D, dtype=BF), some(g, 1, 2, L, D), torch.zeros(1, 2, L, dtype=torch.uint8)
    dev, ctx, out = on_device(ref), ctx_of(ref, L, 4), torch.empty(1, 4, L, D, dtype=BF, device=DEV)
    if call == "turn":
        ag.ag_q8_prefill_attn(ctx, q.to(DEV), k.to(DEV), v.to(DEV), f.to(DEV), None, 0.1, dev, out)
    else:
        one = lambda x: x[:, :, 0].contiguous().to(DEV)  # noqa: E731
        step = torch.empty(1, 4, D, dtype=BF, device=DEV)
        ag.ag_q8_decode_attn(ctx, one(q), one(k), one(v), one(f), None, 0.1, dev, step)
        out[:, :, 0] = step
    check_out(out, R.attend(ref, q.double(), k.double(), v, f != 0, 0.1))

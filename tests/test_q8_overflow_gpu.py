"""Scores that overflow 32 bits, in the attention of prompts over the paged 8-bit cache."""
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
from gpu_util import DEV, ensure_built
from test_q8_gpu import BF, ctx_of, gen, on_device, some

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

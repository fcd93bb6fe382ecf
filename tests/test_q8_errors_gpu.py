"""The sticky device error of the calls over the paged 8-bit cache."""
import pytest
import torch

import paper_2410_12876_amd as ag
import q8_reference as R
from gpu_util import DEV, ensure_built
from test_q8_gpu import ctx_of, gen, on_device, some

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def test_missing_room_and_a_position_outside_the_table_are_both_reported():
    g, D, L = gen(1), 64, 100
    ref = R.Cache(1, 2, D, 2, 1, g, [10, 60])
    dev, ctx = on_device(ref), ctx_of(ref, L, 2)
    pos = torch.arange(L, dtype=torch.int32).view(1, 1, L).clone()
    pos[0, 0, 3] = 500
    rope = ag.Rope(R.table(200, D).to(DEV), pos.to(DEV))
    for _ in range(2):
        ag.ag_q8_append(ctx, some(g, 1, 2, L, D).to(DEV), some(g, 1, 2, L, D).to(DEV), None, rope, dev)
        for status in (ag.AG_ECAPACITY, ag.AG_EINVAL):
            with pytest.raises(ag.AgError) as e:
                ctx.poll_error()
            assert e.value.status == status
        ctx.poll_error()

"""What the teacher says makes its row non-finite where it is not finite itself, also of a token that the policy rules out."""
import math

import pytest
import torch

from paper_2603_01501_b200 import binding as gb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("said", [math.nan, math.inf], ids=str)
@pytest.mark.parametrize("vocab", [500, 60000])
@pytest.mark.parametrize("kind", ["top", "forward", "reverse"])
def test_not_finite_where_the_policy_has_nothing(kind, vocab, said):
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(4, vocab, generator=gen, device="cuda")
    ids = torch.rand(4, vocab, generator=gen, device="cuda").topk(9, 1).indices
    values = torch.log_softmax(torch.randn(4, 9, generator=gen, device="cuda"), 1) - 0.1
    low = torch.tensor([-300.0, -1e30, -1e30, -1e30], device="cuda")
    x.scatter_(1, ids[:, 3:4], low[:, None])                       # its share of the policy is 0
    keep = x[2].gather(0, ids[2])
    x[2] = -math.inf                                                # and there is no rest
    x[2].scatter_(0, ids[2], keep)
    values[:3, 3] = said
    for got in (gb.gac_distill(x, ids.to(torch.int32), values, kind), gb.gac_distill(x, ids.to(torch.int32), values, kind, grad=True)[0]):
        assert not bool(got[:3].isfinite().any()) and math.isfinite(float(got[3])), got

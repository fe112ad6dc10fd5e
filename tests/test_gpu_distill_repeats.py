"""Of several entries with one id the first counts: what the others say moves nothing, however large it is."""
import math

import pytest
import torch

from paper_2603_01501_b200 import binding as gb

import distill_far_ref as ref
from packed_ref import within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("said", [-3.0, 3.0, 2000.0, 1e30, math.inf, math.nan], ids=str)
@pytest.mark.parametrize("temperature", [0.001, 0.01, 1.0])
@pytest.mark.parametrize("kind", ["top", "forward", "reverse"])
@pytest.mark.parametrize("size", [(6, 500), (6, 60000), (4000, 500), (700, 30000)], ids=str)
def test_repeated_entries_say_nothing(size, kind, temperature, said):
    tokens, vocab = size
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(tokens, vocab, generator=gen, device="cuda") * temperature
    ids = (torch.randint(0, vocab, (tokens, 1), generator=gen, device="cuda") + (vocab // 40) * torch.arange(40, device="cuda")) % vocab
    values = torch.log_softmax(torch.randn(tokens, 40, generator=gen, device="cuda"), 1) - 0.1
    if kind == "top":
        values = values * temperature
    ids[0, 20:] = ids[0, :20]                  # pairs all over the row
    ids[1, 1:] = ids[1, :1]                    # one token throughout
    ids[2, 7] = ids[2, 3]                      # one pair
    ids[3, 0] = -1                             # what is absent does not come first
    ids[3, 30] = ids[3, 2]
    values[3, 2] = -math.inf
    ids[3, 31] = ids[3, 2]
    values[0, 20:] = values[1, 1:] = values[2, 7] = values[3, 31] = said
    w = 0.5 + torch.rand(tokens, generator=gen, device="cuda")
    ids = ids.to(torch.int32)
    want = ref.distill(x[:6], ids[:6], values[:6], kind, temperature, w[:6])
    loss, grad = gb.gac_distill(x, ids, values, kind, temperature, weights=w, grad=True)
    for got in (gb.gac_distill(x, ids, values, kind, temperature), loss):
        within(got[:6], *want["loss"], "loss")
    within(grad[:6], *want["grad"], "grad")
    low = values.clone()
    low[0, 20:] = low[1, 1:] = low[2, 7] = low[3, 31] = -30.0
    other = gb.gac_distill(x, ids, low, kind, temperature, weights=w, grad=True)
    within(other[0][:6], *want["loss"], "loss")
    within(other[1][:6], *want["grad"], "grad")
    assert torch.equal(other[0][4:], loss[4:]) and torch.equal(other[1][4:], grad[4:])
    if kind != "top" or tokens > 1000:          # whole rows; of parts of a row the sums may be told in another order
        assert torch.equal(other[0], loss) and torch.equal(other[1], grad)

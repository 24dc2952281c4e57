"""More tokens than one launch has threads for."""
import pytest
import torch

from layer_cases import DEV
from paper_2504_15299_amd import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("given", [True, False])
def test_tokens_of_more_than_one_launch(given):
    """Two experts, of which the token's one value says which, at its own bit-width."""
    T = (1 << 26) + 5
    want = torch.randint(0, 2, (T,), device=DEV, dtype=torch.int32,
                         generator=torch.Generator(DEV).manual_seed(1))
    x = (want * 2 - 1).float().view(T, 1)
    Wg = torch.tensor([[-1.0], [1.0]], device=DEV)
    table = torch.tensor([[3, 5]], dtype=torch.uint8, device=DEV)
    if given:
        r = api.route_scored(x * Wg.view(1, 2), 1, None, table, "sigmoid")
    else:
        r = api.route_scored(None, 1, None, table, "sigmoid", x=x, Wg=Wg)
    assert torch.equal(r.topk_idx.view(-1), want) and (r.topk_w == 1).all()
    assert torch.equal(r.topk_bits.view(-1), (3 + 2 * want).to(torch.uint8))
    ones = int(want.sum())
    hist = torch.zeros((2, 7), dtype=torch.int32)
    hist[0, 1], hist[1, 3] = T - ones, ones
    assert torch.equal(r.hist.cpu(), hist) and int(r.flags) == 0
    # the tokens of either expert in order
    perm = r.perm.long()
    assert not want[perm[:T - ones]].any() and want[perm[T - ones:]].all()
    for part in (perm[:T - ones], perm[T - ones:]):
        assert (part[1:] > part[:-1]).all()
    assert torch.equal(r.slot_of[perm].long(), torch.arange(T, device=DEV))

"""Tokens whose choice is looked for among more tokens than one list holds, against the
plain form in binary64."""
import numpy as np
import pytest
import torch

from layer_cases import DEV
from paper_2504_15299_amd import api
from test_gpu_sample import BF, F32, gpu, normal, run

pytestmark = pytest.mark.gpu

LIST = 512      # tokens that one list holds


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V,std", [(1500, 1e-3), (32000, 0.003), (50257, 0.02), (131072, 0.1)])
def test_top_p_in_bins_of_many_tokens(V, std, dtype):
    """Top-p over flat rows, whose bins (of 4/256 in units of log2) hold more than a
    list: the search starts over, with an empty list that every wave has seen full.  Many
    rows, twice: equal calls give equal tokens."""
    x = normal(24, V, dtype, std)
    width = 4 / 256 * np.log(2)
    top = x.float().amax(1, keepdim=True)
    assert all(torch.bincount(((t - r) / width).long()).max() > LIST
               for t, r in zip(top, x.float()))
    rng = np.random.default_rng(V)
    u, p = rng.random(24), rng.uniform(0.3, 0.95, 24)
    want = run(x, u, None, None, p)[0]
    many = x.repeat(40, 1).to(DEV)
    for _ in range(3):
        got, _ = api.sample(many, gpu(np.tile(u, 40), F32), top_p=gpu(np.tile(p, 40), F32))
        assert (got.view(40, 24).cpu().numpy() == want).all()


@pytest.mark.parametrize("dtype", [F32, BF])
def test_top_p_of_equal_logits(dtype):
    """All tokens in one bin, and of one key."""
    u = np.array([0.0, 0.25, 0.5, 0.75] * 64)
    x = torch.zeros((256, 4096), dtype=dtype)
    tokens, probs = api.sample(gpu(x), gpu(u, F32), top_p=gpu([0.5] * 256, F32))
    assert tokens.tolist() == [int(a * 2048) for a in u] and (probs == 2.0 ** -11).all()

"""NaN logits among masked ones: chosen last, and with a weight that says so."""
import numpy as np
import pytest

from paper_2504_15299_amd import api
from test_gpu_route_scored import gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T", [4, 100])
def test_rows_without_a_finite_logit(T, renorm, scoring):
    x = np.random.default_rng(0).standard_normal((T, 8)).astype(np.float32)
    x[1] = np.nan
    x[2] = -np.inf
    x[2, [1, 5]] = np.nan
    x[3] = -np.inf
    table = gpu(np.full((1, 8), 4, np.uint8))

    def route(k):
        r = api.route_scored(gpu(x), k, None, table, scoring, renorm=renorm)
        return r.topk_idx.cpu().numpy()[1:4], r.topk_w.cpu().numpy()[1:4]

    idx, w = route(3)
    assert idx.tolist() == [[0, 1, 2], [0, 2, 3], [0, 1, 2]]
    assert np.isnan(w[0]).all() and (w[1:] == 0).all()
    idx, w = route(8)
    assert idx.tolist() == [list(range(8)), [0, 2, 3, 4, 6, 7, 1, 5], list(range(8))]
    assert np.isnan(w[0]).all() and (w[2] == 0).all()
    # (a sum with a NaN in it is one)
    assert np.isnan(w[1, 6:]).all()
    assert (np.isnan(w[1, :6]) if renorm else w[1, :6] == 0).all()


@pytest.mark.parametrize("T", [4, 100])
def test_scores_beside_a_nan_do_not_depend_on_it(T):
    x = np.random.default_rng(1).standard_normal((T, 8)).astype(np.float32)
    x[1, 6] = np.nan
    x[2, :4], x[2, 6] = np.inf, np.nan
    table = gpu(np.full((1, 8), 4, np.uint8))
    r = api.route_scored(gpu(x), 8, None, table, renorm=False)
    idx, w = r.topk_idx.cpu().numpy(), r.topk_w.cpu().numpy()
    for t in (1, 2):
        assert idx[t, 7] == 6 and np.isnan(w[t, 7])
    e = np.exp(np.delete(x[1], 6).astype(np.float64))
    e = np.sort(e / e.sum())[::-1]
    assert (np.abs(w[1, :7] - e) <= 2.0 ** -24 * (1 + 1e-6) * e).all()
    assert w[2, :7].tolist() == [0.25] * 4 + [0.0] * 3

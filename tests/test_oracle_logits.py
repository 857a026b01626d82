"""The 64-bit definitions of the operators on logits, checked against differences, closed forms and brute force."""
import numpy as np
import pytest

from oracle import logits as ol


def _problem(seed, rows=4, V=23, k=5):
    rng = np.random.default_rng(seed)
    z = rng.normal(0, 2, (rows, V))
    index = np.stack([rng.choice(V, k, replace=False) for _ in range(rows)])
    value = np.log(rng.dirichlet(np.ones(k + 2), rows)[:, :k])
    return rng, z, index, value


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [0.7, 1.0, 2.5])
@pytest.mark.parametrize("double", [False, True])
def test_distill_gradient_is_the_losses_difference(tail, tau, double):
    rng, z, index, value = _problem(1)
    if double:
        index[:, 3] = index[:, 0]  # one column listed twice
    index[1, 2] = -1               # and an entry that is none
    w = rng.uniform(0.5, 2, z.shape[0])
    got = ol.distill(z, index, value, w, tau, tail)["grad"]
    eps = 1e-5
    for v in range(z.shape[1]):
        d = np.zeros(z.shape[1])
        d[v] = eps
        up, down = (ol.distill(z + s * d, index, value, w, tau, tail)["loss"] for s in (1, -1))
        # central differences: an error of eps^2 and of 2^-53 * |loss| / eps
        assert np.allclose((up - down) / (2 * eps), got[:, v], rtol=0, atol=1e-8)


def test_distill_against_closed_forms():
    _, z, _, _ = _problem(2, V=7)
    rows = np.arange(z.shape[0])
    index = np.tile(np.arange(7), (z.shape[0], 1))
    log_q = z - ol.log_sum_exp(z)[:, None]
    same = ol.distill(z, index, log_q, tail=True)
    assert np.allclose(same["loss"], 0, atol=1e-14) and np.allclose(same["grad"], 0, atol=1e-14)
    one_hot = ol.distill(z, index[:, :1] + 3, np.zeros((len(rows), 1)))
    assert np.allclose(one_hot["loss"], -log_q[:, 3])  # a certain teacher: the cross entropy
    # any constant on the values leaves the listed distribution alone
    a, b = (ol.distill(z, index[:, :4], log_q[:, :4] + c) for c in (0.0, 3.5))
    assert np.allclose(a["loss"], b["loss"]) and np.allclose(a["grad"], b["grad"])
    assert np.allclose(a["grad"].sum(1), 0, atol=1e-14)


def test_distill_rows_that_hold_nothing():
    _, z, index, value = _problem(3)
    none = np.full_like(index, -1)
    for tail in (False, True):
        got = ol.distill(z, none, value, tail=tail)
        assert np.allclose(got["loss"], 0) and np.allclose(got["grad"], 0)
    z[0] = -np.inf
    assert ol.distill(z, index, value)["loss"][0] == np.inf
    assert (ol.distill(z, index, value, np.zeros(4))["loss"] == 0).all()


def test_topk_orders_by_value_then_column():
    x = np.array([[1.0, 3.0, 3.0, -np.inf, 0.0, -0.0, 2.0], [-np.inf] * 7, [np.nan, 1, 2, 3, 4, 5, 6]])
    index, logp, lse = ol.topk(x, 6)
    assert index.tolist() == [[1, 2, 6, 0, 4, 5], [-1] * 6, [6, 5, 4, 3, 2, 1]]
    assert np.isclose(np.exp(logp[0]).sum(), 1) and (logp[1] == -np.inf).all() and np.isnan(logp[2]).all()
    assert lse[1] == -np.inf and np.isnan(lse[2])


def test_constrain_by_hand():
    x = np.array([[2.0, -2.0, 1.0, 0.5, 0.0]])
    got = ol.constrain(x, history=[[0, 1, 1, 2, 2, 2, 9, -1]], prompt_len=[3], theta=[2.0], frequency=[0.25], presence=[0.5],
                       biases=[[(3, 1.0), (3, 0.5), (7, 9.0)]], allowed=[np.array([1, 1, 1, 1, 0], bool)])
    assert got.tolist() == [[1.0, -4.0, 0.5 - (0.75 + 0.5), 2.0, -np.inf]]

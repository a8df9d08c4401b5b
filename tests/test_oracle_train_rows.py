"""The plain scoring and training operators: gradients against differences, the sort against numpy's."""
import numpy as np
import pytest

from oracle import train_rows as tr


def differences(f, x, step=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        g[i] = (f(a) - f(b)) / (2 * step)
    return g


@pytest.mark.parametrize("temperature", [1.0, 0.6, 1.7])
def test_logprobs_gradient(temperature):
    rng = np.random.default_rng(1)
    x, tokens = 2 * rng.standard_normal((5, 7)), np.array([3, 0, -1, 6, 2])
    g, h, z = rng.standard_normal((3, 5))

    def loss(v):
        lp, ent, lse, _, _ = tr.logprobs(v, tokens, temperature)
        return np.sum(g * lp + h * ent + z * lse)
    got, size = tr.logprobs_grad(x, tokens, temperature, g, h, z)
    assert np.max(np.abs(got - differences(loss, x))) < 1e-8
    assert np.all(size + 1e-15 >= np.abs(got)) and not got[2].any()


def test_logprobs_of_masked_logits():
    x = np.array([[0.0, -np.inf, 0.0], [-np.inf, -np.inf, -np.inf], [1.0, np.nan, 2.0], [np.inf, 0.0, 0.0]])
    lp, ent, lse, best, ids = tr.logprobs(x, np.array([0, 1, 0, 1]), top=3)
    assert np.isclose(lp[0], -np.log(2)) and np.isclose(ent[0], np.log(2)) and ids[0].tolist() == [0, 2, 1]
    assert np.isnan(lp[1:]).all() and np.isnan(ent[1:]).all() and (ids[1:] == -1).all() and np.isnan(best[1:]).all()
    assert lse[1] == -np.inf and np.isnan(lse[2:]).all()
    lowest = np.full((1, 4), np.finfo(np.float32).min, dtype=np.float64)
    assert np.allclose(tr.logprobs(lowest, np.array([2]))[0], -np.log(4))


def test_embed_gradient():
    rng = np.random.default_rng(2)
    table, tokens, g = rng.standard_normal((4, 3)), np.array([2, -1, 0, 2, 2]), rng.standard_normal((5, 3))
    got, _, rows = tr.embed_grad(g, tokens, 4, 1.5)
    assert np.allclose(got, differences(lambda t: np.sum(g * tr.embed(t, tokens, 1.5)), table), atol=1e-8)
    assert rows.tolist() == [1, 0, 3, 0]


@pytest.mark.parametrize("align", [1, 4])
def test_experts(align):
    rng = np.random.default_rng(3)
    n, k, e, d = 6, 3, 5, 4
    ids = rng.integers(-1, e + 1, size=(n, k))
    starts, source, position = tr.expert_sort(ids, e, align)
    flat = ids.reshape(-1)
    there = (flat >= 0) & (flat < e)
    order = np.argsort(np.where(there, flat, e), kind="stable")[:there.sum()]
    assert source[source >= 0].tolist() == order.tolist()
    assert all(position.reshape(-1)[a] == p for p, a in enumerate(source) if a >= 0) and (position.reshape(-1)[~there] == -1).all()
    assert all(s % align == 0 for s in starts) and len(source) >= starts[-1]
    x, w, g_out, g_packed = rng.standard_normal((n, d)), rng.standard_normal((n, k)), rng.standard_normal((n, d)), rng.standard_normal((len(source), d))
    packed = tr.expert_gather(x, source, k)
    g_x, _ = tr.expert_combine(g_packed, position)
    assert np.allclose(g_x, differences(lambda v: np.sum(g_packed * tr.expert_gather(v, source, k)), x), atol=1e-8)
    of_packed, of_weights, _ = tr.expert_combine_grad(g_out, packed, source, position, w)
    assert np.allclose(of_packed, differences(lambda v: np.sum(g_out * tr.expert_combine(v, position, w)[0]), packed), atol=1e-8)
    assert np.allclose(of_weights, differences(lambda v: np.sum(g_out * tr.expert_combine(packed, position, v)[0]), w), atol=1e-8)

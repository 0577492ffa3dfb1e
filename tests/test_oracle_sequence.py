"""Pins of the sequence operators' oracle by values that do not come from it:
central differences, an independent library's autograd, closed forms."""
import numpy as np
import pytest
import torch

import oracle


def _rng(*key):
    return np.random.default_rng([404, *key])


def _difference(f, x, g, eps=1e-6):
    """The directional derivative of f at x along g, by central differences."""
    return (f(x + eps * g) - f(x - eps * g)) / (2 * eps)


@pytest.mark.parametrize("coupled", [False, True])
@pytest.mark.parametrize("lens", [None, (4, 0, 7)])
def test_gated_scan_gradient(coupled, lens):
    r = _rng(1, int(coupled), lens is None)
    T, B, H = 7, 3, 4
    z, x = r.standard_normal((T, B, H)), r.standard_normal((T, B, H))
    h0, dhs, dhT = r.standard_normal((B, H)), r.standard_normal((T, B, H)), r.standard_normal((B, H))

    def loss(z, x, h0):
        h, hs = oracle.gated_scan(z, x, h0, lens, coupled)
        return (hs * dhs).sum() + (h[-1] * dhT).sum()

    dz, dx, dh0 = oracle.gated_scan_vjp(z, x, h0, lens, coupled, dhs, dhT)
    for name, grad, f in (("z", dz, lambda v: loss(v, x, h0)), ("x", dx, lambda v: loss(z, v, h0)),
                          ("h0", dh0, lambda v: loss(z, x, v))):
        at = {"z": z, "x": x, "h0": h0}[name]
        g = r.standard_normal(at.shape)
        want = _difference(f, at, g)
        assert abs((grad * g).sum() - want) <= 1e-7 * max(1.0, abs(want)), name

    # the same loss by the library's autograd, sequences cut to their lengths
    tz, tx, th = (torch.tensor(v, requires_grad=True) for v in (z, x, h0))
    total = 0.0
    for b in range(B):
        h = th[b]
        for t in range(T if lens is None else lens[b]):
            a = torch.sigmoid(tz[t, b])
            h = a * h + ((1 - a) * tx[t, b] if coupled else tx[t, b])
            total = total + (h * torch.tensor(dhs[t, b])).sum()
        total = total + (h * torch.tensor(dhT[b])).sum()
    total.backward()
    for got, t in ((dz, tz), (dx, tx), (dh0, th)):
        np.testing.assert_allclose(got, t.grad.numpy(), rtol=1e-12, atol=1e-13)


def test_gated_scan_closed_forms():
    T, B, H = 9, 1, 2
    x = _rng(2).standard_normal((T, B, H))
    half = np.zeros((T, B, H))                  # a = 1/2: a geometric sum
    h, _ = oracle.gated_scan(half, x, None, None, False)
    want = sum(0.5 ** (T - 1 - t) * x[t] for t in range(T))
    np.testing.assert_allclose(h[-1], want, rtol=1e-14)
    open_, shut = np.full((T, B, H), np.inf), np.full((T, B, H), -np.inf)
    h, hs = oracle.gated_scan(open_, x, np.ones((B, H)), None, True)
    assert (hs == 1).all()                      # nothing enters
    h, hs = oracle.gated_scan(shut, x, np.ones((B, H)), None, True)
    assert (hs == x).all()                      # nothing stays


@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_token_scores_against_the_library(scale):
    r = _rng(3)
    z = r.standard_normal((5, 11)) * 3
    z[1, 2:6] = -np.inf
    tokens = np.array([0, 10, -1, 3, 7])
    dlogp, dent = r.standard_normal(5), r.standard_normal(5)
    s = oracle.token_scores(z, tokens, scale, 4)
    t = torch.tensor(z, requires_grad=True)
    lp = torch.log_softmax(t * scale, 1)
    p = lp.exp()
    ent = -torch.where(p > 0, p * torch.where(p > 0, lp, 0.0), 0.0).sum(1)
    given = torch.stack([lp[i, c] if c >= 0 else lp.new_zeros(()) for i, c in enumerate(tokens)])
    np.testing.assert_allclose(s["logp"], given.detach(), rtol=1e-13, atol=1e-14)
    np.testing.assert_allclose(s["entropy"], ent.detach(), rtol=1e-13)
    np.testing.assert_allclose(s["lse"], torch.logsumexp(t * scale, 1).detach(), rtol=1e-13)
    v, i = lp.topk(4, dim=1)
    assert (s["top_ids"] == i.numpy()).all()
    np.testing.assert_allclose(s["top_logp"], v.detach(), rtol=1e-13)
    got = oracle.token_scores_vjp(z, tokens, scale, dlogp, dent)
    (given * torch.tensor(dlogp)).sum().backward(retain_graph=True)
    by_logp = t.grad.clone()
    np.testing.assert_allclose(oracle.token_scores_vjp(z, tokens, scale, dlogp, None), by_logp,
                               rtol=1e-12, atol=1e-14)
    # the entropy by differences (rows without masked classes)
    rows = [0, 2, 3, 4]
    g = r.standard_normal(z.shape)
    g[1] = 0

    def loss(v):
        o = oracle.token_scores(v, tokens, scale, 0)
        return (o["logp"] * dlogp)[rows].sum() + (o["entropy"] * dent)[rows].sum()

    want = _difference(loss, z, g)
    assert abs((got * g).sum() - want) <= 1e-7 * max(1.0, abs(want))


def test_token_scores_special_rows():
    z = np.array([[-np.inf] * 4, [1.0, 1.0, 2.0, 1.0], [0.0, np.nan, 1.0, 2.0], [np.inf, 0, 0, 0]])
    s = oracle.token_scores(z, [0, 9, 0, 0], 1.0, 3)
    assert s["lse"][0] == s["logp"][0] == -np.inf and s["entropy"][0] == 0
    assert s["top_ids"].tolist() == [[0, 1, 2], [2, 0, 1], [3, 2, 0], [0, 1, 2]]
    assert np.isnan(s["logp"][1]) and np.isfinite(s["lse"][1])
    assert np.isnan(s["lse"][2:]).all() and np.isnan(s["top_logp"][2:]).all()
    uniform = oracle.token_scores(np.zeros((1, 8)), [3], 1.0, 0)
    np.testing.assert_allclose([uniform["logp"][0], uniform["entropy"][0]], [-np.log(8), np.log(8)])


def test_embedding_is_the_product_of_one_hot_rows():
    r = _rng(4)
    V, E = 6, 3
    table, ids = r.standard_normal((V, E)), np.array([5, 0, -1, 5, 2, 6])
    hot = np.zeros((len(ids), V))
    for i, v in enumerate(ids):
        if 0 <= v < V:
            hot[i, v] = 1
    out = oracle.embedding(table, ids, 0.5)
    np.testing.assert_allclose(out[:5], 0.5 * hot[:5] @ table)
    assert np.isnan(out[5]).all() and (out[2] == 0).all()
    dout = r.standard_normal((len(ids), E))
    d, mag, cnt = oracle.embedding_grad(dout, ids, V, 0.5)
    np.testing.assert_allclose(d, 0.5 * hot.T @ dout)
    np.testing.assert_allclose(mag, 0.5 * hot.T @ np.abs(dout))
    assert cnt.tolist() == [1, 0, 1, 0, 0, 2]

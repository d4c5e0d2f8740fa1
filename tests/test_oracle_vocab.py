"""Pins of the float64 oracle of the operators over discrete values: finite differences and
autograd of the losses, the sums' closed forms, limits of the sampling rules."""

import numpy as np
import pytest
import torch

from oracle import vocab


def test_embedding_gradient_is_the_adjoint_of_the_lookup():
    rng = np.random.default_rng(0)
    ids = rng.integers(-2, 9, (3, 4, 5))
    table, d = rng.normal(size=(7, 6)), rng.normal(size=(3, 4, 5, 6))
    out = vocab.embed_forward(ids, table, 1.7)
    g = vocab.embed_backward(ids, d, 7, 1.7)
    assert np.isclose((out * d).sum(), (table * g).sum())
    assert np.all(out[(ids < 0) | (ids >= 7)] == 0)
    onehot = (ids[..., None] == np.arange(7)).astype(float)
    assert np.allclose(out, 1.7 * onehot @ table)
    assert np.array_equal(vocab.embed_forward(ids, table, 1.7, base=d), out + d)


ROWS = [(0, 1.0, 1.0), (1, 1.0, 1.0), (0, 2.0, 0.5), (1, 2.0, 0.3), (1, 0.5, 0.0)]


@pytest.mark.parametrize("tail,tau,alpha", ROWS)
def test_distillation_gradient_against_differences(tail, tau, alpha):
    rng = np.random.default_rng(5)
    V, k = 9, 4
    s, t = rng.normal(size=V), 2 * rng.normal(size=V)
    idx = np.argsort(-t)[:k]
    lse = np.log(np.exp(t / tau).sum())
    args = (idx, t[idx], lse, 2, tau, alpha, tail)
    _, g = vocab.distill_row(s, *args)
    for v in range(V):
        h = np.zeros(V)
        h[v] = 1e-6
        diff = (vocab.distill_row(s + h, *args)[0] - vocab.distill_row(s - h, *args)[0]) / 2e-6
        assert abs(diff - g[v]) < 1e-7
    assert abs(g.sum()) < 1e-12          # a shift of all logits changes nothing


@pytest.mark.parametrize("tail,tau", [(0, 1.0), (1, 3.0)])
def test_distillation_of_all_logits_is_the_whole_divergence(tail, tau):
    """With every class among the entries the loss is tau^2 KL(p || q), and 0 for equal logits."""
    rng = np.random.default_rng(6)
    s, t = rng.normal(size=12), rng.normal(size=12)
    lse = np.log(np.exp(t / tau).sum())
    L, g = vocab.distill_row(s, np.arange(12), t, lse, -1, tau, 1.0, tail)
    S = torch.tensor(s, requires_grad=True)
    p = torch.softmax(torch.tensor(t) / tau, 0)
    ref = tau * tau * (p * (torch.log(p) - torch.log_softmax(S / tau, 0))).sum()
    ref.backward()
    assert np.isclose(L, ref.item()) and np.allclose(g, S.grad.numpy())
    L0, g0 = vocab.distill_row(t, np.arange(12), t, lse, -1, tau, 1.0, tail)
    assert abs(L0) < 1e-12 and np.abs(g0).max() < 1e-12


def test_distillation_rows_that_say_nothing():
    s = np.array([0.3, -np.inf, 1.0])
    assert vocab.distill_row(s, [-1, 7], [1.0, 2.0], 0.0, -1, 1.0, 1.0, 0)[0] == 0.0
    L, g = vocab.distill_row(s, [-1, 7], [1.0, 2.0], 0.0, -1, 1.0, 1.0, 1)
    assert abs(L) < 1e-12 and np.abs(g).max() < 1e-12   # all mass is outside, on both sides
    assert vocab.distill_row(np.full(3, -np.inf), [0], [1.0], 0.0, 0, 1.0, 0.5, 1)[0] == 0.0
    a = vocab.distill_row(s, [0, 0, 2], [1.0, 9.0, 2.0], 0.0, -1, 1.0, 1.0, 0)
    b = vocab.distill_row(s, [0, 2], [1.0, 2.0], 0.0, -1, 1.0, 1.0, 0)
    assert a[0] == b[0] and np.array_equal(a[1], b[1])   # the first of a repeated class counts


def test_distillation_weights():
    rng = np.random.default_rng(7)
    s = rng.normal(size=(3, 5))
    idx, top = np.tile([0, 3], (3, 1)), rng.normal(size=(3, 2))
    loss, rows, g = vocab.distill_loss(s, idx, top, None, None, np.array([1.0, 0.0, 3.0]), None,
                                       1.0, 1.0, 0)
    assert np.isclose(loss, (rows[0] + 3 * rows[2]) / 4) and rows[1] == 0 and not g[1].any()
    loss, _, g = vocab.distill_loss(s, idx, top, None, None, np.zeros(3), None, 1.0, 1.0, 0)
    assert loss == 0 and not g.any()


def test_sampling_follows_the_probabilities():
    """Over an even grid of u the draws' shares are the kept probabilities to a grid step."""
    s = np.array([0.0, 2.0, -1.0, 2.0, 1.0])
    us = (np.arange(4000) + 0.5) / 4000
    for kw, kept in ((dict(), [0, 1, 2, 3, 4]), (dict(top_k=2), [1, 3]), (dict(top_k=1), [1]),
                     (dict(top_p=0.5), [1, 3]), (dict(min_p=0.3), [1, 3, 4]),
                     (dict(top_k=4, top_p=0.99), [0, 1, 3, 4]), (dict(temperature=0.0), [1])):
        p = np.zeros(5)
        p[kept] = np.exp(s[kept] / 1.0)
        p /= p.sum()
        draws = [vocab.sample_row(s, u=u, **kw) for u in us]
        share = np.bincount([t for t, _ in draws], minlength=5) / len(us)
        assert np.abs(share - p).max() <= 1 / 2000, kw
        for t, lp in draws[::100]:
            assert np.isclose(lp, np.log(p[t]), atol=1e-12)


def test_sampling_edges():
    inf = np.inf
    assert vocab.sample_row(np.full(4, -inf)) == (-1, -inf)
    assert vocab.sample_row([]) == (-1, -inf)
    assert vocab.sample_row([np.nan, 1.0], u=0.9)[0] == 1
    assert vocab.sample_row([inf, 1.0, inf], u=0.6) == (2, pytest.approx(-np.log(2)))
    assert vocab.sample_row([1.0, 1.0, 1.0], top_k=2, u=0.99)[0] == 1    # ties: lowest index
    assert vocab.sample_row([1.0, 1.0, 1.0, 1.0], top_p=0.5, u=0.99)[0] == 1
    assert vocab.sample_row([1.0, 5.0], top_p=0.0, u=0.99)[0] == 1
    assert vocab.sample_row([1.0, 1.0], u=float("nan"))[0] == 0
    assert vocab.sample_row([1.0, 1.0], u=7.0)[0] == 1
    assert vocab.sample_row([1.0, 1.0], min_p=2.0, u=0.9)[0] == 0


@pytest.mark.parametrize("mode", ["target", "mean"])
def test_decoder_backward_for_a_given_gradient(mode):
    """The decoder's backward fed with the cross entropy's gradient is decode_loss's, and it is the
    derivative of sum(dlog * logits)."""
    from oracle import ends
    rng = np.random.default_rng(2)
    B, R, C, E, Hd, K = 2, 6, 4, 5, 7, 3
    n_train, n_feat, n_class = np.array([2, 4]), np.array([4, 2]), np.array([3, 2])
    P = ends.unpack_ends_params(rng.normal(size=ends.ends_param_count(E, 1, Hd, K)), E, 1, Hd, K)
    Y = rng.normal(size=(B, R, C + 1, E))
    y = np.stack([rng.integers(0, c, R) for c in n_class])
    _, dY, dP, logits = ends.decode_loss(Y, y, n_train, n_feat, n_class, C, P, mode)
    assert np.array_equal(logits, ends.decode_logits(Y, n_train, n_feat, C, P, mode))
    lab = np.concatenate([y[b][n_train[b]:] for b in range(B)])
    nc = np.repeat(n_class, R - n_train)
    z = np.where(np.arange(K) < nc[:, None], logits, -np.inf)
    dlog = np.exp(z - z.max(1, keepdims=True))
    dlog = dlog / dlog.sum(1, keepdims=True)
    dlog[np.arange(len(lab)), lab] -= 1
    dlog /= len(lab)
    gY, gP = ends.decode_backward(Y, n_train, n_feat, C, P, mode, dlog)
    assert np.allclose(gY, dY) and all(np.allclose(gP[k], dP[k]) for k in gP)
    d = rng.normal(size=Y.shape)
    h = 1e-6
    f = lambda t: (dlog * ends.decode_logits(Y + t * d, n_train, n_feat, C, P, mode)).sum()  # noqa: E731
    assert abs((f(h) - f(-h)) / (2 * h) - (gY * d).sum()) < 1e-8

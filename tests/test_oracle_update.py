"""Pins of oracle/update.py: closed forms, central differences, torch's autograd in float64."""
import numpy as np
import pytest
import torch

from oracle import update as U


def _case(seed, rows=6, vocab=9):
    r = np.random.default_rng(seed)
    z = r.normal(size=(rows, vocab)) * 2
    y = r.integers(0, vocab, rows)
    l = U.log_softmax(z)[np.arange(rows), y]
    return r, z, y, l


def test_no_move_gives_the_policy_gradient():
    """l == l_old == l_ref: ratio 1, nothing clipped, no KL; the gradient is that of -sum A l."""
    r, z, y, l = _case(0)
    a = r.normal(size=6)
    lp, stats, g = U.policy_loss(z, y, l, a, lp_ref=l, kl_coef=0.3)
    np.testing.assert_allclose(lp, l, rtol=1e-14)
    np.testing.assert_allclose(stats, [-a.sum(), -a.sum(), 0.0, 0.0], atol=1e-12)
    p = np.exp(U.log_softmax(z))
    want = -a[:, None] * (np.eye(9)[y] - p)
    np.testing.assert_allclose(g, want, atol=1e-13)
    np.testing.assert_allclose(g.sum(1), 0.0, atol=1e-13)


@pytest.mark.parametrize("kl_coef", [0.0, 0.2])
def test_gradient_against_differences(kl_coef):
    """Rows inside the range, above it and below it, with advantages of both signs."""
    r, z, y, l = _case(1)
    moved, a = np.array([0.05, 0.5, 0.5, -0.5, -0.5, -0.1]), np.array([1.0, 1.5, -1.5, 0.7, -0.7, -1.0])
    w, ref = r.uniform(0.2, 1.0, 6), l + r.normal(size=6) * 0.4
    args = dict(lp_ref=ref, weight=w, kl_coef=kl_coef)
    _, stats, g = U.policy_loss(z, y, l - moved, a, **args)
    assert stats[3] == pytest.approx(w[1] + w[4])       # cut: too likely and good, too unlikely and bad
    h = 1e-6
    for i in np.ndindex(z.shape):
        up, dn = z.copy(), z.copy()
        up[i] += h
        dn[i] -= h
        d = (U.policy_loss(up, y, l - moved, a, **args)[1][0] - U.policy_loss(dn, y, l - moved, a, **args)[1][0]) / (2 * h)
        assert abs(d - g[i]) < 1e-8


def test_gradient_against_autograd():
    r, z, y, l = _case(2, rows=40, vocab=17)
    old, ref, a, w = l - 0.3 * r.normal(size=40), l + 0.3 * r.normal(size=40), r.normal(size=40), r.uniform(size=40) * (r.uniform(size=40) > 0.3)
    lp, stats, g = U.policy_loss(z, y, old, a, lp_ref=ref, weight=w, clip_low=0.1, clip_high=0.3, kl_coef=0.07, grad_scale=5.0)
    t = torch.tensor(z, requires_grad=True)
    tl = torch.log_softmax(t, 1)[torch.arange(40), torch.tensor(y)]
    rho, ta = torch.exp(tl - torch.tensor(old)), torch.tensor(a)
    x = torch.tensor(ref) - tl
    row = -torch.minimum(rho * ta, rho.clamp(0.9, 1.3) * ta) + 0.07 * (torch.exp(x) - x - 1)
    loss = (torch.tensor(w) * row).sum()
    (5.0 * loss).backward()
    assert stats[0] == pytest.approx(loss.item(), abs=1e-13)
    np.testing.assert_allclose(g, t.grad.numpy(), atol=1e-13)
    np.testing.assert_allclose(lp, np.where(w != 0, tl.detach().numpy(), 0.0), atol=1e-13)


def test_embedding_and_its_gradient_are_adjoint():
    """<embed(T), D> = <T, embed_grad(D)> for every T and D; padded rows give and take nothing."""
    r = np.random.default_rng(3)
    tok = np.array([4, -1, 0, 4, 4, 6, -1])
    T, D = r.normal(size=(7, 5)), r.normal(size=(7, 5))
    out, g = U.embed(T, tok, 1.7), U.embed_grad(D, tok, 7, 1.7)
    assert (out * D).sum() == pytest.approx((T * g).sum(), rel=1e-13)
    assert not out[1].any() and not g[1].any()
    np.testing.assert_allclose(U.embed_grad(D, tok, 7, 1.7, start=T), T + g)
    np.testing.assert_allclose(g[4], 1.7 * (D[0] + D[3] + D[4]))


def test_norm_and_clipping():
    t = [np.array([3.0]), np.array([[0.0, 4.0]]), np.array([])]
    assert U.grad_norm(t) == 5.0
    assert U.clip_factor(5.0, 1.0) == 0.2 and U.clip_factor(5.0, 5.0) == 1.0 and U.clip_factor(0.0, 1.0) == 1.0
    assert U.clip_factor(np.inf, 1.0) == 1.0 and U.clip_factor(np.nan, 1.0) == 1.0

"""The Actor's update in float64, from its formulas.  TEST INFRASTRUCTURE ONLY.

The clipped policy loss with a KL term towards the Reference (the paper trains with PPO and prints no formula; this is
the reading the product follows too), for row r with log-probability l of its token:

    rho = exp(l - l_old),  policy = -min(rho A, clamp(rho, 1 - lo, 1 + hi) A)
    x = l_ref - l,         kl = exp(x) - x - 1     (zero where the two agree, never negative)
    loss = sum over the rows of w (policy + kl_coef kl)

the embedding lookup with scaling and its gradient, and clipping by the global 2-norm.
"""
import numpy as np


def log_softmax(z):
    z = np.asarray(z, np.float64)
    m = z.max(-1, keepdims=True)
    return z - m - np.log(np.exp(z - m).sum(-1, keepdims=True))


def policy_loss(logits, tokens, lp_old, adv, lp_ref=None, weight=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0, grad_scale=1.0):
    """Returns lp [rows], stats [4] = (loss, policy, kl, clipped weight), dlogits [rows, vocab].  Rows of weight 0 or a
    negative token are left out."""
    rows, vocab = np.shape(logits)
    lp, grad, stats = np.zeros(rows), np.zeros((rows, vocab)), np.zeros(4)
    for r in range(rows):
        w = 1.0 if weight is None else float(weight[r])
        y = int(tokens[r])
        if y < 0 or w == 0.0:
            continue
        logp = log_softmax(logits[r])
        l, a = logp[y], float(adv[r])
        rho = np.exp(l - float(lp_old[r]))
        held = min(max(rho, 1.0 - clip_low), 1.0 + clip_high)
        cut = rho * a > held * a
        policy, slope = -min(rho * a, held * a), 0.0 if cut else -rho * a
        kl = 0.0
        if lp_ref is not None:
            x = float(lp_ref[r]) - l
            kl = np.expm1(x) - x
            slope -= kl_coef * np.expm1(x)
        lp[r] = l
        stats += w * np.array([policy + kl_coef * kl, policy, kl, float(cut)])
        onehot = np.arange(vocab) == y
        grad[r] = grad_scale * w * slope * (onehot - np.exp(logp))
    return lp, stats, grad


def embed(table, tokens, scale=1.0):
    out = np.zeros((len(tokens), np.shape(table)[1]))
    for r, v in enumerate(tokens):
        if v >= 0:
            out[r] = scale * np.asarray(table[v], np.float64)
    return out


def embed_grad(dout, tokens, vocab, scale=1.0, start=None):
    """The table's gradient, added to `start` if given."""
    out = np.zeros((vocab, np.shape(dout)[1])) if start is None else np.array(start, np.float64)
    for r, v in enumerate(tokens):
        if 0 <= v < vocab:
            out[v] += scale * np.asarray(dout[r], np.float64)
    return out


def grad_norm(tensors):
    return float(np.sqrt(sum((np.asarray(t, np.float64) ** 2).sum() for t in tensors)))


def clip_factor(norm, max_norm):
    return max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0

"""The output layer's operators and the orthogonalised update in 64 bits, from their formulas (CPU; no code shared with the library)."""
import math

import torch

F64 = torch.float64
USUAL = (3.4445, -4.7750, 2.0315)


def score(x, w, target):
    """float64 x [T, H], w [V, H]; target: int64 [T] -> (logits, logprob, entropy, stats)."""
    z = x @ w.t()
    m = z.max(dim=1).values
    d = z - m[:, None]
    log_sum = torch.log(torch.exp(d).sum(dim=1))
    lp = d - log_sum[:, None]
    entropy = -(torch.exp(lp) * lp).sum(dim=1)
    has = (target >= 0) & (target < w.shape[0])
    given = lp.gather(1, target.clamp(0, w.shape[0] - 1)[:, None])[:, 0]
    return z, torch.where(has, given, torch.zeros_like(given)), entropy, torch.stack((m, log_sum), dim=1)


def logits_grad(z, target, stats, entropy, g_logprob, g_entropy):
    """-> c [T, V]; rows without weight are 0 whatever z holds."""
    V = z.shape[1]
    lp = z - stats[:, :1] - stats[:, 1:]
    p = torch.exp(lp)
    has = (target >= 0) & (target < V)
    a = torch.where(has, g_logprob, torch.zeros_like(g_logprob))
    hot = torch.zeros_like(z)
    hot[has, target[has]] = 1.0
    c = a[:, None] * (hot - p)
    if g_entropy is not None:
        c = c - g_entropy[:, None] * p * (lp + entropy[:, None])
    none = (a == 0) & ((g_entropy == 0) if g_entropy is not None else True)
    return torch.where(none[:, None], torch.zeros_like(c), c), none


def orthogonal(g, steps, coefficients=None):
    """float64 [R, C] -> the last X."""
    norm = torch.sqrt((g * g).sum())
    x = g / norm if float(norm) else g
    for i in range(steps):
        a, b, c = coefficients[i] if coefficients else USUAL
        q = x @ x.t()
        x = a * x + b * (q @ x) + c * (q @ (q @ x))
    return x


def step(g, momentum, x, mu, nesterov, steps, coefficients, eta, shrink):
    """-> (momentum, x) after the step; momentum may be None."""
    u = g
    if momentum is not None:
        momentum = mu * momentum + g
        u = g + mu * momentum if nesterov else momentum
    return momentum, shrink * x - eta * orthogonal(u, steps, coefficients)


def finite(t):
    return bool(torch.isfinite(t).all()) and not math.isnan(float(t.sum()))

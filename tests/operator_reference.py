"""The operators on activations and on logits in 64 bits, from their formulas (CPU; no code shared with the library)."""
import math

import torch

F64 = torch.float64


def scale_bytes(v, group):
    """v: float64 [T, K] -> E8M0 bytes [T, ceil(K/group)]."""
    T, K = v.shape
    out = torch.zeros(T, -(-K // group), dtype=torch.int64)
    for g in range(out.shape[1]):
        most = v[:, g * group:(g + 1) * group].abs().amax(dim=1)
        for t in range(T):
            m = float(most[t])
            if not math.isfinite(m) or bool(torch.isnan(v[t, g * group:(g + 1) * group]).any()):
                out[t, g] = 255
                continue
            b = 1
            if m > 0:
                b = max(1, math.frexp(m)[1] - 8 + 127)          # too small by at least one, then the smallest that fits
                while m > 127 * 2.0 ** (b - 127):
                    b += 1
            out[t, g] = b
    return out


def code(v, scales, group):
    """Nearest whole multiples of the scales, ties to even -> int64 [T, K]."""
    s = scales.repeat_interleave(group, dim=1)[:, :v.shape[1]]
    q = torch.round(v / torch.exp2((s - 127).to(F64)))
    q = torch.where(s == 249, q.clamp(-63, 63), q)              # 64 at the largest scale would be 2^128
    return torch.where(s == 255, torch.zeros_like(q), q).to(torch.int64)


def decode(codes, scales, group):
    """Codes and bytes of any integer type -> float64 values."""
    s = scales.to(torch.int64).repeat_interleave(group, dim=1)[:, :codes.shape[1]]
    v = codes.to(F64) * torch.exp2((s - 127).to(F64))
    return torch.where(s == 255, torch.full_like(v, math.nan), v)


def norm(h, weight, eps):
    """-> (rstd, y) of the float64 stream h."""
    rstd = 1.0 / torch.sqrt((h * h).mean(dim=1) + eps)
    return rstd, h * rstd[:, None] * weight


def norm_grad(dy, h, weight, rstd, dh):
    n = h * rstd[:, None]
    g = dy * weight
    dx = rstd[:, None] * (g - n * (g * n).mean(dim=1, keepdim=True))
    return (dx if dh is None else dx + dh), (dy * n).sum(dim=0)


def token_logprob(x, target):
    """-> (logprob, entropy, stats, log p) of float64 logits."""
    m = x.amax(dim=1, keepdim=True)
    empty = m == -math.inf
    d = x - torch.where(empty, torch.zeros_like(m), m)
    log_sum = torch.log(torch.exp(d).sum(dim=1, keepdim=True))
    logp = torch.where(empty, torch.full_like(x, -math.inf), d - log_sum)
    p = torch.exp(logp)
    entropy = -torch.where(p == 0, torch.zeros_like(p), p * logp).sum(dim=1)
    none = (target < 0) | (target >= x.shape[1])
    given = logp.gather(1, torch.where(none, torch.zeros_like(target), target).long()[:, None])[:, 0]
    stats = torch.cat((m, torch.where(empty, torch.zeros_like(m), log_sum)), dim=1)
    return torch.where(none, torch.zeros_like(given), given), entropy, stats, logp


def top(x, k):
    """Indices of the k largest, of equal ones the lowest index first; a NaN counts as -inf."""
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    return torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]


def token_logprob_grad(x, target, g_logprob, g_entropy):
    _, entropy, _, logp = token_logprob(x, target)
    p = torch.exp(logp)
    has = (target >= 0) & (target < x.shape[1])
    a = torch.where(has, g_logprob, torch.zeros_like(g_logprob))[:, None]
    inner = torch.where(p == 0, torch.zeros_like(p), p * (logp + entropy[:, None]))
    dx = -a * p - g_entropy[:, None] * inner
    rows = torch.arange(x.shape[0])[has]
    dx[rows, target[has].long()] += a[has, 0]
    return dx

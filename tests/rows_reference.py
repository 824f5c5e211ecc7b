"""Plain 64-bit forms of the operators between sparse rows and dense rows, on
the CPU: entries are (row, column, value) triples, everything is float64."""
import math

import torch


def f64(t):
    return t.detach().cpu().double()


def lookup(rows, cols, vals, W, m, scale):
    """scale A W and the sum of the terms' magnitudes."""
    ok = (cols >= 0) & (cols < W.shape[0])
    r, c, v = rows[ok], cols[ok], vals[ok]
    out = torch.zeros((m, W.shape[1]), dtype=torch.float64)
    mag = torch.zeros_like(out)
    term = W[c] * v[:, None] * scale
    out.index_add_(0, r, term)
    mag.index_add_(0, r, term.abs())
    return out, mag


def lookup_grad(rows, cols, vals, G, v, scale):
    ok = (cols >= 0) & (cols < v)
    return lookup(cols[ok], rows[ok], vals[ok], G, v, scale)


def layer_norm(x, g, b, eps):
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + eps)
    return (x - mean) * rstd * g + b, mean[:, 0], rstd[:, 0]


def layer_norm_grad(dy, x, mean, rstd, g):
    h = (x - mean[:, None]) * rstd[:, None]
    a = dy * g
    dx = rstd[:, None] * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def distill_row(s, cols, vals, T):
    """(loss, gradient, q, p as a dense row, magnitude of the loss's terms) of one row."""
    V = s.numel()
    zero = torch.zeros(V, dtype=torch.float64)
    ok = (cols >= 0) & (cols < V)
    c, t = cols[ok], vals[ok]
    if c.numel() == 0 or bool((t == -math.inf).all()) or bool((s == -math.inf).all()):
        return 0.0, zero, zero, zero, 0.0
    logq = torch.log_softmax(s / T, 0)
    logp = torch.log_softmax(t / T, 0)
    p = logp.exp()
    term = torch.where(p == 0, 0.0, p * (logp - logq[c]))
    dense = zero.index_add(0, c, p)
    mag = torch.where(p == 0, 0.0, p * (logp.abs() + logq[c].abs())).sum()
    return float(T * T * term.sum()), T * (logq.exp() - dense), logq.exp(), dense, float(mag)

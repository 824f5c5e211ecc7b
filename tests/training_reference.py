"""Plain 64-bit forms of a training step's operators, on the CPU."""
import torch


def cross_entropy(x, w, t, scale, weight=None):
    """x, w in float64.  A dict of the results and of the magnitudes that bound their errors."""
    V = w.shape[0]
    z = scale * (x @ w.T)
    zmag = abs(scale) * (x.abs() @ w.abs().T)  # of the terms of each logit
    lse = torch.logsumexp(z, 1)
    named = (t >= 0) & (t < V)
    col = t.clamp(0, V - 1)
    hit = z.gather(1, col[:, None])[:, 0]
    loss = torch.where(named, lse - hit, 0.0)
    out = dict(loss=loss, lse=lse, hit=hit, zmag=zmag.amax(1), named=named)
    if weight is None:
        return out
    wt = torch.where(named, weight, 0.0)
    used = wt != 0
    q = torch.where(used[:, None], torch.exp(z - lse[:, None]) * wt[:, None], 0.0)
    g = q.clone()
    rows = torch.nonzero(used)[:, 0]
    g[rows, col[rows]] = wt[rows] * torch.expm1(hit[rows] - lse[rows])
    xs = torch.where(used[:, None], x, 0.0)
    out.update(dx=scale * (g @ w), dw=scale * (g.T @ xs), dx_mag=abs(scale) * (g.abs() @ w.abs()),
               dw_mag=abs(scale) * (g.abs().T @ xs.abs()), q_dx=abs(scale) * (q.abs() @ w.abs()),
               q_dw=abs(scale) * (q.abs().T @ xs.abs()), w_abs=abs(scale) * w.abs().sum(0), x_abs=abs(scale) * xs.abs().sum(0),
               used=used)
    return out

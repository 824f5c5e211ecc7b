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


def block_norm(x, b, gate, scale, post, pre, normed, eps):
    """Everything in float64; gate: one row per row of x.  (y, h, r1, r2, scale * gate * u)."""
    r1 = 1.0 / torch.sqrt(b.square().mean(1, keepdim=True) + eps) if normed else torch.ones_like(b[:, :1])
    term = scale * gate * (b * r1 * post)
    y = x + term
    r2 = 1.0 / torch.sqrt(y.square().mean(1, keepdim=True) + eps)
    return y, y * r2 * pre, r1, r2, term


def block_norm_grad(dy, dh, y, b, r1, r2, gate, scale, post, pre, normed, per, k):
    """Results in float64, each with a bound of its error in units of 2^-24: sums
    of n terms count k (along a row) or n + 8 (over rows) of their magnitudes."""
    m, d = y.shape
    n2, n1 = y * r2, b * r1
    a = dh * pre
    m2, m2_abs = (a * n2).mean(1, keepdim=True), (a * n2).abs().mean(1, keepdim=True)
    Y = dy + r2 * (a - n2 * m2)
    eY = k * (dy.abs() + r2 * (a.abs() + n2.abs() * m2_abs))
    f = scale * gate * post
    c, ec = f * Y, f.abs() * eY + 4 * (f * Y).abs()
    if normed:
        m1, m1_abs = (c * n1).mean(1, keepdim=True), (c * n1).abs().mean(1, keepdim=True)
        db = r1 * (c - n1 * m1)
        edb = r1 * (ec + n1.abs() * (ec * n1.abs()).mean(1, keepdim=True) + k * (c.abs() + n1.abs() * m1_abs))
    else:
        db, edb = c, ec + 2 * c.abs()

    def over(t, rows):
        return t.view(m // rows, rows, d).sum(1)

    g = scale * Y * n1 * post
    eg = (scale * n1 * post).abs() * eY + 4 * g.abs()
    p = scale * gate * Y * n1
    ep = (scale * gate * n1).abs() * eY + 4 * p.abs()
    q = dh * n2
    return dict(dx=(Y, eY), db=(db, edb), dgate=(over(g, per), over(eg + (per + 8) * g.abs(), per)),
                dpost=(p.sum(0), (ep + (m + 8) * p.abs()).sum(0)), dpre=(q.sum(0), ((m + 8) * q.abs()).sum(0)))


ADAM_BLOCK = 256


def adamw(w, g, m, v, lr, step, betas, eps, decay):
    """A step in float64: (w, m, v)."""
    b1, b2 = betas
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return w - lr * decay * w - lr * (m / (1 - b1 ** step)) / ((v / (1 - b2 ** step)).sqrt() + eps), m, v


def adam_decode(mc, vc, ms, vs):
    n = mc.numel()
    block = torch.arange(n) // ADAM_BLOCK
    q = mc.double() / 127
    return q * q.abs() * ms.double()[block], (vc.double() / 255) ** 4 * vs.double()[block]


def adam_encode(m, v):
    """(codes of m, of v, scales) of float64 values."""
    n = m.numel()
    blocks = -(-n // ADAM_BLOCK)
    pad = torch.zeros((2, blocks * ADAM_BLOCK), dtype=torch.float64)
    pad[0, :n], pad[1, :n] = m.abs(), v
    ms, vs = pad.view(2, blocks, ADAM_BLOCK).amax(2).float()
    block = torch.arange(n) // ADAM_BLOCK
    S, R = ms.double()[block], vs.double()[block]
    mc = torch.where(S > 0, (127 * (m.abs() / S).sqrt()).round().clamp(max=127), 0.0).nan_to_num(0.0) * m.sign()
    vc = torch.where(R > 0, (255 * (v / R) ** 0.25).round().clamp(max=255), 0.0).nan_to_num(0.0)
    vc = torch.where((v > 0) & (R > 0), vc.clamp(min=1), vc)
    return mc.to(torch.int8), vc.to(torch.uint8), ms, vs

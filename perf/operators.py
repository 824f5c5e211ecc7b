"""Cases of the operators between sparse rows and dense rows, forward and backward.

A case is one call of a model whose inputs and targets are sparse rows over
many columns: the lookup of tokens (or of weighted bags of columns, a CSR) in a
table of dense rows and the gradient of that table, the layer norm of the rows
looked up and its gradient, and the loss that distils a teacher's stored top
entries of each row into logits over all columns, alone or with its gradient.

`run` computes a pass either in plain torch operations in 32 bits (`own` false)
or by the library's calls (`own` true).
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5
_sp = None


def _library():
    global _sp
    if _sp is None:
        import paper_2608_09713_amd
        _sp = paper_2608_09713_amd
    return _sp


def listed():
    return [
        # the tokens of one decoding step of a small batch: latency
        dict(name="embed_step", op="embed", rows="tokens", N=8, V=32000, D=2048, dtype="bf16"),
        # the tokens of a batch of long prompts or of a training step
        dict(name="embed_prompt", op="embed", rows="tokens", N=65536, V=131072, D=4096, dtype="bf16"),
        # the table's gradient of a training step: Zipf-like tokens, some padding, most table rows unnamed
        dict(name="embed_grad_tokens", op="embed_grad", rows="tokens", N=65536, V=131072, D=4096, dtype="bf16"),
        # the same for weighted bags of columns (ragged k-mer rows, some of them empty), odd sizes
        dict(name="embed_grad_bags", op="embed_grad", rows="bags", N=65537, V=200003, D=250, d=24, dtype="f32"),
        # the norm of one decoding step's rows: latency
        dict(name="layer_norm_step", op="layer_norm", N=16, D=4096, dtype="bf16", pdtype="bf16"),
        # the norm of a training batch
        dict(name="layer_norm_batch", op="layer_norm", N=65536, D=4096, dtype="bf16", pdtype="bf16"),
        # odd rows of 16 bits with parameters in 32
        dict(name="layer_norm_grad_odd", op="layer_norm_grad", N=8191, D=1001, dtype="f16", pdtype="f32"),
        # the backward pass of a training batch with wide rows
        dict(name="layer_norm_grad_batch", op="layer_norm_grad", N=32768, D=8192, dtype="bf16", pdtype="bf16"),
        # the loss of a few held-out positions
        dict(name="distill_few", op="distill", teacher="top", N=4, V=32000, K=16, T=2.0, dtype="bf16"),
        # the loss over many rows of an odd width, against ragged similarity rows
        dict(name="distill_rows", op="distill", teacher="csr", N=8192, V=65537, K=48, T=0.5, dtype="f32"),
        # loss and gradient against ragged rows, 32 bits, odd sizes
        dict(name="distill_grad_csr", op="distill_grad", teacher="csr", N=1001, V=50021, K=96, T=1.0, dtype="f32"),
        # loss and gradient of a training step over a large vocabulary
        dict(name="distill_grad_step", op="distill_grad", teacher="top", N=4096, V=131072, K=64, T=2.0, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi] spread over its logarithm, odd more often than not."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.6 and n > 4:
        n |= 1
    return min(hi, max(lo, n))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "layer_norm", "layer_norm_grad", "distill", "distill_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("embed", "embed_grad"):
        rows = rng.choice(["tokens", "tokens", "bags"])
        if rows == "tokens":
            case = dict(op=op, rows=rows, N=_log(rng, 1, 65536), V=_log(rng, 256, 131072), D=_log(rng, 16, 4096),
                        dtype=dtype)
        else:
            case = dict(op=op, rows=rows, N=_log(rng, 16, 65536), V=_log(rng, 256, 200003), D=_log(rng, 16, 250),
                        d=rng.randint(2, 24), dtype=dtype)
        if dtype == "f32" and rows == "tokens":
            case["D"] = min(case["D"], 2047)
    elif op in ("layer_norm", "layer_norm_grad"):
        case = dict(op=op, N=_log(rng, 1, 65536), D=_log(rng, 16, 8192), dtype=dtype,
                    pdtype=rng.choice([dtype, "f32"]))
    else:
        case = dict(op=op, teacher=rng.choice(["top", "csr"]), N=_log(rng, 1, 8192), V=_log(rng, 1024, 131072),
                    K=_log(rng, 1, 128), T=rng.choice([0.5, 1.0, 2.0, 4.0]), dtype=dtype)
    while work(case)["bytes"] > 1.6e9:
        case["N"] = max(1, int(case["N"] * 0.7))
    return case


# ---- inputs

def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1_000_003 + stream) & 0x7FFFFFFFFFFF)
    return g


def _normal(shape, dtype, g, scale=1.0, shift=0.0):
    return torch.randn(shape, device=DEV, generator=g).mul_(scale).add_(shift).to(dtype)


def _spread(N, width, most, g):
    """(lengths, columns, kept): per row up to `most` distinct ascending columns
    of [0, width), a random number of them (0 for some rows)."""
    most = min(most, width)
    step = width // most
    lens = torch.randint(0, most + 1, (N, 1), device=DEV, generator=g)
    at = torch.arange(most, device=DEV)[None, :]
    cols = at * step + torch.randint(0, step, (N, most), device=DEV, generator=g)
    first = torch.randint(0, most, (N, 1), device=DEV, generator=g)
    kept = (at - first).remainder(most) < lens
    return lens[:, 0], cols, kept


def _csr(N, width, most, g, values):
    lens, cols, kept = _spread(N, width, most, g)
    row_ptr = torch.zeros(N + 1, dtype=torch.int64, device=DEV)
    row_ptr[1:] = lens.cumsum(0)
    return row_ptr, cols[kept].int(), values(cols.shape)[kept].contiguous()


def prepare(case, seed):
    op, dt = case["op"], DTYPE[case["dtype"]]
    N = case["N"]
    state = dict(case)
    if op in ("embed", "embed_grad"):
        V, D = case["V"], case["D"]
        state["scale"] = math.sqrt(D)
        if case["rows"] == "tokens":
            # log-uniform ranks (a few tokens make up most of a text), labelled
            # by the seed; one position in 32 is padding (-1)
            g = _gen(seed, 1)
            rank = (float(V) ** torch.rand(N, dtype=torch.float64, device=DEV, generator=g)).long().sub_(1).clamp_(0, V - 1)
            label = torch.randperm(V, device=DEV, generator=g)
            state["tokens"] = label[rank].masked_fill_(torch.rand(N, device=DEV, generator=g) < 1 / 32, -1)
        else:
            g = _gen(seed, 2)
            state["scale"] = 1.0 / case["d"]
            state["csr"] = _csr(N, V, 2 * case["d"], g,
                                lambda shape: 1.0 - torch.rand(shape, device=DEV, generator=g))
        if op == "embed":
            state["weight"] = _normal((V, D), dt, _gen(seed, 3), 0.02)
        else:
            state["grad"] = _normal((N, D), dt, _gen(seed, 4), 1.0 / 64)
    elif op in ("layer_norm", "layer_norm_grad"):
        D, pt = case["D"], DTYPE[case["pdtype"]]
        g = _gen(seed, 5)
        x = torch.randn((N, D), device=DEV, generator=g)
        x.mul_(torch.rand((N, 1), device=DEV, generator=g).mul_(3).add_(0.25))
        x.add_(torch.randn((N, 1), device=DEV, generator=g).mul_(0.5))
        state["x"] = x.to(dt)
        state["weight"] = _normal((D,), pt, _gen(seed, 6), 0.1, 1.0)
        state["bias"] = _normal((D,), pt, _gen(seed, 7), 0.1)
        if op == "layer_norm_grad":
            state["grad"] = _normal((N, D), dt, _gen(seed, 8), 1.0 / 64)
            x = state["x"].float()
            state["mean"] = x.mean(1)
            state["rstd"] = 1.0 / torch.sqrt((x - state["mean"][:, None]).square().mean(1) + EPS)
    else:
        V, T = case["V"], case["T"]
        usable = V - V // 128  # (the rest pads the table to a round size: masked)
        K = min(case["K"], usable)
        g = _gen(seed, 9)
        logits = torch.randn((N, V), device=DEV, generator=g).mul_(2.0)
        logits[:, usable:] = -math.inf
        if case["teacher"] == "top":
            # a teacher's K largest logits, descending, at columns in no order
            step = usable // K
            cols = torch.arange(K, device=DEV) * step + torch.randint(0, step, (N, K), device=DEV, generator=g)
            cols = cols.gather(1, torch.rand((N, K), device=DEV, generator=g).argsort(1))
            values = torch.randn((N, K), device=DEV, generator=g).mul_(2.0).add_(8.0).sort(1, descending=True).values
            logits.scatter_add_(1, cols, values.mul(0.5))  # (the student has learnt some of it)
            state["top"] = (values.to(dt), cols)
        else:
            # similarities of other rows in (0, 1], ragged, some rows without any
            state["csr"] = _csr(N, usable, 2 * K, g,
                                lambda shape: 1.0 - torch.rand(shape, device=DEV, generator=g))
        state["logits"] = logits.to(dt)
        if case["op"] == "distill_grad":
            w = torch.full((N,), 1.0 / N, device=DEV)
            state["row_weight"] = w.masked_fill_(torch.rand(N, device=DEV, generator=g) < 1 / 16, 0.0)
    return state


# ---- a pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    sp = _sp or _library()
    op = state["op"]
    if op in ("embed", "embed_grad"):
        rows = state.get("tokens")
        if rows is None:
            row_ptr, cols, values = state["csr"]
            rows = sp.DeviceCSR(state["N"], state["V"], row_ptr, cols, values, cols.numel())
        if op == "embed":
            return sp.embed(rows, state["weight"], state["scale"])
        return sp.embed_grad(rows, state["grad"], state["V"], state["scale"])
    if op == "layer_norm":
        return sp.layer_norm(state["x"], state["weight"], state["bias"], EPS)
    if op == "layer_norm_grad":
        return sp.layer_norm_grad(state["grad"], state["x"], state["mean"], state["rstd"], state["weight"],
                                  state["bias"])
    teacher = state.get("top")
    if teacher is None:
        row_ptr, cols, values = state["csr"]
        teacher = sp.DeviceCSR(state["N"], state["V"], row_ptr, cols, values, cols.numel())
    if op == "distill":
        return sp.distill(state["logits"], teacher, state["T"])
    return sp.distill_grad(state["logits"], teacher, state["T"], state["row_weight"])


def _entry_rows(row_ptr, n):
    N = row_ptr.numel() - 1
    return torch.repeat_interleave(torch.arange(N, device=row_ptr.device), row_ptr[1:] - row_ptr[:-1], output_size=n)


def _run_plain(state):
    op = state["op"]
    if op in ("embed", "embed_grad"):
        V, D, scale = state["V"], state["D"], state["scale"]
        tokens = state.get("tokens")
        if op == "embed":
            W = state["weight"]
            if tokens is not None:
                valid = ((tokens >= 0) & (tokens < V))[:, None]
                return (W[tokens.clamp(0, V - 1)].float() * scale).masked_fill_(~valid, 0.0).to(W.dtype)
            row_ptr, cols, values = state["csr"]
            rows = _entry_rows(row_ptr, cols.numel())
            out = torch.zeros((state["N"], D), device=W.device)
            out.index_add_(0, rows, W[cols].float() * values[:, None])
            return (out * scale).to(W.dtype)
        G = state["grad"]
        out = torch.zeros((V, D), device=G.device)
        if tokens is not None:
            valid = ((tokens >= 0) & (tokens < V))[:, None]
            out.index_add_(0, tokens.clamp(0, V - 1), G.float().masked_fill(~valid, 0.0))
        else:
            row_ptr, cols, values = state["csr"]
            rows = _entry_rows(row_ptr, cols.numel())
            out.index_add_(0, cols, G[rows].float() * values[:, None])
        return (out * scale).to(G.dtype)
    if op == "layer_norm":
        x = state["x"].float()
        mean = x.mean(1)
        c = x - mean[:, None]
        rstd = 1.0 / torch.sqrt(c.square().mean(1) + EPS)
        y = c * rstd[:, None] * state["weight"].float() + state["bias"].float()
        return y.to(state["x"].dtype), mean, rstd
    if op == "layer_norm_grad":
        g, x = state["grad"].float(), state["x"].float()
        rstd = state["rstd"][:, None]
        h = (x - state["mean"][:, None]) * rstd
        a = g * state["weight"].float()
        dx = rstd * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
        return (dx.to(state["x"].dtype), (g * h).sum(0).to(state["weight"].dtype), g.sum(0).to(state["bias"].dtype))
    s, T = state["logits"], state["T"]
    N, V = s.shape
    z = s.float()
    z = (z - z.max(1, keepdim=True).values) / T
    lse = z.exp().sum(1).log()
    if "top" in state:
        values, cols = state["top"]
        t = values.float()
        t = (t - t.max(1, keepdim=True).values) / T
        logp = t - t.exp().sum(1, keepdim=True).log()
        p = logp.exp()
        loss = T * T * (p * (logp - z.gather(1, cols) + lse[:, None])).sum(1)
        mass = torch.ones_like(lse)
        flat = (torch.arange(N, device=s.device)[:, None] * V + cols).view(-1)
    else:
        row_ptr, cols, values = state["csr"]
        rows = _entry_rows(row_ptr, cols.numel())
        t = values / T  # (similarities in (0, 1]: no maximum is needed)
        total = torch.zeros_like(lse).index_add_(0, rows, t.exp())
        logp = t - total.log()[rows]
        p = logp.exp()
        loss = torch.zeros_like(lse).index_add_(0, rows, p * (logp - z[rows, cols.long()] + lse[rows])) * (T * T)
        mass = (total > 0).float()
        flat = rows * V + cols
    if op == "distill":
        return loss
    w = state["row_weight"]
    grad = z.sub_(lse[:, None]).exp_().mul_(mass[:, None])
    grad.view(-1).index_add_(0, flat, p.reshape(-1), alpha=-1.0)
    return loss, grad.mul_((w * T)[:, None]).to(s.dtype)


# ---- the definition in 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    with torch.no_grad():
        if op in ("embed", "embed_grad"):
            return _exact_embed(state, op)
        if op in ("layer_norm", "layer_norm_grad"):
            return _exact_norm(state, op)
        return _exact_distill(state, op)


def _exact_embed(state, op):
    N, V, D, scale = state["N"], state["V"], state["D"], state["scale"]
    if "tokens" in state:
        cols = state["tokens"]
        rows = torch.arange(N, device=DEV)
        weight = torch.ones(N, dtype=torch.float64, device=DEV)
        named = (cols >= 0) & (cols < V)
        rows, cols, weight = rows[named], cols[named], weight[named]
    else:
        row_ptr, cols, values = state["csr"]
        rows = torch.bucketize(torch.arange(cols.numel(), device=DEV), row_ptr[1:], right=True)
        cols, weight = cols.long(), values.double()
    source, target, src, height = ((state["weight"], rows, cols, N) if op == "embed" else
                                   (state["grad"], cols, rows, V))
    # sums of each target row's entries as differences of a running sum over
    # the entries in the order of their targets
    order = torch.argsort(target, stable=True)
    end = torch.bincount(target, minlength=height).cumsum(0)
    out = torch.empty((height, D), dtype=torch.float64, device=DEV)
    step = max(1, int(2.0e8 // max(order.numel() + height, 1)))
    for c in range(0, D, step):
        part = source[:, c:c + step].double()[src[order]] * weight[order][:, None]
        total = torch.zeros((order.numel() + 1, part.shape[1]), dtype=torch.float64, device=DEV)
        torch.cumsum(part, 0, out=total[1:])
        out[:, c:c + step] = total[end]
        out[1:, c:c + step] -= total[end[:-1]]
    return out.mul_(scale)


def _exact_norm(state, op):
    x, w = state["x"], state["weight"].double()
    N, D = x.shape
    step = max(1, int(1.0e8 // D))
    if op == "layer_norm":
        y, means, rstds = [], [], []
        for r in range(0, N, step):
            part = x[r:r + step].double()
            mean = part.sum(1) / D
            var = ((part - mean[:, None]) ** 2).sum(1) / D
            rstd = (var + EPS) ** -0.5
            y.append((part - mean[:, None]) * rstd[:, None] * w + state["bias"].double())
            means.append(mean)
            rstds.append(rstd)
        return torch.cat(y), torch.cat(means), torch.cat(rstds)
    # y = w h + b, h = (x - mean) rstd: dx by the chain rule through mean and rstd
    dx, dw, db = [], 0.0, 0.0
    for r in range(0, N, step):
        g = state["grad"][r:r + step].double()
        rstd = state["rstd"][r:r + step].double()[:, None]
        c = x[r:r + step].double() - state["mean"][r:r + step].double()[:, None]
        dh = g * w
        d_rstd = (dh * c).sum(1, keepdim=True)
        d_var = d_rstd * (-0.5) * rstd ** 3
        d_c = dh * rstd + d_var * 2.0 * c / D
        d_mean = -(dh * rstd).sum(1, keepdim=True)
        dx.append(d_c + d_mean / D)
        dw = dw + (g * c * rstd).sum(0)
        db = db + g.sum(0)
    return torch.cat(dx), dw, db


def _exact_distill(state, op):
    s, T = state["logits"], state["T"]
    N, V = s.shape
    if "top" in state:
        values, cols = state["top"]
        K = cols.shape[1]
        starts = torch.arange(N + 1) * K
        values, cols = values.reshape(-1).double(), cols.reshape(-1)
    else:
        row_ptr, cols, values = state["csr"]
        starts = row_ptr.cpu()
        values, cols = values.double(), cols.long()
    loss = torch.zeros(N, dtype=torch.float64, device=DEV)
    grad = torch.empty((N, V), dtype=torch.float64, device=DEV) if op == "distill_grad" else None
    step = max(1, int(6.0e7 // V))
    for r in range(0, N, step):
        n = min(step, N - r)
        a, b = int(starts[r]), int(starts[r + n])
        lens = (starts[r + 1:r + n + 1] - starts[r:r + n]).to(DEV)
        # the teacher as a dense block of logits, -inf where it has no entry
        row = torch.repeat_interleave(torch.arange(n, device=DEV), lens, output_size=b - a)
        teacher = torch.full((n, V), -math.inf, dtype=torch.float64, device=DEV)
        teacher[row, cols[a:b]] = values[a:b] / T
        logq = torch.log_softmax(s[r:r + n].double() / T, 1)
        named = lens > 0
        logp = torch.log_softmax(teacher, 1)
        p = logp.exp().masked_fill_(~named[:, None], 0.0)
        term = torch.where(p > 0, p * (logp - logq), 0.0)
        loss[r:r + n] = term.sum(1) * (T * T)
        if grad is not None:
            scale = (state["row_weight"][r:r + n].double() * T * named)[:, None]
            grad[r:r + n] = (logq.exp() - p) * scale
    return loss if grad is None else (loss, grad)


# ---- what a pass cannot do without

def _named_rows(case):
    """Rows of the table that a pass's rows name, expected."""
    N, V = case["N"], case["V"]
    if case["rows"] == "bags":
        E = N * case["d"]
        return V * -math.expm1(-E / V)
    k = torch.arange(1, V + 1, dtype=torch.float64)
    p = torch.log((k + 1) / k) / math.log(V)
    return float(-torch.expm1(torch.log1p(-p.clamp_(max=1 - 1e-12)) * N).sum())


def work(case):
    op, N, es = case["op"], case["N"], BYTES[case["dtype"]]
    if op in ("embed", "embed_grad"):
        V, D = case["V"], case["D"]
        E = N if case["rows"] == "tokens" else N * case["d"]
        ids = 8 * N if case["rows"] == "tokens" else 8 * (N + 1) + 8 * E
        rows = min(_named_rows(case), E) + N if op == "embed" else N + V
        return dict(bytes=int(ids + rows * D * es), flops=int(2 * E * D))
    if op == "layer_norm":
        return dict(bytes=2 * N * case["D"] * es + 2 * case["D"] * BYTES[case["pdtype"]] + 8 * N,
                    flops=8 * N * case["D"])
    if op == "layer_norm_grad":
        return dict(bytes=3 * N * case["D"] * es + 3 * case["D"] * BYTES[case["pdtype"]] + 8 * N,
                    flops=15 * N * case["D"])
    V, K = case["V"], case["K"]
    teacher = N * K * (8 + es) if case["teacher"] == "top" else 8 * (N + 1) + N * K * 8
    if op == "distill":
        return dict(bytes=N * V * es + teacher + 4 * N, flops=5 * N * V)
    return dict(bytes=2 * N * V * es + teacher + 8 * N, flops=8 * N * V)

"""Cases of a training step's operators around the sparse ones: the cross entropy
of a linear layer over many columns with its gradient, the norms before and
after a block fused with its gate and residual scale with their gradient, and an
AdamW step over many tensors.

`run` computes a pass either in plain torch operations in 32 bits (`own` false)
or by the library's calls (`own` true).
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
LR, BETAS, ADAM_EPS, DECAY, STEP = 1e-3, (0.9, 0.999), 1e-8, 0.01, 100
BLOCK = 256  # elements that share a scale in 8-bit states
_sp = None


def _library():
    global _sp
    if _sp is None:
        import paper_2608_09713_amd
        _sp = paper_2608_09713_amd
    return _sp


def listed():
    return [
        # the score of one token of a sequence that is being decoded: latency, and one reading of the layer
        dict(name="ce_token", op="ce", N=1, V=32000, D=2048, dtype="bf16"),
        # the scores of an evaluation batch over a large vocabulary
        dict(name="ce_batch", op="ce", N=8192, V=131072, D=4096, dtype="bf16"),
        # 32 bits, odd sizes throughout
        dict(name="ce_odd", op="ce", N=1001, V=50021, D=250, dtype="f32"),
        # loss and gradients of a training step over a large vocabulary
        dict(name="ce_grad_step", op="ce_grad", N=4096, V=131072, D=4096, dtype="bf16"),
        # the same with odd sizes in IEEE 16 bits (rows that start on no boundary)
        dict(name="ce_grad_odd", op="ce_grad", N=2047, V=50021, D=1001, dtype="f16"),
        # the rows of one decoding step between two blocks: latency
        dict(name="norm_step", op="norm", N=16, D=4096, gate="vector", post=True, dtype="bf16", pdtype="bf16"),
        # the same of a batch of prompts, a gate for each sequence
        dict(name="norm_batch", op="norm", N=32768, D=4096, gate="group", post=True, dtype="bf16", pdtype="bf16"),
        # the backward pass of odd rows, parameters in 32 bits, block without its own norm
        dict(name="norm_grad_odd", op="norm_grad", N=8191, D=1001, gate="vector", post=False, dtype="f16", pdtype="f32"),
        # the backward pass of a training batch with wide rows and a gate for every element
        dict(name="norm_grad_batch", op="norm_grad", N=16384, D=8192, gate="full", post=True, dtype="bf16", pdtype="bf16"),
        # many small tensors, states in 32 bits: launches
        dict(name="adamw_many", op="adamw", count=160, n=2_000_003, bits=32, master=False, dtype="f32"),
        # a model's step: 16-bit parameters with copies in 32, states in 32
        dict(name="adamw_step", op="adamw", count=48, n=160_000_000, bits=32, master=True, dtype="bf16"),
        # the same with states in 8 bits
        dict(name="adamw_8bit", op="adamw", count=12, n=64_000_000, bits=8, master=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi] spread over its logarithm, odd more often than not."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.6 and n > 4:
        n |= 1
    return min(hi, max(lo, n))


def draw(rng):
    op = rng.choice(["ce", "ce_grad", "norm", "norm_grad", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("ce", "ce_grad"):
        case = dict(op=op, N=_log(rng, 1, 8192), V=_log(rng, 256, 131072), D=_log(rng, 16, 4096), dtype=dtype)
        # (a drawn case in 32 bits has an eighth of the products)
        most = (4.0e11 if dtype == "f32" else 3.2e12) * (1 if op == "ce" else 1.0 / 3)
        while 2.0 * case["N"] * case["V"] * case["D"] > most:
            case["N"] = max(1, int(case["N"] * 0.7))
        return case
    if op in ("norm", "norm_grad"):
        case = dict(op=op, N=_log(rng, 1, 65536), D=_log(rng, 16, 8192), gate=rng.choice(["none", "vector", "group", "full"]),
                    post=rng.random() < 0.6, dtype=dtype, pdtype=rng.choice([dtype, "f32"]))
        while work(case)["bytes"] > 1.0e9:
            case["N"] = max(1, int(case["N"] * 0.7))
        return case
    bits = rng.choice([32, 32, 8])
    return dict(op=op, count=_log(rng, 1, 12 if bits == 8 else 200), n=_log(rng, 10_000, 64_000_000), bits=bits,
                master=dtype != "f32" and rng.random() < 0.5, dtype=dtype)


# ---- inputs

def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1_000_003 + stream) & 0x7FFFFFFFFFFF)
    return g


def _normal(shape, dtype, g, scale=1.0, shift=0.0):
    return torch.randn(shape, device=DEV, generator=g).mul_(scale).add_(shift).to(dtype)


def _groups(case):
    """Rows of the gate: the largest number up to 8 that divides the rows evenly, for a gate of each sequence."""
    N = case["N"]
    return {"none": 0, "vector": 1, "group": max(g for g in range(1, 9) if N % g == 0), "full": N}[case["gate"]]


def _sizes(case):
    """Elements of each tensor, spread over three decades as a model's vectors and matrices are."""
    rng = random.Random(case["count"] * 1_000_003 + case["n"])
    share = [10.0 ** rng.uniform(0, 3) for _ in range(case["count"])]
    return [max(1, int(case["n"] * s / sum(share))) for s in share]


def prepare(case, seed):
    op, dt = case["op"], DTYPE[case["dtype"]]
    state = dict(case)
    if op in ("ce", "ce_grad"):
        N, V, D = case["N"], case["V"], case["D"]
        g = _gen(seed, 1)
        # logits of deviation 2, and of the target up to 16 more: some rows have learnt theirs
        W = _normal((V, D), dt, g, 2.0 / math.sqrt(D))
        rank = (float(V) ** torch.rand(N, dtype=torch.float64, device=DEV, generator=g)).long().sub_(1).clamp_(0, V - 1)
        t = torch.randperm(V, device=DEV, generator=g)[rank]
        x = torch.randn((N, D), device=DEV, generator=g)
        x += W[t].float() * (torch.rand((N, 1), device=DEV, generator=g) * 4.0)
        if N > 1:
            t.masked_fill_(torch.rand(N, device=DEV, generator=g) < 1 / 32, -1)  # (padding)
        state["x"], state["W"], state["targets"] = x.to(dt), W, t
        if op == "ce_grad":
            # the mean over the rows (times a loss scale for IEEE 16 bits), some rows left out
            w = torch.full((N,), (1024.0 if case["dtype"] == "f16" else 1.0) / N, device=DEV)
            state["row_weight"] = w.masked_fill_(torch.rand(N, device=DEV, generator=g) < (1 / 16 if N > 1 else 0), 0.0)
        return state
    if op in ("norm", "norm_grad"):
        N, D, pt = case["N"], case["D"], DTYPE[case["pdtype"]]
        g, G = _gen(seed, 2), _groups(case)
        state["scale"] = 0.5
        state["block"] = (torch.randn((N, D), device=DEV, generator=g)
                          * (torch.rand((N, 1), device=DEV, generator=g) * 3 + 0.25)).to(dt)
        state["gate"] = _normal((G, D) if G != 1 else (D,), dt if case["gate"] == "full" else pt, g, 0.5, 0.5) if G else None
        state["post_weight"] = _normal((D,), pt, g, 0.1, 1.0) if case["post"] else None
        state["pre_weight"] = _normal((D,), pt, g, 0.1, 1.0)
        x = _normal((N, D), dt, g, 2.0)
        if op == "norm":
            state["x"] = x
            return state
        state["y"] = x
        state["dy"], state["dh"] = _normal((N, D), dt, g, 1.0 / 64), _normal((N, D), dt, g, 1.0 / 64)
        state["rstd_post"] = 1.0 / torch.sqrt(state["block"].float().square().mean(1) + EPS) if case["post"] else None
        state["rstd_pre"] = 1.0 / torch.sqrt(x.float().square().mean(1) + EPS)
        return state
    sizes = _sizes(case)
    n = sum(sizes)
    state["sizes"] = sizes
    g = _gen(seed, 3)

    def split(t, lengths=sizes):
        return list(torch.split(t, lengths))

    master = _normal((n,), torch.float32, g, 0.02)
    p = master.to(dt)
    grad = _normal((n,), dt, g, 1e-2)
    state["flat"] = dict(p=p, grad=grad)
    if case["master"]:
        state["flat"]["master"] = master
    if case["bits"] == 32:
        state["flat"]["m"] = _normal((n,), torch.float32, g, 3e-3)
        state["flat"]["v"] = torch.rand((n,), device=DEV, generator=g).mul_(2e-4).add_(1e-6)
        return dict(state, views={k: split(t) for k, t in state["flat"].items()})
    # 8 bits: codes, and a scale for each block of a tensor; every block has an element of its scale
    blocks = [-(-s // BLOCK) for s in sizes]
    at = torch.tensor([0] + blocks).cumsum(0)[:-1].mul_(BLOCK).to(DEV)
    start = torch.tensor([0] + sizes).cumsum(0)[:-1].to(DEV)
    shift = torch.repeat_interleave(at - start, torch.tensor(sizes, device=DEV), output_size=n)
    state["place"] = torch.arange(n, device=DEV) + shift  # (of each element among whole blocks)
    first = state["place"] % BLOCK == 0
    mc = torch.randn((n,), device=DEV, generator=g).mul_(50).round_().clamp_(-127, 127).masked_fill_(first, 127.0)
    vc = torch.rand((n,), device=DEV, generator=g).mul_(254).add_(1).round_().clamp_(1, 255).masked_fill_(first, 255.0)
    B = sum(blocks)
    state["flat"].update(
        m=mc.to(torch.int8), v=vc.to(torch.uint8),
        m_scale=torch.rand((B,), device=DEV, generator=g).mul_(5e-3).add_(5e-3),
        v_scale=torch.rand((B,), device=DEV, generator=g).mul_(2e-4).add_(1e-4))
    views = {k: split(t, blocks if k.endswith("scale") else sizes) for k, t in state["flat"].items()}
    return dict(state, views=views)


# ---- a pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    sp = _sp or _library()
    op = state["op"]
    if op == "ce":
        return sp.linear_cross_entropy(state["x"], state["W"], state["targets"])
    if op == "ce_grad":
        return sp.linear_cross_entropy_grad(state["x"], state["W"], state["targets"], row_weight=state["row_weight"])
    if op == "norm":
        return sp.block_norm(state["x"], state["block"], state["gate"], state["scale"], state["post_weight"],
                             state["pre_weight"], norm_block=state["post"], eps=EPS)
    if op == "norm_grad":
        return sp.block_norm_grad(state["dy"], state["dh"], state["y"], state["block"], state["rstd_post"],
                                  state["rstd_pre"], state["gate"], state["scale"], state["post_weight"],
                                  state["pre_weight"])
    plan = state.get("plan")
    if plan is None:  # (a training program makes it once, for the tensors that it keeps)
        v = state["views"]
        none = [None] * len(v["p"])
        states = list(map(sp.AdamState, v["m"], v["v"], v.get("m_scale", none), v.get("v_scale", none)))
        plan = state["plan"] = sp.adamw_plan(v["p"], v["grad"], states, v.get("master"))
    plan.step(LR, STEP, BETAS, ADAM_EPS, DECAY)
    flat = state["flat"]
    if state["bits"] == 32:
        return flat["p"], flat.get("master"), flat["m"], flat["v"]
    return flat["p"], flat.get("master"), sp.adam_values(plan.states)


def _run_plain(state):
    op = state["op"]
    if op in ("ce", "ce_grad"):
        x, W, t = state["x"].float(), state["W"].float(), state["targets"]
        z = x @ W.t()
        top = z.max(1, keepdim=True).values
        lse = (z - top).exp_().sum(1).log_().add_(top[:, 0])
        valid = (t >= 0) & (t < W.shape[0])
        col = t.clamp(0, W.shape[0] - 1)[:, None]
        loss = (lse - z.gather(1, col)[:, 0]).masked_fill_(~valid, 0.0)
        if op == "ce":
            return loss, lse
        q = z.sub_(lse[:, None]).exp_()
        q.scatter_add_(1, col, torch.full_like(col, -1.0, dtype=torch.float32))
        q.mul_((state["row_weight"] * valid)[:, None])
        return loss, (q @ W).to(state["x"].dtype), (q.t() @ x).to(state["W"].dtype)
    if op in ("norm", "norm_grad"):
        dt, s = state["block"].dtype, state["scale"]
        b = state["block"].float()
        N, D = b.shape
        gate, post, pre = state["gate"], state["post_weight"], state["pre_weight"].float()
        G = 1 if gate is None or gate.dim() == 1 else gate.shape[0]
        gain = torch.full((1, D), s, device=DEV) if gate is None else gate.float().view(G, D) * s

        def spread(a):  # a row of the gate for every row
            return a.repeat_interleave(N // G, 0)

        if op == "norm":
            rstd_post = None
            if state["post"]:
                rstd_post = 1.0 / torch.sqrt(b.square().mean(1) + EPS)
                b = b * rstd_post[:, None] * post.float()
            y = state["x"].float() + spread(gain) * b
            rstd_pre = 1.0 / torch.sqrt(y.square().mean(1) + EPS)
            return y.to(dt), (y * rstd_pre[:, None] * pre).to(dt), rstd_post, rstd_pre
        dh, r2 = state["dh"].float(), state["rstd_pre"][:, None]
        n2 = state["y"].float() * r2
        a = dh * pre
        dy = state["dy"].float() + r2 * (a - n2 * (a * n2).mean(1, keepdim=True))
        dpre = (dh * n2).sum(0)
        du = spread(gain) * dy
        n1 = b * state["rstd_post"][:, None] if state["post"] else b
        u = n1 * post.float() if state["post"] else n1
        dgate = None
        if gate is not None:
            dgate = (dy * u * s).view(G, N // G, D).sum(1).view(gate.shape).to(gate.dtype)
        db, dpost = du, None
        if state["post"]:
            dpost = (du * n1).sum(0).to(post.dtype)
            c = du * post.float()
            db = state["rstd_post"][:, None] * (c - n1 * (c * n1).mean(1, keepdim=True))
        return dy.to(dt), db.to(dt), dgate, dpost, dpre.to(state["pre_weight"].dtype)
    flat = state["flat"]
    (b1, b2), p = BETAS, flat["p"]
    c1, c2 = 1.0 - b1 ** STEP, 1.0 - b2 ** STEP
    wide = flat.get("master")
    w = p.float() if wide is None else wide
    if state["bits"] == 32:
        g = flat["grad"].float()
        m = flat["m"].mul_(b1).add_(g * (1.0 - b1))
        v = flat["v"].mul_(b2).add_(g * g * (1.0 - b2))
        w = w - LR * DECAY * w - LR * ((m / c1) / ((v / c2).sqrt() + ADAM_EPS))
        out = (m, v)
    else:
        # (in 64 bits: a value next to a border between two codes goes to the one that is nearer)
        g, place = flat["grad"].double(), state["place"]
        block = place // BLOCK
        m = flat["m"].double() / 127.0
        m = m * m.abs() * flat["m_scale"].double()[block]
        v = (flat["v"].double() / 255.0) ** 4 * flat["v_scale"].double()[block]
        m = b1 * m + (1.0 - b1) * g
        v = b2 * v + (1.0 - b2) * (g * g)
        w = (w.double() * (1.0 - LR * DECAY) - LR * ((m / c1) / ((v / c2).sqrt() + ADAM_EPS))).float()
        whole = torch.zeros((2, flat["m_scale"].numel() * BLOCK), dtype=torch.float64, device=DEV)
        whole[0, place], whole[1, place] = m.abs(), v
        ms, vs = whole.view(2, -1, BLOCK).amax(2).float()
        mc = (127.0 * (m.abs() / ms.double()[block]).sqrt()).round().clamp(max=127.0).nan_to_num(0.0) * m.sign()
        vc = (255.0 * (v / vs.double()[block]).sqrt().sqrt()).round().clamp(1.0, 255.0).nan_to_num(0.0) * (v > 0)
        flat["m"].copy_(mc)
        flat["v"].copy_(vc)
        flat["m_scale"].copy_(ms)
        flat["v_scale"].copy_(vs)
        mv = ((mc / 127.0) * (mc / 127.0).abs() * ms.double()[block]).float()
        vv = ((vc / 255.0) ** 4 * vs.double()[block]).float()
        out = list(zip(torch.split(mv, state["sizes"]), torch.split(vv, state["sizes"])))
    if wide is not None:
        wide.copy_(w)
    p.copy_(w)
    return (p, wide, *out) if state["bits"] == 32 else (p, wide, out)


# ---- the definition in 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    with torch.no_grad():
        if case["op"] in ("ce", "ce_grad"):
            return _exact_ce(state, case["op"])
        if case["op"] in ("norm", "norm_grad"):
            return _exact_norm(state, case["op"])
        return _exact_adamw(state)


def _exact_ce(state, op):
    x, W, t = state["x"].double(), state["W"].double(), state["targets"]
    N, V = x.shape[0], W.shape[0]
    loss, lses, dx, dW = [], [], [], torch.zeros_like(W) if op == "ce_grad" else None
    step = max(1, int(1.5e8 // V))
    for r in range(0, N, step):
        part, col = x[r:r + step], t[r:r + step]
        named = (col >= 0) & (col < V)
        logq = torch.matmul(part, W.transpose(0, 1))
        lse = torch.logsumexp(logq, 1)
        logq -= lse[:, None]
        hot = torch.nonzero(named)[:, 0]
        row_loss = torch.zeros_like(lse)
        row_loss[hot] = -logq[hot, col[hot]]
        loss.append(row_loss)
        lses.append(lse)
        if dW is not None:
            q = logq.exp_()
            q[hot, col[hot]] = torch.expm1(-row_loss[hot])
            q *= (state["row_weight"][r:r + step].double() * named)[:, None]
            dx.append(torch.matmul(q, W))
            dW += torch.matmul(q.transpose(0, 1).contiguous(), part)
    if dW is None:
        return torch.cat(loss), torch.cat(lses)
    return torch.cat(loss), torch.cat(dx), dW


def _exact_norm(state, op):
    N, D = state["block"].shape
    gate, s, normed = state["gate"], state["scale"], state["post"]
    G = 1 if gate is None or gate.dim() == 1 else gate.shape[0]
    table = torch.ones((1, D), device=DEV, dtype=torch.float64) if gate is None else gate.double().view(G, D)
    post = state["post_weight"].double() if normed else None
    pre = state["pre_weight"].double()
    step = max(1, int(4.0e7 // D))
    parts, dgate, dpost, dpre = [], torch.zeros((G, D), device=DEV, dtype=torch.float64), 0.0, 0.0
    for r in range(0, N, step):
        rows = torch.arange(r, min(N, r + step), device=DEV)
        b, owner = state["block"][rows].double(), rows // (N // G)
        k = table[owner] * s
        if op == "norm":
            rp = (b.square().sum(1) / D + EPS) ** -0.5 if normed else None
            u = b * rp[:, None] * post if normed else b
            y = state["x"][rows].double() + k * u
            rq = (y.square().sum(1) / D + EPS) ** -0.5
            parts.append((y, y * rq[:, None] * pre, rp, rq))
            continue
        # h = y q pre with q = (mean y^2 + eps)^-1/2, so dq/dy = -q^3 y / D; the same for the block's norm
        y, q = state["y"][rows].double(), state["rstd_pre"][rows].double()[:, None]
        dh = state["dh"][rows].double()
        dq = (dh * pre * y).sum(1, keepdim=True)
        dy = state["dy"][rows].double() + dh * pre * q - dq * q ** 3 * y / D
        dpre = dpre + (dh * y * q).sum(0)
        if normed:
            p = state["rstd_post"][rows].double()[:, None]
            du = dy * k
            dp = (du * post * b).sum(1, keepdim=True)
            db = du * post * p - dp * p ** 3 * b / D
            dpost = dpost + (du * b * p).sum(0)
            u = b * p * post
        else:
            db, u = dy * k, b
        if gate is not None:
            dgate.index_add_(0, owner, dy * u * s)
        parts.append((dy, db))
    whole = [None if c[0] is None else torch.cat(c) for c in zip(*parts)]
    if op == "norm":
        return tuple(whole)
    return whole[0], whole[1], None if gate is None else dgate.view(gate.shape), dpost if normed else None, dpre


def _exact_adamw(state):
    flat = state["flat"]
    g = flat["grad"].double()
    p = (flat["master"] if "master" in flat else flat["p"]).double()
    if state["bits"] == 32:
        m, v = flat["m"].double(), flat["v"].double()
    else:
        block = torch.div(state["place"], BLOCK, rounding_mode="floor")
        code = flat["m"].double()
        m = code.sign() * (code / 127) ** 2 * flat["m_scale"].double()[block]
        v = (flat["v"].double() / 255).square().square() * flat["v_scale"].double()[block]
    m += (g - m) * (1 - BETAS[0])
    v += (g.square() - v) * (1 - BETAS[1])
    unbiased_m, unbiased_v = m / -math.expm1(STEP * math.log(BETAS[0])), v / -math.expm1(STEP * math.log(BETAS[1]))
    p -= LR * (DECAY * p + unbiased_m / (unbiased_v ** 0.5 + ADAM_EPS))
    wide = p if "master" in flat else None
    if state["bits"] == 32:
        return p, wide, m, v
    # the block's largest, in 32 bits, is its scale; borders lie half-way between two codes
    count = flat["m_scale"].numel()
    ms = torch.zeros(count, dtype=torch.float64, device=DEV).index_reduce_(0, block, m.abs(), "amax").float().double()[block]
    vs = torch.zeros(count, dtype=torch.float64, device=DEV).index_reduce_(0, block, v, "amax").float().double()[block]
    mc = torch.floor(127 * (m.abs() / ms) ** 0.5 + 0.5).clamp_(max=127)
    vc = torch.floor(255 * (v / vs) ** 0.25 + 0.5).clamp_(1, 255)
    m, v = m.sign() * (mc / 127) ** 2 * ms, (vc / 255) ** 4 * vs
    return p, wide, list(zip(torch.split(m, state["sizes"]), torch.split(v, state["sizes"])))


# ---- what a pass cannot do without

def work(case):
    op, es = case["op"], BYTES[case["dtype"]]
    if op in ("ce", "ce_grad"):
        N, V, D = case["N"], case["V"], case["D"]
        if op == "ce":
            return dict(bytes=(N + V) * D * es + 16 * N, flops=2 * N * V * D + 4 * N * V)
        return dict(bytes=2 * (N + V) * D * es + 16 * N, flops=6 * N * V * D + 6 * N * V)
    if op in ("norm", "norm_grad"):
        N, D, G = case["N"], case["D"], _groups(case)
        ps = BYTES[case["pdtype"]]
        gate = G * D * (es if case["gate"] == "full" else ps)
        params = (2 if case["post"] else 1) * D * ps
        if op == "norm":
            return dict(bytes=4 * N * D * es + gate + params + 8 * N, flops=12 * N * D)
        return dict(bytes=6 * N * D * es + 2 * gate + 2 * params + 8 * N, flops=28 * N * D)
    n = sum(_sizes(case))
    per = 2 * es + es + (8 if case["master"] else 0) + (16 if case["bits"] == 32 else 4 + 16.0 / BLOCK)
    if case["master"]:
        per -= es  # (the parameter itself is written only)
    if case["bits"] == 8:
        per += 8  # (the states' values are returned in 32 bits)
    return dict(bytes=int(n * per), flops=14 * n)

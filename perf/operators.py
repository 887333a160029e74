"""The operators around the gradient codec, as they are measured: from a language model's logits to
the gradient that is sent (token log probabilities, entropy, top alternatives, and their backward
pass), and from the averaged gradient that comes back to the weights (Newton-Schulz
orthogonalisation of matrix updates, alone and with its momentum and weight update).

``run`` computes an operator either in plain torch operations in 32 bits, or, where ``own`` is
true, through this package's calls.  ``exact`` restates the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}

# Coefficients (a, b, c) of X <- a X + b (X X^T) X + c (X X^T)^2 X, five times, as the Muon
# optimiser uses them.
QUINTIC = (3.4445, -4.7750, 2.0315)
STEPS = 5

# Matrices of one layer of the language model whose gradient the framework's largest workload
# has (24 such layers), and of ResNet-50, its convolutions as (outputs, inputs x kernel area).
LM_LAYER = ((1024, 4096), (4096, 1024), (1024, 3072), (1024, 1024))


def resnet50_matrices():
    shapes, inplanes = [(64, 3 * 49)], 64
    for planes, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
        for block in range(blocks):
            shapes += [(planes, inplanes), (planes, planes * 9), (planes * 4, planes)]
            if block == 0:
                shapes.append((planes * 4, inplanes))
            inplanes = planes * 4
    return shapes + [(1000, 2048)]


def matrices(case):
    """(rows, cols) of every matrix of a case, in the order in which they lie in the flat vector."""
    if case["model"] == "lm":
        return [s for _ in range(case["layers"]) for s in LM_LAYER]
    if case["model"] == "resnet50":
        return resnet50_matrices()
    return [(case["rows"], case["cols"])] * case["count"]


def layout(case):
    """Offsets of the matrices and the length of the flat vector; "gap" entries (biases, norms)
    lie behind each matrix, so that most do not start on a 16-byte boundary where it is odd."""
    offsets, at = [], 0
    for r, c in matrices(case):
        offsets.append(at)
        at += r * c + case["gap"]
    return offsets, at


def listed():
    return [
        # serving: the log probability of one sampled token and its 20 best alternatives
        dict(name="logprob, one token", op="logprob", rows=1, vocab=50257, stride=50257, dtype="bf16",
             top=20, temperature=0.8, masked=0.0),
        # a small decoding batch over a large vocabulary; two thirds of it ruled out by a grammar
        dict(name="logprob, 24 tokens, masked", op="logprob", rows=24, vocab=128001, stride=128008, dtype="f16",
             top=5, temperature=1.0, masked=0.67),
        # scoring a prompt: every token's log probability with alternatives
        dict(name="logprob, 2047 tokens, top 8", op="logprob", rows=2047, vocab=50257, stride=50257, dtype="bf16",
             top=8, temperature=1.0, masked=0.0),
        # forward pass of a training step: losses and entropies, rows padded to a multiple of 64
        dict(name="logprob, training forward", op="logprob", rows=4096, vocab=50257, stride=50304, dtype="f32",
             top=0, temperature=1.0, masked=0.0),
        # its backward pass on a small batch, odd sizes
        dict(name="logprob grad, 129 tokens", op="grad", rows=129, vocab=32003, stride=32003, dtype="f32",
             temperature=0.7, entropy=True),
        # and on a full one, with a weight on the entropy
        dict(name="logprob grad, 8192 tokens", op="grad", rows=8192, vocab=50257, stride=50257, dtype="bf16",
             temperature=1.0, entropy=True),
        # one small matrix: latency
        dict(name="orthogonalize, 96x160", op="orth", model="one", rows=96, cols=160, count=1, gap=0,
             src="bf16", dst="bf16"),
        # one square matrix of a language model's attention
        dict(name="orthogonalize, 1024x1024", op="orth", model="one", rows=1024, cols=1024, count=1, gap=0,
             src="bf16", dst="bf16"),
        # a few tall matrices of odd sizes, kept in 32 bits throughout
        dict(name="orthogonalize, 3 of 1537x611", op="orth", model="one", rows=1537, cols=611, count=3, gap=77,
             src="f32", dst="f32"),
        # one rank's share of a language model: momentum, then the update that the ranks exchange
        dict(name="update, two lm layers", op="update", model="lm", layers=2, gap=4096, dst="bf16"),
        # the whole language model on one GPU
        dict(name="update, 24 lm layers", op="update", model="lm", layers=24, gap=4096, dst="bf16"),
        # a convolutional model's 54 matrices of 24 shapes, stepped with 32-bit weights
        dict(name="step, resnet50", op="step", model="resnet50", gap=131),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprob", "logprob", "grad", "orth", "orth", "update", "step"])
    if op in ("logprob", "grad"):
        vocab = _log(rng, 1000, 160000)
        dtype = rng.choice(["f32", "bf16", "f16"])
        rows = _log(rng, 1, max(1, min(8192, 250_000_000 // vocab)))
        case = dict(op=op, rows=rows, vocab=vocab, stride=vocab + rng.choice([0, 0, 1, 7, -vocab % 64]),
                    dtype=dtype, temperature=rng.choice([1.0, 1.0, 0.6, 1.3]))
        if op == "logprob":
            return dict(case, top=rng.choice([0, 0, 1, 5, 8, 20, 32]), masked=rng.choice([0.0, 0.0, 0.5]))
        return dict(case, entropy=rng.choice([True, False]))
    if op == "orth":
        rows, cols = _log(rng, 24, 2500), _log(rng, 24, 5000)
        if rng.random() < 0.5:
            rows, cols = cols, rows
        small = min(rows, cols)
        most = 3e12 / (60.0 * small * small * max(rows, cols))
        wide = rng.random() < 0.4
        return dict(op=op, model="one", rows=rows, cols=cols, count=_log(rng, 1, max(1.0, min(48.0, most))),
                    gap=rng.choice([0, 0, 64, 77]), src="f32" if wide else rng.choice(["bf16", "f16"]),
                    dst="f32" if wide else rng.choice(["bf16", "f16"]))
    if op == "update":
        return dict(op=op, model="lm", layers=rng.randint(1, 20), gap=rng.choice([0, 1024, 4096, 4099]),
                    dst=rng.choice(["bf16", "f16"]))
    return dict(op=op, model="resnet50", gap=rng.randint(0, 2048))


# ---- what a user's program has in hand before the call -------------------------------------------

def _logits(case, gen):
    """Logits as a trained language model gives them: a broad bulk, one token that stands out in
    most rows, and for constrained decoding a share of the vocabulary at minus infinity."""
    rows, vocab = case["rows"], case["vocab"]
    full = torch.empty(rows, case["stride"], dtype=DTYPES[case["dtype"]], device="cuda")
    x = full[:, :vocab]
    for at in range(0, rows, 1024):
        part = torch.randn(min(1024, rows - at), vocab, generator=gen, device="cuda").mul_(2.5)
        best = torch.randint(0, vocab, (part.shape[0], 1), generator=gen, device="cuda")
        lift = 8.0 + 3.0 * torch.randn(part.shape[0], 1, generator=gen, device="cuda")
        part.scatter_add_(1, best, lift)
        if case.get("masked"):
            keep = torch.rand(vocab, generator=gen, device="cuda") >= case["masked"]
            part.masked_fill_(~keep, -math.inf)
        x[at:at + part.shape[0]] = part
    # a target is the best token half the time; one row in sixteen is padding (a negative target)
    any_token = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    coin = torch.rand(rows, generator=gen, device="cuda")
    targets = torch.where(coin < 0.5, x.float().argmax(1) if rows <= 1024 else any_token, any_token)
    if case.get("masked"):
        targets = x.float().argmax(1)   # a sampled token is one that the grammar allows
    if rows > 16:
        targets = torch.where(coin > 15 / 16, torch.full_like(targets, -100), targets)
    return x, targets


def _gradients(case, gen):
    """The flat gradient: per matrix a few strong directions over noise, as gradients of trained
    models have; entries between the matrices are other parameters'."""
    shapes, (offsets, length) = matrices(case), layout(case)
    flat = torch.randn(length, generator=gen, device="cuda").mul_(1e-4)
    for (r, c), at in zip(shapes, offsets):
        rank = min(8, r, c)
        left = torch.randn(r, rank, generator=gen, device="cuda") * (0.7 ** torch.arange(rank, device="cuda"))
        right = torch.randn(rank, c, generator=gen, device="cuda")
        flat[at:at + r * c].view(r, c).addmm_(left, right, alpha=2e-4)
    return flat


class _Plan:
    """The orthogonaliser's handle and workspace, which a program makes once for its model."""

    def __init__(self, case):
        import paper_1806_08054_b200 as ecq
        self.ecq = ecq
        shapes, (offsets, _) = matrices(case), layout(case)
        self.handle = ecq.ecq_muon_create(offsets, [s[0] for s in shapes], [s[1] for s in shapes],
                                          scales=[_scale(*s) for s in shapes])
        self.workspace = torch.empty(ecq.ecq_muon_workspace_bytes(self.handle), dtype=torch.uint8, device="cuda")
        ecq.ecq_muon_bind(self.handle, self.workspace)

    def __del__(self):
        self.ecq.ecq_muon_destroy(self.handle)


def _scale(rows, cols):
    """Factor of a matrix's update that makes its entries about 0.2 in size, whatever its shape."""
    return 0.2 * math.sqrt(max(rows, cols))


HYPER = dict(mu=0.95, lr=3e-4, decay=0.1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = {"case": case}
    if case["op"] in ("logprob", "grad"):
        x, targets = _logits(case, gen)
        rows = case["rows"]
        state.update(x=x, targets=targets)
        if case["op"] == "logprob":
            for name in ("logprob", "entropy", "lse"):
                state[name] = torch.empty(rows, device="cuda")
            if case["top"]:
                state["top_logprob"] = torch.empty(rows, case["top"], device="cuda")
                state["top_index"] = torch.empty(rows, case["top"], dtype=torch.int32, device="cuda")
            return state
        # the forward pass's results, and the loss's derivatives: a mean over the tokens, weighted
        # by advantages, less a small share of the entropy
        lse, ent = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        for at in range(0, rows, 1024):
            z = x[at:at + 1024].double() / case["temperature"]
            lse[at:at + 1024] = torch.logsumexp(z, 1)
            logp = torch.log_softmax(z, 1)
            ent[at:at + 1024] = -(logp.exp() * logp).sum(1)
        state.update(lse=lse, entropy=ent, d_x=torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda"))
        state["d_logprob"] = torch.randn(rows, generator=gen, device="cuda") / rows
        state["d_entropy"] = torch.full((rows,), -0.01 / rows, device="cuda") if case["entropy"] else None
        return state
    _, length = layout(case)
    state["grad"] = _gradients(case, gen)
    if case["op"] == "orth":
        state["grad"] = state["grad"].to(DTYPES[case["src"]])
        state["out"] = torch.zeros(length, dtype=DTYPES[case["dst"]], device="cuda")
    else:
        state["momentum"] = _gradients(case, gen).mul_(8.0)
        if case["op"] == "update":
            state["out"] = torch.zeros(length, dtype=DTYPES[case["dst"]], device="cuda")
        else:
            state["params"] = 0.02 * torch.randn(length, generator=gen, device="cuda")
    if own:   # the handle is the framework's own; the plain form needs none
        state["plan"] = _Plan(case)
    return state


# ---- plain forms ---------------------------------------------------------------------------------

def _plain_logprob(s):
    case, x, y = s["case"], s["x"], s["targets"]
    z = x.float() * (1.0 / case["temperature"])
    top = z.max(dim=1, keepdim=True).values
    d = z - top
    e = torch.exp(d)
    total = e.sum(dim=1, keepdim=True)
    logp = d - torch.log(total)
    out = {"lse": (top + torch.log(total))[:, 0]}
    out["entropy"] = -torch.where(e > 0, e * logp, 0.0).sum(dim=1) / total[:, 0]
    picked = torch.gather(logp, 1, y.clamp(min=0)[:, None])[:, 0]
    out["logprob"] = torch.where(y >= 0, picked, 0.0)
    if case["top"]:
        # unique keys: the value's order, then the lower index first
        bits = (x.float() + 0.0).view(torch.int32).to(torch.int64)
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        key = order * (1 << 32) - torch.arange(case["vocab"], device=x.device)
        index = torch.topk(key, case["top"], dim=1).indices
        value = torch.gather(logp, 1, index)
        out["top_index"] = torch.where(value > -math.inf, index, -1).to(torch.int32)
        out["top_logprob"] = value
    return out


def _plain_grad(s):
    case, x, y = s["case"], s["x"], s["targets"]
    scale = 1.0 / case["temperature"]
    logp = x.float() * scale - s["lse"][:, None]
    p = torch.exp(logp)
    g = torch.where(y >= 0, s["d_logprob"], 0.0)
    d = -g[:, None] * p
    if s["d_entropy"] is not None:
        d = d - s["d_entropy"][:, None] * torch.where(p > 0, p * (logp + s["entropy"][:, None]), 0.0)
    d.scatter_add_(1, y.clamp(min=0)[:, None], g[:, None])
    return (d * scale).to(x.dtype)


def _newton_schulz(x):
    """Of a batch of matrices [count, rows, cols]."""
    x = x / x.square().sum(dim=(1, 2), keepdim=True).sqrt()
    tall = x.shape[1] > x.shape[2]
    x = x.mT if tall else x
    a, b, c = QUINTIC
    for _ in range(STEPS):
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.mT if tall else x


def _groups(case):
    """Matrices of one shape together, each with the entries that they hold of the flat vector."""
    shapes, (offsets, _) = matrices(case), layout(case)
    return [(shape, [o for s, o in zip(shapes, offsets) if s == shape]) for shape in dict.fromkeys(shapes)]


def _orthogonalize(flat, out, case, newton_schulz, write):
    for (r, c), offsets in _groups(case):
        x = torch.stack([flat[o:o + r * c].view(r, c) for o in offsets])
        for o, y in zip(offsets, newton_schulz(x)):
            write(out[o:o + r * c].view(r, c), y, r, c)


def _plain_step(s):
    """Momentum (Nesterov's), orthogonalisation, and the update itself or the weights stepped by it."""
    case, mu, lr = s["case"], HYPER["mu"], HYPER["lr"]
    if case["op"] == "orth":
        _orthogonalize(s["grad"].float(), s["out"], case, _newton_schulz, lambda out, y, r, c: out.copy_(y))
        return s["out"]
    if "spans" not in s:
        covered = torch.zeros(s["grad"].numel(), dtype=torch.bool, device="cuda")
        for (r, c), offsets in _groups(case):
            for o in offsets:
                covered[o:o + r * c] = True
        s["spans"] = covered
    s["momentum"].copy_(torch.where(s["spans"], mu * s["momentum"] + s["grad"], s["momentum"]))
    u = s["grad"] + mu * s["momentum"]
    if case["op"] == "update":
        _orthogonalize(u, s["out"], case, _newton_schulz, lambda out, y, r, c: out.copy_(_scale(r, c) * y))
        return {"momentum": s["momentum"], "update": s["out"]}
    _orthogonalize(u, s["params"], case, _newton_schulz,
                   lambda p, y, r, c: p.mul_(1 - lr * HYPER["decay"]).sub_(y, alpha=lr * _scale(r, c)))
    return {"momentum": s["momentum"], "params": s["params"]}


# ---- one pass ------------------------------------------------------------------------------------

def run(state):
    s, case = state, state["case"]
    if not own:
        if case["op"] == "logprob":
            return _plain_logprob(s)
        return _plain_grad(s) if case["op"] == "grad" else _plain_step(s)
    import paper_1806_08054_b200 as ecq
    if case["op"] == "logprob":
        ecq.ecq_token_logprob(s["x"], s["targets"], s["logprob"], s["entropy"], s["lse"], s.get("top_logprob"),
                              s.get("top_index"), temperature=case["temperature"])
        return {k: s[k] for k in ("logprob", "entropy", "lse", "top_logprob", "top_index") if k in s}
    if case["op"] == "grad":
        ecq.ecq_token_logprob_grad(s["x"], s["targets"], s["lse"], s["entropy"], s["d_logprob"], s["d_entropy"],
                                   s["d_x"], temperature=case["temperature"])
        return s["d_x"]
    if case["op"] == "orth":
        ecq.ecq_muon_orthogonalize(s["plan"].handle, s["grad"], s["out"])
        return s["out"]
    ecq.ecq_muon_step(s["plan"].handle, s["grad"], s["momentum"], params=s.get("params"), update=s.get("out"), **HYPER)
    if case["op"] == "update":
        return {"momentum": s["momentum"], "update": s["out"]}
    return {"momentum": s["momentum"], "params": s["params"]}


def work(case):
    if case["op"] in ("logprob", "grad"):
        entries, size = case["rows"] * case["vocab"], DTYPES[case["dtype"]].itemsize
        if case["op"] == "grad":
            return {"bytes": 2 * entries * size + case["rows"] * (20 + 4 * case["entropy"]), "flops": 8 * entries}
        return {"bytes": entries * size + case["rows"] * (20 + 8 * case["top"]), "flops": 6 * entries}
    # symmetric products counted once: X X^T and (X X^T)^2, then the product with X
    flops = entries = 0
    for r, c in matrices(case):
        m, n = min(r, c), max(r, c)
        flops += STEPS * (m * m * n + m * m * m + 2 * m * m * n)
        entries += r * c
    if case["op"] == "orth":
        return {"bytes": entries * (DTYPES[case["src"]].itemsize + DTYPES[case["dst"]].itemsize), "flops": flops}
    return {"bytes": entries * (12 + (2 if case["op"] == "update" else 8)), "flops": flops}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("logprob", "grad"):
        tau, x, y = float(case["temperature"]), s["x"], s["targets"]
        parts = []
        for at in range(0, case["rows"], 512):
            z = x[at:at + 512].to(torch.float64) / tau
            logp = z - torch.logsumexp(z, dim=1, keepdim=True)
            p = logp.exp()
            plogp = torch.nan_to_num(p * logp, nan=0.0)
            entropy = -plogp.sum(1)
            t = y[at:at + 512]
            if case["op"] == "grad":
                one_hot = torch.zeros_like(p)
                real = t >= 0
                one_hot[torch.arange(len(t), device="cuda")[real], t[real]] = 1.0
                d = s["d_logprob"][at:at + 512, None].double() * real[:, None] * (one_hot - p)
                if case["entropy"]:
                    d -= s["d_entropy"][at:at + 512, None].double() * (plogp + p * entropy[:, None])
                parts.append((d / tau,))
                continue
            lp = torch.where(t >= 0, logp[torch.arange(len(t), device="cuda"), t.clamp(min=0)], 0.0)
            part = (entropy, lp, torch.logsumexp(z, dim=1))
            if case["top"]:
                part += (logp.sort(dim=1, descending=True).values[:, :case["top"]],)
            parts.append(part)
        whole = [torch.cat(v) for v in zip(*parts)]
        if case["op"] == "grad":
            return whole[0]
        out = {"entropy": whole[0], "logprob": whole[1], "lse": whole[2]}
        if case["top"]:
            out.update(top_logprob=whole[3], top_index=None)
        return out

    def polar(g):
        """The quintic iteration from its definition, one matrix."""
        x = g / torch.linalg.matrix_norm(g)
        for _ in range(STEPS):
            if x.shape[0] <= x.shape[1]:
                gram = x @ x.T
                x = QUINTIC[0] * x + QUINTIC[1] * (gram @ x) + QUINTIC[2] * (gram @ (gram @ x))
            else:
                gram = x.T @ x
                x = QUINTIC[0] * x + QUINTIC[1] * (x @ gram) + QUINTIC[2] * ((x @ gram) @ gram)
        return x

    shapes, (offsets, length) = matrices(case), layout(case)
    grad = s["grad"].double()
    if case["op"] == "orth":
        result, momentum = torch.zeros_like(grad), None
    else:
        momentum = s["momentum"].double()
        result = s["params"].double() if case["op"] == "step" else torch.zeros_like(grad)
    for (r, c), at in zip(shapes, offsets):
        here = slice(at, at + r * c)
        g = grad[here]
        if momentum is not None:
            momentum[here] = HYPER["mu"] * momentum[here] + g
            g = g + HYPER["mu"] * momentum[here]
        o = polar(g.view(r, c)).reshape(-1)
        if case["op"] == "orth":
            result[here] = o
        elif case["op"] == "update":
            result[here] = 0.2 * max(r, c) ** 0.5 * o
        else:
            result[here] = (1 - HYPER["lr"] * HYPER["decay"]) * result[here] - HYPER["lr"] * 0.2 * max(r, c) ** 0.5 * o
    if case["op"] == "orth":
        return result
    return {"momentum": momentum, "update" if case["op"] == "update" else "params": result}

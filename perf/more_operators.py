"""The operators of a language model's layer in 8 bits, as they are measured: the root-mean-square
norm with the residual's addition and its gradient, matrices stored in 8 bits with a scale for each
block of 128 (both ways round) and restored, the gated activation that keeps its inputs in 8 bits and
its gradient from them, and the product of two such matrices.

``run`` computes an operator either in plain torch operations in 32 bits, or, where ``own`` is true,
through this package's calls.  ``exact`` restates the definitions in 64 bits.

A matrix in 8 bits is a pair (q, scales): q [rows, cols] in e4m3 or e5m2, and for each 128 consecutive
columns of a row a power of two, the smallest with which the block's largest magnitude is in the
type's range, as the byte exponent + 127.  The bytes lie in groups of 128 rows and four blocks:
((row // 128) * ceil(blocks / 4) + block // 4) * 512 + row % 32 * 16 + row % 128 // 32 * 4 + block % 4.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn,
          "e5m2": torch.float8_e5m2}
LARGEST = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
EPS = 1e-6


def listed():
    return [
        # generating: one token's residual and norm, and the projection that takes the norm's 8 bits
        dict(name="norm and product, one token", op="norm_product", rows=1, cols=1024, n=4096, dtype="bf16"),
        # forward pass of a training step, residual stream in bf16, kept in 8 bits for the backward pass
        dict(name="norm, 8192 tokens", op="norm", rows=8192, cols=4096, stride=4096, dtype="bf16", residual=True, kept=True),
        # its backward pass from what was kept in 8 bits
        dict(name="norm grad, 8192 tokens", op="norm_grad", rows=8192, cols=4096, stride=4096, dtype="bf16", saved="e4m3",
             joined=True),
        # a small batch in 32 bits of an odd width
        dict(name="norm grad, 515 tokens", op="norm_grad", rows=515, cols=1537, stride=1537, dtype="f32", saved="f32",
             joined=False),
        # a gradient stored both ways round, for the products with the weights and with the activations
        dict(name="store, 8192x4096", op="store", rows=8192, cols=4096, stride=4096, dtype="bf16", to="e4m3"),
        # odd sizes in 32 bits, with the wider range
        dict(name="store, 1001x2049", op="store", rows=1001, cols=2049, stride=2051, dtype="f32", to="e5m2"),
        # forward pass of the gated activation: 8 bits for the next product, both inputs kept in 8 bits
        dict(name="gate, 8192x4096", op="gate", rows=8192, cols=4096, dtype="bf16"),
        # its gradient from the kept inputs, a small batch
        dict(name="gate grad, 777x2816", op="gate_grad", rows=777, cols=2816, dtype="bf16"),
        # forward product of a training step
        dict(name="product, 8192x4096x1024", op="product", m=8192, n=4096, k=1024, a="e4m3", b="e4m3", d="bf16", add=False),
        # gradient of a weight matrix: few entries, a long sum over the tokens, added to the flat gradient
        dict(name="product, 1024x1024x8192", op="product", m=1024, n=1024, k=8192, a="e5m2", b="e4m3", d="f32", add=True),
        # odd sizes
        dict(name="product, 1000x2049x1537", op="product", m=1000, n=2049, k=1537, a="e4m3", b="e4m3", d="f16", add=False),
        # backward pass of a whole gated layer
        dict(name="layer backward, 4096 tokens", op="layer", rows=4096, cols=1024, hidden=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_product", "norm", "norm", "norm_grad", "norm_grad", "store", "store", "gate", "gate_grad",
                     "product", "product", "product", "layer"])
    plain = ["f32", "bf16", "bf16", "f16"]
    if op == "norm_product":
        return dict(op=op, rows=_log(rng, 1, 64), cols=_log(rng, 128, 8192), n=_log(rng, 64, 8192), dtype=rng.choice(["bf16", "f16"]))
    if op == "product":
        m, n = _log(rng, 1, 8192), _log(rng, 16, 8192)
        k = _log(rng, 16, max(32, min(16384, 3.4e10 / (m * n))))
        d = rng.choice(["f32", "bf16", "bf16", "f16", "e4m3"])
        return dict(op=op, m=m, n=n, k=k, a=rng.choice(["e4m3", "e4m3", "e5m2"]), b="e4m3", d=d,
                    add=d == "f32" and rng.random() < 0.6)
    if op == "layer":
        return dict(op=op, rows=_log(rng, 64, 4096), cols=64 * rng.randint(2, 16), hidden=_log(rng, 256, 4096))
    cols = _log(rng, 64, 12000)
    rows = _log(rng, 1, max(1, min(8192, 3.3e7 / cols)))
    if op in ("gate", "gate_grad"):
        return dict(op=op, rows=rows, cols=cols, dtype=rng.choice(plain))
    case = dict(op=op, rows=rows, cols=cols, stride=cols + rng.choice([0, 0, 0, 3, -cols % 64]), dtype=rng.choice(plain))
    if op == "norm":
        return dict(case, residual=rng.random() < 0.7, kept=rng.random() < 0.5)
    if op == "norm_grad":
        return dict(case, saved=rng.choice([case["dtype"], "e4m3"]), joined=rng.random() < 0.7)
    return dict(case, to=rng.choice(["e4m3", "e4m3", "e5m2"]))


# ---- 8 bits in plain operations ------------------------------------------------------------------

def _blocks(x):
    """[rows, blocks, 128], with zeros behind the last column."""
    rows, cols = x.shape
    return torch.nn.functional.pad(x, (0, -cols % 128)).view(rows, -1, 128)


def _quantise(x, dtype):
    """Entries in 8 bits and the blocks' exponents, of a matrix in 32 bits."""
    v = _blocks(x)
    mantissa, exponent = torch.frexp(v.abs().amax(2))
    limit, shift = math.frexp(LARGEST[dtype])
    e = exponent - shift + (mantissa > limit)
    e = torch.where(mantissa == 0, -127, e).clamp(min=-127)
    return (v * torch.exp2(-e.float())[:, :, None]).to(dtype).view(x.shape[0], -1)[:, :x.shape[1]], e


def _scaled(q, e):
    return (_blocks(q.float()) * torch.exp2(e.float())[:, :, None]).view(q.shape[0], -1)[:, :q.shape[1]]


def _round8(x, dtype=torch.float8_e4m3fn):
    """The values that a matrix's entries stand for once it is stored in 8 bits."""
    return _scaled(*_quantise(x, dtype))


def _exponents(scales, rows, cols):
    """The blocks' exponents from the scale bytes."""
    blocks = -(-cols // 128)
    groups = scales.view(-(-rows // 128), -(-blocks // 4), 32, 4, 4).permute(0, 3, 2, 1, 4)
    return groups.reshape(groups.shape[0] * 128, -1)[:rows, :blocks].int() - 127


def _values(pair):
    q, scales = pair
    return _scaled(q, _exponents(scales, *q.shape))


def _pair(rows, cols, dtype):
    """Room for a matrix in 8 bits: rows begin on 16-byte boundaries."""
    q = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8, device="cuda").view(dtype)[:, :cols]
    return q, torch.zeros(-(-rows // 128) * -(-cols // 512) * 512, dtype=torch.uint8, device="cuda")


def _stored(x, dtype=torch.float8_e4m3fn):
    """A matrix in 8 bits as a program has it in hand."""
    rows, cols = x.shape
    pair = _pair(rows, cols, dtype)
    q, e = _quantise(x, dtype)
    pair[0].view(torch.uint8).copy_(q.view(torch.uint8))
    whole = torch.zeros(-(-rows // 128) * 128, -(-cols // 512) * 4, dtype=torch.uint8, device="cuda")
    whole[:rows, :e.shape[1]] = (e + 127).to(torch.uint8)
    pair[1].copy_(whole.view(-1, 4, 32, whole.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1))
    return pair


# ---- what a user's program has in hand before the call -------------------------------------------

def _activations(rows, cols, gen, size=1.0):
    """Activations as a trained model has them: a few channels are much larger than the others, and
    tokens differ in size."""
    channel = torch.exp(0.5 * torch.randn(cols, generator=gen, device="cuda"))
    channel[torch.randint(0, cols, (max(1, cols // 200),), generator=gen, device="cuda")] *= 20
    token = size * torch.exp(0.3 * torch.randn(rows, 1, generator=gen, device="cuda"))
    return torch.randn(rows, cols, generator=gen, device="cuda") * channel * token


def _gradients(rows, cols, gen):
    """Gradients: small, of very different sizes from token to token."""
    return _activations(rows, cols, gen, 1e-4) * torch.exp(torch.randn(rows, 1, generator=gen, device="cuda"))


def _weights(rows, cols, gen):
    return torch.randn(rows, cols, generator=gen, device="cuda") / math.sqrt(cols)


def _room(rows, cols, dtype, stride=None):
    return torch.zeros(rows, stride or cols, dtype=dtype, device="cuda")[:, :cols]


def _given(x, dtype, stride=None):
    return _room(*x.shape, dtype, stride).copy_(x)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, s, e4m3 = case["op"], {"case": case}, torch.float8_e4m3fn
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"] = _stored(_activations(m, k, gen), DTYPES[case["a"]])
        s["b"] = _stored(_weights(n, k, gen), DTYPES[case["b"]])
        s["add"] = torch.randn(m, n, generator=gen, device="cuda") if case["add"] else None
        if case["d"] == "e4m3":
            s.update(d=_pair(m, n, e4m3), out=_room(m, n, torch.bfloat16))
        else:
            s["d"] = _room(m, n, DTYPES[case["d"]])
        return s
    rows, cols = case["rows"], case["cols"]
    if op == "layer":
        hidden = case["hidden"]
        x = _activations(rows, cols, gen).div_(4)
        s["x"] = _stored(x)
        s["gate"], s["up"] = (_stored(x @ _weights(hidden, cols, gen).T) for _ in range(2))
        s["d_y"] = _gradients(rows, cols, gen).to(torch.bfloat16)
        # weights as the backward pass takes them, transposed: [cols, hidden] twice, [hidden, cols]
        s["w_gate_t"], s["w_up_t"] = _stored(_weights(cols, hidden, gen)), _stored(_weights(cols, hidden, gen))
        s["w_down_t"] = _stored(_weights(hidden, cols, gen))
        for name, r, c in (("d_y8", rows, cols), ("d_y8_t", cols, rows), ("x_t", cols, rows), ("h_t", hidden, rows),
                           ("d_gate", rows, hidden), ("d_gate_t", hidden, rows), ("d_up", rows, hidden),
                           ("d_up_t", hidden, rows)):
            s[name] = _pair(r, c, e4m3)
        s.update(d_h=_room(rows, hidden, torch.bfloat16), part=_room(rows, cols, torch.float32),
                 d_x=_room(rows, cols, torch.bfloat16), d_w_gate=_room(hidden, cols, torch.bfloat16),
                 d_w_up=_room(hidden, cols, torch.bfloat16), d_w_down=_room(cols, hidden, torch.bfloat16))
        return s
    dtype = DTYPES[case["dtype"]]
    if op in ("gate", "gate_grad"):
        gate, up = _activations(rows, cols, gen), _activations(rows, cols, gen)
        if op == "gate":
            s.update(gate=gate.to(dtype), up=up.to(dtype))
            for name in ("h", "gate8", "up8"):
                s[name] = _pair(rows, cols, e4m3)
                s[name + "_out"] = _room(rows, cols, torch.bfloat16)
        else:
            s.update(gate=_stored(gate), up=_stored(up), d_h=_gradients(rows, cols, gen).to(dtype),
                     d_gate=_room(rows, cols, dtype), d_up=_room(rows, cols, dtype))
        return s
    if op == "store":
        to = DTYPES[case["to"]]
        s.update(x=_given(_gradients(rows, cols, gen), dtype, case["stride"]), q=_pair(rows, cols, to), q_t=_pair(cols, rows, to),
                 out=_room(rows, cols, torch.bfloat16), out_t=_room(cols, rows, torch.bfloat16))
        return s
    s["weight"] = 1.0 + 0.2 * torch.randn(cols, generator=gen, device="cuda")
    x = _activations(rows, cols, gen)
    if op == "norm_grad":
        s["s"] = _stored(x) if case["saved"] == "e4m3" else _given(x, dtype, case["stride"])
        values = _values(s["s"]) if case["saved"] == "e4m3" else s["s"].float()
        s["rstd"] = (values.double().square().mean(1) + EPS).rsqrt().float()
        s["d_out"] = _given(_gradients(rows, cols, gen), dtype, case["stride"])
        s["d_sum"] = _given(_gradients(rows, cols, gen), dtype, case["stride"]) if case["joined"] else None
        s.update(d_x=_room(rows, cols, dtype, case["stride"]), d_weight=torch.zeros(cols, device="cuda"))
        if own:   # scratch memory of the framework's call; the plain form needs none
            import paper_1806_08054_b200 as ecq
            s["workspace"] = torch.empty(ecq.ecq_act8_norm_grad_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        return s
    stride = case.get("stride")
    s["x"] = _given(x, dtype, stride)
    s["residual"] = _given(_activations(rows, cols, gen, 3.0), dtype, stride) if case.get("residual", True) else None
    s.update(sum=_room(rows, cols, dtype, stride), y=_pair(rows, cols, e4m3), rstd=torch.zeros(rows, device="cuda"))
    if op == "norm_product":
        s.update(w=_stored(_weights(case["n"], cols, gen)), d=_room(rows, case["n"], dtype))
    else:
        s["y_out"] = _room(rows, cols, torch.bfloat16)
        if case["kept"]:
            s.update(sum8=_pair(rows, cols, e4m3), sum8_out=_room(rows, cols, torch.bfloat16))
    return s


# ---- plain forms ---------------------------------------------------------------------------------

def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _gate_gradient(gate, up, d_h):
    sig = _sigmoid(gate)
    return d_h * up * sig * (1.0 + gate * (1.0 - sig)), d_h * gate * sig


def _plain(s):
    case = s["case"]
    op, bf16 = case["op"], torch.bfloat16
    if op == "product":
        d = _values(s["a"]) @ _values(s["b"]).T
        if s["add"] is not None:
            d = d + s["add"]
        return _round8(d).to(bf16) if case["d"] == "e4m3" else d.to(DTYPES[case["d"]])
    if op == "layer":
        d_y, gate, up, x = s["d_y"].float(), _values(s["gate"]), _values(s["up"]), _values(s["x"])
        d_h = (_round8(d_y) @ _values(s["w_down_t"]).T).to(bf16).float()
        d_gate, d_up = _gate_gradient(gate, up, d_h)
        h_t, x_t = _round8((gate * _sigmoid(gate) * up).T), _round8(x.T)
        d_x = _round8(d_gate) @ _values(s["w_gate_t"]).T + _round8(d_up) @ _values(s["w_up_t"]).T
        return {"d_x": d_x.to(bf16), "d_w_gate": (_round8(d_gate.T) @ x_t.T).to(bf16),
                "d_w_up": (_round8(d_up.T) @ x_t.T).to(bf16), "d_w_down": (_round8(d_y.T) @ h_t.T).to(bf16)}
    if op == "store":
        x, to = s["x"].float(), DTYPES[case["to"]]
        return {"out": _round8(x, to).to(bf16), "out_t": _round8(x.T, to).to(bf16)}
    if op == "gate":
        gate, up = s["gate"].float(), s["up"].float()
        return {"h": _round8(gate * _sigmoid(gate) * up).to(bf16), "gate8": _round8(gate).to(bf16), "up8": _round8(up).to(bf16)}
    if op == "gate_grad":
        d_gate, d_up = _gate_gradient(_values(s["gate"]), _values(s["up"]), s["d_h"].float())
        return {"d_gate": d_gate.to(s["d_h"].dtype), "d_up": d_up.to(s["d_h"].dtype)}
    if op == "norm_grad":
        x = _values(s["s"]) if case["saved"] == "e4m3" else s["s"].float()
        normed, d_out = x * s["rstd"][:, None], s["d_out"].float()
        g = d_out * s["weight"]
        d_x = s["rstd"][:, None] * (g - normed * (g * normed).mean(1, keepdim=True))
        if s["d_sum"] is not None:
            d_x = d_x + s["d_sum"].float()
        return {"d_x": d_x.to(s["d_x"].dtype), "d_weight": (d_out * normed).sum(0)}
    total = s["x"].float()
    if s["residual"] is not None:
        total = total + s["residual"].float()
    rstd = 1.0 / torch.sqrt(total.square().mean(1) + EPS)
    y = _round8(total * rstd[:, None] * s["weight"])
    if op == "norm_product":
        return {"sum": total.to(s["x"].dtype), "d": (y @ _values(s["w"]).T).to(s["x"].dtype)}
    out = {"sum": total.to(s["x"].dtype), "rstd": rstd, "y": y.to(bf16)}
    if case["kept"]:
        out["sum8"] = _round8(total).to(bf16)
    return out


# ---- one pass ------------------------------------------------------------------------------------

def run(state):
    s, case = state, state["case"]
    if not own:
        return _plain(s)
    import paper_1806_08054_b200 as ecq
    op = case["op"]
    if op == "product":
        ecq.ecq_act8_product(s["a"], s["b"], s["d"], add=s["add"])
        if case["d"] != "e4m3":
            return s["d"]
        ecq.ecq_act8_load(s["d"], s["out"])
        return s["out"]
    if op == "layer":
        ecq.ecq_act8_store(s["d_y"], s["d_y8"], s["d_y8_t"])
        ecq.ecq_act8_product(s["d_y8"], s["w_down_t"], s["d_h"])
        ecq.ecq_act8_gate(s["gate"], s["up"], out8_t=s["h_t"])
        ecq.ecq_act8_gate_grad(s["gate"], s["up"], s["d_h"], d_gate8=s["d_gate"], d_gate8_t=s["d_gate_t"], d_up8=s["d_up"],
                               d_up8_t=s["d_up_t"])
        ecq.ecq_act8_product(s["d_gate"], s["w_gate_t"], s["part"])
        ecq.ecq_act8_product(s["d_up"], s["w_up_t"], s["d_x"], add=s["part"])
        ecq.ecq_act8_store(s["x"], None, s["x_t"])
        ecq.ecq_act8_product(s["d_gate_t"], s["x_t"], s["d_w_gate"])
        ecq.ecq_act8_product(s["d_up_t"], s["x_t"], s["d_w_up"])
        ecq.ecq_act8_product(s["d_y8_t"], s["h_t"], s["d_w_down"])
        return {k: s[k] for k in ("d_x", "d_w_gate", "d_w_up", "d_w_down")}
    if op == "store":
        # stored in the forward or the backward pass, restored where the values are wanted
        ecq.ecq_act8_store(s["x"], s["q"], s["q_t"])
        ecq.ecq_act8_load(s["q"], s["out"])
        ecq.ecq_act8_load(s["q_t"], s["out_t"])
        return {"out": s["out"], "out_t": s["out_t"]}
    if op == "gate":
        ecq.ecq_act8_gate(s["gate"], s["up"], out8=s["h"], gate8=s["gate8"], up8=s["up8"])
        for name in ("h", "gate8", "up8"):
            ecq.ecq_act8_load(s[name], s[name + "_out"])
        return {"h": s["h_out"], "gate8": s["gate8_out"], "up8": s["up8_out"]}
    if op == "gate_grad":
        ecq.ecq_act8_gate_grad(s["gate"], s["up"], s["d_h"], d_gate=s["d_gate"], d_up=s["d_up"])
        return {"d_gate": s["d_gate"], "d_up": s["d_up"]}
    if op == "norm_grad":
        ecq.ecq_act8_norm_grad(s["s"], s["weight"], s["rstd"], s["d_out"], s["d_x"], s["d_weight"], s["workspace"],
                               d_sum=s["d_sum"])
        return {"d_x": s["d_x"], "d_weight": s["d_weight"]}
    ecq.ecq_act8_norm(s["x"], s["residual"], s["weight"], eps=EPS, sum=s["sum"], out8=s["y"], sum8=s.get("sum8"), rstd=s["rstd"])
    if op == "norm_product":
        ecq.ecq_act8_product(s["y"], s["w"], s["d"])
        return {"sum": s["sum"], "d": s["d"]}
    ecq.ecq_act8_load(s["y"], s["y_out"])
    out = {"sum": s["sum"], "rstd": s["rstd"], "y": s["y_out"]}
    if case["kept"]:
        ecq.ecq_act8_load(s["sum8"], s["sum8_out"])
        out["sum8"] = s["sum8_out"]
    return out


def work(case):
    """Inputs read and outputs written once; where values are restored from 8 bits that the pass has
    stored, those written, read and restored to 16 bits."""
    op, b8, restored = case["op"], 1 + 1 / 128, 2 * (1 + 1 / 128) + 2
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        out = restored if case["d"] == "e4m3" else DTYPES[case["d"]].itemsize + (4 if case["add"] else 0)
        return {"bytes": int((m + n) * k * b8 + m * n * out), "flops": 2 * m * n * k}
    rows, cols = case["rows"], case["cols"]
    n = rows * cols
    if op == "layer":
        hidden = case["hidden"]
        inputs = n * (2 + b8) + 2 * rows * hidden * b8 + 3 * cols * hidden * b8
        return {"bytes": int(inputs + 2 * n + 6 * cols * hidden), "flops": 12 * n * hidden}
    size = DTYPES[case["dtype"]].itemsize
    if op == "store":
        return {"bytes": int(n * (size + 2 * restored)), "flops": 4 * n}
    if op == "gate":
        return {"bytes": int(n * (2 * size + 3 * restored)), "flops": 12 * n}
    if op == "gate_grad":
        return {"bytes": int(n * (2 * b8 + 3 * size)), "flops": 12 * n}
    if op == "norm_grad":
        saved = b8 if case["saved"] == "e4m3" else size
        return {"bytes": int(n * (saved + (3 if case["joined"] else 2) * size) + 4 * rows + 8 * cols), "flops": 10 * n}
    if op == "norm_product":
        return {"bytes": int(n * (3 * size) + 4 * cols + case["n"] * (cols * b8 + rows * size)), "flops": n * (6 + 2 * case["n"])}
    through = (3 if case["residual"] else 2) * size + (2 if case["kept"] else 1) * restored
    return {"bytes": int(n * through + 4 * (rows + cols)), "flops": 8 * n}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _eight(x, mantissa=3, lowest=-6, largest=448.0):
    """x, in 64 bits, as it is held in 8 bits: per 128 columns a power of two, then the nearest value
    of the type, ties to the even one."""
    rows, cols = x.shape
    out = torch.empty_like(x)
    for at in range(0, cols, 128):
        part = x[:, at:at + 128]
        big = part.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(big / largest))
        e = torch.where(big > largest * torch.exp2(e), e + 1, torch.where(big <= largest * torch.exp2(e - 1), e - 1, e))
        unit = torch.exp2(torch.where(big > 0, e, -127.0).clamp(min=-127))
        v = part / unit
        power = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** lowest)))
        power = torch.where(torch.exp2(power) > v.abs().clamp(min=2.0 ** lowest), power - 1, power)
        step = torch.exp2(power - mantissa)
        out[:, at:at + 128] = torch.round(v / step) * step * unit
    return out


def _bf16(x):
    return x.to(torch.bfloat16).double()


def _exact_values(pair):
    q, scales = pair
    rows, cols = q.shape
    r, b = torch.arange(rows, device="cuda")[:, None], torch.arange(cols, device="cuda")[None, :] // 128
    at = ((r // 128) * -(-cols // 512) + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4
    return q.to(torch.float64) * torch.exp2(scales[at].double() - 127)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "product":
        d = _exact_values(s["a"]).matmul(_exact_values(s["b"]).T)
        if case["add"]:
            d += s["add"]
        return _eight(d) if case["d"] == "e4m3" else d
    if op in ("gate", "gate_grad", "layer"):
        gate, up = (_exact_values(s[k]) if op != "gate" else s[k].double() for k in ("gate", "up"))
        silu = gate / (1 + torch.exp(-gate))
        if op == "gate":
            return {"h": _eight(silu * up), "gate8": _eight(gate), "up8": _eight(up)}
        slope = torch.sigmoid(gate) + silu * (1 - torch.sigmoid(gate))
        if op == "gate_grad":
            d_h = s["d_h"].double()
            return {"d_gate": d_h * up * slope, "d_up": d_h * silu}
        d_y, x = s["d_y"].double(), _exact_values(s["x"])
        d_h = _bf16(_eight(d_y).matmul(_exact_values(s["w_down_t"]).T))
        d_gate, d_up = d_h * up * slope, d_h * silu
        d_x = _eight(d_gate).matmul(_exact_values(s["w_gate_t"]).T)
        d_x += _eight(d_up).matmul(_exact_values(s["w_up_t"]).T)
        tokens = _eight(x.T.contiguous()).T
        return {"d_x": d_x, "d_w_gate": _eight(d_gate.T.contiguous()).matmul(tokens),
                "d_w_up": _eight(d_up.T.contiguous()).matmul(tokens),
                "d_w_down": _eight(d_y.T.contiguous()).matmul(_eight((silu * up).T.contiguous()).T)}
    if op == "store":
        kind = (3, -6, 448.0) if case["to"] == "e4m3" else (2, -14, 57344.0)
        x = s["x"].double()
        return {"out": _eight(x, *kind), "out_t": _eight(x.T.contiguous(), *kind)}
    if op == "norm_grad":
        x = _exact_values(s["s"]) if case["saved"] == "e4m3" else s["s"].double()
        rstd, g = s["rstd"].double()[:, None], s["d_out"].double() * s["weight"].double()
        d_x = rstd * g - x * rstd ** 3 * (g * x).sum(1, keepdim=True) / case["cols"]
        if case["joined"]:
            d_x += s["d_sum"].double()
        return {"d_x": d_x, "d_weight": (s["d_out"].double() * x * rstd).sum(0)}
    total = s["x"].double()
    if s["residual"] is not None:
        total = total + s["residual"].double()
    rstd = (total.square().sum(1) / case["cols"] + EPS) ** -0.5
    y = _eight(total * rstd[:, None] * s["weight"].double())
    if op == "norm_product":
        return {"sum": total, "d": y.matmul(_exact_values(s["w"]).T)}
    out = {"sum": total, "rstd": rstd, "y": y}
    if case["kept"]:
        out["sum8"] = _eight(total)
    return out

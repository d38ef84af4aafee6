"""More operators of a training step, as measured cases.

What lies between the last block of a model and its updated weights, and between
one block and the next: the head's matrix product with the cross entropy of labels
and both gradients, in pieces of the vocabulary so that the logits are never kept;
the norm after a block, its gate, the scaled residual and the norm before the next
block in one pass, forward and backward; and AdamW over a list of tensors where
they lie, with its moments in 32 or in 8 bits.  Every case is one pass through one
of them.

`run` computes the plain form (elementary torch operations in 32 bits, rounded
once at the end) or, with `own` set, makes the calls of
``paper_2509_21271_b200.operators`` and ``paper_2509_21271_b200.tensor_adamw``.
`exact` states the definitions once more in 64 bits.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-5
LR, BETA1, BETA2, ADAM_EPS, DECAY, MAX_NORM = 1e-3, 0.9, 0.999, 1e-8, 0.01, 1.0
FIRST_STEP = 10            # steps that the moments have behind them
SEED = 20250925
BLOCK = 256                # elements that share an 8-bit moment's scale


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def _entropy(name, rows, vocab, cols, dtype, out, masked, grad_scale):
    """`out`: type of the table's gradient; empty for the loss alone."""
    return {"op": "entropy", "name": name, "rows": rows, "vocab": vocab, "cols": cols, "dtype": dtype, "out": out,
            "masked": masked, "grad_scale": grad_scale}


def _norm(op, name, rows, cols, dtype, param, kind, post, groups, scale):
    """`groups`: gates [groups, cols], one for rows / groups rows each; 0 for none."""
    return {"op": op, "name": name, "rows": rows, "cols": cols, "dtype": dtype, "param": param, "kind": kind,
            "post": post, "groups": groups, "scale": scale}


def _adamw(name, tensors, size, layers, vocab, bits, grad, copy, stochastic, clip):
    """`tensors`: what the list looks like, see `_sizes`."""
    return {"op": "adamw", "name": name, "tensors": tensors, "size": size, "layers": layers, "vocab": vocab, "bits": bits,
            "grad": grad, "copy": copy, "stochastic": stochastic, "clip": clip}


def listed():
    return [
        # one short answer, 768 wide: the table is read and its gradient written for 63 tokens
        _entropy("entropy_short_answer", 63, 50257, 768, "bf16", "bf16", 0.0, 1.0),
        # an odd batch in fp16 under a loss scale, into an fp32 gradient arena
        _entropy("entropy_ragged", 1025, 50257, 1600, "fp16", "fp32", 0.1, 65536.0),
        # a packed batch of the 8B-parameter stack with its prompts masked
        _entropy("entropy_batch", 8192, 128256, 4096, "bf16", "bf16", 0.3, 1.0),
        # losses alone, as in an evaluation with the 1B-parameter stack
        _entropy("entropy_loss_alone", 4095, 128256, 2048, "bf16", "", 0.0, 1.0),
        # one token between two blocks of the 8B-parameter stack: the cost of a call
        _norm("norm_forward", "norm_forward_one_token", 1, 4096, "bf16", "bf16", "rms", True, 1, 1.0),
        # 8 x 4096 tokens of a micro-batch, a learned gate per channel
        _norm("norm_forward", "norm_forward_long", 32768, 4096, "bf16", "bf16", "rms", True, 1, 1.0),
        # a short ragged micro-batch in fp16: residual and layer norm only, fp32 master weights
        _norm("norm_backward", "norm_backward_ragged", 2047, 768, "fp16", "fp32", "layer", False, 0, 1.0),
        # 16 sequences of 2048 tokens, each with a gate of its own, scaled residuals
        _norm("norm_backward", "norm_backward_long", 32768, 2048, "bf16", "fp32", "layer", True, 16, 0.875),
        # the norms of a small stack: many tiny tensors, where latency counts
        _adamw("adamw_norm_weights", "norms", 768, 12, 0, 32, "bf16", "bf16", False, False),
        # a stack of 24 layers, 1024 wide, moments in 32 bits, gradients clipped
        _adamw("adamw_stack", "stack", 1024, 24, 50257, 32, "bf16", "bf16", False, True),
        # tensors of odd sizes, fp32 gradients, 8-bit moments rounded to the nearest code
        _adamw("adamw_8bit_ragged", "odd", 333331, 12, 0, 8, "fp32", "fp16", False, True),
        # the 1B-parameter stack with 8-bit moments, rounded stochastically
        _adamw("adamw_8bit_large", "stack", 2048, 16, 128256, 8, "bf16", "bf16", True, True),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng):
    if rng.random() < 0.6:
        return rng.choice([512, 768, 1024, 1536, 2048, 2560, 4096, 5120, 8192])
    return _between(rng, 65, 8192)


def draw(rng):
    op = rng.choice(["entropy", "entropy", "norm_forward", "norm_backward", "adamw", "adamw"])
    if op == "entropy":
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        vocab = rng.choice([50257, 128256, _between(rng, 1000, 160000)])
        cols = min(_width(rng), 5120)
        rows = _between(rng, 1, min(8192, (1 << 42) // (vocab * cols)))
        out = rng.choice(["", dtype, dtype, "fp32"])
        case = _entropy("", rows, vocab, cols, dtype, out, rng.choice([0.0, rng.uniform(0.05, 0.6)]),
                        65536.0 if dtype == "fp16" else 1.0)
    elif op == "adamw":
        bits = rng.choice([8, 8, 32])
        tensors = rng.choice(["norms", "stack", "odd"])
        size = {"norms": _between(rng, 64, 8192), "stack": _between(rng, 2, 64) * 32,
                "odd": _between(rng, 1, 4000000)}[tensors]
        layers = rng.randint(1, 16)
        case = _adamw("", tensors, size, layers, rng.choice([50257, 128256, _between(rng, 1000, 128256)]), bits,
                      rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.choice(["bf16", "fp16", ""]),
                      bits == 8 and rng.random() < 0.7, rng.random() < 0.7)
    else:
        cols = _width(rng)
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        post = rng.random() < 0.6
        groups = rng.choice([0, 1, rng.randint(2, 16)])
        rows = _between(rng, 1, min(65536, (1 << 27) // cols))
        if groups > 1:
            rows = max(groups, rows // groups * groups)
        case = _norm(op, "", rows, cols, dtype, rng.choice([dtype, "fp32"]), rng.choice(["rms", "layer"]), post, groups,
                     rng.choice([1.0, rng.uniform(0.25, 1.5)]))
    case.pop("name")
    return case


def _sizes(case):
    """Elements of each tensor of an AdamW case's list."""
    kind, d, layers, vocab = case["tensors"], case["size"], case["layers"], case["vocab"]
    if kind == "norms":                                   # weight and bias of two norms a layer, and the last ones
        return [d] * (4 * layers + 2)
    if kind == "odd":                                     # from one element to `size`, hardly one a multiple of 8
        return [max(1, d * (k * k % (layers + 1)) // (layers + 1) + k) for k in range(layers)] + [1, 7, d]
    per_layer = [d * d, d * d // 4, d * d // 4, d * d, 4 * d * d, 4 * d * d, 4 * d * d, d, d]
    return [vocab * d] + per_layer * layers + [d]


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _fill(t, g, scale, at=0.0):
    """Normal values into a matrix of any type, some rows at a time."""
    step = max(1, (1 << 27) // t.shape[1])
    for lo in range(0, t.shape[0], step):
        part = t[lo:lo + step]
        part.copy_(torch.randn(part.shape, generator=g, device=DEVICE).mul_(scale).add_(at))
    return t


def _empty(rows, cols, t):
    return torch.empty(rows, cols, dtype=t, device=DEVICE)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["op"] == "adamw":
        _handle(s)
    return s


def _inputs(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed * 1_000_003 + 29)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEVICE)  # noqa: E731
    s = {"case": case}
    if case["op"] == "entropy":
        rows, vocab, cols, t = case["rows"], case["vocab"], case["cols"], TYPES[case["dtype"]]
        # logits of a spread of about 1.3; the label's is raised by up to 8, as a trained head's is
        s["table"] = _fill(_empty(vocab, cols, t), g, 1.3 / math.sqrt(cols))
        labels = torch.randint(vocab, (rows,), generator=g, device=DEVICE)
        raised = torch.rand(rows, 1, generator=g, device=DEVICE) * (8.0 / 1.69)
        s["hidden"] = (rand(rows, cols) + raised * s["table"][labels].float()).to(t)
        gone = min(int(rows * case["masked"]), rows)
        masked = torch.randperm(rows, generator=g, device=DEVICE)[:gone]
        weight = torch.ones(rows, device=DEVICE)
        weight[masked] = 0.0
        labels[masked[: gone // 2]] = -100                # prompts, and what pads the batch
        s["weight"], s["labels"] = weight / max(rows - gone, 1), labels
        s["loss"], s["row_loss"] = torch.empty(1, device=DEVICE), torch.empty(rows, device=DEVICE)
        if case["out"]:
            s["dhidden"], s["dtable"] = _empty(rows, cols, t), _empty(vocab, cols, TYPES[case["out"]])
    elif case["op"] == "adamw":
        _prepare_adamw(s, g)
    else:
        rows, cols, t, pt = case["rows"], case["cols"], TYPES[case["dtype"]], TYPES[case["param"]]
        weight, bias = lambda: (1.0 + 0.1 * rand(cols)).to(pt), lambda: (0.1 * rand(cols)).to(pt)  # noqa: E731
        layer = case["kind"] == "layer"
        s["x"], s["block"] = _fill(_empty(rows, cols, t), g, 1.5, 0.1), _fill(_empty(rows, cols, t), g, 0.7, -0.05)
        s["weight"], s["bias"] = weight(), bias() if layer else None
        s["post_weight"] = weight() if case["post"] else None
        s["post_bias"] = bias() if case["post"] and layer else None
        n = case["groups"]
        s["gate"] = None if n == 0 else (0.5 + 0.2 * rand(cols)).to(pt) if n == 1 else (0.5 + 0.2 * rand(n, cols)).to(pt)
        s["h"], s["y"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["stats"] = torch.empty(4, rows, device=DEVICE)
        if case["op"] == "norm_backward":
            done = _plain_norm_forward(s)
            s["h"].copy_(done["h"])
            s["stats"].copy_(done["stats"])
            del done
            s["dh"], s["dy"] = _fill(_empty(rows, cols, t), g, 0.02), _fill(_empty(rows, cols, t), g, 0.05)
            s["dx"], s["dblock"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    return s


def _prepare_adamw(s, g):
    case = s["case"]
    sizes = _sizes(case)
    padded = [-(-n // BLOCK) * BLOCK for n in sizes]
    total = sum(padded)
    live = torch.zeros(total // BLOCK, BLOCK, dtype=torch.bool, device=DEVICE)
    at, where = 0, []
    for n, room in zip(sizes, padded):
        live.view(-1)[at:at + n] = True
        where.append((at, n))
        at += room
    # the tensors are cut out of one buffer, each from a multiple of 256 elements; what lies between them is zero
    flat = lambda t, scale: _fill(torch.empty(total // BLOCK, BLOCK, dtype=t, device=DEVICE), g, scale).mul_(live)  # noqa: E731
    s["param"] = flat(torch.float32, 0.02)
    s["grad"] = flat(TYPES[case["grad"]], 1e-3)
    s["copy"] = torch.zeros_like(s["param"], dtype=TYPES[case["copy"]]) if case["copy"] else None
    m, v = flat(torch.float32, 2e-4), flat(torch.float32, 1e-3).square_()
    s["t"] = FIRST_STEP
    if case["bits"] == 8:
        half = torch.full((), 1 << 18, dtype=torch.int32, device=DEVICE)
        s["m"], s["m_scale"] = _encode(m, 10, half, True)
        s["v"], s["v_scale"] = _encode(v, 18, half, False)
    else:
        s["m"], s["v"] = m, v
    s["where"] = where


def _handle(s):
    """The optimizer that a program keeps, with the moments in place."""
    from paper_2509_21271_b200.tensor_adamw import TensorAdamW
    case = s["case"]
    views = lambda t: [t.view(-1)[a:a + n] for a, n in s["where"]]  # noqa: E731
    opt = TensorAdamW(views(s["param"]), views(s["grad"]), copies=views(s["copy"]) if case["copy"] else None,
                      state_bits=case["bits"])
    for name in ("m", "v", "m_scale", "v_scale") if case["bits"] == 8 else ("m", "v"):
        getattr(opt, name).view(-1).copy_(s.pop(name).view(-1))
    opt.set_step(FIRST_STEP)
    s["opt"], s["hp"] = opt, _HParams()


class _HParams:
    lr, beta1, beta2, eps, weight_decay, max_grad_norm = LR, BETA1, BETA2, ADAM_EPS, DECAY, MAX_NORM


# --------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------

def _plain_entropy(s):
    case = s["case"]
    h, w = s["hidden"].float(), s["table"].float()
    live = (s["weight"] != 0) & (s["labels"] >= 0) & (s["labels"] < case["vocab"])
    at = torch.where(live, s["labels"], torch.zeros_like(s["labels"]))[:, None]
    z = h @ w.t()
    top = z.amax(1, keepdim=True)
    picked = z.gather(1, at)
    z.sub_(top).exp_()
    total = z.sum(1, keepdim=True)
    zero = torch.zeros_like(s["weight"])
    row = torch.where(live, (top + total.log() - picked)[:, 0], zero)
    weight = torch.where(live, s["weight"], zero)
    out = {"loss": (weight * row).sum().reshape(1), "row_loss": row}
    if case["out"]:
        z.div_(total)
        z.scatter_add_(1, at, torch.full_like(top, -1.0))
        z.mul_((weight * case["grad_scale"])[:, None])
        out["dhidden"] = (z @ w).to(s["hidden"].dtype)
        out["dtable"] = (z.t() @ h).to(s["dtable"].dtype)
    return out


def _plain_stats(x, layer):
    mean = x.mean(1, keepdim=True) if layer else torch.zeros_like(x[:, :1])
    c = x - mean
    return mean, ((c * c).mean(1, keepdim=True) + EPS).rsqrt()


def _by_group(s, rows):
    """The gates of all rows, as a matrix that broadcasts over them."""
    gate = s["gate"]
    return 1.0 if gate is None else gate.float().reshape(-1, 1, rows.shape[1]).expand(
        -1, rows.shape[0] // max(s["case"]["groups"], 1), -1).reshape(rows.shape)


def _plain_norm_forward(s):
    case = s["case"]
    layer = case["kind"] == "layer"
    x, u, t = s["x"].float(), s["block"].float(), s["x"].dtype
    zero, one = torch.zeros_like(x[:, :1]), torch.ones_like(x[:, :1])
    post_mean, post_rstd = _plain_stats(u, layer) if case["post"] else (zero, one)
    if case["post"]:
        u = (u - post_mean) * post_rstd * s["post_weight"].float()
        u = u + s["post_bias"].float() if layer else u
    h = x * case["scale"] + _by_group(s, u) * u
    h = h.to(t)                          # the residual stream as it is stored, and as the next norm sees it
    mean, rstd = _plain_stats(h.float(), layer)
    y = (h.float() - mean) * rstd * s["weight"].float()
    y = y + s["bias"].float() if layer else y
    return {"h": h, "y": y.to(t), "stats": torch.cat([post_mean, post_rstd, mean, rstd], 1).t()}


def _plain_norm_backward(s):
    case = s["case"]
    layer, post, t, pt = case["kind"] == "layer", case["post"], s["x"].dtype, s["weight"].dtype
    post_mean, post_rstd, mean, rstd = (r[:, None] for r in s["stats"])
    h, dy = s["h"].float(), s["dy"].float()
    hat = (h - mean) * rstd
    e = dy * s["weight"].float()
    out = {"dweight": (dy * hat).sum(0).to(pt)}
    if layer:
        out["dbias"] = dy.sum(0).to(pt)
    inner = e - e.mean(1, keepdim=True) if layer else e
    total = s["dh"].float() + rstd * (inner - hat * (e * hat).mean(1, keepdim=True))
    out["dx"] = (total * case["scale"]).to(t)
    block, gate = s["block"].float(), _by_group(s, total)
    bhat = (block - post_mean) * post_rstd
    du = total * gate
    if case["groups"]:
        u = bhat * s["post_weight"].float() if post else block
        u = u + s["post_bias"].float() if post and layer else u
        per = (total * u).reshape(case["groups"], -1, total.shape[1]).sum(1)
        out["dgate"] = per.reshape(s["gate"].shape).to(pt)
    if not post:
        out["dblock"] = du.to(t)
        return out
    out["dpost_weight"] = (du * bhat).sum(0).to(pt)
    if layer:
        out["dpost_bias"] = du.sum(0).to(pt)
    e = du * s["post_weight"].float()
    inner = e - e.mean(1, keepdim=True) if layer else e
    out["dblock"] = (post_rstd * (inner - bhat * (e * bhat).mean(1, keepdim=True))).to(t)
    return out


# An 8-bit moment: 4 bits of fraction, 3 bits of exponent and a sign (m) or 4 bits of exponent (v), in units of its
# block's scale 2^(s - 127), s a byte: 0 for a block of zeros, 255 for one that is not finite.  With f fraction and e
# exponent bits it stands for f units where e is 0, for (16 + f) 2^(e - 1) otherwise: the bit pattern of an fp32 number
# of that many units of 2^-130, cut off 19 bits above its end, so that adding 2^18 (or a random number) first rounds.

def _decode(code, scale, signed):
    k = (code & 127) if signed else code
    k = k.to(torch.int32)
    units = torch.where(k < 16, k, (16 + (k & 15)) << ((k >> 4) - 1).clamp_(min=0)).float()
    units = torch.where(code >= 128, -units, units) if signed else units
    factor = torch.exp2((scale.to(torch.float32) - 127.0).clamp_(min=-126.0))
    return units * torch.where(scale == 255, torch.full_like(factor, math.nan), factor)[:, None]


def _encode(x, top, noise, signed):
    """Codes and scales of blocks: `top` = 10 or 18 binades above a unit are the largest code's."""
    bits = x.abs().view(torch.int32)
    most = bits.amax(1)
    exponent = most >> 23
    scale = (exponent + ((most & 0x7FFFFF) > 0x780000) - top).clamp_(min=1)
    scale = torch.where(exponent == 255, 255, torch.where(most == 0, 0, scale))
    up = ((254 - scale.clamp(min=1, max=253)) << 23).view(torch.float32)        # 1 over the scale
    y = ((x.abs() * up[:, None]) * 2.0 ** -130).view(torch.int32)
    code = (y + noise) >> 19
    code = code | ((x.view(torch.int32) < 0).to(torch.int32) << 7) if signed else torch.where(x > 0, code.clamp_(min=1), code)
    code = torch.where((scale == 255)[:, None], torch.zeros_like(code), code)
    return code.to(torch.uint8), scale.to(torch.uint8)


def _mix(x):
    """MurmurHash3's 32-bit finalizer, on whole numbers below 2^32."""
    x = x ^ (x >> 16)
    x = (x * 0x85EBCA6B) & 0xFFFFFFFF
    x = x ^ (x >> 13)
    x = (x * 0xC2B2AE35) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _noise(case, t, shape):
    """What is added to 19 bits below a code: 2^18, or 16 random bits of the seed, the step and the element."""
    if not case["stochastic"]:
        half = torch.full((), 1 << 18, dtype=torch.int32, device=DEVICE)
        return half, half
    key = _mix((_mix((SEED & 0xFFFFFFFF) + 0) ^ _mix((SEED >> 32) ^ 0x9E3779B9)) ^ (t & 0xFFFFFFFF))
    key = _mix(key)                                       # elements 0 to 2^32 - 1
    x = _mix(torch.arange(shape[0] * shape[1], device=DEVICE) ^ key).view(shape)
    return (((x & 0xFFFF) << 3) + 4).to(torch.int32), (((x >> 16) << 3) + 4).to(torch.int32)


def _plain_adamw(s):
    case = s["case"]
    s["t"] += 1
    t = s["t"]
    eight = case["bits"] == 8
    f32 = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    g = s["grad"].float()
    out = {}
    if case["clip"]:
        norm = g.double().square().sum().sqrt()
        coef = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0).float()
        out["norm"] = norm.float().reshape(1)
        g = g * coef
    m = _decode(s["m"], s["m_scale"], True) if eight else s["m"]
    v = _decode(s["v"], s["v_scale"], False) if eight else s["v"]
    m = m * f32(BETA1) + g * f32(1.0 - BETA1)
    v = v * f32(BETA2) + g * f32(1.0 - BETA2) * g
    u = m / (v.sqrt() * f32(1.0 / math.sqrt(1.0 - BETA2 ** t)) + f32(ADAM_EPS))
    s["param"].sub_(s["param"] * f32(LR * DECAY) + u * f32(LR / (1.0 - BETA1 ** t)))
    del g, u
    out["param"] = s["param"]
    if case["copy"]:
        out["copy"] = s["copy"].copy_(s["param"])
    if eight:
        noise = _noise(case, t, m.shape)
        s["m"], s["m_scale"] = _encode(m, 10, noise[0], True)
        s["v"], s["v_scale"] = _encode(v, 18, noise[1], False)
        del noise
        out["m"], out["v"] = (_decode(s[k], s[k + "_scale"], k == "m").to(torch.bfloat16) for k in ("m", "v"))
    else:
        out["m"], out["v"] = s["m"].copy_(m), s["v"].copy_(v)
    return out


PLAIN = {"entropy": _plain_entropy, "norm_forward": _plain_norm_forward, "norm_backward": _plain_norm_backward,
         "adamw": _plain_adamw}


# --------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------

def _own(s):
    from paper_2509_21271_b200 import operators as ops
    case = s["case"]
    op = case["op"]
    if op == "entropy":
        grads = bool(case["out"])
        loss, row, dhidden, dtable = ops.linear_cross_entropy(
            s["hidden"], s["table"], s["labels"], s["weight"], grad_scale=case["grad_scale"],
            dhidden=s["dhidden"] if grads else False, dtable=s["dtable"] if grads else False, loss=s["loss"],
            row_loss=s["row_loss"])
        out = {"loss": loss, "row_loss": row}
        return {**out, "dhidden": dhidden, "dtable": dtable} if grads else out
    if op == "norm_forward":
        h, y, stats = ops.residual_norm_forward(
            s["x"], s["block"], s["gate"], s["post_weight"], s["post_bias"], s["weight"], s["bias"], kind=case["kind"],
            post=case["post"], scale=case["scale"], eps=EPS, h=s["h"], y=s["y"], stats=s["stats"])
        return {"h": h, "y": y, "stats": stats}
    if op == "norm_backward":
        got = ops.residual_norm_backward(
            s["dy"], s["dh"], s["h"], s["block"], s["stats"], s["gate"], s["post_weight"], s["post_bias"], s["weight"],
            kind=case["kind"], post=case["post"], scale=case["scale"], dx=s["dx"], dblock=s["dblock"])
        names = ("dx", "dblock", "dgate", "dpost_weight", "dpost_bias", "dweight", "dbias")
        return {k: x for k, x in zip(names, got) if x is not None}
    opt = s["opt"]
    stats = opt.step(s["hp"], clip=case["clip"], seed=SEED if case["stochastic"] else None)
    out = {"param": s["param"]}
    if case["clip"]:
        out["norm"] = stats[:1]
    if case["copy"]:
        out["copy"] = s["copy"]
    m, v = opt.moments()
    out["m"], out["v"] = m.view(s["param"].shape), v.view(s["param"].shape)
    return out


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["case"]["op"]](state)


# --------------------------------------------------------------------------
# bytes and operations that a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "entropy":
        rows, vocab, cols, b = case["rows"], case["vocab"], case["cols"], SIZE[case["dtype"]]
        live = rows - min(int(rows * case["masked"]), rows)
        total = (live + vocab) * cols * b + 16 * rows
        if case["out"]:
            total += rows * cols * b + vocab * cols * SIZE[case["out"]]
        # the logits, and two products with their gradient
        return {"bytes": total, "flops": (6 if case["out"] else 2) * live * vocab * cols}
    if op == "adamw":
        n = sum(_sizes(case))
        state = 16 if case["bits"] == 32 else 8 + 4 / BLOCK       # moments read and written; 8-bit ones returned as bf16
        copy = SIZE[case["copy"]] if case["copy"] else 0
        # clipped gradients are read for their norm before any of them is used
        return {"bytes": int(n * ((2 if case["clip"] else 1) * SIZE[case["grad"]] + 8 + copy + state)), "flops": 16 * n}
    rows, cols, b, pb = case["rows"], case["cols"], SIZE[case["dtype"]], SIZE[case["param"]]
    layer = case["kind"] == "layer"
    vectors = case["groups"] + (1 + layer) * (1 + case["post"])
    if op == "norm_forward":
        return {"bytes": 4 * rows * cols * b + vectors * cols * pb + 16 * rows, "flops": 16 * rows * cols}
    matrices = 6 if case["post"] or case["groups"] else 5         # the block's output takes part in gradients of gate and norm
    return {"bytes": matrices * rows * cols * b + 2 * vectors * cols * pb + 16 * rows, "flops": 32 * rows * cols}


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return {"entropy": _exact_entropy, "adamw": _exact_adamw}.get(case["op"], _exact_norm)(s)


def _exact_entropy(s):
    case = s["case"]
    rows, vocab = case["rows"], case["vocab"]
    table = s["table"].double()
    row = torch.zeros(rows, dtype=torch.float64, device=DEVICE)
    if case["out"]:
        dhidden = torch.zeros(s["hidden"].shape, dtype=torch.float64, device=DEVICE)
        dtable = torch.zeros_like(table)
    weight = s["weight"].double() * ((s["labels"] >= 0) & (s["labels"] < vocab))
    (index,) = torch.nonzero(weight, as_tuple=True)
    for part in index.split(1024):
        hidden, label = s["hidden"][part].double(), s["labels"][part]
        logp = torch.log_softmax(torch.einsum("nd,vd->nv", hidden, table), 1)
        here = torch.arange(part.numel(), device=DEVICE)
        row[part] = -logp[here, label]
        if case["out"]:
            p = logp.exp_()
            p[here, label] -= 1.0
            p *= (weight[part] * case["grad_scale"])[:, None]
            dhidden[part] = p.mm(table)
            dtable += p.t().mm(hidden)
    out = {"loss": (weight * row).sum().reshape(1), "row_loss": row}
    return {**out, "dhidden": dhidden, "dtable": dtable} if case["out"] else out


def _exact_norm(s):
    case = s["case"]
    layer, post, groups = case["kind"] == "layer", case["post"], case["groups"]
    rows, cols = s["x"].shape
    f = lambda name: s[name].to(torch.float64)  # noqa: E731

    def statistics(a):
        m = a.sum(1) / cols if layer else torch.zeros(rows, dtype=torch.float64, device=DEVICE)
        return m, 1.0 / torch.sqrt((a - m[:, None]).square().sum(1) / cols + EPS)

    def affine(a, m, r, w, b):
        unit = (a - m[:, None]) * r[:, None]
        return torch.addcmul(f(b), unit, f(w)) if layer else unit * f(w)

    gate = torch.ones(1, 1, cols, dtype=torch.float64, device=DEVICE) if groups == 0 else f("gate").view(groups, 1, cols)
    grouped = lambda a: a.view(max(groups, 1), -1, cols)  # noqa: E731
    if case["op"] == "norm_forward":
        block = f("block")
        pm, pr = statistics(block) if post else (torch.zeros(rows, device=DEVICE).double(), torch.ones(rows, device=DEVICE).double())
        u = affine(block, pm, pr, "post_weight", "post_bias") if post else block
        h = f("x") * case["scale"] + (grouped(u) * gate).view(rows, cols)
        # the stored residual is what is normed: its rounding is part of the definition
        seen = h.to(torch.float32).to(s["x"].dtype).to(torch.float64)
        m, r = statistics(seen)
        return {"h": h, "y": affine(seen, m, r, "weight", "bias"), "stats": torch.stack([pm, pr, m, r])}
    pm, pr, m, r = (a[:, None] for a in f("stats"))
    dy = f("dy")
    unit = (f("h") - m) * r
    through = lambda e, unit, r: r * (e - unit * (e * unit).sum(1, keepdim=True) / cols - (e.sum(1, keepdim=True) / cols if layer else 0.0))  # noqa: E731
    out = {"dweight": torch.einsum("rc,rc->c", dy, unit)}
    if layer:
        out["dbias"] = torch.ones(rows, dtype=torch.float64, device=DEVICE) @ dy
    dh = f("dh") + through(dy * f("weight"), unit, r)
    out["dx"] = dh * case["scale"]
    block = f("block")
    unit = (block - pm) * pr
    du = (grouped(dh) * gate).view(rows, cols)
    u = (affine(block, pm[:, 0], pr[:, 0], "post_weight", "post_bias") if post else block)
    if groups:
        out["dgate"] = torch.einsum("grc,grc->gc", grouped(dh), grouped(u)).view(s["gate"].shape)
    if not post:
        return {**out, "dblock": du}
    out["dpost_weight"] = torch.einsum("rc,rc->c", du, unit)
    if layer:
        out["dpost_bias"] = torch.ones(rows, dtype=torch.float64, device=DEVICE) @ du
    return {**out, "dblock": through(du * f("post_weight"), unit, pr)}


def _exact_adamw(s):
    """The update in 64 bits.  8-bit moments have no such value: which of two codes is taken is a choice of the rounding."""
    case = s["case"]
    t = FIRST_STEP + 1
    out = {}
    g = s["grad"].double()
    if case["clip"]:
        norm = torch.linalg.vector_norm(g)
        out["norm"] = norm.reshape(1)
        g *= min(1.0, MAX_NORM / (float(norm) + 1e-6))
    m, v = s["m"], s["v"]
    if case["bits"] == 8:
        m, v = _decode(m, s["m_scale"], True), _decode(v, s["v_scale"], False)
    m, v = torch.lerp(g, m.double(), BETA1), torch.lerp(g.square_(), v.double(), BETA2)
    out["m"], out["v"] = (m.clone(), v.clone()) if case["bits"] == 32 else (None, None)
    u = m.div_(1.0 - BETA1 ** t).div_(v.div_(1.0 - BETA2 ** t).sqrt_().add_(ADAM_EPS))
    out["param"] = s["param"].double().mul_(1.0 - LR * DECAY).sub_(u.mul_(LR))
    if case["copy"]:
        out["copy"] = out["param"]
    return out

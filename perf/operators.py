"""The operators at both ends of a training step, as measured cases.

A fine-tuning step that ends in the bucketed AdamW update begins and ends with
operators that move memory rather than multiply matrices: the token embedding
and its gradient, the layer norms between the blocks with the gradients of
their weights, and the loss on the logits (distillation from a teacher's top
logits, or a clipped policy loss with a KL term), whose gradient is as large
as the logits themselves.  Every case is one pass through one of them.

`run` computes the plain form (elementary torch operations in 32 bits, rounded
once at the end) or, with `own` set, makes the calls of
``paper_2509_21271_b200.operators``.  `exact` states the definitions once more
in 64 bits.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-5
CLIP_LOW, CLIP_HIGH = 0.2, 0.28


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def _norm(op, name, rows, cols, dtype, param):
    return {"op": op, "name": name, "rows": rows, "cols": cols, "dtype": dtype, "param": param}


def _embedding(op, name, tokens, cols, vocab, dtype, out, scaled, ids):
    return {"op": op, "name": name, "tokens": tokens, "cols": cols, "vocab": vocab,
            "dtype": dtype, "out": out, "scaled": scaled, "ids": ids}


def _distill(name, rows, vocab, pad, top, dtype, masked, temperature, grad_scale):
    return {"op": "distill", "name": name, "rows": rows, "vocab": vocab, "pad": pad, "top": top,
            "dtype": dtype, "masked": masked, "temperature": temperature, "grad_scale": grad_scale}


def _policy(name, rows, vocab, pad, dtype, masked, temperature, kl, grad_scale):
    return {"op": "policy", "name": name, "rows": rows, "vocab": vocab, "pad": pad, "dtype": dtype,
            "masked": masked, "temperature": temperature, "kl": kl, "grad_scale": grad_scale}


def listed():
    return [
        # one token through a norm of the small GPT-style stack: the cost of a call
        _norm("norm_forward", "norm_forward_one_row", 1, 768, "bf16", "bf16"),
        # the 8 x 4096 tokens of a micro-batch through a norm of the 8B-parameter stack
        _norm("norm_forward", "norm_forward_long", 32768, 4096, "bf16", "fp32"),
        # a short ragged micro-batch in fp16 with the fp32 master weights
        _norm("norm_backward", "norm_backward_ragged", 2047, 768, "fp16", "fp32"),
        # 16 x 2048 tokens through a norm of the 1B-parameter stack
        _norm("norm_backward", "norm_backward_long", 32768, 2048, "bf16", "bf16"),
        # 8 x 1024 tokens of the small GPT-style stack
        _embedding("embedding_forward", "embedding_forward_small", 8192, 768, 50257, "bf16", "bf16", False, "int64"),
        # a long packed batch of odd length, scaled by sqrt(width)
        _embedding("embedding_forward", "embedding_forward_long", 32767, 4096, 128256, "fp16", "fp16", True, "int32"),
        # the same 8 x 1024 tokens backward, into the bf16 gradient arena
        _embedding("embedding_backward", "embedding_backward_small", 8192, 768, 50257, "bf16", "bf16", False, "int64"),
        # 16 x 2048 tokens backward into an fp32 gradient arena
        _embedding("embedding_backward", "embedding_backward_long", 32768, 2048, 128256, "bf16", "fp32", True, "int64"),
        # one short answer distilled in fp16 under a loss scale; rows start at odd addresses
        _distill("distill_short", 63, 50257, 0, 16, "fp16", 0.0, 2.0, 65536.0),
        # 4096 tokens of a batch, some of them prompt, 64 teacher logits each
        _distill("distill_long", 4096, 128256, 0, 64, "bf16", 0.2, 1.0, 1.0),
        # one sampled answer, fp32 logits cut out of a padded vocabulary
        _policy("policy_one_answer", 129, 50257, 47, "fp32", 0.0, 1.0, 0.05, 1.0),
        # a packed batch of sampled answers with their prompts masked
        _policy("policy_long", 8191, 128256, 0, "bf16", 0.3, 0.7, 0.02, 1.0),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng):
    if rng.random() < 0.6:
        return rng.choice([512, 768, 1024, 1536, 2048, 2560, 4096, 5120, 8192])
    return _between(rng, 33, 8192)


def draw(rng):
    op = rng.choice(["norm_forward", "norm_backward", "embedding_forward", "embedding_backward", "distill", "policy"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("norm_forward", "norm_backward"):
        cols = _width(rng)
        rows = _between(rng, 1, min(65536, (1 << 28) // cols))
        case = _norm(op, "", rows, cols, dtype, rng.choice([dtype, "fp32"]))
    elif op in ("embedding_forward", "embedding_backward"):
        cols = _width(rng)
        vocab = rng.choice([50257, 128256, _between(rng, 1000, 128256)])
        vocab = min(vocab, (1 << 29) // cols)
        tokens = _between(rng, 1, min(65536, (1 << 28) // cols))
        out = dtype if op == "embedding_forward" else rng.choice([dtype, "fp32"])
        case = _embedding(op, "", tokens, cols, vocab, dtype, out, rng.random() < 0.5, rng.choice(["int32", "int64"]))
    else:
        vocab = rng.choice([50257, 128256, _between(rng, 1000, 160000)])
        rows = _between(rng, 1, min(8191, (1 << 31) // (vocab * SIZE[dtype])))
        masked = rng.choice([0.0, rng.uniform(0.05, 0.6)])
        pad = rng.choice([0, 0, rng.randint(1, 127)])
        scale = 65536.0 if dtype == "fp16" else 1.0
        temperature = rng.choice([1.0, rng.uniform(0.5, 4.0)])
        if op == "distill":
            case = _distill("", rows, vocab, pad, _between(rng, 1, 256), dtype, masked, temperature, scale)
        else:
            case = _policy("", rows, vocab, pad, dtype, masked, temperature, rng.choice([0.0, 0.05]), scale)
    case.pop("name")
    return case


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _tokens(g, n, vocab):
    """Token ids with the 1/rank frequencies of text, the ranks scattered over the vocabulary."""
    u = torch.rand(n, generator=g, device=DEVICE, dtype=torch.float64)
    rank = torch.exp(u * math.log(vocab + 1)).long().sub_(1).clamp_(0, vocab - 1)
    step = next(p for p in (48271, 16807, 69621) if math.gcd(p, vocab) == 1)
    return (rank * step + 17) % vocab


def _weights(g, rows, masked):
    """1 / (rows that count) each, zero for the masked rows."""
    w = torch.ones(rows, device=DEVICE)
    gone = min(int(rows * masked), rows)
    w[torch.randperm(rows, generator=g, device=DEVICE)[:gone]] = 0.0
    return w / max(rows - gone, 1)


def _logits(g, case):
    """[rows, vocab] cut out of rows of vocab + pad elements."""
    t = TYPES[case["dtype"]]
    full = torch.empty(case["rows"], case["vocab"] + case["pad"], dtype=t, device=DEVICE)
    for lo in range(0, case["rows"], 1024):
        part = full[lo:lo + 1024]
        part.copy_(torch.randn(part.shape, generator=g, device=DEVICE).mul_(2.0))
    return full[:, :case["vocab"]], torch.empty_like(full)[:, :case["vocab"]]


def _off_the_bounds(d):
    """Log ratios no nearer than 1e-3 to where the clipped loss has its kinks (the slope jumps there)."""
    for bound in (-math.log(1.0 - CLIP_LOW), -math.log(1.0 + CLIP_HIGH)):
        d = torch.where((d - bound).abs() < 1e-3, d + 2e-3, d)
    return d


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed * 1_000_003 + 17)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEVICE)  # noqa: E731
    op = case["op"]
    s = {"case": case}
    if op in ("norm_forward", "norm_backward"):
        rows, cols, t, pt = case["rows"], case["cols"], TYPES[case["dtype"]], TYPES[case["param"]]
        s["x"] = (rand(rows, cols) * 1.5 + 0.3 * rand(rows, 1)).to(t)
        s["weight"] = (1.0 + 0.1 * rand(cols)).to(pt)
        s["bias"] = (0.1 * rand(cols)).to(pt)
        s["out"] = torch.empty_like(s["x"])
        s["mean"] = torch.empty(rows, device=DEVICE)
        s["rstd"] = torch.empty(rows, device=DEVICE)
        if op == "norm_backward":
            s["dy"] = (rand(rows, cols) * 0.05).to(t)
            x = s["x"].float()
            s["mean"].copy_(x.mean(1))
            s["rstd"].copy_((x.var(1, unbiased=False) + EPS).rsqrt())
            s["dweight"] = torch.empty_like(s["weight"])
            s["dbias"] = torch.empty_like(s["bias"])
    elif op in ("embedding_forward", "embedding_backward"):
        n, cols, vocab, t = case["tokens"], case["cols"], case["vocab"], TYPES[case["dtype"]]
        s["ids"] = _tokens(g, n, vocab).to(torch.int32 if case["ids"] == "int32" else torch.int64)
        s["scale"] = math.sqrt(cols) if case["scaled"] else 1.0
        if op == "embedding_forward":
            s["table"] = (rand(vocab, cols) * 0.02).to(t)
            s["out"] = torch.empty(n, cols, dtype=t, device=DEVICE)
        else:
            s["dout"] = (rand(n, cols) * 0.01).to(t)
            s["dtable"] = torch.empty(vocab, cols, dtype=TYPES[case["out"]], device=DEVICE)
    else:
        rows, vocab, t = case["rows"], case["vocab"], TYPES[case["dtype"]]
        s["logits"], s["grad"] = _logits(g, case)
        s["weight"] = _weights(g, rows, case["masked"])
        s["loss"] = torch.empty(1, device=DEVICE)
        s["row_loss"] = torch.empty(rows, device=DEVICE)
        if op == "distill":
            k = min(case["top"], vocab)
            u = torch.rand(rows, k, generator=g, device=DEVICE, dtype=torch.float64)
            at = torch.arange(k, device=DEVICE, dtype=torch.float64)
            ids = ((at + u) * (vocab / k)).long().clamp_(0, vocab - 1)   # one of each k-th of the vocabulary
            teacher = rand(rows, k) * 2.0 + 9.0
            s["logits"].scatter_(1, ids, (teacher + 0.7 * rand(rows, k)).to(t))
            s["teacher_ids"] = ids.to(torch.int32)
            s["teacher_logits"] = teacher.to(t)
        else:
            s["tokens"] = torch.randint(vocab, (rows,), generator=g, device=DEVICE)
            s["logits"].scatter_(1, s["tokens"][:, None], (rand(rows, 1) * 2.0 + 12.0).to(t))
            logp = torch.empty(rows, device=DEVICE)
            for lo in range(0, rows, 1024):
                z = s["logits"][lo:lo + 1024].float() / case["temperature"]
                at = s["tokens"][lo:lo + 1024, None]
                logp[lo:lo + 1024] = z.gather(1, at)[:, 0] - torch.logsumexp(z, 1)
            s["old_logp"] = logp + _off_the_bounds(0.15 * rand(rows))
            s["ref_logp"] = logp + 0.3 * rand(rows)
            s["advantage"] = rand(rows)
            s["logp"] = torch.empty(rows, device=DEVICE)
    return s


# --------------------------------------------------------------------------
# the plain forms, and the framework's calls
# --------------------------------------------------------------------------

def _plain_norm_forward(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = ((c * c).mean(1, keepdim=True) + EPS).rsqrt()
    y = c * rstd * s["weight"].float() + s["bias"].float()
    return {"y": y.to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}


def _plain_norm_backward(s):
    x, dy = s["x"].float(), s["dy"].float()
    rstd = s["rstd"][:, None]
    xhat = (x - s["mean"][:, None]) * rstd
    g = dy * s["weight"].float()
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xhat).sum(0).to(s["weight"].dtype),
            "dbias": dy.sum(0).to(s["bias"].dtype)}


def _plain_embedding_forward(s):
    return {"out": (s["table"][s["ids"]].float() * s["scale"]).to(s["table"].dtype)}


def _plain_embedding_backward(s):
    dtable = torch.zeros(s["dtable"].shape, device=DEVICE)
    dtable.index_add_(0, s["ids"], s["dout"].float())
    return {"dtable": (dtable * s["scale"]).to(s["dtable"].dtype)}


def _plain_softmax(s):
    """Softmax of the rows of logits / temperature, and the logarithm of its denominator with the maximum."""
    z = s["logits"].float() * (1.0 / s["case"]["temperature"])
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    return z, e / total, top + total.log()


def _plain_distill(s):
    tau = s["case"]["temperature"]
    w, ids = s["weight"][:, None], s["teacher_ids"].long()
    z, q, lse = _plain_softmax(s)
    a = s["teacher_logits"].float() * (1.0 / tau)
    a = a - a.amax(1, keepdim=True)
    p = a.exp()
    total = p.sum(1, keepdim=True)
    p, logp = p / total, a - total.log()
    row = (tau * tau) * (p * (logp - (z.gather(1, ids) - lse))).sum(1)
    row = torch.where(s["weight"] != 0, row, torch.zeros_like(row))
    grad = q.scatter_add_(1, ids, -p) * (w * (tau * s["case"]["grad_scale"]))
    return {"loss": (s["weight"] * row).sum().reshape(1), "row_loss": row, "grad": grad.to(s["logits"].dtype)}


def _plain_policy(s):
    case, w, at = s["case"], s["weight"], s["tokens"][:, None]
    z, q, lse = _plain_softmax(s)
    logp = (z.gather(1, at) - lse)[:, 0]
    adv = s["advantage"]
    ratio = (logp - s["old_logp"]).exp()
    free, held = ratio * adv, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * adv
    d = s["ref_logp"] - logp
    row = case["kl"] * (d.exp() - d - 1.0) - torch.minimum(free, held)
    slope = case["kl"] * (1.0 - d.exp()) - torch.where(free <= held, free, torch.zeros_like(free))
    zero = torch.zeros_like(row)
    row, logp = torch.where(w != 0, row, zero), torch.where(w != 0, logp, zero)
    c = (w * slope * (case["grad_scale"] / case["temperature"]))[:, None]
    grad = (q * -c).scatter_add_(1, at, c)
    return {"loss": (w * row).sum().reshape(1), "row_loss": row, "logp": logp, "grad": grad.to(s["logits"].dtype)}


PLAIN = {"norm_forward": _plain_norm_forward, "norm_backward": _plain_norm_backward,
         "embedding_forward": _plain_embedding_forward, "embedding_backward": _plain_embedding_backward,
         "distill": _plain_distill, "policy": _plain_policy}


def _own(s):
    from paper_2509_21271_b200 import operators as ops
    case = s["case"]
    op = case["op"]
    if op == "norm_forward":
        y, mean, rstd = ops.layer_norm_forward(s["x"], s["weight"], s["bias"], EPS, out=s["out"],
                                               mean=s["mean"], rstd=s["rstd"])
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_backward":
        dx, dweight, dbias = ops.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"],
                                                     dx=s["out"], dweight=s["dweight"], dbias=s["dbias"])
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    if op == "embedding_forward":
        return {"out": ops.embedding_forward(s["ids"], s["table"], s["scale"], out=s["out"])}
    if op == "embedding_backward":
        return {"dtable": ops.embedding_backward(s["ids"], s["dout"], s["dtable"], s["scale"])}
    if op == "distill":
        loss, row, grad = ops.distill_loss(s["logits"], s["teacher_ids"], s["teacher_logits"], s["weight"],
                                           temperature=case["temperature"], grad_scale=case["grad_scale"],
                                           grad=s["grad"], loss=s["loss"], row_loss=s["row_loss"])
        return {"loss": loss, "row_loss": row, "grad": grad}
    loss, row, logp, grad = ops.policy_loss(s["logits"], s["tokens"], s["advantage"], s["weight"],
                                            old_logp=s["old_logp"], ref_logp=s["ref_logp"],
                                            temperature=case["temperature"], clip_low=CLIP_LOW,
                                            clip_high=CLIP_HIGH, kl_coef=case["kl"],
                                            grad_scale=case["grad_scale"], grad=s["grad"],
                                            loss=s["loss"], row_loss=s["row_loss"], logp=s["logp"])
    return {"loss": loss, "row_loss": row, "logp": logp, "grad": grad}


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["case"]["op"]](state)


# --------------------------------------------------------------------------
# bytes and operations that a pass cannot do without
# --------------------------------------------------------------------------

def _distinct(n, vocab):
    """How many different ids `n` tokens of the 1/rank distribution have, on average."""
    r = torch.arange(1, vocab + 1, dtype=torch.float64)
    p = ((r + 1) / r).log() / math.log(vocab + 1)
    return float((1.0 - torch.exp(n * torch.log1p(-p))).sum())


def work(case):
    op = case["op"]
    if op in ("norm_forward", "norm_backward"):
        rows, cols, b, pb = case["rows"], case["cols"], SIZE[case["dtype"]], SIZE[case["param"]]
        if op == "norm_forward":
            return {"bytes": 2 * rows * cols * b + 2 * cols * pb + 8 * rows, "flops": 7 * rows * cols}
        return {"bytes": 3 * rows * cols * b + 3 * cols * pb + 8 * rows, "flops": 15 * rows * cols}
    if op in ("embedding_forward", "embedding_backward"):
        n, cols, b = case["tokens"], case["cols"], SIZE[case["dtype"]]
        ids = n * (4 if case["ids"] == "int32" else 8)
        if op == "embedding_forward":
            return {"bytes": ids + (_distinct(n, case["vocab"]) + n) * cols * b, "flops": n * cols}
        return {"bytes": ids + n * cols * b + case["vocab"] * cols * SIZE[case["out"]], "flops": 2 * n * cols}
    rows, vocab, b = case["rows"], case["vocab"], SIZE[case["dtype"]]
    live = rows - min(int(rows * case["masked"]), rows)
    total = (live + rows) * vocab * b + 8 * rows
    if op == "distill":
        total += live * min(case["top"], vocab) * (4 + b)
    else:
        total += live * (8 + 12) + 4 * rows
    return {"bytes": total, "flops": 8 * live * vocab}


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    f = lambda name: s[name].to(torch.float64)  # noqa: E731
    op = case["op"]
    if op == "norm_forward":
        x = f("x")
        n = x.shape[1]
        mean = x.sum(1) / n
        var = (x - mean[:, None]).pow(2).sum(1) / n
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = torch.addcmul(f("bias"), (x - mean[:, None]) / torch.sqrt(var + EPS)[:, None], f("weight"))
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_backward":
        # y_i = w_i u_i + b_i with u = (x - mean) * rstd: the Jacobian of u applied to w * dy
        n = s["x"].shape[1]
        u = (f("x") - f("mean")[:, None]) * f("rstd")[:, None]
        v = f("dy") * f("weight")
        along = (u * v).sum(1, keepdim=True) / n
        dx = (v - u * along - v.sum(1, keepdim=True) / n) * f("rstd")[:, None]
        ones = torch.ones(1, u.shape[0], dtype=torch.float64, device=DEVICE)
        return {"dx": dx, "dweight": (ones @ (u * f("dy")))[0], "dbias": (ones @ f("dy"))[0]}
    if op == "embedding_forward":
        return {"out": torch.index_select(s["table"], 0, s["ids"]).to(torch.float64) * s["scale"]}
    if op == "embedding_backward":
        order = torch.argsort(s["ids"], stable=True)
        ids = s["ids"][order].long()
        first = torch.ones_like(ids, dtype=torch.bool)
        first[1:] = ids[1:] != ids[:-1]
        segment = first.cumsum(0) - 1
        sums = torch.zeros(int(segment[-1]) + 1, case["cols"], dtype=torch.float64, device=DEVICE)
        sums.index_put_((segment,), s["dout"][order].to(torch.float64), accumulate=True)
        out = torch.zeros(case["vocab"], case["cols"], dtype=torch.float64, device=DEVICE)
        out[ids[first]] = sums * s["scale"]
        return {"dtable": out}
    rows, tau = case["rows"], case["temperature"]
    grad = torch.zeros(rows, case["vocab"], dtype=torch.float64, device=DEVICE)
    row = torch.zeros(rows, dtype=torch.float64, device=DEVICE)
    logp = torch.zeros(rows, dtype=torch.float64, device=DEVICE)
    for lo in range(0, rows, 512):
        r = slice(lo, min(lo + 512, rows))
        w = f("weight")[r]
        logq = torch.log_softmax(s["logits"][r].to(torch.float64) / tau, 1)
        q = logq.exp()
        live = (w != 0).to(torch.float64)
        if op == "distill":
            ids = s["teacher_ids"][r].long()
            t = torch.log_softmax(s["teacher_logits"][r].to(torch.float64) / tau, 1)
            row[r] = live * tau * tau * (t.exp() * (t - torch.gather(logq, 1, ids))).sum(1)
            target = torch.zeros_like(q).scatter_add_(1, ids, t.exp())
            grad[r] = (q - target) * (case["grad_scale"] * tau * w)[:, None]
        else:
            here = torch.arange(w.numel(), device=DEVICE)
            at = s["tokens"][r]
            lp = logq[here, at]
            adv, old, ref = f("advantage")[r], f("old_logp")[r], f("ref_logp")[r]
            ratio = torch.exp(lp - old)
            bounded = torch.minimum(torch.maximum(ratio, ratio.new_tensor(1.0 - CLIP_LOW)),
                                    ratio.new_tensor(1.0 + CLIP_HIGH))
            gain = torch.minimum(ratio * adv, bounded * adv)
            kl = torch.expm1(ref - lp) - (ref - lp)
            row[r] = live * (case["kl"] * kl - gain)
            logp[r] = live * lp
            past = ((adv > 0) & (ratio > 1.0 + CLIP_HIGH)) | ((adv < 0) & (ratio < 1.0 - CLIP_LOW))
            slope = -case["kl"] * torch.expm1(ref - lp) - torch.where(past, torch.zeros_like(adv), ratio * adv)
            c = slope * w * case["grad_scale"] / tau
            part = q.neg_()
            part[here, at] += 1.0
            grad[r] = part * c[:, None]
    loss = (f("weight") * row).sum().reshape(1)
    out = {"loss": loss, "row_loss": row, "grad": grad}
    if op == "policy":
        out["logp"] = logp
    return out

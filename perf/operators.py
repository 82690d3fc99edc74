"""Cases that stand for what a program that trains or serves a language model has libbns do around its last layers.

* ``rms_forward``: the residual's addition and the root-mean-square norm, with an output in the inputs' type or in 8 bits
  (e4m3) with scales, and ``rms_backward``, its gradients.
* ``head_forward``: softmax cross entropy from the hidden states and the vocabulary's matrix, without keeping the logits, and
  ``head_backward``, the gradients of both.
* ``distill_forward``: the loss against a teacher's top logits, with the logits' gradient from the same pass, and
  ``distill_backward``, the gradient on its own from what the forward pass kept.

Where ``own`` is false, ``run`` computes them with elementary torch operations in 32 bits; where it is true, it calls the
library.  ``exact`` computes the same in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0
SMALLEST_SCALE = 2.0 ** -126
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ----------------------------------------------------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of a served model: the norm in front of an 8-bit product, one scale for the token
        dict(name="rms_token_e4m3", op="rms_forward", rows=1, width=4096, dtype="bf16", residual=True, out="e4m3", group=0, pow2=False),
        # a prompt in 8 bits, a power-of-two scale for every 32 elements
        dict(name="rms_prompt_e4m3", op="rms_forward", rows=8192, width=5120, dtype="bf16", residual=True, out="e4m3", group=32, pow2=True),
        # training, one block of a mid-sized model
        dict(name="rms_train_backward", op="rms_backward", rows=16384, width=4096, dtype="bf16", residual=True),
        # a small research model in 32 bits, a width that is no multiple of anything
        dict(name="rms_odd_backward", op="rms_backward", rows=777, width=1001, dtype="f32", residual=False),
        # scoring a handful of tokens against a mid-sized vocabulary (the matrix is read once)
        dict(name="head_few_tokens", op="head_forward", tokens=16, width=2048, vocab=50257, dtype="bf16", ignored=0.0),
        # a training step's loss: thousands of tokens, a large vocabulary
        dict(name="head_train", op="head_forward", tokens=4096, width=4096, vocab=131072, dtype="bf16", ignored=0.1),
        # a small model in 32 bits: ragged in every size
        dict(name="head_ragged_backward", op="head_backward", tokens=1021, width=1000, vocab=32003, dtype="f32", ignored=0.3),
        # the gradients of the training step above: the largest case
        dict(name="head_train_backward", op="head_backward", tokens=4096, width=4096, vocab=131072, dtype="bf16", ignored=0.1),
        # distillation on a small batch, a vocabulary whose rows begin on odd addresses
        dict(name="distill_odd", op="distill_forward", tokens=64, vocab=50257, k=20, dtype="bf16", tau=2.0, missing=0.1),
        # a training step of distillation
        dict(name="distill_train", op="distill_forward", tokens=4096, vocab=131072, k=64, dtype="bf16", tau=1.0, missing=0.0),
        # the gradient on its own, as an autograd graph asks for it, logits in 32 bits
        dict(name="distill_backward_f32", op="distill_backward", tokens=2048, vocab=50304, k=32, dtype="f32", tau=1.5, missing=0.1),
        # a few rows of a large vocabulary
        dict(name="distill_rows_backward", op="distill_backward", tokens=7, vocab=100003, k=100, dtype="bf16", tau=4.0, missing=0.2),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _size(rng, low, high, multiple):
    """A size between the two, spread over its logarithm; two times out of three a multiple as models have them."""
    n = _log(rng, low, high)
    if rng.random() < 2 / 3:
        n = min(high, max(multiple, round(n / multiple) * multiple))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["rms_forward", "rms_backward", "head_forward", "head_backward", "distill_forward", "distill_backward"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "rms_forward":
        out = rng.choice(["same", "e4m3"])
        group = rng.choice([0, 32, 64, 128]) if out == "e4m3" else 0
        return dict(op=op, rows=_log(rng, 1, 16384), width=_size(rng, 64, 8192, 64), dtype=dtype, residual=rng.random() < 0.7, out=out, group=group,
                    pow2=out == "e4m3" and rng.random() < 0.5)
    if op == "rms_backward":
        return dict(op=op, rows=_log(rng, 1, 16384), width=_size(rng, 64, 8192, 64), dtype=dtype, residual=rng.random() < 0.7)
    if op.startswith("head"):
        most = (4096 * 4096 * 131072) // (4 if dtype == "f32" else 1)
        while True:
            c = dict(op=op, tokens=_log(rng, 1, 4096), width=_size(rng, 64, 4096, 64), vocab=_size(rng, 1000, 131072, 128), dtype=dtype,
                     ignored=rng.choice([0.0, 0.1, 0.5]))
            if c["tokens"] * c["width"] * c["vocab"] <= most:
                return c
    return dict(op=op, tokens=_log(rng, 1, 2048 if dtype == "f32" else 4096), vocab=_size(rng, 1000, 131072, 128), k=_log(rng, 1, 128), dtype=dtype,
                tau=rng.choice([1.0, 2.0, 4.0]), missing=rng.choice([0.0, 0.1]))


def work(case):
    op, size = case["op"], 4 if case["dtype"] == "f32" else 2
    if op.startswith("rms"):
        n, rows, width = case["rows"] * case["width"], case["rows"], case["width"]
        if op == "rms_forward":
            y = n * size
            if case["out"] == "e4m3":
                y = n + 4 * rows * (-(-width // case["group"]) if case["group"] else 1)
            return {"bytes": n * size * (3 if case["residual"] else 1) + y + 4 * width + 4 * rows, "flops": 5 * n}
        return {"bytes": n * size * (4 if case["residual"] else 3) + 8 * width + 4 * rows, "flops": 10 * n}
    if op.startswith("head"):
        t, d, v = case["tokens"], case["width"], case["vocab"]
        once = (t + v) * d * size + 8 * t
        # backward: the logits again, as they are not kept, and one product for each gradient
        return {"bytes": once + 8 * t, "flops": 2 * t * d * v} if op == "head_forward" else {"bytes": 2 * once, "flops": 6 * t * d * v}
    n, teacher = case["tokens"] * case["vocab"], case["tokens"] * case["k"] * 12
    return {"bytes": 2 * n * size + teacher + 12 * case["tokens"], "flops": 6 * n}


# ----------------------------------------------------------------------------------------------------------------------
# what a program holds before the call
# ----------------------------------------------------------------------------------------------------------------------
def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    op = case["op"]
    if op.startswith("rms"):
        rows, width = case["rows"], case["width"]
        s = {"weight": 1 + normal(width, std=0.1, dtype=torch.float32)}
        # the residual stream of a trained model: rows of very different size, a few channels far larger than the others
        large = torch.where(uniform(width) < 0.005, 20.0, 1.0)
        stream = (normal(rows, width, dtype=torch.float32) * large * torch.exp(normal(rows, 1, dtype=torch.float32))).to(dt)
        if op == "rms_forward":
            s["x"], s["residual"] = (normal(rows, width, std=0.5), stream) if case["residual"] else (stream, None)
            return s
        s["x"] = stream
        s["rstd"] = torch.rsqrt(stream.float().square().mean(1) + EPS)
        s["dy"] = normal(rows, width, std=1e-2)
        s["dsum"] = normal(rows, width, std=1e-2) if case["residual"] else None
        return s
    if op.startswith("head"):
        t, d, v = case["tokens"], case["width"], case["vocab"]
        weight = normal(v, d, std=0.02)
        right = torch.randint(0, v, (t,), generator=g, device="cuda")
        # a trained model: for most tokens the right logit stands out by some amount
        ahead = 8 * uniform(t, 1) / (0.02 ** 2 * d)
        hidden = (normal(t, d, dtype=torch.float32) + ahead * weight[right].float()).to(dt)
        targets = torch.where(uniform(t) < case["ignored"], -100, right)
        s = {"hidden": hidden, "weight": weight, "targets": targets}
        if op == "head_backward":
            s["lse"] = torch.logsumexp(hidden.float() @ weight.float().T, 1)
            s["dloss"] = torch.full((t,), 1.0 / max(1, t), device="cuda")
        return s
    t, v, k = case["tokens"], case["vocab"], min(case["k"], case["vocab"])
    logits = normal(t, v, std=2.0)
    # the teacher's largest logits and where they are: in places that differ within a row
    start, step = torch.randint(0, v, (t, 1), generator=g, device="cuda"), max(1, v // k)
    ids = (start + step * torch.arange(k, device="cuda")) % v
    ids = torch.where(uniform(t, k) < case["missing"], -1, ids)
    teacher = 12.0 - 8.0 * uniform(t, k).sort(1).values
    s = {"logits": logits, "ids": ids, "teacher": teacher, "dloss": torch.full((t,), 1.0 / t, device="cuda") * (0.5 + uniform(t))}
    if op == "distill_backward":
        s["lse"] = torch.logsumexp(logits.float() / case["tau"], 1)
    return s


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if own:
        state.update(_buffers(case, state))
    return state


def _buffers(case, s):
    """What a program of the library keeps for its calls: the description of the problem, outputs and workspace."""
    from paper_1810_10962_amd import bns

    op = case["op"]
    f32 = lambda *shape: torch.empty(*shape, dtype=torch.float32, device="cuda")  # noqa: E731
    if op.startswith("rms"):
        rows, width = case["rows"], case["width"]
        if op == "rms_forward":
            rms = bns.make_rms(rows, width, case["dtype"], out=case["out"], group=case["group"], pow2_scales=case["pow2"], eps=EPS)
            e4m3 = case["out"] == "e4m3"
            return {"rms": rms, "sum": torch.empty_like(s["x"]) if case["residual"] else None, "rstd": f32(rows),
                    "y": torch.empty(rows, width, dtype=torch.float8_e4m3fn if e4m3 else s["x"].dtype, device="cuda"),
                    "scales": f32(rows, -(-width // case["group"]) if case["group"] else 1) if e4m3 else None}
        rms = bns.make_rms(rows, width, case["dtype"], eps=EPS)
        return {"rms": rms, "dx": torch.empty_like(s["x"]), "dweight": f32(width),
                "workspace": torch.empty(bns.bns_rms_workspace_bytes(rms), dtype=torch.uint8, device="cuda")}
    if op.startswith("head"):
        head = bns.make_head(case["tokens"], case["width"], case["vocab"], case["dtype"])
        got = {"head": head, "workspace": torch.empty(bns.bns_head_workspace_bytes(head), dtype=torch.uint8, device="cuda")}
        if op == "head_forward":
            return {**got, "loss": f32(case["tokens"]), "lse": f32(case["tokens"])}
        return {**got, "dhidden": torch.empty_like(s["hidden"]), "dweight": torch.empty_like(s["weight"])}
    return {"distill": bns.make_distill(case["tokens"], case["vocab"], s["ids"].shape[1], case["dtype"], temperature=case["tau"]),
            "loss": f32(case["tokens"]), "lse_out": f32(case["tokens"]), "dlogits": torch.empty_like(s["logits"])}


# ----------------------------------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state["case"], state)


def _own_rms_forward(case, s):
    from paper_1810_10962_amd import bns

    bns.bns_rms_forward(s["rms"], s["x"], s["residual"], s["weight"], s["sum"], s["y"], s["scales"], s["rstd"])
    return {"y": s["y"], "scales": s["scales"], "sum": s["sum"], "rstd": s["rstd"]}


def _own_rms_backward(case, s):
    from paper_1810_10962_amd import bns

    bns.bns_rms_backward(s["rms"], s["x"], s["weight"], s["rstd"], s["dy"], s["dsum"], s["dx"], s["dweight"], s["workspace"])
    return {"dx": s["dx"], "dweight": s["dweight"]}


def _own_head_forward(case, s):
    from paper_1810_10962_amd import bns

    bns.bns_head_forward(s["head"], s["hidden"], s["weight"], s["targets"], s["loss"], s["lse"], s["workspace"])
    return {"loss": s["loss"], "lse": s["lse"]}


def _own_head_backward(case, s):
    from paper_1810_10962_amd import bns

    bns.bns_head_backward(s["head"], s["hidden"], s["weight"], s["targets"], s["lse"], s["dloss"], s["dhidden"], s["dweight"], s["workspace"])
    return {"dhidden": s["dhidden"], "dweight": s["dweight"]}


def _own_distill_forward(case, s):
    from paper_1810_10962_amd import bns

    bns.bns_distill_forward(s["distill"], s["logits"], s["ids"], s["teacher"], s["dloss"], s["loss"], s["lse_out"], s["dlogits"])
    return {"loss": s["loss"], "lse": s["lse_out"], "dlogits": s["dlogits"]}


def _own_distill_backward(case, s):
    from paper_1810_10962_amd import bns

    bns.bns_distill_backward(s["distill"], s["logits"], s["ids"], s["teacher"], s["lse"], s["dloss"], s["dlogits"])
    return {"dlogits": s["dlogits"]}


def _plain_rms_forward(case, s):
    x = s["x"].float()
    if case["residual"]:
        x = x + s["residual"].float()
    rstd = torch.rsqrt((x * x).mean(1) + EPS)
    y = x * rstd[:, None] * s["weight"]
    scales = None
    if case["out"] == "e4m3":
        rows, width = y.shape
        group = case["group"] or width
        y = torch.nn.functional.pad(y, (0, -width % group)).view(rows, -1, group)
        scales = (y.abs().amax(2) / E4M3_MAX).clamp(min=SMALLEST_SCALE)
        if case["pow2"]:
            mantissa, exponent = torch.frexp(scales)
            scales = torch.ldexp(torch.ones_like(scales), torch.where(mantissa == 0.5, exponent - 1, exponent))
        y = (y / scales[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).view(rows, -1)[:, :width].to(torch.float8_e4m3fn)
    else:
        y = y.to(s["x"].dtype)
    return {"y": y, "scales": scales, "sum": x.to(s["x"].dtype) if case["residual"] else None, "rstd": rstd}


def _plain_rms_backward(case, s):
    x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    normed = x * rstd
    wdy = dy * s["weight"]
    dx = rstd * (wdy - normed * (wdy * normed).mean(1, keepdim=True))
    if case["residual"]:
        dx = dx + s["dsum"].float()
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * normed).sum(0)}


def _plain_head_forward(case, s):
    z = s["hidden"].float() @ s["weight"].float().T
    top = z.amax(1, keepdim=True)
    right = s["targets"].clamp(min=0)[:, None]
    at = torch.gather(z, 1, right)[:, 0]
    lse = torch.log(torch.exp(z - top).sum(1)) + top[:, 0]
    return {"loss": torch.where(s["targets"] >= 0, lse - at, 0.0), "lse": lse}


def _plain_head_backward(case, s):
    hidden, weight = s["hidden"].float(), s["weight"].float()
    g = torch.exp(hidden @ weight.T - s["lse"][:, None])
    valid = s["targets"] >= 0
    g.scatter_add_(1, s["targets"].clamp(min=0)[:, None], torch.full_like(s["lse"], -1.0)[:, None])
    g = g * torch.where(valid, s["dloss"], 0.0)[:, None]
    return {"dhidden": (g @ weight).to(s["hidden"].dtype), "dweight": (g.T @ hidden).to(s["weight"].dtype)}


def _teacher(case, s):
    valid = s["ids"] >= 0
    u = torch.where(valid, s["teacher"] / case["tau"], -torch.inf)
    q = torch.exp(u - u.amax(1, keepdim=True))
    q = torch.where(valid, q / q.sum(1, keepdim=True), 0.0)
    some = valid.any(1)
    return valid, torch.where(some[:, None], q, 0.0), some


def _distill_gradient(case, s, z, lse, q, some):
    dz = torch.exp(z - lse[:, None]) * some[:, None]
    dz.scatter_add_(1, s["ids"].clamp(min=0), -q)
    return (dz * (case["tau"] * s["dloss"])[:, None]).to(s["logits"].dtype)


def _plain_distill_forward(case, s):
    tau = case["tau"]
    z = s["logits"].float() / tau
    top = z.amax(1, keepdim=True)
    lse = torch.log(torch.exp(z - top).sum(1)) + top[:, 0]
    valid, q, some = _teacher(case, s)
    logp = torch.gather(z, 1, s["ids"].clamp(min=0)) - lse[:, None]
    kl = torch.where(q > 0, q * (torch.log(q) - logp), 0.0).sum(1)
    return {"loss": tau * tau * torch.where(some, kl, 0.0), "lse": lse, "dlogits": _distill_gradient(case, s, z, lse, q, some)}


def _plain_distill_backward(case, s):
    _, q, some = _teacher(case, s)
    return {"dlogits": _distill_gradient(case, s, s["logits"].float() / case["tau"], s["lse"], q, some)}


_own = {"rms_forward": _own_rms_forward, "rms_backward": _own_rms_backward, "head_forward": _own_head_forward,
        "head_backward": _own_head_backward, "distill_forward": _own_distill_forward, "distill_backward": _own_distill_backward}
_plain = {"rms_forward": _plain_rms_forward, "rms_backward": _plain_rms_backward, "head_forward": _plain_head_forward,
          "head_backward": _plain_head_backward, "distill_forward": _plain_distill_forward, "distill_backward": _plain_distill_backward}


# ----------------------------------------------------------------------------------------------------------------------
# the definition, in 64 bits
# ----------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in _inputs(case, seed).items()}
    return {"rms_forward": _exact_rms_forward, "rms_backward": _exact_rms_backward, "head_forward": _exact_head, "head_backward": _exact_head,
            "distill_forward": _exact_distill, "distill_backward": _exact_distill}[case["op"]](case, s)


def _exact_rms_forward(case, s):
    total = s["x"] if s["residual"] is None else s["x"] + s["residual"]
    norm = (total.pow(2).sum(1) / case["width"] + EPS).sqrt()
    y = total / norm.unsqueeze(1) * s["weight"]
    scales = None
    if case["out"] == "e4m3":
        group = case["group"] or case["width"]
        scales = torch.stack([part.abs().amax(1) for part in y.split(group, 1)], 1) / E4M3_MAX
        scales = torch.where(scales < SMALLEST_SCALE, torch.full_like(scales, SMALLEST_SCALE), scales)
        if case["pow2"]:
            scales = 2.0 ** torch.ceil(torch.log2(scales))
        y = y / scales.repeat_interleave(group, 1)[:, :case["width"]]
    return {"y": y, "scales": scales, "sum": total if s["residual"] is not None else None, "rstd": 1 / norm}


def _exact_rms_backward(case, s):
    # J = (rstd I - rstd^3 x x^T / width) for each row, applied to w dy
    r, wdy = s["rstd"].unsqueeze(1), s["dy"] * s["weight"]
    dx = r * wdy - r ** 3 / case["width"] * (s["x"] * wdy).sum(1, keepdim=True) * s["x"]
    return {"dx": dx if s["dsum"] is None else dx + s["dsum"], "dweight": torch.mv((s["dy"] * s["x"]).t(), s["rstd"])}


def _exact_head(case, s):
    counts = s["targets"] != -100
    rows = torch.arange(case["tokens"], device="cuda")[counts]
    z = torch.mm(s["hidden"], s["weight"].t())
    if case["op"] == "head_forward":
        lse = torch.logsumexp(z, 1)
        loss = torch.zeros_like(lse)
        loss[rows] = lse[rows] - z[rows, s["targets"][rows]]
        return {"loss": loss, "lse": lse}
    z = z.sub_(s["lse"].unsqueeze(1)).exp_()
    z[rows, s["targets"][rows]] -= 1
    z *= (s["dloss"] * counts).unsqueeze(1)
    return {"dhidden": torch.mm(z, s["weight"]), "dweight": torch.mm(z.t(), s["hidden"])}


def _exact_distill(case, s):
    tau, ids = case["tau"], s["ids"]
    u = (s["teacher"] / tau).masked_fill(ids < 0, -math.inf)
    logq = torch.log_softmax(u, 1)
    none = (ids < 0).all(1)
    q = logq.exp().masked_fill((ids < 0) | none.unsqueeze(1), 0.0)
    z = s["logits"] / tau
    lse = torch.logsumexp(z, 1) if case["op"] == "distill_forward" else s["lse"]
    logp = z - lse.unsqueeze(1)
    spread = torch.zeros_like(z).scatter_add_(1, ids.clamp(min=0), q)
    dz = (logp.exp() * q.sum(1, keepdim=True) - spread) * (tau * s["dloss"]).unsqueeze(1)
    if case["op"] == "distill_backward":
        return {"dlogits": dz}
    loss = tau ** 2 * (torch.xlogy(q, q) - q * logp.gather(1, ids.clamp(min=0))).sum(1)
    return {"loss": loss, "lse": lse, "dlogits": dz}

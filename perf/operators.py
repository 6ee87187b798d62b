"""The operators that distil a classifier from a quantized teacher's largest logits, as cases whose speed can be measured.

A teacher that only answers keeps its classifier in 8-bit integers, the largest logits of each row are kept (with the
log-sum-exp of all others), and a student learns from them and from labels.  Kinds of case, one per operator:
  fc       fc_i8_fwd: rows are quantized, multiplied with 8-bit weights in integers and scaled back (the weights have been
           quantized once, as a program does when it loads them).
  topk     topk_rows: the k largest logits of every row, their classes, and the log-sum-exp of the rest.
  distill  distill_fwd_bwd: the loss of student logits against a teacher's entries, mixed with the cross-entropy of labels, and
           (with "grad") its gradient.

`listed()` names the cases that are always looked at, `draw(rng)` gives others of the same ranges, `prepare` / `run` are one pass,
`work` is what a pass cannot do without, and `exact` the outputs from the definitions in 64 bits.  `own`: run the library's kernels
instead of the operators' plain forms.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def listed():
    return [
        # The classifier of ResNet-50 for a single image: latency.
        {"name": "fc 1 x 2048 -> 1000", "kind": "fc", "rows": 1, "cin": 2048, "cout": 1000, "x": "bf16", "y": "f32", "bias": True},
        # One token through a large projection: the weights are read once, 64 MB of them.
        {"name": "fc 1 x 8192 -> 8192", "kind": "fc", "rows": 1, "cin": 8192, "cout": 8192, "x": "bf16", "y": "bf16", "bias": False},
        # Odd sizes in every direction, float in and out: a ragged head in a check run.
        {"name": "fc 1001 x 2047 -> 4099, float", "kind": "fc", "rows": 1001, "cin": 2047, "cout": 4099, "x": "f32", "y": "f32", "bias": True},
        # A 1x1 convolution of ResNet-50 as a product over pixels: 1024 -> 256 at 14x14, batch 256, which memory bounds.
        {"name": "fc 50176 x 1024 -> 256", "kind": "fc", "rows": 50176, "cin": 1024, "cout": 256, "x": "bf16", "y": "bf16", "bias": True},
        # A large prompt through a large projection, which the matrix cores bound.
        {"name": "fc 8192 x 8192 -> 8192", "kind": "fc", "rows": 8192, "cin": 8192, "cout": 8192, "x": "bf16", "y": "bf16", "bias": False},
        # One worker's batch of ImageNet logits.
        {"name": "topk 40 x 1000, 8", "kind": "topk", "rows": 40, "classes": 1000, "k": 8, "x": "f32", "temperature": 2.0},
        # A single row of a large vocabulary: one row has to fill the card.
        {"name": "topk 1 x 131072, 64", "kind": "topk", "rows": 1, "classes": 131072, "k": 64, "x": "bf16", "temperature": 1.0},
        # A teacher's pass over a long batch, an odd number of classes, many entries.
        {"name": "topk 4096 x 50001, 100", "kind": "topk", "rows": 4096, "classes": 50001, "k": 100, "x": "bf16", "temperature": 2.0},
        # One worker's batch of ImageNet logits with label smoothing: the loss beside the classifier, a chain of short launches.
        {"name": "distill 40 x 1000, 8", "kind": "distill", "rows": 40, "classes": 1000, "k": 8, "x": "f32", "temperature": 4.0, "alpha": 0.5,
         "smoothing": 0.1, "tail": True, "ragged": False, "grad": True},
        # A few rows of a large vocabulary, truncated entries without the teacher's tail.
        {"name": "distill 7 x 131072, 32", "kind": "distill", "rows": 7, "classes": 131072, "k": 32, "x": "bf16", "temperature": 1.0, "alpha": 1.0,
         "smoothing": 0.0, "tail": False, "ragged": True, "grad": True},
        # Validation: the loss alone, an odd number of classes.
        {"name": "distill 4096 x 50001, loss", "kind": "distill", "rows": 4096, "classes": 50001, "k": 100, "x": "bf16", "temperature": 2.0,
         "alpha": 0.7, "smoothing": 0.0, "tail": True, "ragged": True, "grad": False},
        # A training step's loss and gradient over a long batch of a large vocabulary: the largest.
        {"name": "distill 2048 x 131072, 64", "kind": "distill", "rows": 2048, "classes": 131072, "k": 64, "x": "bf16", "temperature": 2.0,
         "alpha": 0.7, "smoothing": 0.0, "tail": True, "ragged": True, "grad": True},
    ]


def _between(rng, lo, hi):
    """Spread over the logarithm of the range; a third of them multiples of 64 (as far as the range has them), the rest as they fall."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n > 64 and rng.random() < 1 / 3:
        n -= n % 64
    return max(lo, min(hi, n))


def draw(rng):
    kind = rng.choice(("fc", "topk", "distill"))
    if kind == "fc":
        rows, cin, cout = _between(rng, 1, 50176), _between(rng, 64, 8192), _between(rng, 64, 16384)
        while rows * cin * cout > 8192 ** 3 or rows * cout > 1 << 28:
            rows = max(1, rows // 2 - 1)
        return {"kind": kind, "rows": rows, "cin": cin, "cout": cout, "x": rng.choice(("bf16", "bf16", "f32")), "y": rng.choice(("bf16", "f32")),
                "bias": rng.random() < 0.5}
    rows, classes, k = _between(rng, 1, 4096), _between(rng, 256, 131072), _between(rng, 1, 128)
    while rows * classes > 1 << 28:
        rows = max(1, rows // 2 - 1)
    case = {"kind": kind, "rows": rows, "classes": classes, "k": k, "x": rng.choice(("bf16", "f32")), "temperature": rng.choice((1.0, 2.0, 4.0))}
    if kind == "distill":
        if case["x"] == "f32":
            case["rows"] = max(1, rows // 2)
        case.update(tail=rng.random() < 0.7, smoothing=rng.choice((0.0, 0.1)), ragged=rng.random() < 0.5, grad=rng.random() < 0.8)
        # (the divergence of cells that hold nearly the same on both sides is a difference far below its terms: with a tail, labels go along)
        case["alpha"] = rng.choice((0.3, 0.5, 0.7) if case["tail"] else (0.3, 0.7, 1.0))
    return case


# ------------------------------------------------------------------ inputs
def _quantized_weights(w):
    """8-bit rows, zeros up to a multiple of 64 bytes, and a scale for each row: as quant_rows_i8 lays them out."""
    n, k = w.shape
    a = w.abs().amax(1).clamp(min=2.0 ** -100)
    c = torch.full_like(a, 127.0)
    q = torch.zeros((n, (k + 63) // 64 * 64), dtype=torch.int8, device=w.device)
    q[:, :k] = torch.round(w * (c / a)[:, None]).to(torch.int8)
    return q, a / c


def _logits(g, rows, classes):
    """A trained classifier's logits: most classes near the row's floor, a few far above it."""
    z = torch.randn((rows, classes), device="cuda", generator=g)
    z *= 1.6
    peaks = min(classes, 24)
    at = torch.randint(0, classes, (rows, peaks), device="cuda", generator=g)
    z.scatter_add_(1, at, torch.rand((rows, peaks), device="cuda", generator=g) * 9.0)
    return z


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case}
    if case["kind"] == "fc":
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        x = torch.randn((rows, cin), device="cuda", generator=g)
        x *= torch.exp(0.5 * torch.randn((1, cin), device="cuda", generator=g))  # channels differ in size, tokens as well
        x *= torch.exp(0.5 * torch.randn((rows, 1), device="cuda", generator=g))
        w = torch.randn((cout, cin), device="cuda", generator=g) * (cin ** -0.5)
        state["x"] = x.to(DTYPES[case["x"]])
        state["w"], state["w_scale"] = _quantized_weights(w)
        state["bias"] = torch.randn(cout, device="cuda", generator=g) if case["bias"] else None
        return state
    rows, classes, k, t = case["rows"], case["classes"], case["k"], case["temperature"]
    z = _logits(g, rows, classes)
    if case["kind"] == "topk":
        state["logits"] = z.to(DTYPES[case["x"]])
        return state
    state["values"], at = torch.topk(z, min(k, classes), dim=1)
    if case["tail"]:
        state["tail"] = torch.logsumexp((z / t).scatter_(1, at, -math.inf), 1)
    else:
        state["tail"] = None
    if case["ragged"]:  # a row keeps 1 to k entries, the others are marked as absent
        kept = torch.randint(1, at.shape[1] + 1, (rows, 1), device="cuda", generator=g)
        absent = torch.arange(at.shape[1], device="cuda")[None, :] >= kept
        if case["tail"]:  # what is cut off belongs to the tail
            cut = torch.logsumexp((state["values"] / t).masked_fill(~absent, -math.inf), 1)
            state["tail"] = torch.logaddexp(state["tail"], cut)
        at = at.masked_fill(absent, -1)
    state["indices"] = at.to(torch.int32)
    state["labels"] = torch.randint(0, classes, (rows,), device="cuda", generator=g).to(torch.int32)
    counted = torch.rand(rows, device="cuda", generator=g) < 0.95  # the others are padding
    counted[0] = True
    state["weight"] = counted.float() / counted.sum()
    z *= 0.8
    z += 0.6 * torch.randn((rows, classes), device="cuda", generator=g)
    state["logits"] = z.to(DTYPES[case["x"]])
    return state


# ------------------------------------------------------------- plain forms
def _plain_fc(x, w, w_scale, bias, dtype):
    x = x.float()
    a = x.abs().amax(1).clamp(min=2.0 ** -100)
    c = torch.full_like(a, 127.0)
    q = torch.round(x * (c / a)[:, None])
    y = torch.matmul(q, w[:, :x.shape[1]].float().t()) * (a / c)[:, None] * w_scale
    return (y if bias is None else y + bias).to(dtype)


def _lse(u):
    """log(sum(exp(u))) of every row; -inf where the row holds nothing else."""
    m = u.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    return torch.log(torch.exp(u - m).sum(1)) + m[:, 0]


def _plain_topk(logits, k, temperature):
    x = logits.float()
    values, at = torch.sort(x, dim=1, descending=True, stable=True)
    values, at = values[:, :k], at[:, :k]
    return values, at.to(torch.int32), _lse((x / temperature).scatter(1, at, -math.inf))


def _plain_distill(state):
    case, logits = state["case"], state["logits"]
    t, alpha, ls = case["temperature"], case["alpha"], case["smoothing"]
    z = logits.float()
    n, c = z.shape
    w = state["weight"]
    # the teacher's cells: its entries and the tail
    present = state["indices"] >= 0
    at = torch.where(present, state["indices"], torch.zeros_like(state["indices"])).long()
    v = torch.where(present, state["values"] / t, torch.full_like(state["values"], -math.inf))
    tail = torch.full((n,), -math.inf, device=z.device) if state["tail"] is None else state["tail"]
    cells = torch.cat([v, tail[:, None]], 1)
    logp = cells - _lse(cells)[:, None]
    p = torch.exp(logp)
    # the student's
    u = z / t
    total = _lse(u)
    top = torch.zeros((n, c), dtype=torch.int32, device=z.device).scatter_add_(1, at, present.to(torch.int32)) > 0
    rest = _lse(torch.where(top, torch.full_like(u, -math.inf), u))
    logq = torch.cat([u.gather(1, at), rest[:, None]], 1) - total[:, None]
    kl = torch.where(p > 0, p * (logp - logq), torch.zeros_like(p)).sum(1)
    row = alpha * t * t * kl
    if alpha < 1:
        logs = z - _lse(z)[:, None]
        label = state["labels"].long()[:, None]
        row = row + (1 - alpha) * (-(1 - ls) * logs.gather(1, label)[:, 0] - ls / c * logs.sum(1))
    row = torch.where(w != 0, row, torch.zeros_like(row))
    loss = (w * row).sum().reshape(1)
    if not case["grad"]:
        return loss, row
    pr, qr = p[:, -1:], torch.exp(rest - total)[:, None]
    d = torch.where(top, torch.exp(u - total[:, None]), torch.exp(u - rest[:, None]) * (qr - pr))
    d.scatter_add_(1, at, -p[:, :-1])
    d *= alpha * t
    if alpha < 1:
        d += (1 - alpha) * (torch.exp(logs) - ls / c)
        d.scatter_add_(1, label, torch.full((n, 1), -(1 - alpha) * (1 - ls), device=z.device))
    return loss, row, (d * w[:, None]).to(logits.dtype)


def run(state):
    case = state["case"]
    if not own:
        if case["kind"] == "fc":
            return _plain_fc(state["x"], state["w"], state["w_scale"], state["bias"], DTYPES[case["y"]])
        if case["kind"] == "topk":
            return _plain_topk(state["logits"], case["k"], case["temperature"])
        return _plain_distill(state)
    import paper_1903_12650_amd as rn
    if case["kind"] == "fc":
        return rn.fc_i8_fwd(state["x"], state["w"], state["w_scale"], state["bias"], dtype=DTYPES[case["y"]])
    if case["kind"] == "topk":
        return rn.topk_rows(state["logits"], case["k"], case["temperature"])
    out = rn.distill_fwd_bwd(state["logits"], state["values"], state["indices"], state["tail"], state["labels"], temperature=case["temperature"],
                             alpha=case["alpha"], label_smoothing=case["smoothing"], row_weight=state["weight"], grad=case["grad"])
    return out if case["grad"] else out[:2]


def work(case):
    if case["kind"] == "fc":
        m, k, n = case["rows"], case["cin"], case["cout"]
        return {"bytes": m * k * SIZE[case["x"]] + n * k + 4 * n * (2 if case["bias"] else 1) + m * n * SIZE[case["y"]], "flops": 2 * m * n * k}
    n, c, k = case["rows"], case["classes"], min(case["k"], case["classes"])
    if case["kind"] == "topk":
        return {"bytes": n * c * SIZE[case["x"]] + 8 * n * k + 4 * n, "flops": 4 * n * c}
    entries = 8 * n * k + (4 * n if case["tail"] else 0) + 12 * n
    return {"bytes": n * c * SIZE[case["x"]] * (2 if case["grad"] else 1) + entries, "flops": n * c * (12 if case["grad"] else 6)}


# ------------------------------------------------ the definitions in 64 bits
def _exact_distill(case, s):
    t, alpha, ls = case["temperature"], case["alpha"], case["smoothing"]
    z = s["logits"].double().requires_grad_(case["grad"])
    n, c = z.shape
    entry = s["indices"] >= 0
    at = s["indices"].long().clamp(min=0)
    member = torch.zeros((n, c + 1), dtype=torch.bool, device=z.device)
    member.scatter_(1, torch.where(entry, at, c), True)
    member = member[:, :c]
    teacher = (s["values"].double() / t).masked_fill(~entry, -math.inf)
    student = torch.log_softmax(z / t, 1)
    q = student.gather(1, at).masked_fill(~entry, 0.0)
    if s["tail"] is not None:
        teacher = torch.cat([teacher, s["tail"].double()[:, None]], 1)
        q = torch.cat([q, torch.logsumexp(student.masked_fill(member, -math.inf), 1, keepdim=True)], 1)
    logp = torch.log_softmax(teacher, 1)
    p = logp.exp()
    row = alpha * t * t * (p * (logp.masked_fill(p == 0, 0.0) - q)).sum(1)
    if alpha < 1:
        logs = torch.log_softmax(z, 1)
        row = row - (1 - alpha) * ((1 - ls) * logs.gather(1, s["labels"].long()[:, None])[:, 0] + ls * logs.mean(1))
    w = s["weight"].double()
    loss = (w * row).sum().reshape(1)
    row = row * (w != 0)
    if not case["grad"]:
        return loss, row
    loss.backward()
    return loss.detach(), row.detach(), z.grad


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "fc":
        x = s["x"].double()
        a = x.abs().amax(1, keepdim=True)
        y = torch.round(127.0 * x / a) @ s["w"][:, :case["cin"]].double().T
        y = y * (a / 127.0) * s["w_scale"].double()
        return y if s["bias"] is None else y + s["bias"].double()
    if case["kind"] == "topk":
        x = s["logits"].double()
        order = torch.argsort(-x, dim=1, stable=True)[:, :case["k"]]
        return x.gather(1, order), order, torch.logsumexp((x / case["temperature"]).scatter(1, order, -math.inf), 1)
    return _exact_distill(case, s)

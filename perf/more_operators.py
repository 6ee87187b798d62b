"""The operators that train a classifier in 8-bit floating point behind a dropout, as cases whose speed can be measured.

Matrices are held in 8-bit floating point with a power of two for every 128 numbers along the axis that a product sums over; a dropout's
mask is a function of a seed, the number of the call and the element's place, and is never stored.  Kinds of case, one per operator:
  dropout  dropout_fwd (with a residual where there is one) and, in a training pass, dropout_bwd.
  quant    quant_blocks_f8: a matrix quantized along its rows and, transposed, along its columns, in one call.
  matmul   matmul_f8: the product of two quantized matrices, scaled back.
  fwd      fc_f8_fwd: rows are dropped out and quantized, and multiplied with quantized weights; a training pass keeps the rows
           quantized along the batch.
  bwd      fc_f8_bwd: the gradients of input, weights and bias from the output's gradient and what was kept.

`listed()` names the cases that are always looked at, `draw(rng)` gives others of the same ranges, `prepare` / `run` are one pass,
`work` is what a pass cannot do without, and `exact` the outputs from the definitions in 64 bits.  `own`: run the library's kernels
instead of the operators' plain forms.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def listed():
    return [
        # The features in front of ResNet-50's classifier, one worker's batch: latency.
        {"name": "dropout 40 x 2048", "kind": "dropout", "rows": 40, "cols": 2048, "x": "bf16", "p": 0.2, "residual": False, "back": False},
        # Both directions of a dropout with a residual on the activations of a block, batch 256 at 14x14, which memory bounds.
        {"name": "dropout 50176 x 1024, trained", "kind": "dropout", "rows": 50176, "cols": 1024, "x": "bf16", "p": 0.1, "residual": True, "back": True},
        # Odd sizes: a gradient in float, kept in the format with the wider range.
        {"name": "quant 1001 x 2047, float", "kind": "quant", "rows": 1001, "cols": 2047, "x": "f32", "format": "e5m2"},
        # The weights of a large projection after an update, for the forward and the backward pass.
        {"name": "quant 8192 x 8192", "kind": "quant", "rows": 8192, "cols": 8192, "x": "bf16", "format": "e4m3"},
        # The classifier's product of one worker's batch: few rows, the weights are what is read.
        {"name": "matmul 40 x 2048 -> 1000", "kind": "matmul", "rows": 40, "cin": 2048, "cout": 1000, "format": "e4m3", "y": "f32", "bias": True},
        # Odd sizes in every direction, a gradient's product.
        {"name": "matmul 1001 x 2047 -> 4099", "kind": "matmul", "rows": 1001, "cin": 2047, "cout": 4099, "format": "e5m2", "y": "f32", "bias": False},
        # A large batch through a large projection, which the matrix cores bound: the largest.
        {"name": "matmul 8192 x 8192 -> 8192", "kind": "matmul", "rows": 8192, "cin": 8192, "cout": 8192, "format": "e4m3", "y": "bf16", "bias": False},
        # A single image's answer.
        {"name": "fwd 1 x 2048 -> 1000", "kind": "fwd", "rows": 1, "cin": 2048, "cout": 1000, "x": "bf16", "y": "f32", "bias": True, "p": 0.0, "train": False},
        # A training pass through a projection with dropout.
        {"name": "fwd 8192 x 4096 -> 4096, trained", "kind": "fwd", "rows": 8192, "cin": 4096, "cout": 4096, "x": "bf16", "y": "bf16", "bias": True,
         "p": 0.1, "train": True},
        # The classifier's gradients of one worker's batch, from gradients of logits in float.
        {"name": "bwd 40 x 2048 -> 1000", "kind": "bwd", "rows": 40, "cin": 2048, "cout": 1000, "x": "f32", "y": "bf16", "p": 0.2, "format": "e4m3"},
        # A 1x1 convolution of ResNet-50 as a product over pixels: 1024 -> 256 at 14x14, batch 256: a long sum into small weights.
        {"name": "bwd 50176 x 1024 -> 256", "kind": "bwd", "rows": 50176, "cin": 1024, "cout": 256, "x": "bf16", "y": "bf16", "p": 0.0, "format": "e5m2"},
        # The gradients of the projection above.
        {"name": "bwd 8192 x 4096 -> 4096", "kind": "bwd", "rows": 8192, "cin": 4096, "cout": 4096, "x": "bf16", "y": "bf16", "p": 0.1, "format": "e4m3"},
    ]


def _between(rng, lo, hi):
    """Spread over the logarithm of the range; a third of them multiples of 64 (as far as the range has them), the rest as they fall."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n > 64 and rng.random() < 1 / 3:
        n -= n % 64
    return max(lo, min(hi, n))


def draw(rng):
    kind = rng.choice(("dropout", "quant", "matmul", "fwd", "fwd", "bwd", "bwd"))
    if kind in ("dropout", "quant"):
        rows, cols = _between(rng, 1, 65536), _between(rng, 1 if kind == "dropout" else 16, 16384)
        while rows * cols > 1 << 26:
            rows = max(1, rows // 2 - 1)
        case = {"kind": kind, "rows": rows, "cols": cols, "x": rng.choice(("bf16", "bf16", "f32"))}
        if kind == "quant":
            case["format"] = rng.choice(("e4m3", "e4m3", "e5m2"))
        else:
            case.update(p=rng.choice((0.0, 0.1, 0.2, 0.5)), residual=rng.random() < 0.5, back=rng.random() < 0.5)
        return case
    rows, cin, cout = _between(rng, 1, 50176), _between(rng, 64, 8192), _between(rng, 64, 16384)
    while rows * cin * cout > (8192 ** 3 if kind == "matmul" else 8192 ** 3 // 4) or rows * max(cin, cout) > 1 << 27:
        rows = max(1, rows // 2 - 1)
    case = {"kind": kind, "rows": rows, "cin": cin, "cout": cout, "y": rng.choice(("bf16", "f32"))}
    if kind != "bwd":
        case["bias"] = rng.random() < 0.5
    if kind != "fwd":
        case["format"] = rng.choice(("e4m3", "e4m3", "e5m2"))
    if kind != "matmul":
        case.update(x=rng.choice(("bf16", "bf16", "f32")), p=rng.choice((0.0, 0.1, 0.2, 0.5)))
    if kind == "fwd":
        case["train"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------ inputs
def _values(g, rows, cols):
    """Channels differ in size, rows (images, tokens) as well."""
    x = torch.randn((rows, cols), device="cuda", generator=g)
    x *= torch.exp(0.5 * torch.randn((1, cols), device="cuda", generator=g))
    x *= torch.exp(0.5 * torch.randn((rows, 1), device="cuda", generator=g))
    return x


def _gradient(g, rows, cols):
    """Small, of very different sizes from row to row, most of it near zero."""
    x = torch.randn((rows, cols), device="cuda", generator=g)
    x *= x.abs()
    x *= torch.exp(torch.randn((rows, 1), device="cuda", generator=g)) * (1e-3 / rows)
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case, "seed": 100000 + seed}  # (the dropout's)
    kind = case["kind"]
    if kind == "dropout":
        state["x"] = _values(g, case["rows"], case["cols"]).to(DTYPES[case["x"]])
        state["residual"] = _values(g, case["rows"], case["cols"]).to(DTYPES[case["x"]]) if case["residual"] else None
        state["dy"] = _gradient(g, case["rows"], case["cols"]).to(DTYPES[case["x"]]) if case["back"] else None
        return state
    if kind == "quant":
        make = _gradient if case["format"] == "e5m2" else _values
        state["x"] = make(g, case["rows"], case["cols"]).to(DTYPES[case["x"]])
        return state
    rows, cin, cout = case["rows"], case["cin"], case["cout"]
    w = torch.randn((cout, cin), device="cuda", generator=g) * (cin ** -0.5)
    if kind == "matmul":
        make = _gradient if case["format"] == "e5m2" else _values
        state["a"], state["a_scale"] = _quantized(make(g, rows, cin), case["format"])
        state["w"], state["w_scale"] = _quantized(w, "e4m3")
    elif kind == "fwd":
        state["x"] = _values(g, rows, cin).to(DTYPES[case["x"]])
        state["w"], state["w_scale"] = _quantized(w, "e4m3")
    else:
        state["dy"] = _gradient(g, rows, cout).to(DTYPES[case["x"]])
        state["wt"], state["wt_scale"] = _quantized(w.t(), "e4m3")
        x = _values(g, rows, cin)
        if case["p"]:
            x = x * (torch.rand((rows, cin), device="cuda", generator=g) >= case["p"]) / (1 - case["p"])
        state["xt"], state["xt_scale"] = _quantized(x.t(), "e4m3")
    if kind != "bwd":
        state["bias"] = torch.randn(cout, device="cuda", generator=g) if case["bias"] else None
    return state


# ------------------------------------------------------------- plain forms
def _power(e):
    """2^e, exactly (a power function may be a unit in the last place off)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantized(x, fmt):
    """Rows of x in blocks of 128: 8-bit numbers (zeros up to a multiple of 128) and the powers' exponents + 127, four blocks of a
    row side by side, rows behind one another."""
    m, k = x.shape
    blocks, groups = (k + 127) // 128, (k + 511) // 512
    v = torch.zeros((m, blocks * 128), device=x.device)
    v[:, :k] = x
    v = v.view(m, blocks, 128)
    fraction, power = torch.frexp(v.abs().amax(2).clamp(min=2.0 ** -100))
    e = power - (9 if fmt == "e4m3" else 16) + (fraction > 0.875).to(power.dtype)
    q = (v * _power(-e)[:, :, None]).to(FORMATS[fmt]).view(m, blocks * 128)
    scale = torch.zeros((m, groups * 4), dtype=torch.uint8, device=x.device)
    scale[:, :blocks] = (e + 127).to(torch.uint8)
    return q, scale.view(m, groups, 4).transpose(0, 1).contiguous()


def _dequantized(q, scale):
    m, k = q.shape
    e = scale.transpose(0, 1).reshape(m, -1)[:, :k // 128].to(torch.int32) - 127
    return (q.float().view(m, k // 128, 128) * _power(e)[:, :, None]).view(m, k)


def _threshold(p):
    return int(round(p * 65536))


def _kept(rows, cols, p, seed, call=0):
    """[r >= t] of every element: r 16 bits of Philox4x32-10, 8 elements of a row from one counter."""
    per_row = (cols + 7) // 8
    b = torch.arange(rows * per_row, device="cuda")
    mask = 0xffffffff
    c0, c1, c2, c3 = b & mask, (b >> 32) | 0x80000000, torch.full_like(b, call & mask), torch.full_like(b, call >> 32)
    k0, k1 = seed & mask, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & mask) ^ c1 ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ c3 ^ k1, p0 & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    words = torch.stack((c0, c1, c2, c3), 1)
    r = torch.stack((words & 0xffff, words >> 16), 2).view(rows, per_row * 8)[:, :cols]
    return r >= _threshold(p)


def _dropped(x, p, seed):
    """In 32 bits."""
    t = _threshold(p)
    x = x.float() * (65536 / (65536 - t))
    return torch.where(_kept(x.shape[0], x.shape[1], p, seed), x, torch.zeros_like(x))


def _plain(state):
    case, seed = state["case"], state["seed"]
    kind = case["kind"]
    if kind == "dropout":
        y = _dropped(state["x"], case["p"], seed)
        if case["residual"]:
            y = y + state["residual"].float()
        y = y.to(state["x"].dtype)
        return (y, _dropped(state["dy"], case["p"], seed).to(y.dtype)) if case["back"] else y
    if kind == "quant":
        x = state["x"].float()
        return _quantized(x, case["format"]) + _quantized(x.t(), case["format"])
    if kind == "matmul":
        y = torch.matmul(_dequantized(state["a"], state["a_scale"]), _dequantized(state["w"], state["w_scale"]).t())
        return (y if state["bias"] is None else y + state["bias"]).to(DTYPES[case["y"]])
    if kind == "fwd":
        x = _dropped(state["x"], case["p"], seed) if case["p"] else state["x"].float()
        y = torch.matmul(_dequantized(*_quantized(x, "e4m3")), _dequantized(state["w"], state["w_scale"]).t())
        y = (y if state["bias"] is None else y + state["bias"]).to(DTYPES[case["y"]])
        return (y,) + _quantized(x.t(), "e4m3") if case["train"] else y
    dy = state["dy"].float()
    dx = torch.matmul(_dequantized(*_quantized(dy, case["format"])), _dequantized(state["wt"], state["wt_scale"]).t())
    if case["p"]:
        dx = _dropped(dx, case["p"], seed)
    dw = torch.matmul(_dequantized(*_quantized(dy.t(), case["format"])), _dequantized(state["xt"], state["xt_scale"]).t())
    return dx.to(DTYPES[case["y"]]), dw, dy.double().sum(0).float()


def run(state):
    if not own:
        return _plain(state)
    import paper_1903_12650_amd as rn
    case = state["case"]
    kind = case["kind"]
    drop = rn.Dropout(case["p"], state["seed"]) if case.get("p") or kind == "dropout" else None
    if kind == "dropout":
        y = rn.dropout_fwd(state["x"], drop, state["residual"])
        return (y, rn.dropout_bwd(state["dy"], drop)) if case["back"] else y
    if kind == "quant":
        return rn.quant_blocks_f8(state["x"], FORMATS[case["format"]], rows=True, columns=True)
    if kind == "matmul":
        return rn.matmul_f8(case["cin"], state["a"], state["a_scale"], state["w"], state["w_scale"], state["bias"], dtype=DTYPES[case["y"]])
    if kind == "fwd":
        return rn.fc_f8_fwd(state["x"], state["w"], state["w_scale"], state["bias"], dtype=DTYPES[case["y"]], dropout=drop, save=case["train"])
    return rn.fc_f8_bwd(state["dy"], state["wt"], state["wt_scale"], state["xt"], state["xt_scale"], dtype=DTYPES[case["y"]], dropout=drop,
                        format=FORMATS[case["format"]])


def work(case):
    kind = case["kind"]
    if kind == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * SIZE[case["x"]] * (2 + (1 if case["residual"] else 0) + (2 if case["back"] else 0)), "flops": n * (2 if case["back"] else 1)}
    if kind == "quant":
        n = case["rows"] * case["cols"]
        return {"bytes": n * SIZE[case["x"]] + 2 * (n + n // 128), "flops": 2 * n}
    m, k, n = case["rows"], case["cin"], case["cout"]
    f8 = lambda a, b: a * b + a * b // 128  # noqa: E731
    if kind == "bwd":
        return {"bytes": m * n * SIZE[case["x"]] + f8(n, k) + f8(m, k) + m * k * SIZE[case["y"]] + 4 * n * k + 4 * n, "flops": 4 * m * n * k}
    out = m * n * SIZE[case["y"]] + f8(n, k) + (4 * n if case["bias"] else 0)
    if kind == "fwd":
        return {"bytes": out + m * k * SIZE[case["x"]] + (f8(m, k) if case["train"] else 0), "flops": 2 * m * n * k}
    return {"bytes": out + f8(m, k), "flops": 2 * m * n * k}


# ------------------------------------------------ the definitions in 64 bits
def _two(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_numbers(x, fmt):
    """The 8-bit numbers that stand for x (double; along rows) and their exponents, from the grid of the format."""
    m, k = x.shape
    digits, lowest, largest = (3, -6, 448.0) if fmt == "e4m3" else (2, -14, 57344.0)
    pad = torch.nn.functional.pad(x, (0, -k % 128)).reshape(m, -1, 128)
    a = pad.abs().amax(2, keepdim=True).clamp(min=2.0 ** -100)
    e = torch.floor(torch.log2(a / largest)) - 1
    for _ in range(2):
        e = torch.where(largest * _two(e) < a, e + 1, e)
    v = pad / _two(e)
    size = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -40)))
    size = torch.where(_two(size) > v.abs(), size - 1, size).clamp(min=lowest)
    step = _two(size - digits)
    return (torch.round(v / step) * step).reshape(m, -1), e[:, :, 0]


def _exact_scaled(x, fmt):
    q, e = _exact_numbers(x, fmt)
    return (q.reshape(e.shape + (128,)) * _two(e)[:, :, None]).reshape(q.shape)


def _exact_value(q, scale):
    """What a quantized matrix stands for."""
    m, k = q.shape
    e = torch.cat(list(scale), 1)[:, :k // 128].double() - 127
    return (q.double().reshape(m, -1, 128) * _two(e)[:, :, None]).reshape(m, k)


def _exact_kept(rows, cols, p, seed):
    b = np.arange(rows * -(-cols // 8), dtype=np.uint64)
    low, up = np.uint64(0xffffffff), np.uint64(32)
    c = [b & low, (b >> up) | np.uint64(1 << 31), np.zeros_like(b), np.zeros_like(b)]
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for i in range(10):
        even, odd = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        k = [np.uint64((key[0] + i * 0x9E3779B9) % 2 ** 32), np.uint64((key[1] + i * 0xBB67AE85) % 2 ** 32)]
        c = [(odd >> up) ^ c[1] ^ k[0], odd & low, (even >> up) ^ c[3] ^ k[1], even & low]
    words = np.stack([w.astype(np.uint32) for w in c], 1)
    r = words.astype("<u4").view("<u2").reshape(rows, -1)[:, :cols]
    return torch.from_numpy(r >= np.rint(p * 65536)).cuda()


def _exact_dropped(x, p, seed):
    return x.double() * (65536.0 / (65536.0 - _threshold(p))) * _exact_kept(x.shape[0], x.shape[1], p, seed)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "dropout":
        y = _exact_dropped(s["x"], case["p"], s["seed"])
        y = y if s["residual"] is None else y + s["residual"].double()
        return (y, _exact_dropped(s["dy"], case["p"], s["seed"])) if case["back"] else y
    if kind == "quant":
        x = s["x"].double()
        return _exact_numbers(x, case["format"])[0], None, _exact_numbers(x.T.contiguous(), case["format"])[0], None
    if kind == "matmul":
        y = _exact_value(s["a"], s["a_scale"]) @ _exact_value(s["w"], s["w_scale"]).T
        return y if s["bias"] is None else y + s["bias"].double()
    if kind == "fwd":
        x = s["x"].double()
        if case["p"]:  # (what is quantized is a number in 32 bits, times the 32-bit factor)
            factor = torch.tensor(65536.0 / (65536.0 - _threshold(case["p"])), device="cuda")
            x = (s["x"].float() * factor).double() * _exact_kept(case["rows"], case["cin"], case["p"], s["seed"])
        y = _exact_scaled(x, "e4m3") @ _exact_value(s["w"], s["w_scale"]).T
        y = y if s["bias"] is None else y + s["bias"].double()
        return (y, _exact_numbers(x.T.contiguous(), "e4m3")[0], None) if case["train"] else y
    dy = s["dy"].double()
    dx = _exact_scaled(dy, case["format"]) @ _exact_value(s["wt"], s["wt_scale"]).T
    if case["p"]:
        dx = _exact_dropped(dx, case["p"], s["seed"])
    dw = _exact_scaled(dy.T.contiguous(), case["format"]) @ _exact_value(s["xt"], s["xt_scale"]).T
    return dx, dw, dy.sum(0)

"""Plain 64-bit forms of the operators that distil a classifier from a quantized teacher's largest logits, from their definitions
(include/rn50_hip.h: quant_rows_i8, matmul_i8, topk_rows, distill_fwd_bwd)."""
import numpy as np


def row_bytes(K):
    return (K + 63) // 64 * 64


def quant_rows(x):
    """q [M, row_bytes(K)] int8 and scale [M] float; the definition's roundings to float included."""
    x = np.asarray(x, np.float32)
    M, K = x.shape
    a = np.maximum(np.abs(x).max(1), np.float32(2.0 ** -100))
    finite = np.isfinite(x).all(1)
    with np.errstate(all="ignore"):
        inv = np.where(finite, np.float32(127) / a, np.float32(0)).astype(np.float32)
        scale = np.where(finite, a / np.float32(127), np.float32(np.nan)).astype(np.float32)
        t = (np.where(finite[:, None], x, 0) * inv[:, None]).astype(np.float32)
    q = np.zeros((M, row_bytes(K)), np.int8)
    q[:, :K] = np.rint(t).astype(np.int8)
    return q, scale


def matmul_i8(q, q_scale, w, w_scale, bias=None):
    """(y in 64 bits, the magnitude its roundings go by)."""
    acc = q.astype(np.float64) @ w.astype(np.float64).T  # (sums below 2^31: exact)
    y = acc * np.asarray(q_scale, np.float64)[:, None] * np.asarray(w_scale, np.float64)[None, :]
    size = np.abs(y)
    if bias is not None:
        y, size = y + bias, size + np.abs(bias)
    return y, size


def lse(u, axis=1):
    """log(sum(exp(u))) along an axis, -inf where there is nothing else, +inf where one is (and none is NaN)."""
    with np.errstate(all="ignore"):
        m = u.max(axis, keepdims=True) if u.shape[axis] else np.full([1 if i == axis % u.ndim else s for i, s in enumerate(u.shape)], -np.inf)
        m = np.where(np.isinf(m), 0.0, m)
        return np.squeeze(np.log(np.exp(u - m).sum(axis, keepdims=True)) + m, axis)


def topk_rows(x, k, temperature):
    """values, indices, tail log-sum-exp.  NaN first, then descending; equal logits by class; (-inf, -1) past the last."""
    x = np.asarray(x, np.float64)
    N, C = x.shape
    values, indices, tail = np.full((N, k), -np.inf), np.full((N, k), -1, np.int32), np.empty(N)
    for n in range(N):
        rank = np.where(np.isnan(x[n]), np.inf, x[n])
        order = np.lexsort((np.arange(C), -rank, ~np.isnan(x[n])))
        got = order[:k]
        values[n, :len(got)], indices[n, :len(got)] = x[n, got], got
        rest = np.delete(x[n], got)
        tail[n] = lse(rest[None] / temperature)[0] if rest.size else -np.inf
    return values, indices, tail


def distill(z, t_values, t_indices, t_tail=None, labels=None, temperature=1.0, alpha=1.0, label_smoothing=0.0, row_weight=None, grad_scale=1.0):
    """loss, row_loss [N], dlogits [N, C] and, per element of dlogits, the size of the terms that it is the sum of."""
    z = np.asarray(z, np.float64)
    N, C = z.shape
    T, ls = float(temperature), float(label_smoothing)
    w = np.full(N, 1.0 / N) if row_weight is None else np.asarray(row_weight, np.float64)
    rows, grad, size = np.zeros(N), np.zeros((N, C)), np.zeros((N, C))
    for n in range(N):
        if w[n] == 0 or (z[n] == -np.inf).all():
            continue
        with np.errstate(all="ignore"):
            entries = {}
            for j in range(0 if t_values is None else t_values.shape[1]):
                c = int(t_indices[n, j])
                if 0 <= c < C and c not in entries:
                    entries[c] = float(t_values[n, j]) / T
            zn = z[n] - z[n].max()  # (nothing depends on a shift of the row; what follows must not lose the classes beside a large one)
            u = zn / T
            tau = -np.inf if t_tail is None else float(t_tail[n])
            if alpha > 0:
                at = np.array(list(entries), np.int64)
                cells = np.array(list(entries.values()) + [tau])
                rest = np.ones(C, bool)
                rest[at] = False
                if not (cells == -np.inf).all():
                    Z, lam = lse(u[None])[0], lse(u[rest][None])[0] if rest.any() else -np.inf
                    cells = cells - cells.max()
                    logp = cells - lse(cells[None])[0]
                    p = np.exp(logp)
                    logq = np.append(u[at], lam) - Z
                    rows[n] += alpha * T * T * np.where(p == 0, 0.0, p * (logp - logq)).sum()
                    q, pr, qr = np.exp(u - Z), p[-1], np.exp(lam - Z)
                    share = np.zeros(C)  # exp(u - lam), about the rest's own largest: beside a large one lam loses the logarithm of how many there are
                    if rest.any() and u[rest].max() != -np.inf:
                        share[rest] = np.exp(u[rest] - u[rest].max())
                        share /= share.sum()
                    d = np.where(rest, share * (qr - pr), q)
                    d[at] -= p[:-1]
                    s = np.where(rest, share * (qr + pr), q)
                    s[at] += p[:-1]
                    grad[n] += alpha * T * d
                    size[n] += alpha * T * s
            if alpha < 1 and labels is not None and 0 <= labels[n] < C:
                logs = zn - lse(zn[None])[0]
                y = np.full(C, ls / C)
                y[labels[n]] += 1 - ls
                rows[n] += (1 - alpha) * -np.where(y == 0, 0.0, y * logs).sum()
                grad[n] += (1 - alpha) * (np.exp(logs) - y)
                size[n] += (1 - alpha) * (np.exp(logs) + y)
            grad[n] *= grad_scale * w[n]
            size[n] *= abs(grad_scale * w[n])
    with np.errstate(all="ignore"):
        loss = float(np.sum(np.where(w == 0, 0.0, w * rows)))
    return loss, rows, grad, size

"""The 64-bit forms of quantized products, largest logits and the distillation loss, pinned by closed forms, brute force, central
differences and the cross-entropy oracle (no GPU)."""
import numpy as np
import pytest

import oracle as orc
from oracle import distill as od

RNG = np.random.default_rng(7)


def _case(N=5, C=23, k=6, tail=True, seed=0):
    r = np.random.default_rng(seed)
    t = r.normal(size=(N, C)) * 2
    return r.normal(size=(N, C)) * 2, t, *od.topk_rows(t, k, 1.7)


def test_quantized_rows_stay_within_half_a_step_and_rows_of_zeros_are_zeros():
    x = RNG.normal(size=(6, 71)).astype(np.float32)
    x[2] = 0
    x[3] *= 1e-38
    q, s = od.quant_rows(x)
    assert q.shape == (6, 128) and not q[:, 71:].any() and not q[2].any()
    assert (np.abs(q[:, :71] * s[:, None].astype(np.float64) - x) <= s[:, None] * (0.5 + 1e-4)).all()
    assert (np.abs(q[[0, 1, 4, 5]]).max(1) == 127).all()
    x[1, 5] = np.nan
    x[4, 0] = np.inf
    q, s = od.quant_rows(x)
    assert np.isnan(s[[1, 4]]).all() and not q[[1, 4]].any() and np.isfinite(s[[0, 2, 3, 5]]).all()


def test_product_of_quantized_rows_is_near_the_product():
    x, w = RNG.normal(size=(4, 300)).astype(np.float32), RNG.normal(size=(7, 300)).astype(np.float32)
    y, _ = od.matmul_i8(*od.quant_rows(x), *od.quant_rows(w))
    assert np.abs(y - x.astype(np.float64) @ w.T).max() < 0.03 * np.sqrt(300)


def test_largest_logits_against_brute_force():
    x = np.round(RNG.normal(size=(8, 40)) * 2) / 2  # many ties
    x[1, 3] = np.nan
    x[2] = -np.inf
    x[3, :38] = -np.inf
    v, i, tail = od.topk_rows(x, 9, 2.0)
    for n in range(8):
        left = list(range(40))
        for j in range(9):
            best = max(left, key=lambda c: (np.isnan(x[n, c]), x[n, c] if not np.isnan(x[n, c]) else 0, -c))
            assert i[n, j] == best
            left.remove(best)
        with np.errstate(divide="ignore"):
            np.testing.assert_allclose(tail[n], np.log(np.exp(x[n, left] / 2.0).sum()), rtol=1e-12)
    v, i, tail = od.topk_rows(x[:, :3], 5, 1.0)
    assert (i[:, 3:] == -1).all() and np.isneginf(v[:, 3:]).all() and np.isneginf(tail).all()


def test_without_entries_it_is_the_cross_entropy():
    z, labels = RNG.normal(size=(6, 11)).astype(np.float32), np.arange(6, dtype=np.int32)
    want = orc.xent_fwd_bwd(z, labels, 0.1)
    loss, rows, grad, _ = od.distill(z, None, None, labels=labels, alpha=0.0, label_smoothing=0.1)
    for got, w in ((loss, want[0]), (rows, want[1]), (grad, want[2])):
        np.testing.assert_allclose(got, w, rtol=2e-6, atol=1e-7)


def test_all_classes_as_entries_is_the_divergence_of_the_two_softmaxes():
    z, t, *_ = _case()
    T = 3.0
    v, i, tail = od.topk_rows(t, 23, T)
    for tl in (None, tail):
        loss, rows, grad, _ = od.distill(z, v, i, tl, temperature=T)
        p = np.exp(t / T - od.lse(t / T)[:, None])
        q = np.exp(z / T - od.lse(z / T)[:, None])
        np.testing.assert_allclose(rows, T * T * (p * np.log(p / q)).sum(1), rtol=1e-10)
        np.testing.assert_allclose(grad, T * (q - p) / 5, atol=1e-12)
    assert np.abs(od.distill(t, v, i, temperature=T)[1]).max() < 1e-12


def test_the_tail_is_one_cell():
    """Merging classes into a cell: the divergence of the merged distributions, at most the whole one."""
    z, t, v, i, tail = _case(k=4)
    T = 1.7
    _, rows, _, _ = od.distill(z, v, i, tail, temperature=T)
    p, q = np.exp(t / T - od.lse(t / T)[:, None]), np.exp(z / T - od.lse(z / T)[:, None])
    for n in range(5):
        top = i[n]
        P, Q = np.append(p[n, top], np.delete(p[n], top).sum()), np.append(q[n, top], np.delete(q[n], top).sum())
        np.testing.assert_allclose(rows[n], T * T * (P * np.log(P / Q)).sum(), rtol=1e-10)
        assert rows[n] <= T * T * (p[n] * np.log(p[n] / q[n])).sum()


@pytest.mark.parametrize("tail, alpha, ls, T", [(True, 1.0, 0.0, 1.0), (True, 0.6, 0.1, 2.5), (False, 1.0, 0.0, 4.0), (False, 0.3, 0.2, 0.7),
                                                (True, 0.0, 0.1, 2.0)])
def test_gradient_against_central_differences(tail, alpha, ls, T):
    z, t, v, i, tl = _case(N=3, C=9, k=3)
    i = i.copy()
    i[1, 1] = -1            # an absent entry
    i[2, 2] = i[2, 0]       # one that appears again
    w = np.array([0.5, 1.25, 0.25])
    labels = np.array([i[0, 0], 8, -3])
    f = lambda zz: od.distill(zz, v, i, tl if tail else None, labels, T, alpha, ls, w, 1.0)
    _, _, grad, size = f(z)
    assert (np.abs(grad) <= size + 1e-15).all()
    h = 1e-5
    for n in range(3):
        for c in range(9):
            zp, zm = z.copy(), z.copy()
            zp[n, c] += h
            zm[n, c] -= h
            assert abs((f(zp)[0] - f(zm)[0]) / (2 * h) - grad[n, c]) < 1e-8


def test_rows_that_have_nothing():
    z, t, v, i, tail = _case(N=4, C=9, k=3)
    z[0] = -np.inf
    i[1] = -1
    w = np.array([0.25, 0.25, 0.0, 0.25])
    z[2] = np.nan
    loss, rows, grad, _ = od.distill(z, v, i, None, row_weight=w)
    assert rows[0] == rows[1] == rows[2] == 0 and not grad[:3].any() and rows[3] > 0 and np.isfinite(loss)
    # a teacher that is sure of a class the student rules out
    z[3, i[3, 0]] = -np.inf
    assert np.isposinf(od.distill(z, v, i, None, row_weight=w)[0])


def test_the_rest_of_a_row_with_more_infinities_than_places():
    x = np.random.default_rng(3).normal(size=(4, 9))
    x[0, [1, 4, 6]] = np.inf             # one is left
    x[1, [1, 4]] = np.inf                # none is
    x[2, [1, 4, 6]], x[2, 8] = np.inf, np.nan  # a NaN takes a place
    x[3, [0, 1, 2]], x[3, 5] = np.nan, np.inf  # and here one is left
    v, i, tail = od.topk_rows(x, 2, 2.0)
    assert i.tolist() == [[1, 4], [1, 4], [8, 1], [0, 1]]
    assert np.isposinf(tail[0]) and np.isfinite(tail[1]) and np.isposinf(tail[2]) and np.isnan(tail[3])
    np.testing.assert_allclose(tail[1], np.log(np.exp(np.delete(x[1], [1, 4]) / 2).sum()), rtol=1e-12)


def test_a_rest_of_equal_logits_far_below_shares_the_tail():
    low = float(np.finfo(np.float32).min)
    z = np.full((2, 9), low)
    z[0, 3], z[1, [2, 5]] = 1.0, 2.0
    i, v, tail = np.array([[3, -1], [2, 5]]), np.ones((2, 2)), np.array([0.5, 0.25])
    _, _, grad, _ = od.distill(z, v, i, tail, row_weight=np.ones(2))
    for n, (inside, others) in enumerate((([3], 8), ([2, 5], 7))):
        pr = np.exp(tail[n]) / (np.exp(tail[n]) + len(inside) * np.e)
        np.testing.assert_allclose(np.delete(grad[n], inside), -pr / others, rtol=1e-12)
        np.testing.assert_allclose(grad[n].sum(), 0, atol=1e-12)

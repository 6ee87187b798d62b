"""Quantized rows and products, largest logits, and the distillation loss with its gradient, against their 64-bit forms.

Where the bounds come from (eps = 2^-24, half a unit in the last place of a float):
 - quantized rows: the definition's roundings are part of it: bit for bit;
 - products: the sum is exact, then one rounding of the sum to float, two products and an addition: 5 eps of the terms' size; one
   more rounding (2^-8 of the result) in bfloat16;
 - sums of exponentials: every term's argument has three roundings, each eps of the argument's own size, on average at most ln C of
   it (the mean of max - u under the softmax is at most its entropy); the exponential itself 2 eps; an addition or a rescaling of
   the running sum 4 eps, and no kernel adds more than C / 64 + 64 terms one after another: `sum_error`;
 - log-sum-exp: that, and one rounding of the result;  losses: four log-probabilities, weighted by at most one each;
 - gradients: sum_error, and the element's own exponentials, whose arguments have three roundings: of the size of its terms;
   one more rounding in bfloat16."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import distill as od

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def rn():
    import paper_1903_12650_amd as rn
    return rn


def sum_error(C):
    return EPS * (4 * (C / 64 + 64) + 5 * np.log(C + 1) + 16)


def spread(t, extra):
    """The same matrix with rows `extra` elements further apart."""
    wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan") if t.is_floating_point() else -7, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def f64(t):
    return t.detach().double().cpu().numpy()


# ----------------------------------------------------------- quantized rows
QUANT = [(1, 1), (1, 2048), (3, 7), (5, 64), (40, 2048), (2, 65), (300, 255), (9, 1000), (7, 8192), (4, 8200), (2, 20011), (1, 131071), (2049, 130)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M, K", QUANT)
def test_quantized_rows(rn, M, K, dtype):
    g = torch.Generator().manual_seed(M * 131 + K)
    x = (torch.randn(M, K, generator=g) * torch.exp(2 * torch.randn(M, 1, generator=g))).to(dtype)
    if M > 2:
        x[1] = 0
    for src in (x.cuda(), spread(x.cuda(), 1), spread(x.cuda(), 8)):
        q, s = rn.quant_rows_i8(src)
        want_q, want_s = od.quant_rows(x.float().numpy())
        assert q.shape == (M, rn.quant_i8_row_bytes(K))
        assert np.array_equal(s.cpu().numpy(), want_s) and np.array_equal(q.cpu().numpy(), want_q)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_quantized_rows_of_extreme_values(rn, dtype):
    big = torch.finfo(dtype).max
    tiny = 1e-40 if dtype == F32 else 2.0 ** -133
    x = torch.randn(12, 517)
    x[0, 516] = float("inf")
    x[1, 0] = float("-inf")
    x[2, 300] = float("nan")
    x[3] = torch.sign(x[3]) * big
    x[4] *= tiny
    x[5] = 0
    x[5, 100] = -big
    x[6] = -0.0
    x[7, 511] = 2.0 ** -101
    x[7, :511] = 0
    x[7, 512:] = 0
    x = x.to(dtype)
    q, s = rn.quant_rows_i8(x.cuda())
    want_q, want_s = od.quant_rows(x.float().numpy())
    np.testing.assert_array_equal(s.cpu().numpy(), want_s)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)
    assert np.isnan(want_s[:3]).all() and np.isfinite(want_s[3:]).all()
    w = torch.randn(33, 517).cuda()
    y = rn.fc_i8_fwd(x.cuda(), *rn.quant_rows_i8(w))  # the rows with such values are NaN, whole; no other is (3 and 5 may pass the largest float)
    assert torch.isnan(y[:3]).all() and not torch.isnan(y[3:]).any() and torch.isfinite(y[4]).all() and torch.isfinite(y[6:]).all()


# ----------------------------------------------------------------- products
PRODUCTS = [(1, 1, 1), (1, 1000, 2048), (1, 17, 64), (2, 33, 100), (3, 5, 4099), (7, 256, 512), (16, 129, 1000), (17, 1000, 2048), (40, 1000, 2048),
            (33, 96, 640), (64, 64, 64), (65, 130, 128), (127, 255, 192), (129, 257, 320), (256, 256, 256), (257, 300, 65), (300, 513, 1025),
            (515, 258, 2047), (1001, 777, 448), (20, 8193, 130), (64, 8200, 320), (49, 8192, 1000),
            (4, 300, 4096), (5, 300, 4096), (2, 77, 8192), (3, 77, 8192), (16, 40, 1024), (16, 40, 1025), (9, 70, 1777), (13, 33, 5)]


def product_bound(size, want, out):
    return 5 * EPS * size + (2.0 ** -8 * 1.01 * np.abs(want) if out == BF16 else 0) + 1e-44


@pytest.mark.parametrize("x_type, y_type, bias", [(BF16, F32, True), (F32, F32, False), (BF16, BF16, True), (F32, BF16, False)])
@pytest.mark.parametrize("M, N, K", PRODUCTS)
def test_products(rn, M, N, K, x_type, y_type, bias):
    g = torch.Generator().manual_seed(M + 1000 * N + K)
    x = (torch.randn(M, K, generator=g) * torch.exp(torch.randn(M, 1, generator=g))).to(x_type)
    w = torch.randn(N, K, generator=g)
    b = torch.randn(N, generator=g).cuda() if bias else None
    wq, ws = rn.quant_rows_i8(w.cuda())
    want, size = od.matmul_i8(*od.quant_rows(x.float().numpy()), wq.cpu().numpy(), ws.cpu().numpy(), None if b is None else f64(b))
    bound = product_bound(size, want, y_type)
    y = rn.fc_i8_fwd(x.cuda(), wq, ws, b, dtype=y_type)
    assert y.dtype == y_type and y.shape == (M, N)
    assert (np.abs(f64(y) - want) <= bound).all()
    # in two calls, and into rows that lie further apart, whose gaps stay as they are: the same
    q, s = rn.quant_rows_i8(spread(x.cuda(), 3))
    assert torch.equal(rn.matmul_i8(K, q, s, wq, ws, b, y_type), y)
    for extra in (1, 8):
        wide = torch.full((M, N + extra), 5.0, dtype=y_type, device="cuda")
        rn.fc_i8_fwd(spread(x.cuda(), extra), wq, ws, b, y=wide[:, :N])
        assert torch.equal(wide[:, :N], y) and bool((wide[:, N:] == 5.0).all())


@pytest.mark.parametrize("x_type, y_type, bias", [(BF16, F32, True), (F32, BF16, False)])
@pytest.mark.parametrize("M, N, K", [(2900, 3900, 70), (2817, 3841, 641), (4097, 4100, 130), (1500, 3900, 193), (1409, 3844, 1000), (1000, 2100, 193)])
def test_products_of_many_tiles(rn, M, N, K, x_type, y_type, bias):
    test_products(rn, M, N, K, x_type, y_type, bias)


@pytest.mark.parametrize("M, N", [(1, 3), (5, 70), (70, 5), (200, 130)])
def test_longest_sums_do_not_overflow(rn, M, N):
    K = 131071
    q = torch.full((M, rn.quant_i8_row_bytes(K)), -128, dtype=torch.int8, device="cuda")
    q[:, K:] = 0
    w = torch.full((N, q.shape[1]), -128, dtype=torch.int8, device="cuda")
    w[:, K:] = 0
    w[N - 1] = 127
    one = lambda n: torch.ones(n, device="cuda")
    y = rn.matmul_i8(K, q, one(M), w, one(N))
    want = np.full((M, N), np.float32(128 * 128 * K), np.float32)
    want[:, N - 1] = np.float32(-128 * 127 * K)
    assert np.array_equal(y.cpu().numpy(), want)
    with pytest.raises(rn.Rn50Error) as e:
        rn.quant_rows_i8(torch.zeros(1, K + 1, device="cuda"))
    assert e.value.code == -2


def test_nan_scales_stay_in_their_rows_and_columns(rn):
    x, w = torch.randn(130, 200), torch.randn(140, 200)
    x[77, 3] = float("nan")
    w[101, 5] = float("inf")
    y = rn.fc_i8_fwd(x.cuda(), *rn.quant_rows_i8(w.cuda()))
    bad = torch.zeros(130, 140, dtype=torch.bool)
    bad[77], bad[:, 101] = True, True
    assert torch.equal(torch.isnan(y).cpu(), bad)


# ----------------------------------------------------------- largest logits
def check_topk(rn, x, k, temperature, tail=True):
    values, indices, t = rn.topk_rows(x, k, temperature, tail)
    wv, wi, wt = od.topk_rows(f64(x), k, temperature)
    assert values.dtype == F32 and indices.dtype == torch.int32 and values.shape == indices.shape == (x.shape[0], k)
    np.testing.assert_array_equal(indices.cpu().numpy(), wi)
    np.testing.assert_array_equal(values.cpu().numpy(), wv.astype(np.float32))
    if not tail:
        assert t is None
        return
    t = f64(t)
    same = np.isnan(wt) == np.isnan(t)
    assert same.all() and (np.isinf(wt) == np.isinf(t)).all() and (t[np.isinf(wt)] == wt[np.isinf(wt)]).all()
    fine = np.isfinite(wt)
    assert (np.abs(t[fine] - wt[fine]) <= sum_error(x.shape[1]) + 2 * EPS * np.abs(wt[fine])).all()


TOPK = [(1, 1, 1), (3, 5, 8), (40, 1000, 8), (2, 256, 256), (5, 257, 256), (9, 255, 1), (4, 1024, 100), (33, 4096, 32), (3, 8195, 64), (1, 50001, 100),
        (2, 65537, 17), (6, 40000, 256), (1, 131072, 64), (3, 300001, 128), (200, 2500, 10), (130, 33000, 50),
        (1, 81933, 256), (7, 98304, 1), (241, 80001, 30), (9, 306, 75), (5, 1025, 200), (3, 2500, 256), (3, 1024, 256)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N, C, k", TOPK)
def test_largest_logits(rn, N, C, k, dtype):
    g = torch.Generator().manual_seed(N * 7 + C + k)
    x = (torch.randn(N, C, generator=g) * 2).to(dtype).cuda()
    check_topk(rn, x, k, 2.0)
    check_topk(rn, spread(x, 1), k, 0.5)
    check_topk(rn, spread(x, 8), k, 1.0, tail=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("C, k", [(1000, 7), (1000, 256), (2100, 256), (5000, 64), (70000, 100), (70000, 256), (100003, 100), (100003, 256)])
def test_largest_logits_of_awkward_rows(rn, C, k, dtype):
    g = torch.Generator().manual_seed(C + k)
    low = torch.finfo(dtype).min
    x = torch.randn(16, C, generator=g)
    x[0] = float("-inf")                                   # nothing is left
    x[1] = float("-inf")
    x[1, C - 3] = 1.0                                      # one class is left
    x[2] = low
    x[2, ::C // 5] = 2.0
    x[3] = 0.25                                            # all equal
    x[4] = torch.round(x[4])                               # a handful of values
    x[5] = torch.arange(C) / C                             # ascending
    x[6] = -torch.arange(C) / C
    x[7, 5] = float("nan")
    x[7, C - 1] = float("nan")
    x[8, 11] = float("inf")
    x[9, C // 2:C // 2 + k] += 50                          # all in one place
    x[10, ::2], x[10, 1::2] = 0.0, -0.0
    x[11] = float("nan")
    x[12, :k + 40] = 9.0                                   # more ties at the top than places
    x[13, 64:] = float("-inf")
    x[14] = x[14] * 1e-38
    x[15] = x[15].sign() * torch.finfo(dtype).max
    check_topk(rn, x.to(dtype).cuda(), k, 1.0)
    one = x.to(dtype).cuda()
    for n in (0, 3, 9, 12):
        check_topk(rn, one[n:n + 1], k, 1.0)               # the forms for few rows


# ------------------------------------------------------- distillation loss
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("C, k", [(4001, 64), (9000, 256), (50001, 100), (50001, 256), (131072, 256)])
def test_largest_logits_that_lie_side_by_side(rn, C, k, dtype):
    """Rows in the order of their classes' frequency: the vectors that hold the largest logits hold more than are kept as candidates."""
    g = torch.Generator().manual_seed(C * 3 + k)
    x = torch.randn(14, C, generator=g)
    rank = torch.log(torch.arange(1, C + 1).float())
    x[0] = x[0].sort(descending=True)[0]
    x[1] = x[1].sort()[0]
    x[2] = x[2] - rank                                     # the largest on both sides of zero
    x[3] = x[3] * 0.01 - rank * 0.1
    x[4] = x[4] * 2 - rank * 2 + 9
    x[5, 300:1400] = 5 + x[5, 300:1400] * 1e-3             # a hair apart
    x[6, 300:1400] = 5 + torch.round(x[6, 300:1400] * 8) / 64  # and equal
    x[7, 300:1400], x[7, 310] = 7.0, 1e30
    x[8, C - 1200:] = -1e-3 * x[8, C - 1200:].abs() + 6
    x[9] = torch.where(torch.arange(C) < 1500, x[9].abs() * 1e-20, float("-inf"))
    x[10] = torch.where(torch.arange(C) < 1500, x[10] * 1e-20, -1.0)
    x[11, 100:1200] = torch.linspace(-4, 40, 1100)
    x[11, 1200:] = -5
    x[12] = -3 - x[12].abs()
    x[12, 64:1200] = torch.linspace(1e-9, 1e-6, 1136)
    x[13] = torch.arange(C, 0, -1) * 1e30
    check_topk(rn, x.to(dtype).cuda(), k, 1.0)
    check_topk(rn, spread(x[:6].to(dtype).cuda(), 3), k, 3.0)
    for n in (0, 2, 7):
        check_topk(rn, x[n:n + 1].to(dtype).cuda(), k, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("C, k", [(300, 3), (1001, 8), (4000, 256), (50001, 7), (131072, 64)])
@pytest.mark.parametrize("temperature", [0.03, 1.0])
def test_rests_far_below_the_largest_logits(rn, C, k, dtype, temperature):
    g = torch.Generator().manual_seed(C + 5 * k)
    x = torch.randn(12, C, generator=g)
    for n, gap in enumerate((40, 90, 120, 1000, 1e30)):
        x[n, torch.randperm(C, generator=g)[:k]] += gap    # as many as are taken
        x[5 + n, torch.randperm(C, generator=g)[:max(1, k // 2)]] += gap
    x[10, ::2], x[10, 7] = float("-inf"), 500.0
    x[11, 3:] = float("-inf")                              # a few, or as many as are taken, and nothing else
    check_topk(rn, x.to(dtype).cuda(), k, temperature)
    for n in (1, 3, 10):
        check_topk(rn, x[n:n + 1].to(dtype).cuda(), k, temperature)


def teacher(rn, N, C, k, T, seed, tail=True, absent=False):
    g = torch.Generator().manual_seed(seed)
    t = torch.randn(N, C, generator=g) * 3
    v, i, tl = od.topk_rows(t.numpy(), k, T)
    if absent:
        i = np.where(np.arange(k)[None] >= 1 + np.arange(N)[:, None] % k, -1, i)
    z = 0.7 * t + torch.randn(N, C, generator=g)
    labels = torch.randint(0, C, (N,), generator=g).to(torch.int32)
    f = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(F32).cuda()
    return z, f(v), torch.from_numpy(i).to(torch.int32).cuda(), f(tl) if tail else None, labels.cuda()


def check_distill(rn, z, v, i, tl, labels, T=1.0, alpha=1.0, ls=0.0, w=None, scale=1.0, **more):
    a = dict(temperature=T, alpha=alpha, label_smoothing=ls, row_weight=w, grad_scale=scale)
    keep = z.clone()
    loss, rows, grad = rn.distill_fwd_bwd(z, v, i, tl, labels, **a, **more)
    n64 = lambda t: None if t is None else f64(t)
    host = lambda t: None if t is None else t.cpu().numpy()
    a["row_weight"] = n64(w)
    want_loss, want_rows, want, size = od.distill(f64(keep), n64(v), host(i), n64(tl), host(labels), **a)
    N, C = z.shape
    e = sum_error(C)
    zz = f64(keep)
    finite = np.where(np.isfinite(zz), zz, 0)
    reach = np.abs(finite).max(1) + (np.abs(f64(v)).max(1, initial=0, where=np.isfinite(f64(v))) if v is not None else 0)
    row_bound = alpha * T * T * (4 * e + 8 * EPS * (reach / T + np.log(C + 1))) + (1 - alpha) * (4 * e + 8 * EPS * (reach + np.log(C + 1))) \
        + 2 * EPS * np.abs(np.where(np.isfinite(want_rows), want_rows, 0))
    got_rows = f64(rows)
    assert (np.isfinite(got_rows) == np.isfinite(want_rows)).all(), (got_rows, want_rows)
    ok = np.isfinite(want_rows)
    assert (np.abs(got_rows[ok] - want_rows[ok]) <= row_bound[ok]).all()
    ww = np.full(N, 1.0 / N) if w is None else f64(w)
    if ok.all():
        assert abs(float(loss) - want_loss) <= float((np.abs(ww) * row_bound).sum()) + 2 * EPS * abs(want_loss)
    if grad is None:
        return None
    # an element's exponentials: three roundings of (z - m) / T, of z - m
    away = np.abs(finite.max(1)[:, None] - finite) * max(1.0, 1.0 / T)
    bound = size * (2 * e + EPS * (5 * np.minimum(away, 90) + 16)) + 1e-36
    if z.dtype == BF16:
        bound += 2.0 ** -8 * 1.01 * (np.abs(want) + bound) + 1e-38
    got = f64(grad)
    assert grad.dtype == z.dtype and np.isfinite(got).all()
    off = np.abs(got - want) - bound
    assert (off <= 0).all(), (np.unravel_index(off.argmax(), off.shape), off.max(), got.flat[off.argmax()], want.flat[off.argmax()])
    return loss, rows, grad


SHAPES = [(1, 1, 1), (2, 3, 2), (40, 1000, 8), (5, 257, 256), (3, 1023, 33), (6, 4100, 64), (1, 50001, 100), (2, 70000, 16), (7, 131072, 32), (64, 8192, 50),
          (300, 515, 5), (3, 200003, 20)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail, alpha, ls, T, absent", [(True, 0.5, 0.1, 4.0, False), (False, 1.0, 0.0, 1.0, True), (True, 0.7, 0.0, 2.0, True),
                                                       (True, 1.0, 0.0, 0.5, False), (True, 0.0, 0.1, 1.0, False)])
@pytest.mark.parametrize("N, C, k", SHAPES)
def test_distillation(rn, N, C, k, dtype, tail, alpha, ls, T, absent):
    z, v, i, tl, labels = teacher(rn, N, C, k, T, N + C + k, tail, absent)
    z = z.to(dtype).cuda()
    w = torch.linspace(0.5, 1.5, N).cuda() / N
    if N > 2:
        w[1] = 0
    loss, rows, grad = check_distill(rn, z, v, i, tl, labels, T, alpha, ls, w, 3.0)
    # the loss alone; rows that lie apart; in place
    only = rn.distill_fwd_bwd(z, v, i, tl, labels, T, alpha, ls, w, 3.0, grad=False)
    assert only[2] is None and torch.equal(only[0], loss) and torch.equal(only[1], rows)
    for extra in (1, 8):
        zz = spread(z, extra)
        out = torch.full((N, C + 2 * extra), 5.0, dtype=dtype, device="cuda")
        l2, r2, _ = check_distill(rn, zz, v, i, tl, labels, T, alpha, ls, w, 3.0, dlogits=out[:, :C])
        assert bool((out[:, C:] == 5.0).all())
        if extra == 8:  # (the rows' 16-byte boundaries lie as before: the same sums)
            assert torch.equal(l2, loss) and torch.equal(r2, rows) and torch.equal(out[:, :C], grad)
        l3, r3, _ = rn.distill_fwd_bwd(zz, v, i, tl, labels, T, alpha, ls, w, 3.0, dlogits=zz)
        assert torch.equal(l3, l2) and torch.equal(r3, r2) and torch.equal(zz, out[:, :C])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_without_a_teacher_it_is_the_cross_entropy(rn, dtype):
    z = torch.randn(40, 1000).to(dtype).cuda()
    labels = torch.randint(0, 1000, (40,), dtype=torch.int32).cuda()
    loss, rows, grad = check_distill(rn, z, None, None, None, labels, alpha=0.0, ls=0.1, scale=2.0)
    want = rn.xent_fwd_bwd(z.float(), labels, 0.1, 2.0)
    assert torch.allclose(loss, want[0], rtol=1e-5) and torch.allclose(rows, want[1], rtol=1e-5)
    assert float((grad.float() - want[2]).norm() / want[2].norm()) < (4e-3 if dtype == BF16 else 1e-5)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("C", [700, 60000])
def test_rows_where_something_is_missing(rn, C, dtype):
    N, k, T = 14, 6, 2.0
    low = torch.finfo(dtype).min
    z, v, i, tl, labels = teacher(rn, N, C, k, T, C)
    w = torch.full((N,), 1.0 / N)
    z[0] = float("-inf")                                  # no distribution
    i[1], tl[1] = -1, float("-inf")                       # no teacher
    i[2] = -1                                             # only the teacher's tail
    z[3], w[3] = float("nan"), 0.0                        # padding
    labels[4] = -100                                      # no label
    i[5, 3] = i[5, 0]                                     # an entry twice
    i[6, 2], i[6, 4] = C, 2 ** 31 - 1                     # classes that do not exist
    keep = torch.zeros(C, dtype=torch.bool)
    keep[i[7].cpu().long()] = True
    keep[labels[7].item()] = True
    keep[C // 2] = True
    z[7, ~keep] = float("-inf")                           # the student's mask leaves the entries, the label and one more
    z[8, ~keep] = low                                     # ... and the lowest value as a mask
    z[8, i[8].cpu().long()] = 1.0
    z[8, labels[8].item()] = 0.5
    z[9] = low                                            # all masked alike: a uniform distribution
    v[10] = float("-inf")                                 # entries of no mass: the tail alone
    tl[11] = float("-inf")
    z[12, C // 2:] = float("-inf")
    z[12, i[12].cpu().long()] = 3.0
    z[12, labels[12].item()] = 0.0
    z[13] *= 20                                           # far apart
    check_distill(rn, z.to(dtype).cuda(), v, i, tl, labels, T, 0.6, 0.0, w.cuda())
    for n in (0, 2, 5, 7, 9, 13):                         # the forms for few rows
        s = slice(n, n + 1)
        check_distill(rn, z[s].to(dtype).cuda(), v[s].contiguous(), i[s].contiguous(), tl[s].contiguous(), labels[s].contiguous(), T, 1.0)


@pytest.mark.parametrize("C", [700, 60000])
def test_losses_that_have_no_end(rn, C):
    """A class that the teacher holds possible and the student does not: infinite loss, a gradient without NaN; NaN and +infinity in a
    row make its loss NaN and leave the other rows alone."""
    z, v, i, tl, labels = teacher(rn, 4, C, 5, 1.0, 3)
    z[0, i[0, 2].item()] = float("-inf")
    z[1, C // 3] = float("nan")
    z[2, C // 3] = float("inf")
    loss, rows, grad = rn.distill_fwd_bwd(z.cuda(), v, i, tl)
    rows = rows.cpu()
    assert torch.isposinf(rows[0]) and torch.isnan(rows[1]) and torch.isnan(rows[2]) and torch.isfinite(rows[3])
    assert torch.isfinite(grad[0]).all() and torch.isfinite(grad[3]).all() and torch.isnan(grad[1]).any() and torch.isnan(grad[2]).any()
    _, _, want, _ = od.distill(f64(z), f64(v), i.cpu().numpy(), f64(tl))
    assert np.abs(f64(grad[0]) - want[0]).max() < 1e-5
    # every class of the student's tail is masked while the teacher's tail has mass
    z, v, i, tl, labels = teacher(rn, 2, C, 5, 1.0, 4)
    inside = torch.full((C,), float("-inf"))
    inside[i[0].cpu().long()] = 1.0
    z[0] = inside
    _, rows, grad = rn.distill_fwd_bwd(z.cuda(), v, i, tl)
    assert torch.isposinf(rows[0]) and torch.isfinite(rows[1]) and torch.isfinite(grad).all()


def test_gradient_against_differences_of_the_loss(rn):
    """In float, along directions: the loss of the row's own kernel, two-sided.  Bound: the third derivative's part (h^2) and the loss's
    rounding over 2h."""
    N, C, k, T = 4, 900, 12, 2.0
    z, v, i, tl, labels = teacher(rn, N, C, k, T, 5)
    z = z.cuda()
    a = dict(temperature=T, alpha=0.6, label_smoothing=0.1)
    _, rows, grad = rn.distill_fwd_bwd(z, v, i, tl, labels, **a)
    g = torch.Generator().manual_seed(9)
    h = 2.0 ** -6
    for _ in range(4):
        d = torch.randn(N, C, generator=g).cuda()
        d /= d.abs().max()
        up, down = (rn.distill_fwd_bwd(z + s * h * d, v, i, tl, labels, grad=False, **a)[1] for s in (1, -1))
        want = f64((up.double() - down.double()) / (2 * h))
        got = (f64(grad) * f64(d)).sum(1) * N
        noise = 8 * EPS * np.abs(f64(rows)).max() / h + sum_error(C) / h
        assert (np.abs(got - want) <= noise + h * h * 4).all()


# -------------------------------------------------------- how they are called
@pytest.mark.parametrize("N, ld, used", [(3, 2 ** 30, 5003), (40, 2 ** 26 + 8, 1000)])
def test_rows_past_32_bits(rn, N, ld, used):
    """The last rows start past 2^31 elements and 4 GB."""
    base = torch.empty(N * ld, dtype=BF16, device="cuda")
    x = base.view(N, ld)[:, :used]
    z, v, i, tl, labels = teacher(rn, N, used, 9, 1.0, 1)
    x.copy_(z.to(BF16))
    check_topk(rn, x, 9, 1.0)
    for got, want in zip(rn.quant_rows_i8(x), rn.quant_rows_i8(x.contiguous())):
        assert torch.equal(got, want)
    out = rn.distill_fwd_bwd(x, v, i, tl, labels, alpha=0.5)
    check_distill(rn, x, v, i, tl, labels, alpha=0.5, dlogits=x)
    assert torch.equal(x, out[2])
    w = rn.quant_rows_i8(torch.randn(used, 64, device="cuda"))
    a = torch.randn(N, 64, device="cuda")
    rn.fc_i8_fwd(a, *w, y=x)
    assert torch.equal(x, rn.fc_i8_fwd(a, *w, dtype=BF16))


def test_more_rows_than_one_line_of_the_grid(rn):
    N, C, k = 70001, 9, 3
    z = torch.randn(N, C, device="cuda")
    v, i, tl = rn.topk_rows(torch.randn(N, C, device="cuda"), k)
    w = torch.rand(N, device="cuda") / N
    loss, rows, grad = rn.distill_fwd_bwd(z, v, i, tl, row_weight=w)
    q, s = rn.quant_rows_i8(z)
    values, indices, tail = rn.topk_rows(z, k)
    total = 0.0
    for a, b in ((0, 30000), (30000, 65536), (65536, 65537), (65537, N)):
        part = rn.distill_fwd_bwd(z[a:b], v[a:b], i[a:b], tl[a:b], row_weight=w[a:b])
        assert torch.equal(part[1], rows[a:b]) and torch.equal(part[2], grad[a:b])
        total += float(part[0])
        assert all(torch.equal(x, y[a:b]) for x, y in zip((*rn.quant_rows_i8(z[a:b].contiguous()), *rn.topk_rows(z[a:b], k)), (q, s, values, indices, tail)))
    assert abs(total - float(loss)) < 1e-5 * total


def test_quantized_rows_past_one_line_of_the_grid(rn):
    x = torch.randn(4 * 65536 + 5, 9, device="cuda")
    q, s = rn.quant_rows_i8(x)
    for a, b in ((0, 200000), (200000, 262144), (262144, 262149)):
        assert all(torch.equal(u, v[a:b]) for u, v in zip(rn.quant_rows_i8(x[a:b]), (q, s)))


def test_one_long_row(rn):
    """More classes than 2^25, one row: the forms that share a row among workgroups."""
    C = 2 ** 25 + 37
    x = torch.randn(1, C, device="cuda")
    values, indices, tail = rn.topk_rows(x, 50, 1.0)
    want, at = torch.sort(x[0], descending=True, stable=True)
    assert torch.equal(values[0], want[:50]) and torch.equal(indices[0].long(), at[:50])
    rest = torch.logsumexp(want[50:].double(), 0)
    assert abs(float(tail) - float(rest)) < 1e-4
    loss, row, grad = rn.distill_fwd_bwd(x, values, indices, tail)  # its own teacher
    assert abs(float(loss)) < 1e-4 and float(grad.abs().max()) < 1e-5


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_start_anywhere(rn, dtype):
    z, v, i, tl, labels = teacher(rn, 9, 1001, 7, 2.0, 8)
    z = z.to(dtype).cuda()
    wide = spread(z, 5)
    for r, c in ((1, 0), (2, 1), (3, 2), (0, 3), (4, 4), (1, 7), (5, 997)):
        part = wide[r:, c:1001]
        whole = part.contiguous()
        check_topk(rn, part, 7, 2.0)
        check_topk(rn, whole, 7, 0.5)
        for got, want in zip(rn.quant_rows_i8(part), rn.quant_rows_i8(whole)):
            assert torch.equal(got, want)
        a = (v[r:], (i[r:] - c), tl[r:], labels[r:] - c, 2.0, 0.5, 0.1)  # (entries and labels in front of the part are absent)
        check_distill(rn, part, *a)
        out = torch.full((9, 1009), 5.0, dtype=dtype, device="cuda")
        check_distill(rn, part, *a, dlogits=out[:9 - r, 3:3 + 1001 - c])  # (its rows start elsewhere than the logits')
        assert bool((out[:, :3] == 5.0).all()) and bool((out[:, 3 + 1001 - c:] == 5.0).all()) and bool((out[9 - r:] == 5.0).all())
        w = rn.quant_rows_i8(torch.randn(1001 - c, 70, device="cuda"))
        x = torch.randn(9 - r, 70, device="cuda")
        out = torch.full_like(wide, 5.0)
        rn.fc_i8_fwd(x, *w, y=out[r:, c:1001])
        assert torch.equal(out[r:, c:1001], rn.fc_i8_fwd(x, *w, dtype=dtype))
        out[r:, c:1001] = 5.0
        assert bool((out == 5.0).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("C", [9000, 100003])
def test_long_rows_that_start_anywhere(rn, C, dtype):
    """Streamed rows and slices: entries and labels in front of the first vector, behind the last, and across chunks of classes."""
    g = torch.Generator().manual_seed(C)
    for start in (0, 1, 3, 5, 7):
        wide = torch.randn(3, C + 8, generator=g).mul(3).to(dtype).cuda()
        z = wide[:, start:start + C]
        i = torch.tensor([[0, 1, 2, C - 1, C - 2, C // 2], [C - 1, 65535 % C, 65536 % C, 3, 4, 5], [6, 7, 8, 9, 7, 0]], dtype=torch.int32, device="cuda")
        v = torch.randn(3, 6, generator=g).mul(2).cuda()
        labels = torch.tensor([C - 3, 0, 6], dtype=torch.int32, device="cuda")
        check_distill(rn, z, v, i, torch.tensor([1.0, -2.0, 0.5], device="cuda"), labels, 2.0, 0.5, 0.1)
        check_topk(rn, z, 40, 1.0)
        top = z.clone()
        wide[:, start] = 50.0       # the largest at both ends
        wide[:, start + C - 1] = 50.0
        check_topk(rn, z, 3, 1.0)
        z.copy_(top)


@pytest.mark.parametrize("N, C", [(3, 70000), (200, 3000)])
def test_on_another_stream_and_twice(rn, N, C):
    z, v, i, tl, labels = teacher(rn, N, C, 20, 2.0, 8)
    z = z.to(BF16).cuda()
    x, w = torch.randn(N, 520).cuda(), torch.randn(130, 520).cuda()

    def everything():
        wq, ws = rn.quant_rows_i8(w)
        return [*rn.topk_rows(z, 20, 2.0), *rn.distill_fwd_bwd(z, v, i, tl, labels, 2.0, 0.5, 0.1), wq, ws, rn.fc_i8_fwd(x, wq, ws)]

    want = everything()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = everything()
    stream.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("N, C", [(3, 70000), (40, 1000)])
def test_captured_in_a_graph(rn, N, C):
    z, v, i, tl, labels = teacher(rn, N, C, 20, 2.0, 8)
    z, x, w = z.cuda(), torch.randn(N, 520).cuda(), torch.randn(130, 520).cuda()
    wq, ws = rn.quant_rows_i8(w)

    def everything():
        return [*rn.topk_rows(z, 20, 2.0), *rn.distill_fwd_bwd(z, v, i, tl, labels, 2.0, 0.5, 0.1), rn.fc_i8_fwd(x, wq, ws)]

    everything()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything()
    for seed in range(4):
        z.copy_(torch.randn(N, C, generator=torch.Generator().manual_seed(seed)))
        x.copy_(torch.randn(N, 520, generator=torch.Generator().manual_seed(seed)))
        want = everything()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)


def test_a_workspace_of_the_callers(rn):
    z, v, i, tl, labels = teacher(rn, 3, 70000, 20, 2.0, 8)
    z = z.cuda()
    d = rn.DistillDesc(3, 70000, 20, rn.F32, 70000, 70000, 2.0, 1.0, 0.0, 1.0)
    ws = torch.full((max(256, rn.distill_workspace_bytes(d), rn.topk_rows_workspace_bytes(3, 70000, 20)),), 255, dtype=torch.uint8, device="cuda")
    for a, b in ((rn.topk_rows(z, 20, workspace=ws), rn.topk_rows(z, 20)),
                 (rn.distill_fwd_bwd(z, v, i, tl, temperature=2.0, workspace=ws), rn.distill_fwd_bwd(z, v, i, tl, temperature=2.0))):
        for s, t in zip(a, b):
            assert torch.equal(s, t)
    need = rn.fc_i8_workspace_bytes(3, 70000)
    w = rn.quant_rows_i8(z)
    with pytest.raises(rn.Rn50Error) as e:
        rn.fc_i8_fwd(z, *w, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -3


@pytest.mark.parametrize("call, error", [
    (lambda rn, z, i: rn.topk_rows(z, 0), "rn50"),
    (lambda rn, z, i: rn.topk_rows(z, 257), "rn50"),
    (lambda rn, z, i: rn.topk_rows(z, 3, 0.0), "rn50"),
    (lambda rn, z, i: rn.topk_rows(z, 3, float("nan")), "rn50"),
    (lambda rn, z, i: rn.topk_rows(z[:0], 3), "rn50"),
    (lambda rn, z, i: rn.topk_rows(z.t(), 3), AssertionError),
    (lambda rn, z, i: rn.topk_rows(z[:1].expand(5, 64), 3), "rn50"),         # rows on top of each other
    (lambda rn, z, i: rn.topk_rows(z.half(), 3), TypeError),
    (lambda rn, z, i: rn.topk_rows(z[0], 3), ValueError),
    (lambda rn, z, i: rn.quant_rows_i8(i), TypeError),
    (lambda rn, z, i: rn.quant_rows_i8(z[:, :0]), "rn50"),
    (lambda rn, z, i: rn.distill_fwd_bwd(z, z[:, :3], i), AssertionError),   # entries that are not contiguous
    (lambda rn, z, i: rn.distill_fwd_bwd(z, z[:, :3].contiguous(), i.long()), TypeError),
    (lambda rn, z, i: rn.distill_fwd_bwd(z, z[:, :3].contiguous(), i[:, :2].contiguous()), ValueError),
    (lambda rn, z, i: rn.distill_fwd_bwd(z, z[:, :3].contiguous(), None), TypeError),
    (lambda rn, z, i: rn.distill_fwd_bwd(z, z[:, :3].contiguous(), i, alpha=1.5), "rn50"),
    (lambda rn, z, i: rn.distill_fwd_bwd(z, z[:, :3].contiguous(), i, alpha=float("nan")), "rn50"),
    (lambda rn, z, i: rn.distill_fwd_bwd(z, z[:, :3].contiguous(), i, temperature=-1.0), "rn50"),
    (lambda rn, z, i: rn.distill_fwd_bwd(z, z[:, :3].contiguous(), i, label_smoothing=2.0), "rn50"),
    (lambda rn, z, i: rn.distill_fwd_bwd(z, z[:, :3].contiguous(), i, dlogits=z.bfloat16()), TypeError),
    (lambda rn, z, i: rn.distill_fwd_bwd(z, z[:, :3].contiguous(), i, dlogits=z[:3]), ValueError),
    (lambda rn, z, i: rn.matmul_i8(64, *rn.quant_rows_i8(z), *rn.quant_rows_i8(z[:, :32])), None),   # both are rows of 64 bytes
    (lambda rn, z, i: rn.matmul_i8(65, *rn.quant_rows_i8(z), *rn.quant_rows_i8(z)), ValueError),
    (lambda rn, z, i: rn.fc_i8_fwd(z, z, z[0]), TypeError),
    (lambda rn, z, i: rn.fc_i8_fwd(z, *rn.quant_rows_i8(z), dtype=torch.float16), TypeError),
    (lambda rn, z, i: rn.fc_i8_fwd(z, *rn.quant_rows_i8(z), y=z), ValueError),
    (lambda rn, z, i: rn.fc_i8_fwd(z, *rn.quant_rows_i8(z), bias=z[0, :3].contiguous()), ValueError),
])
def test_what_is_refused(rn, call, error):
    z = torch.randn(5, 64, device="cuda")
    i = torch.zeros(5, 3, dtype=torch.int32, device="cuda")
    if error is None:
        call(rn, z, i)
        return
    with pytest.raises(rn.Rn50Error if error == "rn50" else error):
        call(rn, z, i)
    torch.cuda.synchronize()


def test_the_interface_refuses_before_it_launches(rn):
    """C ABI: every error has its code, and nothing is written."""
    raw, p = rn.raw, ctypes.c_void_p
    out = torch.full((4096,), 3.0, device="cuda")
    o, f, ld = p(out.data_ptr()), ctypes.c_float, ctypes.c_int64
    odd = p(out.data_ptr() + 2)
    z = ctypes.c_size_t(0)
    assert raw.topk_rows(2, 8, 3, 7, o, ld(8), f(1), o, o, None, None, z, None) == -1
    assert raw.topk_rows(2, 8, 3, 0, o, ld(7), f(1), o, o, None, None, z, None) == -1
    assert raw.topk_rows(2, 8, 3, 0, odd, ld(8), f(1), o, o, None, None, z, None) == -4
    assert raw.topk_rows(2, 8, 3, 0, None, ld(8), f(1), o, o, None, None, z, None) == -1
    assert raw.quant_rows_i8(2, 8, 0, o, ld(8), None, o, None) == -1
    assert raw.quant_rows_i8(2, 200000, 0, o, ld(200000), o, o, None) == -2
    assert raw.matmul_i8(2, 2, 8, o, o, o, None, None, 0, o, ld(2), None) == -1
    assert raw.matmul_i8(2, 2, 8, o, o, o, o, None, 0, o, ld(1), None) == -1
    assert raw.fc_i8_fwd(2, 2, 8, 0, o, ld(8), o, o, None, 0, o, ld(2), None, z, None) == -3
    d = rn.DistillDesc(2, 8, 3, 0, 8, 9, 1.0, 1.0, 0.0, 1.0)
    assert raw.distill_fwd_bwd(ctypes.byref(d), o, o, o, None, None, None, o, o, o, None, z, None) == -1   # in place, other rows
    assert raw.distill_fwd_bwd(None, o, o, o, None, None, None, o, o, o, None, z, None) == -1
    assert raw.distill_fwd_bwd(ctypes.byref(d), o, None, o, None, None, None, o, o, None, None, z, None) == -1
    torch.cuda.synchronize()
    assert bool((out == 3.0).all())


def test_the_example_learns(rn):
    from paper_1903_12650_amd import distill_example
    losses = distill_example.run(steps=40)
    assert torch.isfinite(losses).all()
    first, last = float(losses[:4].mean()), float(losses[-4:].mean())
    assert last < 0.8 * first, (first, last)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("C, k", [(300, 5), (1000, 40), (1000, 256), (2500, 256), (5000, 64), (50001, 100), (100003, 7), (100003, 256)])
def test_more_infinities_than_places(rn, C, k, dtype):
    """What is left then has an infinite sum, unless a NaN is left as well."""
    g = torch.Generator().manual_seed(C + k)
    x = torch.randn(12, C, generator=g)
    inf, nan = float("inf"), float("nan")
    some = lambda n: torch.randperm(C, generator=g)[:min(n, C)]
    x[0, some(k + 1)] = inf
    x[1, 5:5 + k + 30] = inf
    x[2] = inf
    x[3, some(k + 1)] = inf
    x[3, C - 2] = nan                                      # one place goes to it
    x[4, some(k + 5)] = nan
    x[4, 3] = inf
    x[5, some(k)] = inf                                    # as many as places: the rest is finite
    x[6] = float("-inf")
    x[6, some(k + 1)] = inf                                # and nothing else
    x[7, C - k - 2:] = inf
    x[8, torch.linspace(0, C - 1, k + 2).long().unique()] = inf  # spread over the row
    x[9, :k + 3] = inf
    x[9, :k - 1] = nan
    x[10, 1], x[10, C - 1] = inf, inf
    check_topk(rn, x.to(dtype).cuda(), k, 1.0)
    check_topk(rn, spread(x.to(dtype).cuda(), 3), k, 0.25)
    check_topk(rn, x.to(dtype).cuda(), 1, 1e30)
    for n in (0, 3, 8):
        check_topk(rn, x[n:n + 1].to(dtype).cuda(), k, 2.0)


@pytest.mark.parametrize("C", [1000, 40000])
def test_one_row_in_place_whatever_its_strides_say(rn, C):
    """A single row has no next one: its gradient may take its place through a view that names another distance."""
    z, v, i, tl, labels = teacher(rn, 1, C, 7, 2.0, C)
    want = rn.distill_fwd_bwd(z.cuda(), v, i, tl, labels, 2.0, 0.5)
    wide = torch.full((1, C + 8), 5.0, device="cuda")
    part = wide[:, :C]
    part.copy_(z)
    view = part[0].unsqueeze(0)
    assert view.data_ptr() == part.data_ptr() and view.stride(0) != part.stride(0)
    got = rn.distill_fwd_bwd(part, v, i, tl, labels, 2.0, 0.5, dlogits=view)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert bool((wide[:, C:] == 5.0).all())


# ----------------------------------------------- every form, every temperature
# Bounds from what the kernels do, one after another (all in units of eps, of a sum's size):
#  - additions: a thread's own terms (`chain`: its share of the row's vectors, and one more), 6 across a wave, at most 16 across a row's waves and
#    14 more across slices;
#  - a term's exponent has four roundings (the difference, log2(e), its division by T, their product), each of the exponent's own size.  A
#    reference lies at most 20 ln 2 < 14 below the largest logit seen, and all moves of a term's reference together are no longer than the way from the
#    term to the largest, and those 14: 2 * 4 * (way + 14); the way is on average at most the softmax's entropy, ln C;
#  - the exponential 2, a move of the reference (its exponential, its product) 3, at most 10 of them.
# Float losses at 131072 classes are held to some 5e-5 of a nat this way.
def chain(C, dtype):
    vec = 8 if dtype == BF16 else 4
    vecs = -(-C // vec)
    threads = 128 if vecs <= 512 else 256 if vecs <= 3072 else 512 if vecs <= 32768 else 1024  # (the fewest that such a row has)
    return vec * -(-vecs // threads) + 1


def sums_of(C, dtype):
    return EPS * (chain(C, dtype) + 36 + 8 * (np.log(C) + 14) + 32)


def row_spread(a):
    """Largest minus smallest finite value of every row."""
    fine = np.isfinite(a)
    return np.where(fine, a, -np.inf).max(1, initial=-1e300) - np.where(fine, a, np.inf).min(1, initial=1e300)


def check_sampled(rn, z, v, i, tl, labels, T, alpha, ls, w, picked, dlogits=None):
    """The picked rows against the oracle; all others have weight 0, and their losses and gradients are zeros."""
    N, C = z.shape
    k = v.shape[1]
    keep = z[picked].double().cpu().numpy()
    dtype = z.dtype
    loss, rows, grad = rn.distill_fwd_bwd(z, v, i, tl, labels, T, alpha, ls, w, 3.0, dlogits=dlogits)
    others = torch.ones(N, dtype=torch.bool, device="cuda")
    others[picked] = False
    assert not rows[others].any() and not grad[others].any() and grad.dtype == dtype
    vv = f64(v)[picked]
    want_loss, want_rows, want, size = od.distill(keep, vv, i.cpu().numpy()[picked], None if tl is None else f64(tl)[picked],
                                                  labels.cpu().numpy()[picked], T, alpha, ls, f64(w)[picked], 3.0)
    e, zs = sums_of(C, dtype), row_spread(keep)
    cells = EPS * (4 + 20 + 2 * (np.log(k + 1) + 1))  # the teacher's sum: four of a lane, the wave's; a rounding of each exponent
    apart = (row_spread(vv) + zs) / T + np.log(k + 2) + np.log(C)  # log p - log q, at most
    row_bound = alpha * T * T * (2 * e + cells + EPS * ((np.log(k + 1) + 3) * apart + 4 * (zs / T + np.log(C)))) \
        + (1 - alpha) * (2 * e + 4 * EPS * (zs + np.log(C))) + 2 * EPS * np.abs(want_rows)
    off = np.abs(f64(rows)[picked] - want_rows) / row_bound
    assert (off <= 1).all(), (off.max(), row_bound.max())
    assert abs(float(loss) - want_loss) <= float((np.abs(f64(w)[picked]) * row_bound).sum()) + 2 * EPS * abs(want_loss)
    away = (keep.max(1)[:, None] - np.where(np.isfinite(keep), keep, keep.max(1)[:, None])) * max(1.0, 1.0 / T)
    bound = size * (2 * e + cells + EPS * (8 * (np.minimum(away, 90) + 14) + 24)) + 1e-36
    if dtype == BF16:
        bound += 2.0 ** -8 * 1.01 * (np.abs(want) + bound) + 1e-38
    got = f64(grad[picked])
    off = np.abs(got - want) / bound
    assert (off <= 1).all(), (np.unravel_index(off.argmax(), off.shape), off.max(), got.flat[off.argmax()], want.flat[off.argmax()])
    return loss, rows, grad


def sampled(rn, N, C, k, dtype, T, seed, rows=5):
    """A few rows with weights; entries and labels at the ends, on both sides of a chunk of 65536 classes, some repeated and some absent."""
    g = torch.Generator().manual_seed(seed)
    picked = sorted({0, N - 1, *(int(j) for j in torch.randint(0, N, (max(1, rows - 2),), generator=g))})
    z = (torch.randn(min(N, 9), C, generator=g) * 2).to(dtype).cuda().repeat(-(-N // 9), 1)[:N].contiguous()
    i = torch.randint(0, C, (N, k), generator=g)
    edges = [c for c in (65535, 65536, 0, C - 1, 65537, C - 2, 1, 65528, 65543, 131071, 131072) if c < C][:k]
    i[:, :len(edges)] = torch.tensor(edges)
    v = torch.randn(N, k, generator=g) * 2
    if k > 2:
        i[0, k - 1] = i[0, 0]            # again, with another value
        i[picked[-1], k - 1] = i[picked[-1], 1]
        i[picked[len(picked) // 2], k // 2] = -1
    tl = torch.randn(N, generator=g) + np.log(C)
    labels = torch.randint(0, C, (N,), generator=g)
    for n, c in zip(picked, (65536 % C, C - 1, int(i[picked[2 % len(picked)], 0]))):
        labels[n] = c
    w = torch.zeros(N)
    w[picked] = torch.linspace(0.5, 1.5, len(picked))
    return z, v.cuda(), i.to(torch.int32).cuda(), (tl / T).cuda(), labels.to(torch.int32).cuda(), w.cuda(), picked


# (rows, bfloat16 classes, float classes, entries): a workgroup's threads and what it holds of a row, or chunks of classes that it streams
FORMS = [(7, 1001, 501, 9), (5, 2040, 1020, 200), (5, 3000, 1500, 20), (5, 3001, 1501, 200), (3, 5001, 2501, 130), (9, 9000, 4500, 64), (3, 25001, 13001, 100),
         (129, 70001, 70001, 64), (130, 131072, 131072, 256), (129, 270001, 132001, 40), (1, 50001, 20001, 256), (6, 131073, 65537, 33), (2, 300007, 150001, 12)]


@pytest.mark.parametrize("T, alpha, ls, tail", [(3.0, 0.6, 0.1, True), (0.3, 0.6, 0.1, True), (2.0, 0.7, 0.1, False), (4.0, 0.5, 0.0, True),
                                               (1.0, 0.4, 0.1, True), (1.5, 1.0, 0.0, True)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N, bf16_classes, float_classes, k", FORMS)
def test_every_form_at_every_temperature(rn, N, bf16_classes, float_classes, k, dtype, T, alpha, ls, tail):
    C = bf16_classes if dtype == BF16 else float_classes
    z, v, i, tl, labels, w, picked = sampled(rn, N, C, k, dtype, T, N + C + k)
    tl = tl if tail else None
    loss, rows, grad = check_sampled(rn, z, v, i, tl, labels, T, alpha, ls, w, picked)
    only = rn.distill_fwd_bwd(z, v, i, tl, labels, T, alpha, ls, w, 3.0, grad=False)
    assert torch.equal(only[0], loss) and torch.equal(only[1], rows)
    # from an odd element on, in place
    wide = torch.full((N, C + 3), 5.0, dtype=dtype, device="cuda")
    part = wide[:, 1:1 + C]
    part.copy_(z)
    check_sampled(rn, part, v, i, tl, labels, T, alpha, ls, w, picked, dlogits=part)
    assert bool((wide[:, 0] == 5.0).all()) and bool((wide[:, 1 + C:] == 5.0).all())


@pytest.mark.parametrize("T", [3.0, 0.7, 20.0])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("C", [700, 60000])
def test_rows_where_something_is_missing_at_other_temperatures(rn, C, dtype, T):
    N, k = 8, 6
    z, v, i, tl, labels = teacher(rn, N, C, k, T, C)
    w = torch.full((N,), 1.0 / N)
    z[0] = float("-inf")
    i[1], tl[1] = -1, float("-inf")
    z[2], w[2] = float("nan"), 0.0
    labels[3] = -100
    i[4, 3] = i[4, 0]
    keep = torch.zeros(C, dtype=torch.bool)
    keep[i[5].cpu().long()] = True
    keep[labels[5].item()] = True
    z[5, ~keep] = float("-inf")
    z[5, C // 2] = 0.5
    z[6] = torch.finfo(dtype).min
    z[7] *= 20
    check_distill(rn, z.to(dtype).cuda(), v, i, tl, labels, T, 0.6, 0.0, w.cuda())


@pytest.mark.parametrize("temperature", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N, C, k", [(7, 1000, 8), (5, 2500, 200), (6, 8195, 64), (5, 50001, 100), (1, 131072, 64), (7, 131073, 33), (241, 80001, 30)])
def test_log_sum_exp_of_the_rest_holds_float(rn, N, C, k, dtype, temperature):
    """The additions: at most C / 1024 vectors a stream and their own numbers, four streams, what is read again, a wave, the waves, slices;
    exponents as above, from references that may be as high as the largest logit, which the rest does not have."""
    g = torch.Generator().manual_seed(N + C + k)
    x = (torch.randn(N, C, generator=g) * 2).to(dtype)
    rows = range(N) if N < 10 else (0, 100, N - 1)
    wv, wi, want = od.topk_rows(x[list(rows)].double().numpy(), k, temperature)
    values, indices, tail = rn.topk_rows(x.cuda(), k, temperature)
    assert np.array_equal(indices[list(rows)].cpu().numpy(), wi)
    above = (wv[:, 0] - wv[:, -1]) / temperature
    bound = EPS * (C / 512 + 64 + 8 * (np.log(C) + 14 + above) + 32 + 2 * np.abs(want))
    off = np.abs(f64(tail)[list(rows)] - want) / bound
    assert (off <= 1).all(), off.max()


@pytest.mark.parametrize("alpha", [0.0, 0.5])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N, C", [(4, 700), (4, 60000), (140, 40000)])
def test_labels_that_smoothing_takes_all_weight_from(rn, N, C, dtype, alpha):
    """label_smoothing = 1: every class has 1 / C, the label no more than the others.  A masked class makes the loss infinite, the label's too."""
    z, v, i, tl, labels = teacher(rn, N, C, 5, 2.0, C)
    z[0, labels[0].item()] = float("-inf")
    z[1, (labels[1].item() + 1) % C] = float("-inf")
    w = torch.zeros(N)
    w[:4] = 0.25
    z = z.to(dtype).cuda()
    _, rows, grad = check_distill(rn, z, v, i, tl, labels, 2.0, alpha, 1.0, w.cuda())
    assert torch.isposinf(rows[:2]).all() and torch.isfinite(rows[2:]).all()
    again = rn.distill_fwd_bwd(z, v, i, tl, (labels + 1) % C, 2.0, alpha, 1.0, w.cuda())
    assert torch.equal(again[1][2:], rows[2:])             # whatever the labels are


@pytest.mark.parametrize("T", [1.0, 2.0, 0.7])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("C", [90, 700, 60000])
def test_a_rest_masked_with_the_lowest_value_shares_the_tail(rn, C, dtype, T):
    """Every class outside the entries is masked alike: they share the teacher's tail evenly.  The loss, T times the tail's probability times
    3.4e38, passes the largest float or does not."""
    z, v, i, tl, labels = teacher(rn, 3, C, 6, T, C)
    z[1] = torch.finfo(dtype).min
    z[1, i[1].cpu().long()] = torch.linspace(-1, 2, 6)
    z[2, C // 2:] = torch.finfo(dtype).min
    z = z.to(dtype).cuda()
    _, rows, grad = rn.distill_fwd_bwd(z, v, i, tl, labels, T, 1.0)
    _, want_rows, want, size = od.distill(f64(z), f64(v), i.cpu().numpy(), f64(tl), labels.cpu().numpy(), T, 1.0)
    e = sum_error(C)
    away = np.abs(f64(z).max(1)[:, None] - f64(z)) * max(1.0, 1.0 / T)
    bound = size * (2 * e + EPS * (5 * np.minimum(away, 90) + 16)) + 1e-36
    if dtype == BF16:
        bound += 2.0 ** -8 * 1.01 * (np.abs(want) + bound) + 1e-38
    assert (np.abs(f64(grad) - want) <= bound).all()
    with np.errstate(over="ignore"):
        np.testing.assert_allclose(rows.cpu().numpy(), want_rows.astype(np.float32), rtol=1e-4)
    rest = torch.ones(C, dtype=torch.bool)
    rest[i[1].cpu().long()] = False
    assert bool((grad[1].cpu()[rest] == grad[1].cpu()[rest][0]).all()) and float(grad[1].cpu()[rest][0]) < 0

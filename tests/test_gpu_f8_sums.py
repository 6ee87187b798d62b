"""The sums of layers in 8-bit floating point where floats would lose what they are made of: a bias's gradient is a sum in 64 bits, rounded
once; a float sum of few rows is folded every 16384 numbers."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def rn():
    import paper_1903_12650_amd as rn
    return rn


# Few tiles of 128x128 (rows and columns by workgroups of their own), more than 256 of them, single rows, rows in the last tile only.
GRADIENTS = [(1, 1), (3, 5), (130, 40), (200, 1001), (1025, 131), (4200, 1030), (40000, 70)]


def bias_gradient(rn, dy):
    dy = dy.cuda()
    got = rn.fc_f8_bwd(dy, None, None, None, None, need_dx=False, need_dw=False)[2]
    _, _, xt, xts = rn.quant_blocks_f8(torch.ones((dy.shape[0], 70), device="cuda"), rows=False, columns=True)
    assert torch.equal(rn.fc_f8_bwd(dy, None, None, xt, xts, need_dx=False)[2], got)  # beside a product, the same
    return got.double().cpu().numpy()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M, N", GRADIENTS)
def test_bias_gradients_are_rounded_once(rn, M, N, dtype):
    """An addition in 64 bits is off by 2^-53 of what it comes to, the result by 2^-24 of itself."""
    g = torch.Generator().manual_seed(M + N)
    dy = (torch.randn(M, N, generator=g) * torch.exp(2 * torch.randn(M, 1, generator=g))).to(dtype)
    want, size = dy.double().sum(0).numpy(), dy.double().abs().sum(0).numpy()
    assert (np.abs(bias_gradient(rn, dy) - want) <= EPS * np.abs(want) + (M + 8) * 2.0 ** -52 * size).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M, N", GRADIENTS)
def test_bias_gradients_that_cancel(rn, M, N, dtype):
    """Whole numbers below 2^53: exact in 64 bits.  Halves that a float next to 2^24 has no room for, and large ones that go again."""
    dy = torch.full((M, N), 0.5)
    dy[0], dy[M - 1] = 2.0 ** 24, -(2.0 ** 24)
    dy[M // 2, ::2] += 2.0 ** 26
    dy[M // 3, ::2] -= 2.0 ** 26
    dy = dy.to(dtype)
    assert np.array_equal(bias_gradient(rn, dy), dy.double().sum(0).float().double().numpy())


def test_bias_gradients_whose_sum_is_in_range_where_its_parts_are_not(rn):
    for M, N in ((6, 40), (300, 70), (4200, 1030)):
        dy = torch.ones(M, N)
        dy[0], dy[1], dy[2], dy[3] = 3e38, 3e38, -3e38, -3e38
        assert np.array_equal(bias_gradient(rn, dy), np.full(N, float(M - 4)))
        dy[4] = 3e38
        dy[3] = 3e38
        assert np.isposinf(bias_gradient(rn, dy)).all()


def long_sum(M, K):
    """[M, K] whose rows come to the sum that is returned: 2^-5 each, which next to 2^24 are lost however many of them up to 32 are added at once, and in front
    of every eighth of the row a block that comes to 2^24."""
    x = torch.full((M, K), 2.0 ** -5, device="cuda")
    for b in range(8):
        x[:, b * (K // 8):b * (K // 8) + 128] = 2.0 ** 17
    return x, 8 * 2.0 ** 24 + (K - 8 * 128) / 32


# A float takes at most 16384 numbers before it is added to the others: next to 2^24 it loses 16384 / 32 = 512 at most.  There are eight sums of 2^24; each of
# the 16 additions of their parts and of the eight's is rounded by at most 2^-24 of 2^27.
LONG_SUM = 8 * 512 + (8 * 16 + 8) * EPS * 2.0 ** 27


@pytest.mark.parametrize("M", [1, 16, 40, 64])
def test_long_float_sums_of_few_rows(rn, M):
    K, N = 1 << 21, 20
    x, want = long_sum(M, K)
    a, sa, _, _ = rn.quant_blocks_f8(x)
    w, sw, _, _ = rn.quant_blocks_f8(torch.ones((N, K), device="cuda"))
    y = rn.matmul_f8(K, a, sa, w, sw).double()
    assert float((y - want).abs().max()) <= LONG_SUM, float(y.min()) - want
    if M <= 16:
        y = rn.fc_f8_fwd(x, w, sw).double()
        assert float((y - want).abs().max()) <= LONG_SUM, float(y.min()) - want


@pytest.mark.parametrize("M", [1, 40])
def test_long_float_sums_of_few_rows_backward(rn, M):
    K, N = 20, 1 << 18
    dy, want = long_sum(M, N)
    _, _, wt, wts = rn.quant_blocks_f8(torch.ones((N, K), device="cuda"), rows=False, columns=True)
    _, _, xt, xts = rn.quant_blocks_f8(torch.ones((M, K), device="cuda"), rows=False, columns=True)
    dx, dw, db = rn.fc_f8_bwd(dy, wt, wts, xt, xts)
    assert float((dx.double() - want).abs().max()) <= LONG_SUM, float(dx.min()) - want
    assert torch.equal(dw, M * dy[0][:, None].expand(N, K)) and torch.equal(db, M * dy[0])

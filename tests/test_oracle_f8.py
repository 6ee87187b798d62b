"""Pins of the 64-bit forms in oracle/f8.py: the formats by torch's own conversions and by exhaustion, blocks by hand, the mask
by known answers, gradients by differences."""
import numpy as np
import pytest
import torch

from oracle import f8, net

FORMATS = {f8.E4M3: torch.float8_e4m3fn, f8.E5M2: torch.float8_e5m2}


@pytest.mark.parametrize("fmt", FORMATS)
def test_values_of_all_codes(fmt):
    want = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(FORMATS[fmt]).double().numpy()
    assert np.array_equal(f8.values(fmt), want, equal_nan=True)
    assert np.nanmax(f8.values(fmt)[np.isfinite(f8.values(fmt))]) == f8.LARGEST[fmt]


@pytest.mark.parametrize("fmt", FORMATS)
def test_rounding_is_to_nearest_ties_to_even(fmt):
    codes = f8.values(fmt)[:128]
    codes = codes[codes <= f8.LARGEST[fmt]]
    assert np.array_equal(f8.encode(codes, fmt), np.arange(len(codes)))
    middle = (codes[1:] + codes[:-1]) / 2
    assert (f8.encode(middle, fmt) % 2 == 0).all() and (f8.encode(-middle, fmt) % 2 == 0).all()
    assert np.array_equal(f8.encode(middle * (1 + 1e-12), fmt), np.arange(1, len(codes)))
    assert np.array_equal(f8.encode(middle * (1 - 1e-12), fmt), np.arange(len(codes) - 1))
    x = (torch.randn(20000, generator=torch.Generator().manual_seed(1)) * 40).clamp(-448, 448)
    assert np.array_equal(f8.encode(x.numpy(), fmt), x.to(FORMATS[fmt]).view(torch.uint8).numpy())


@pytest.mark.parametrize("fmt", FORMATS)
def test_blocks(fmt):
    F = f8.LARGEST[fmt]
    x = np.zeros((9, 700), np.float32)
    x[1, 5] = F                               # just fits
    x[2, 5] = np.nextafter(np.float32(F), np.float32(np.inf))
    x[3, 127] = 1.0
    x[3, 128] = 3.0
    x[4, 600] = 2.0 ** -110                   # below the floor
    x[5, 1] = np.finfo(np.float32).max
    x[6, 0], x[7, 130] = np.inf, np.nan
    x[8] = np.linspace(-5, 5, 700)
    q, s = f8.quant(x, fmt)
    assert q.shape == (9, 768) and s.shape == (2, 9, 4)
    e = s.transpose(1, 0, 2).reshape(9, 8).astype(int) - 127
    top = int(np.log2(F / 1.75))              # F = 1.75 * 2^top
    assert (s[1, :, 2:] == 0).all()
    assert e[0, 0] == -100 - top and e[1, 0] == 0 and e[2, 0] == 1
    assert e[3, 0] == -top and e[3, 1] == 1 - top + 0
    assert e[4, 4] == -100 - top and (q[4] == 0).sum() >= 767
    assert e[5, 0] == 128 - top                # 2^128 (less a rounding) is above 1.75 * 2^127
    assert e[6, 0] == 0 and (q[6, :128] == 0x7F).all() and (q[6, 128:] == 0).all()
    assert e[7, 1] == 0 and (q[7, 128:256] == 0x7F).all() and (q[7, :128] == 0).all()
    assert (q[:, 700:] == 0).all()
    back = f8.stands_for(q, s, fmt)[8, :700]
    blocks = np.abs(np.pad(x[8], (0, 68)).reshape(6, 128)).max(1).repeat(128)[:700]
    assert (np.abs(back - x[8]) <= np.maximum(np.abs(x[8]) * 2.0 ** -(1 + f8._DIGITS[fmt]), blocks * 2.0 ** -13)).all()


def test_every_block_takes_the_least_power():
    g = np.random.Generator(np.random.PCG64(3))
    x = (g.standard_normal((200, 128)) * np.exp(20 * g.standard_normal((200, 1)))).astype(np.float32)
    for fmt in FORMATS:
        e = f8.quant(x, fmt)[1][0, :, 0].astype(int) - 127
        a = np.maximum(np.abs(x).max(1).astype(np.float64), 2.0 ** -100)
        assert (a <= np.ldexp(f8.LARGEST[fmt], e)).all() and (a > np.ldexp(f8.LARGEST[fmt], e - 1)).all()


def test_mask_from_known_answers():
    """The generator's words (pinned by its known-answer vectors in test_oracle_net.py) taken apart element by element."""
    for seed, call, rows, cols in ((0, 0, 3, 20), (2 ** 64 - 1, 2 ** 64 - 1, 2, 8), (0x1234567890, 5 << 32, 1, 9)):
        m = f8.kept(rows, cols, 0.25, seed, call)
        per = (cols + 7) // 8
        for r in range(rows):
            for k in range(cols):
                b = r * per + k // 8
                w = net.philox4x32_10(np.array([[b, 1 << 31, call & 0xFFFFFFFF, call >> 32]], np.uint32), (seed & 0xFFFFFFFF, seed >> 32))[0]
                bits = (int(w[(k % 8) // 2]) >> (16 * (k % 2))) & 0xFFFF
                assert m[r, k] == (bits >= 16384)


def test_mask_shares_and_independence():
    n = 1 << 20
    for p in (0.0, 0.1, 0.5, 0.9):
        share = f8.kept(1024, 1024, p, 7).mean()
        assert abs(share - (1 - p)) < 6 * np.sqrt(p * (1 - p) / n) + 2.0 ** -17
    a, b = f8.kept(512, 512, 0.5, 7, 0), f8.kept(512, 512, 0.5, 7, 1)
    assert abs((a == b).mean() - 0.5) < 6 * 0.5 / 512
    assert np.array_equal(f8.kept(4, 9, 0.5, 3, 2, 5), f8.kept(4, 9, 0.5, 3, 7)) and np.array_equal(f8.kept(4, 9, .5, 3, 2 ** 64 - 1, 2), f8.kept(4, 9, .5, 3, 1))
    assert not f8.kept(8, 8, 1.0, 1).any() and f8.factor(1.0) == 0 and f8.factor(0.5) == 2 and f8.kept(8, 8, 2.0 ** -18, 1).all()


def test_gradients_by_differences():
    """Small whole numbers are quantized exactly: the layer is then linear, and differences of sum(dy * y) are its gradients."""
    g = np.random.Generator(np.random.PCG64(5))
    M, N, K = 5, 6, 130
    x, w, dy = (g.integers(-8, 9, s).astype(np.float32) for s in ((M, K), (N, K), (M, N)))
    drop = (0.5, 11, 3, 0)  # (factor 2: exact)
    def loss(x, w, b):
        y, _, _, _ = f8.fc_fwd(x, *f8.quant(w), b, drop)
        return (dy * y).sum()
    b = np.arange(N, dtype=np.float64)
    _, _, xt, xts = f8.fc_fwd(x, *f8.quant(w), b, drop)
    (dx, _), (dw, _), (db, _) = f8.fc_bwd(dy, *f8.quant(np.ascontiguousarray(w.T)), xt, xts, drop=drop)
    for _ in range(40):
        i, j, k = g.integers(M), g.integers(N), g.integers(K)
        d = np.zeros_like(x); d[i, k] = 1
        assert dx[i, k] == (loss(x + d, w, b) - loss(x - d, w, b)) / 2
        d = np.zeros_like(w); d[j, k] = 1
        assert dw[j, k] == (loss(x, w + d, b) - loss(x, w - d, b)) / 2
        d = np.zeros(N); d[j] = 1
        assert db[j] == (loss(x, w, b + d) - loss(x, w, b - d)) / 2

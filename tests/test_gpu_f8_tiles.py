"""Products in 8-bit floating point bit for bit.

The factors are small whole numbers times a power of two that differs from block to block and row to row: a, w in {-2, .., 2} * 2^{-1, 0, 1}.
Products are multiples of 1/4 up to 16, all eight products that the 8-bit matrix cores add at once share a power (so the smallest is a quarter of
the largest, far above 2^-13 of it), and sums of K <= 2^17 of them are multiples of 1/4 below 2^21: floats hold each of them
in any order.  So a float result is equal to the sum, a bfloat16 one to its rounding, and a product that is lost, doubled or scaled by another
block's power shows."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


@pytest.fixture(scope="module")
def rn():
    import paper_1903_12650_amd as rn
    return rn


def amid(t, fill):
    """The same bytes, contiguous, with others in front and behind."""
    n = t.numel()
    flat = torch.full((n + 8192,), fill, dtype=torch.uint8, device="cuda")
    flat[4096:4096 + n] = t.reshape(-1)
    return flat[4096:4096 + n].view(t.shape)


def whole_numbers(rows, K, fmt, seed):
    """(q, scale, numbers): NaN codes in front of and behind q, NaN scales around scale."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    blocks, groups = (K + 127) // 128, (K + 511) // 512
    n = torch.zeros((rows, blocks * 128), device="cuda")
    n[:, :K] = torch.randint(-2, 3, (rows, K), device="cuda", generator=g).float()
    e = torch.randint(-1, 2, (rows, blocks), device="cuda", generator=g)
    scale = torch.zeros((rows, groups * 4), dtype=torch.uint8, device="cuda")
    scale[:, :blocks] = (e + 127).to(torch.uint8)
    scale = scale.view(rows, groups, 4).transpose(0, 1).contiguous()
    q = amid(n.to(fmt).view(torch.uint8), 0x7F).view(fmt)
    return q, amid(scale, 0xFF), (n.view(rows, blocks, 128) * torch.exp2(e.float())[:, :, None]).view(rows, blocks * 128)


def check_product(rn, M, N, K, fmt, seed=1):
    assert K <= 1 << 17
    a, sa, na = whole_numbers(M, K, fmt, seed)
    w, sw, nw = whole_numbers(N, K, E4M3, seed + 1)
    bias = (torch.arange(N, device="cuda") % 7).float()
    want = torch.matmul(na, nw.t()) + bias
    for y_type in (F32, BF16):
        wide = torch.full((M, N + 3), 5.0, dtype=y_type, device="cuda")
        y = rn.matmul_f8(K, a, sa, w, sw, bias, y=wide[:, :N])
        differ = (y != want.to(y_type)).nonzero()
        assert len(differ) == 0, (y_type, len(differ), differ[0].tolist(), float(y[tuple(differ[0])]), float(want[tuple(differ[0])]))
        assert (wide[:, N:] == 5).all()


# 64x64 tiles by sums of one to four blocks and of more (past the last block their rings ask for nothing), single rows and columns in the last tile.
SMALL = [(65, 65, k) for k in (1, 128, 256, 384, 512, 513, 640, 769, 1000, 1100, 1300, 2000)] + [(300, 200, 500), (193, 257, 2100)]


@pytest.mark.parametrize("fmt", [E4M3, E5M2])
@pytest.mark.parametrize("M, N, K", SMALL)
def test_whole_numbers(rn, M, N, K, fmt):
    check_product(rn, M, N, K, fmt)

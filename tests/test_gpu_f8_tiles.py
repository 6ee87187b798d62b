"""Products in 8-bit floating point by every tile, ring and split, bit for bit.

The factors are small whole numbers times a power of two that differs from block to block and row to row: a, w in {-2, .., 2} * 2^{-1, 0, 1}.
Products are multiples of 1/4 up to 16, all eight products that the 8-bit matrix cores add at once share a power (so the smallest is a quarter of
the largest, far above 2^-13 of it), and sums of K < 2^18 of them are multiples of 1/4 below 2^22: floats hold each of them
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
    assert K < 1 << 18
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
        if fmt == E4M3:  # rows that are quantized on the way: the same numbers
            for x in (na[:, :K], na[:, :K].to(BF16)):
                assert torch.equal(rn.fc_f8_fwd(x, w, sw, bias, dtype=y_type), want.to(y_type))


# Few rows: 16 to 64 of them, 16 or 32 columns a workgroup, a wave with no block, one, several.
FEW = [(1, 40, 128), (1, 1000, 2048), (16, 33, 1100), (17, 70, 700), (33, 1000, 2048), (40, 8200, 1300), (48, 17, 20000), (64, 8201, 1500), (64, 64, 50176),
       (1, 8200, 700), (20, 9000, 1300)]
# Few rows and sums that are folded (more than 131072 numbers), 16 and 32 columns a workgroup.
LONG = [(M, N, 140000) for M in (1, 20, 40, 64) for N in (33, 8200)]
# 64x64 tiles by sums of one to four blocks and of more (past the last block their rings ask for nothing), single rows and columns in the last tile.
SMALL = [(65, 65, k) for k in (1, 128, 256, 384, 512, 513, 640, 769, 1000, 1100, 1300, 2000)] + [(300, 200, 500), (193, 257, 2100)]
# 128x64 tiles with four buffers; 128x128 ones by eight waves with two, by four with four; 128x64 with two, three a unit; 128x128 in many rounds.
MIDDLE = [(1100, 1300, 700), (1025, 1281, 1500), (2000, 1500, 130), (2000, 1500, 1000), (1921, 1409, 1500), (2000, 1500, 4300), (2200, 2100, 130), (2177, 2113, 1500),
          (2200, 2100, 4300), (6100, 4090, 600), (6017, 4097, 1500)]
# 256x256 tiles: sums across groups of scales, ragged, outputs past the caches in float (32 MiB and more) and in both types.
LARGE = [(2900, 2890, 1300), (2900, 2900, 260), (3329, 3085, 1100), (4090, 4000, 520), (7900, 4000, 1100), (8191, 4090, 2047)]
# Sums in parts: few tiles and long sums (512 x 9216 -> 512 in parts of eight blocks), and sums of more than 16384 numbers whatever the tiles.
PARTS = [(130, 70, 7000), (300, 500, 4100), (300, 500, 7168), (500, 510, 9216), (500, 600, 11000), (1024, 2000, 11000), (1000, 1030, 11000), (256, 1024, 50176), (2000, 1500, 20000), (4090, 4090, 16500),
         (65, 9, 100000)]


@pytest.mark.parametrize("fmt", [E4M3, E5M2])
@pytest.mark.parametrize("M, N, K", FEW + LONG + SMALL + MIDDLE + LARGE + PARTS)
def test_whole_numbers(rn, M, N, K, fmt):
    check_product(rn, M, N, K, fmt)


@pytest.mark.parametrize("fmt", [E4M3, E5M2])
@pytest.mark.parametrize("M, N, K", [(40, 1000, 700), (60, 1000, 700), (40, 2900, 300), (12, 300, 5000), (1300, 300, 700), (1100, 2900, 2900), (1024, 4090, 4000), (20000, 256, 1024), (50176, 256, 1000),
                                     (20000, 64, 200)])
def test_layer_of_whole_numbers(rn, M, N, K, fmt):
    """Gradients of a layer of small whole numbers: they are quantized exactly, in either format, and a dropout of one half doubles what it keeps."""
    g = torch.Generator(device="cuda").manual_seed(M + N)
    x, w, dy = (torch.randint(-2, 3, s, device="cuda", generator=g).float() for s in ((M, K), (N, K), (M, N)))
    drop = rn.Dropout(0.5, 7, 1)
    kept = rn.dropout_fwd(torch.ones_like(x), drop)
    _, _, wt, wts = rn.quant_blocks_f8(w, rows=False, columns=True)
    _, _, xt, xts = rn.quant_blocks_f8(x, rows=False, columns=True, dropout=drop)
    want_dx, want_dw, want_db = torch.matmul(dy, w) * kept, torch.matmul(dy.t().contiguous(), x * kept), dy.sum(0)
    for dtype in (F32, BF16):
        dx, dw, db = rn.fc_f8_bwd(dy.to(dtype), wt, wts, xt, xts, dtype=dtype, dropout=drop, format=fmt)
        assert torch.equal(dx, want_dx.to(dtype)) and torch.equal(dw, want_dw) and torch.equal(db, want_db)
        assert torch.equal(rn.fc_f8_bwd(dy.to(dtype), None, None, xt, xts, format=fmt, need_dx=False)[1], want_dw)


@pytest.mark.parametrize("fmt", [E4M3, E5M2])
@pytest.mark.parametrize("M, N, K", [(3, 70, 400), (40, 70, 400), (100, 70, 1000), (300, 90, 400), (1100, 1300, 1000), (2000, 1500, 1500), (2900, 2900, 700)])
def test_nan_blocks(rn, M, N, K, fmt):
    """A block of NaN on either side reaches its row or column and no other, in both formats."""
    x, w = torch.ones((M, K), device="cuda"), torch.ones((N, K), device="cuda")
    x[1, K - 1], x[M - 1, 0], w[5, 3], w[N - 1, 200] = float("nan"), float("inf"), float("-inf"), float("nan")
    a, sa, _, _ = rn.quant_blocks_f8(x, fmt)
    b, sb, _, _ = rn.quant_blocks_f8(w)
    want = torch.full((M, N), float(K), device="cuda")
    want[1], want[M - 1], want[:, 5], want[:, N - 1] = (float("nan"),) * 4
    for y_type in (F32, BF16):
        y = rn.matmul_f8(K, a, sa, b, sb, dtype=y_type)
        assert torch.equal(torch.isnan(y), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(y), torch.nan_to_num(want.to(y_type)))


@pytest.mark.parametrize("M, N, K", [(40, 300, 700), (300, 500, 11000), (1100, 1000, 17000), (2000, 1500, 17000), (17000, 300, 200), (20000, 60, 70)])
def test_workspaces_of_just_what_is_asked_for(rn, M, N, K):
    """Workspaces as large as the sizes say for a call's types and gradients: nothing behind them is touched, and the results are those of the largest."""
    def workspace(size):
        flat = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        return flat[:size], flat[size:]

    def untouched(tail):
        return bool((tail == 0xA5).all())

    x, w, dy = (torch.randint(-2, 3, s, device="cuda").float() for s in ((M, K), (N, K), (M, N)))
    q, s, t, ts = rn.quant_blocks_f8(w, columns=True)
    a, sa, at, ats = rn.quant_blocks_f8(x, columns=True)
    for dtype in (F32, BF16):
        want = torch.matmul(x, w.t()).to(dtype)
        some, tail = workspace(rn.matmul_f8_workspace_bytes(M, N, K, dtype))
        assert torch.equal(rn.matmul_f8(K, a, sa, q, s, dtype=dtype, workspace=some if len(some) else None), want) and untouched(tail)
        some, tail = workspace(rn.fc_f8_fwd_workspace_bytes(M, N, K, dtype))
        assert torch.equal(rn.fc_f8_fwd(x, q, s, dtype=dtype, workspace=some), want) and untouched(tail)
        want = (torch.matmul(dy, w).to(dtype), torch.matmul(dy.t().contiguous(), x), dy.sum(0))
        for need in ((True, True, True), (True, False, False), (False, True, False), (False, False, True), (True, False, True), (True, True, False), (False, True, True)):
            some, tail = workspace(rn.fc_f8_bwd_workspace_bytes(M, N, K, dtype, *need))
            got = rn.fc_f8_bwd(dy, t, ts, at, ats, dtype=dtype, need_dx=need[0], need_dw=need[1], need_db=need[2], workspace=some)
            for g, v, n in zip(got, want, need):
                assert (g is None) != n and (not n or torch.equal(g, v)), (dtype, need)
            assert untouched(tail), (dtype, need)

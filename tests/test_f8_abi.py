"""The host side of dropout and of the products in 8-bit floating point: sizes, and refusals that need no GPU."""
import ctypes

import pytest
import torch

E4M3, E5M2 = 2, 3


class DropoutDesc(ctypes.Structure):
    _fields_ = [("p", ctypes.c_float), ("seed", ctypes.c_uint64), ("call", ctypes.c_uint64), ("step", ctypes.c_void_p)]


def drop(p=0.1, step=None):
    return ctypes.byref(DropoutDesc(p, 1, 2, step))


def test_sizes():
    import paper_1903_12650_amd as rn
    assert [rn.quant_f8_row_bytes(k) for k in (-1, 0, 1, 128, 129, 1000, 1 << 22, (1 << 22) + 1)] == [0, 0, 128, 128, 256, 1024, 1 << 22, 0]
    assert [rn.quant_f8_scale_bytes(3, k) for k in (0, 1, 512, 513, 1 << 22, (1 << 22) + 1)] == [0, 12, 12, 24, 3 * 4 * 8192, 0]
    assert rn.quant_f8_scale_bytes(0, 8) == 0 and rn.quant_f8_scale_bytes(2 ** 31 - 1, 1 << 22) == 4 * 8192 * (2 ** 31 - 1)
    assert rn.fc_f8_fwd_workspace_bytes(40, 1000, 2048) >= 40 * 2048 + 40 * 16 and rn.fc_f8_fwd_workspace_bytes(0, 8, 8) == 0
    assert rn.fc_f8_fwd_workspace_bytes(1 << 20, 8, 1 << 20) > 1 << 40
    assert rn.fc_f8_bwd_workspace_bytes(40, 1000, 2048) >= 40 * 1024 + 1000 * 128 + 4000
    assert rn.fc_f8_bwd_workspace_bytes(1 << 20, 1 << 20, 8) > 2 << 40 and rn.fc_f8_bwd_workspace_bytes(-1, 8, 8) == 0


def test_refusals_come_before_anything_touches_the_device():
    """(a launch attempt without a GPU would be -5)"""
    import paper_1903_12650_amd as rn
    raw, one, odd, far, ld, z = rn.raw, ctypes.c_void_p(256), ctypes.c_void_p(264), ctypes.c_void_p(1 << 20), ctypes.c_int64, ctypes.c_size_t(0)
    big = ctypes.c_size_t(1 << 40)

    def fwd(d=None, M=2, K=8, dtype=0, x=one, ldx=8, r=None, ldr=8, y=far, ldy=8):
        return raw.dropout_fwd(d or drop(), M, K, dtype, x, ld(ldx), r, ld(ldr), y, ld(ldy), None)
    for bad in ({"M": 0}, {"K": -1}, {"dtype": 2}, {"x": None}, {"y": None}, {"ldx": 7}, {"ldy": 7}, {"r": one, "ldr": 7}, {"d": drop(1.5)}, {"d": drop(-0.1)},
                {"d": drop(float("nan"))}, {"y": one, "ldy": 9}, {"r": far, "ldr": 9}):
        assert fwd(**bad) == -1, bad
    assert raw.dropout_fwd(None, 2, 8, 0, one, ld(8), None, ld(8), far, ld(8), None) == -1
    assert raw.dropout_bwd(None, 2, 8, 0, one, ld(8), far, ld(8), None) == -1
    assert fwd(x=ctypes.c_void_p(6)) == -4 and fwd(y=ctypes.c_void_p(258)) == -4 and fwd(d=drop(step=12)) == -4 and fwd(dtype=1, x=ctypes.c_void_p(3)) == -4

    def quant(M=2, K=8, dtype=0, x=one, ldx=8, d=None, fmt=E4M3, q=one, s=one, t=one, ts=one):
        return raw.quant_blocks_f8(M, K, dtype, x, ld(ldx), d, fmt, q, s, t, ts, None)
    for bad in ({"M": 0}, {"K": 0}, {"dtype": 2}, {"fmt": 1}, {"fmt": 4}, {"x": None}, {"ldx": 7}, {"q": None}, {"s": None}, {"t": None}, {"ts": None}, {"d": drop(2)},
                {"q": None, "s": None, "t": None, "ts": None}):
        assert quant(**bad) == -1, bad
    assert quant(q=odd) == -4 and quant(s=odd) == -4 and quant(t=odd) == -4 and quant(ts=odd) == -4 and quant(x=ctypes.c_void_p(6)) == -4
    top = (1 << 22) + 1
    assert quant(K=top, ldx=top) == -2 and quant(M=top) == -2 and quant(M=2 ** 31 - 1, t=None, ts=None) == -2

    def product(M=2, N=2, K=8, fmt=E4M3, a=one, s=one, w=one, ws=one, b=None, yt=0, y=one, ldy=2):
        return raw.matmul_f8(M, N, K, fmt, a, s, w, ws, b, yt, y, ld(ldy), one, big, None)
    for bad in ({"M": 0}, {"N": 0}, {"K": 0}, {"fmt": 0}, {"a": None}, {"s": None}, {"w": None}, {"ws": None}, {"yt": 2}, {"y": None}, {"ldy": 1}):
        assert product(**bad) == -1, bad
    assert product(K=top) == -2 and product(M=1 << 20, N=1 << 20, ldy=1 << 20) == -2
    assert product(N=(1 << 26) + 1, M=1, ldy=1 << 27) == -2
    assert product(a=odd) == -4 and product(ws=odd) == -4 and product(y=ctypes.c_void_p(6)) == -4 and product(b=ctypes.c_void_p(6)) == -4

    def forward(M=2, N=2, K=8, x=one, d=None, w=one, ws=one, b=None, y=one, xt=None, xs=None, work=one, n=big):
        return raw.fc_f8_fwd(M, N, K, 0, x, ld(K), d, w, ws, b, 0, y, ld(N), xt, xs, work, n, None)
    for bad in ({"M": 0}, {"N": 0}, {"K": 0}, {"x": None}, {"w": None}, {"ws": None}, {"y": None}, {"xt": one}, {"xs": one}, {"d": drop(-1)}):
        assert forward(**bad) == -1, bad
    assert forward(n=ctypes.c_size_t(8)) == -3 and forward(work=None) == -3 and forward(work=odd) == -4 and forward(xt=odd, xs=one) == -4
    assert forward(K=top) == -2 and forward(M=top, xt=one, xs=one) == -2

    def backward(M=2, N=2, K=8, dy=one, fmt=E4M3, wt=one, ws=one, xt=one, xs=one, d=None, dxt=0, dx=one, dw=one, db=one, work=one, n=big):
        return raw.fc_f8_bwd(M, N, K, 0, dy, ld(N), fmt, wt, ws, xt, xs, d, dxt, dx, ld(K), dw, db, work, n, None)
    for bad in ({"M": 0}, {"N": 0}, {"K": 0}, {"dy": None}, {"fmt": 7}, {"wt": None}, {"ws": None}, {"xt": None}, {"xs": None}, {"dxt": 2}, {"d": drop(3)},
                {"dx": None, "dw": None, "db": None}):
        assert backward(**bad) == -1, bad
    assert backward(n=z) == -3 and backward(work=odd) == -4 and backward(wt=odd) == -4 and backward(xs=odd) == -4 and backward(dw=ctypes.c_void_p(6)) == -4
    assert backward(M=top) == -2 and backward(N=top) == -2


@pytest.mark.parametrize("call, error", [
    (lambda rn, x: rn.dropout_fwd(x, rn.Dropout(0.1, 1)), AssertionError),                       # host tensors
    (lambda rn, x: rn.dropout_fwd(x.double(), rn.Dropout(0.1, 1)), TypeError),
    (lambda rn, x: rn.dropout_fwd(None, rn.Dropout(0.1, 1)), TypeError),
    (lambda rn, x: rn.dropout_fwd(x[0, 0], rn.Dropout(0.1, 1)), ValueError),
    (lambda rn, x: rn.dropout_bwd(x, rn.Dropout(0.1, 1)), AssertionError),
    (lambda rn, x: rn.quant_blocks_f8(x), AssertionError),
    (lambda rn, x: rn.quant_blocks_f8(x, torch.float16), TypeError),
    (lambda rn, x: rn.quant_blocks_f8(x, "e4m3"), TypeError),
    (lambda rn, x: rn.quant_blocks_f8(x[0]), ValueError),
    (lambda rn, x: rn.quant_blocks_f8(x.half()), TypeError),
    (lambda rn, x: rn.matmul_f8(8, x, x, x, x), TypeError),
    (lambda rn, x: rn.matmul_f8(8, x[0].to(torch.float8_e4m3fn), x, x, x), ValueError),
    (lambda rn, x: rn.matmul_f8(8, x.to(torch.float8_e4m3fn), x, x, x), ValueError),             # rows of 128 bytes are expected
    (lambda rn, x: rn.fc_f8_fwd(x, x, x), AssertionError),
    (lambda rn, x: rn.fc_f8_bwd(x, x, x, x, x), AssertionError),
])
def test_native_calls_refuse_what_they_cannot_take(call, error):
    import paper_1903_12650_amd as rn
    with pytest.raises(error) as e:
        call(rn, torch.zeros(4, 8))
    assert "frame #" not in str(e.value)


@pytest.mark.parametrize("call", [lambda rn, x: rn.matmul_f8(2 ** 32 + 8, x, x, x, x)])
def test_numbers_past_32_bits_are_not_cut(call):
    import paper_1903_12650_amd as rn
    with pytest.raises(OverflowError):
        call(rn, torch.zeros(4, 8))


def test_workspaces_are_what_a_call_uses():
    """A bfloat16 product of many tiles is not split however long its sum: it needs none, and none is asked for.  What is smaller than needed is refused."""
    import paper_1903_12650_amd as rn
    F, B = torch.float32, torch.bfloat16
    sizes = [(M, N, K) for M in (1, 64, 65, 300, 1000, 8192) for N in (9, 500, 2000, 8192) for K in (100, 4200, 8192, 11000, 28672, 100000)]
    for s in sizes:
        assert rn.matmul_f8_workspace_bytes(*s, B) <= rn.matmul_f8_workspace_bytes(*s, F) == rn.matmul_f8_workspace_bytes(*s) == rn.raw.matmul_f8_workspace_bytes(*s)
        assert rn.fc_f8_fwd_workspace_bytes(*s, B) <= rn.fc_f8_fwd_workspace_bytes(*s) == rn.raw.fc_f8_fwd_workspace_bytes(*s)
        most = rn.raw.fc_f8_bwd_workspace_bytes(*s)
        for dtype in (F, B):
            both = rn.fc_f8_bwd_workspace_bytes(*s, dtype)
            assert both <= most
            for need in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
                assert rn.fc_f8_bwd_workspace_bytes(*s, dtype, *need) <= both
    assert rn.matmul_f8_workspace_bytes(8192, 8192, 28672, B) == 0 and rn.matmul_f8_workspace_bytes(8192, 8192, 28672) == 2 * 8192 * 8192 * 4
    assert rn.matmul_f8_workspace_bytes(300, 500, 11000, B) > 0  # (few tiles: split in either type)
    assert rn.fc_f8_fwd_workspace_bytes(8192, 8192, 28672, B) < 8192 * 28672 * 1.1
    assert rn.fc_f8_bwd_workspace_bytes(8192, 28672, 8192, B, need_dw=False) < 8192 * 28672 * 1.1
    assert rn.fc_f8_bwd_workspace_bytes(65536, 8192, 8192, need_dx=False, need_dw=False) == 512 * 8192 * 8
    assert rn.matmul_f8_workspace_bytes(0, 8, 8, B) == rn.fc_f8_fwd_workspace_bytes(8, 8, 0, B) == rn.fc_f8_bwd_workspace_bytes(8, 8, 0, B) == 0
    with pytest.raises(TypeError):
        rn.matmul_f8_workspace_bytes(8, 8, 8, torch.float16)

    raw, one, ld = rn.raw, ctypes.c_void_p(256), ctypes.c_int64
    for s, dtype, code in (((300, 500, 11000), B, 1), ((2000, 1500, 20000), F, 0)):
        M, N, K = s
        less = ctypes.c_size_t(rn.matmul_f8_workspace_bytes(*s, dtype) - 1)
        assert raw.matmul_f8(M, N, K, E4M3, one, one, one, one, None, code, one, ld(N), one, less, None) == -3
        less = ctypes.c_size_t(rn.fc_f8_fwd_workspace_bytes(*s, dtype) - 1)
        assert raw.fc_f8_fwd(M, N, K, 0, one, ld(K), None, one, one, None, code, one, ld(N), None, None, one, less, None) == -3
        for dx, dw, db in ((one, one, one), (one, None, None), (None, one, None), (None, None, one)):
            less = ctypes.c_size_t(rn.fc_f8_bwd_workspace_bytes(*s, dtype, dx is not None, dw is not None, db is not None) - 1)
            assert raw.fc_f8_bwd(M, N, K, 0, one, ld(N), E4M3, one, one, one, one, None, code, dx, ld(K), dw, db, one, less, None) == -3

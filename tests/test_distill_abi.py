"""The host side of the quantized products and the distillation operators: sizes, and refusals that need no GPU."""
import ctypes

import pytest
import torch


def test_sizes():
    import paper_1903_12650_amd as rn
    assert [rn.quant_i8_row_bytes(k) for k in (-1, 0, 1, 64, 65, 1000, 131071, 131072)] == [0, 0, 64, 64, 128, 1024, 131072, 0]
    assert rn.fc_i8_workspace_bytes(40, 2048) >= 40 * 2048 + 40 * 4 and rn.fc_i8_workspace_bytes(0, 64) == 0
    assert rn.fc_i8_workspace_bytes(1 << 20, 131071) > 1 << 32
    d = rn.DistillDesc(4, 1000, 8, rn.F32, 1000, 1000, 1.0, 1.0, 0.0, 1.0)
    assert ctypes.sizeof(d) == 48 and rn.distill_workspace_bytes(d) < 1 << 20


def test_refusals_come_before_anything_touches_the_device():
    """(a launch attempt without a GPU would be -5)"""
    import paper_1903_12650_amd as rn
    raw, one, f, ld, z = rn.raw, ctypes.c_void_p(256), ctypes.c_float, ctypes.c_int64, ctypes.c_size_t(0)
    assert raw.quant_rows_i8(0, 8, 0, one, ld(8), one, one, None) == -1
    assert raw.quant_rows_i8(1, 131072, 0, one, ld(131072), one, one, None) == -2
    assert b"131071" in raw.rn50_last_error()
    assert raw.quant_rows_i8(1, 8, 2, one, ld(8), one, one, None) == -1
    assert raw.quant_rows_i8(2, 8, 0, one, ld(7), one, one, None) == -1
    assert raw.quant_rows_i8(2, 8, 0, ctypes.c_void_p(6), ld(8), one, one, None) == -4
    assert raw.quant_rows_i8(2, 8, 0, one, ld(8), ctypes.c_void_p(8), one, None) == -4
    assert raw.matmul_i8(2, 2, 8, one, None, one, one, None, 0, one, ld(2), None) == -1
    assert raw.matmul_i8(2, 2, 131072, one, one, one, one, None, 0, one, ld(2), None) == -2
    assert raw.matmul_i8(2, 2, 8, one, one, one, one, None, 5, one, ld(2), None) == -1
    assert raw.matmul_i8(1 << 20, 1 << 20, 8, one, one, one, one, None, 0, one, ld(1 << 20), None) == -2
    assert raw.matmul_i8(1, (1 << 26) + 1, 8, one, one, one, one, None, 0, one, ld(1 << 27), None) == -2
    assert raw.fc_i8_fwd(2, 2, 8, 0, one, ld(8), one, one, None, 0, one, ld(2), one, ctypes.c_size_t(8), None) == -3
    assert raw.topk_rows(2, 8, 257, 0, one, ld(8), f(1), one, one, None, None, z, None) == -2
    assert raw.topk_rows(2, 8, 3, 0, one, ld(8), f(float("inf")), one, one, None, None, z, None) == -1
    assert raw.topk_rows(-2, 8, 3, 0, one, ld(8), f(1), one, one, None, None, z, None) == -1
    for bad in ({"temperature": 0.0}, {"alpha": -0.1}, {"label_smoothing": 1.1}, {"N": 0}, {"C": -4}, {"ld": 999}, {"grad_ld": 1}, {"dtype": 9}):
        d = rn.DistillDesc(4, 1000, 8, rn.F32, 1000, 1000, 1.0, 1.0, 0.0, 1.0)
        for name, value in bad.items():
            setattr(d, name, value)
        assert raw.distill_fwd_bwd(ctypes.byref(d), one, one, one, None, None, None, one, one, ctypes.c_void_p(512), None, z, None) == -1, bad
    d = rn.DistillDesc(4, 1000, 300, rn.F32, 1000, 1000, 1.0, 1.0, 0.0, 1.0)
    assert raw.distill_fwd_bwd(ctypes.byref(d), one, one, one, None, None, None, one, one, None, None, z, None) == -2


@pytest.mark.parametrize("call, error", [
    (lambda rn, x: rn.quant_rows_i8(x), AssertionError),                       # host tensors
    (lambda rn, x: rn.quant_rows_i8(x.double()), TypeError),
    (lambda rn, x: rn.quant_rows_i8(x[0]), ValueError),
    (lambda rn, x: rn.quant_rows_i8(None), TypeError),
    (lambda rn, x: rn.topk_rows(x, 3), AssertionError),
    (lambda rn, x: rn.topk_rows(x, "3"), TypeError),
    (lambda rn, x: rn.fc_i8_fwd(x, x, x), AssertionError),
    (lambda rn, x: rn.matmul_i8(8, x, x, x, x), TypeError),
    (lambda rn, x: rn.matmul_i8(8, x[0], x, x, x), ValueError),
    (lambda rn, x: rn.distill_fwd_bwd(x, x, x), AssertionError),
    (lambda rn, x: rn.distill_fwd_bwd(x, None, None, bogus=1), TypeError),
])
def test_native_calls_refuse_what_they_cannot_take(call, error):
    import paper_1903_12650_amd as rn
    with pytest.raises(error) as e:
        call(rn, torch.zeros(4, 8))
    assert "frame #" not in str(e.value)


@pytest.mark.parametrize("call", [
    lambda rn, x: rn.topk_rows(x, 2 ** 32 + 3),
    lambda rn, x: rn.topk_rows(x, -2 ** 32 + 3),
    lambda rn, x: rn.matmul_i8(2 ** 32 + 8, x, x, x, x),
    lambda rn, x: rn.conv_fwd(x[None, None], x[None, None], 2 ** 32 + 1, 0),
])
def test_numbers_past_32_bits_are_not_cut(call):
    import paper_1903_12650_amd as rn
    with pytest.raises(OverflowError):
        call(rn, torch.zeros(4, 8))

"""What the 8-bit matrices' calls refuse before they touch a GPU: no GPU needed."""
import ctypes

import pytest
import torch

import paper_2309_01507_amd as lpmm
from paper_2309_01507_amd import binding as B


def on_cpu(rows=20, cols=130, tile=128):
    return lpmm.new_f8(rows, cols, tile, device="cpu")


def test_sizes():
    assert lpmm.lpmm_f8_sizes(1, 1) == [128, 4]
    assert lpmm.lpmm_f8_sizes(129, 513, 1) == [129 * 640, 5 * 132] and lpmm.lpmm_f8_sizes(129, 513, 128) == [129 * 640, 2 * 8]
    assert lpmm.lpmm_f8_sizes(0, 5, 1) == lpmm.lpmm_f8_sizes(0, 5, 128) == [0, 0]
    for bad in ((1, 0, 1), (-1, 1, 1), (1, 1, 2), (1, 2 ** 22 + 1, 1), (2 ** 30 + 1, 1, 1), (2 ** 27, 128, 1)):
        with pytest.raises(lpmm.LpmmError):
            lpmm.lpmm_f8_sizes(*bad)


def test_matrices_of_another_make():
    good, x = on_cpu(), torch.zeros(3, 130)
    bad = [lpmm.MatF8(20, 130, 128, good.codes.to(torch.int8), good.scales), lpmm.MatF8(20, 130, 128, good.codes, good.scales.to(torch.int32)),
           lpmm.MatF8(20, 130, 128, good.codes[:19], good.scales), lpmm.MatF8(20, 130, 1, good.codes, good.scales),
           lpmm.MatF8(20, 130, 64, good.codes, good.scales), lpmm.MatF8(20, 130, 128, good.codes.t(), good.scales),
           lpmm.MatF8(20, 260, 128, good.codes, good.scales)]
    for m in bad:
        for call in (lambda: lpmm.lpmm_f8_linear(torch.zeros(3, m.cols), m), lambda: lpmm.lpmm_f8_matmul(good, m), lambda: lpmm.lpmm_f8_matmul(m, good),
                     lambda: lpmm.lpmm_f8_dequant(m), lambda: lpmm.lpmm_f8_quant(torch.zeros(20, m.cols), m.tile, m)):
            with pytest.raises((ValueError, lpmm.LpmmError)):
                call()
    for call in (lambda: lpmm.lpmm_f8_quant(x.half()), lambda: lpmm.lpmm_f8_quant(x[0]), lambda: lpmm.lpmm_f8_quant(x.t()),
                 lambda: lpmm.lpmm_f8_quant(x, 128, good), lambda: lpmm.lpmm_f8_quant(x, 1, stream=5), lambda: lpmm.lpmm_f8_quant_both(x, 1, stream=5),
                 lambda: lpmm.lpmm_f8_linear(x[:, :129], good), lambda: lpmm.lpmm_f8_linear(x.double(), good), lambda: lpmm.lpmm_f8_matmul(good, good, torch.float16),
                 lambda: lpmm.f8_linear(x, torch.zeros(20, 131)), lambda: lpmm.f8_linear(x, torch.zeros(130)),
                 lambda: lpmm.lpmm_f8_linear(x, good), lambda: lpmm.lpmm_f8_quant(x), lambda: lpmm.lpmm_f8_dequant(good)):         # the last three: not on a GPU
        with pytest.raises((ValueError, lpmm.LpmmError)):
            call()


def f8(rows, cols, tile, codes=4096, scales=4096):
    return B._F8(codes, scales, rows, cols, tile, 0)


def test_library_refuses():
    """Nothing is launched: no rows, or refused before"""
    L = lpmm.lib()
    at = ctypes.addressof
    a, none = f8(5, 130, 1), f8(0, 130, 1, None, None)
    assert L.lpmm_f8_quant(None, 0, 130, at(none), None) == 0
    assert L.lpmm_f8_quant(None, 0, 129, at(none), None) == L.lpmm_f8_quant(None, 2, 130, at(none), None) == L.lpmm_f8_quant(None, 0, 130, None, None) == -1
    assert L.lpmm_f8_quant(None, 0, 130, at(a), None) == -1, "no input"
    for bad in (f8(5, 130, 1, 4097), f8(5, 130, 1, 4096, 4097), f8(5, 130, 1, None), f8(5, 130, 3), f8(-1, 130, 1), f8(5, 0, 1)):
        assert L.lpmm_f8_quant(4096, 0, 130, at(bad), None) == L.lpmm_f8_dequant(at(bad), 4096, 0, 130, None) == -1
        assert L.lpmm_f8_matmul(at(bad), at(a), 4096, 0, 5, None, 0, None) == L.lpmm_f8_linear(4096, 0, 1, 130, at(bad), 4096, 5, None, 0, None) == -1
    assert L.lpmm_f8_quant_both(4096, 0, 130, at(none), at(f8(130, 5, 1)), None) == -1
    for other in (f8(5, 130, 1), f8(130, 5, 128), f8(130, 6, 1)):
        assert L.lpmm_f8_quant_both(4096, 0, 130, at(a), at(other), None) == -1
    assert L.lpmm_f8_matmul(at(a), at(f8(5, 131, 1)), 4096, 0, 5, None, 0, None) == -1
    assert L.lpmm_f8_matmul(at(none), at(a), None, 0, 5, None, 0, None) == 0
    assert L.lpmm_f8_matmul(at(a), at(a), 4096, 0, 4, None, 0, None) == L.lpmm_f8_matmul(at(a), at(a), 4097, 0, 5, None, 0, None) == -1
    assert L.lpmm_f8_linear(None, 0, 0, 130, at(a), None, 5, None, 0, None) == 0
    assert L.lpmm_f8_linear(None, 0, 2 ** 24, 130, at(a), None, 5, None, 0, None) == -1
    need = L.lpmm_f8_linear_workspace_bytes(100, 5, 130)
    assert need >= 100 * 256
    assert L.lpmm_f8_linear(4096, 0, 100, 130, at(a), 4096, 5, 4096, need - 1, None) == -4
    assert L.lpmm_f8_linear(4096, 0, 100, 130, at(a), 4096, 5, None, need, None) == L.lpmm_f8_linear(4096, 0, 100, 130, at(a), 4096, 5, 4104, need, None) == -1
    assert L.lpmm_f8_linear_workspace_bytes(0, 5, 130) == L.lpmm_f8_linear_workspace_bytes(100, 0, 130) == L.lpmm_f8_matmul_workspace_bytes(5, 5, 0) == 0


def test_library_refuses_training_calls():
    L = lpmm.lib()
    t, n, k = 20, 30, 140
    kept, need = L.lpmm_f8_train_kept_bytes(t, n, k, 3), L.lpmm_f8_train_workspace_bytes(t, n, k)
    assert L.lpmm_f8_train_kept_bytes(t, n, k, 0) == 0 and 0 < L.lpmm_f8_train_kept_bytes(t, n, k, 1) < kept and 0 < L.lpmm_f8_train_kept_bytes(t, n, k, 2) < kept
    assert kept >= 256 * 30 + 140 * 128 and need > 0
    P = 4096

    def forward(x=P, dtype=0, t=t, xs=k, w=P, wd=0, n=n, k=k, ws=k, grads=3, y=P, ys=n, keep=P, keep_bytes=kept, room=P, room_bytes=need):
        return L.lpmm_f8_train_forward(x, dtype, t, xs, w, wd, n, k, ws, grads, y, ys, keep, keep_bytes, room, room_bytes, None)

    def backward(dy=P, dtype=0, t=t, ds=n, n=n, k=k, grads=3, keep=P, keep_bytes=kept, dx=P, xs=k, dw=P, wd=0, ws=k, room=P, room_bytes=need):
        return L.lpmm_f8_train_backward(dy, dtype, t, ds, n, k, grads, keep, keep_bytes, dx, xs, dw, wd, ws, room, room_bytes, None)

    big = 2 ** 22 + 1
    for bad in (dict(t=0), dict(n=0), dict(k=0), dict(t=big), dict(n=big, ys=big), dict(k=big, xs=big, ws=big), dict(grads=4), dict(grads=-1), dict(t=2 ** 22, k=2 ** 22, xs=2 ** 22, ws=2 ** 22),
                dict(x=None), dict(w=None), dict(y=None), dict(x=P + 2), dict(w=P + 1), dict(dtype=2), dict(wd=3), dict(xs=k - 1), dict(ws=k - 1), dict(ys=n - 1),
                dict(keep=None), dict(keep=P + 8), dict(room=None), dict(room=P + 8)):
        assert forward(**bad) == -1, bad
    for bad in (dict(t=0), dict(n=0), dict(k=0), dict(t=big), dict(grads=4), dict(dy=None), dict(dy=P + 2), dict(dtype=2), dict(ds=n - 1), dict(dx=None), dict(xs=k - 1), dict(dw=None),
                dict(wd=2), dict(ws=k - 1), dict(keep=None), dict(keep=P + 8), dict(room=None), dict(room=P + 8)):
        assert backward(**bad) == -1, bad
    assert forward(keep_bytes=kept - 1) == forward(room_bytes=need - 1) == backward(keep_bytes=kept - 1) == backward(room_bytes=need - 1) == -4
    assert backward(grads=0, dx=None, dw=None) == 0, "nothing is wanted"
    assert L.lpmm_f8_train_kept_bytes(0, n, k, 3) == L.lpmm_f8_train_kept_bytes(t, n, k, 4) == L.lpmm_f8_train_workspace_bytes(t, 0, k) == 0


def test_a_cast_of_the_layer():
    layer = lpmm.F8Linear(100, 30, device="cpu")
    assert layer.weight.dtype == torch.float32 and layer.bfloat16().weight.dtype == torch.bfloat16
    copy = lpmm.F8Linear.from_weight(layer.weight)
    assert copy.weight is not layer.weight and copy.weight.requires_grad and (copy.in_features, copy.out_features) == (100, 30)


def test_the_largest_matrices():
    """As the header states them: 2^33 codes, 2^22 columns, and of a matrix with its transpose 2^22 rows"""
    assert lpmm.lpmm_f8_sizes(2 ** 26, 128) == [2 ** 33, 2 ** 26] and lpmm.lpmm_f8_sizes(2 ** 11, 2 ** 22) == [2 ** 33, 2 ** 26]
    for bad in ((2 ** 26 + 1, 128, 1), (2 ** 11 + 1, 2 ** 22, 1), (2 ** 26 + 1, 1, 128)):
        with pytest.raises(lpmm.LpmmError):
            lpmm.lpmm_f8_sizes(*bad)
    L, at = lpmm.lib(), ctypes.addressof
    long = 2 ** 22 + 1
    assert L.lpmm_f8_quant_both(None, 0, 1, at(f8(long, 1, 1)), at(f8(1, long, 1)), None) == -1
    assert L.lpmm_f8_quant_both(None, 0, 1, at(f8(long, 1, 128)), at(f8(1, long, 128)), None) == -1


def test_workspace_of_few_tokens():
    """None where a kernel of their own takes them for either type; that of the tiles next to where results in bf16 take these"""
    need = lpmm.lib().lpmm_f8_linear_workspace_bytes
    assert need(1, 32000, 4096) == need(11, 24576, 4096) == need(12, 24575, 4096) == need(16, 24576, 2048) == need(12, 65537, 4096) == 0
    for t, n, k in ((12, 24576, 4096), (16, 32000, 4096), (16, 65536, 4096), (13, 50257, 2560), (12, 30000, 5120)):
        assert need(t, n, k) >= t * (k + k // 128)

"""CPU checks of the routing and 8-bit entry points: the extension module builds and imports, and arguments are refused before
anything is launched.  No compute calls."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def mok():
    from paper_2609_36070_b200 import build
    build.build()
    from paper_2609_36070_b200 import mok
    return mok


@pytest.fixture(scope="module")
def lib(mok):
    from paper_2609_36070_b200 import build
    return ctypes.CDLL(build.LIB)


class Gate(ctypes.Structure):
    _fields_ = ([("logits", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("logits_stride", ctypes.c_int64)] +
                [(n, ctypes.c_int32) for n in ("T", "E", "k", "type", "score", "n_groups", "topk_groups", "group_top", "renormalise")] +
                [("scale", ctypes.c_float), ("idx", ctypes.c_void_p), ("w", ctypes.c_void_p), ("stream", ctypes.c_void_p)])


class GateBackward(ctypes.Structure):
    _fields_ = ([("logits", ctypes.c_void_p), ("idx", ctypes.c_void_p), ("dw", ctypes.c_void_p), ("stride", ctypes.c_int64),
                 ("d_stride", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("T", "E", "k", "type", "score", "renormalise")] +
                [("scale", ctypes.c_float), ("out", ctypes.c_void_p), ("stream", ctypes.c_void_p)])


class Linear(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("x", "x_codes", "x_scales", "W_codes", "W_scales", "bias")] +
                [(n, ctypes.c_int64) for n in ("x_stride", "codes_stride", "w_stride", "out_stride")] +
                [(n, ctypes.c_int32) for n in ("M", "K", "N", "x_type", "out_type")] +
                [("out", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("stream", ctypes.c_void_p)])


class Experts(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("x", "idx", "w", "gu", "gu_scales", "dn", "dn_scales", "dn_max", "add")] +
                [(n, ctypes.c_int64) for n in ("x_stride", "gu_stride", "dn_stride", "add_stride", "out_stride")] +
                [(n, ctypes.c_int32) for n in ("T", "H", "I", "E", "k", "type")] +
                [("out", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("stream", ctypes.c_void_p)])


A = 1 << 20     # stands for an address: aligned, and never read by a call that is refused


def test_gate_is_refused_before_a_launch(mok, lib):
    good = dict(logits=A, logits_stride=64, T=4, E=64, k=4, type=2, score=1, n_groups=4, topk_groups=2, group_top=2, scale=1.0, idx=A, w=A)
    assert lib.mok_gate(None) == mok.MOK_ERR_NULL
    for change, status in ((dict(logits=None), mok.MOK_ERR_NULL), (dict(idx=None), mok.MOK_ERR_NULL), (dict(E=513), mok.MOK_ERR_SHAPE),
                           (dict(k=33), mok.MOK_ERR_SHAPE), (dict(n_groups=5), mok.MOK_ERR_SHAPE), (dict(topk_groups=5), mok.MOK_ERR_SHAPE),
                           (dict(group_top=3), mok.MOK_ERR_SHAPE), (dict(type=3), mok.MOK_ERR_SHAPE), (dict(score=2), mok.MOK_ERR_SHAPE),
                           (dict(logits_stride=63), mok.MOK_ERR_SHAPE), (dict(T=-1), mok.MOK_ERR_SHAPE), (dict(logits=A + 2), mok.MOK_ERR_ALIGN),
                           (dict(T=0, logits=None), mok.MOK_OK)):
        assert lib.mok_gate(ctypes.byref(Gate(**{**good, **change}))) == status, change
    good = dict(logits=A, idx=A, dw=A, stride=64, d_stride=64, T=4, E=64, k=4, type=2, score=0, scale=1.0, out=A)
    assert lib.mok_gate_backward(None) == mok.MOK_ERR_NULL
    for change, status in ((dict(dw=None), mok.MOK_ERR_NULL), (dict(k=65, E=64), mok.MOK_ERR_SHAPE), (dict(d_stride=3), mok.MOK_ERR_SHAPE),
                           (dict(out=A + 1), mok.MOK_ERR_ALIGN), (dict(T=0), mok.MOK_OK)):
        assert lib.mok_gate_backward(ctypes.byref(GateBackward(**{**good, **change}))) == status, change


def test_8_bit_calls_are_refused_before_a_launch(mok, lib):
    lib.mok_i8_quantize.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong, ctypes.c_void_p,
                                    ctypes.c_longlong, ctypes.c_void_p, ctypes.c_void_p]
    assert lib.mok_i8_quantize(None, 0, 2, 16, 16, A, 16, A, None) == mok.MOK_ERR_NULL
    assert lib.mok_i8_quantize(A, 0, 2, 16, 15, A, 16, A, None) == mok.MOK_ERR_SHAPE
    assert lib.mok_i8_quantize(A, 0, 2, 131073, 1 << 20, A, 1 << 20, A, None) == mok.MOK_ERR_SHAPE
    assert lib.mok_i8_quantize(A + 1, 0, 2, 16, 16, A, 16, A, None) == mok.MOK_ERR_ALIGN
    assert lib.mok_i8_quantize(None, 0, 0, 16, 16, None, 16, None, None) == mok.MOK_OK
    good = dict(x=A, W_codes=A, W_scales=A, x_stride=64, w_stride=64, out_stride=32, M=300, K=64, N=32, x_type=0, out_type=0, out=A,
                workspace=A, workspace_bytes=1 << 20)
    for change, status in ((dict(x=None), mok.MOK_ERR_NULL), (dict(W_scales=None), mok.MOK_ERR_NULL), (dict(N=0), mok.MOK_ERR_SHAPE),
                           (dict(x_stride=63), mok.MOK_ERR_SHAPE), (dict(w_stride=48), mok.MOK_ERR_SHAPE), (dict(out_type=7), mok.MOK_ERR_SHAPE),
                           (dict(w_stride=72), mok.MOK_ERR_ALIGN), (dict(W_codes=A + 8), mok.MOK_ERR_ALIGN), (dict(M=0), mok.MOK_OK),
                           (dict(x=None, x_codes=A), mok.MOK_ERR_SHAPE), (dict(x=None, x_codes=A, codes_stride=64), mok.MOK_ERR_NULL),
                           (dict(x=None, x_codes=A, x_scales=A, codes_stride=72), mok.MOK_ERR_ALIGN)):
        assert lib.mok_i8_linear(ctypes.byref(Linear(**{**good, **change}))) == status, change
    good = dict(x=A, idx=A, w=A, gu=A, gu_scales=A, dn=A, dn_scales=A, dn_max=A, x_stride=64, gu_stride=64, dn_stride=32, out_stride=64,
                T=8, H=64, I=32, E=4, k=2, type=0, out=A, workspace=A, workspace_bytes=0)
    assert lib.mok_i8_experts(None) == mok.MOK_ERR_NULL
    for change, status in ((dict(), mok.MOK_ERR_WORKSPACE), (dict(idx=None), mok.MOK_ERR_NULL), (dict(dn_max=None), mok.MOK_ERR_NULL),
                           (dict(H=60), mok.MOK_ERR_SHAPE), (dict(I=16392, dn_stride=16400), mok.MOK_ERR_SHAPE), (dict(k=5), mok.MOK_ERR_SHAPE),
                           (dict(type=2), mok.MOK_ERR_SHAPE), (dict(gu_stride=48), mok.MOK_ERR_SHAPE), (dict(dn_stride=40), mok.MOK_ERR_ALIGN),
                           (dict(out=A + 8), mok.MOK_ERR_ALIGN), (dict(T=0), mok.MOK_OK)):
        assert lib.mok_i8_experts(ctypes.byref(Experts(**{**good, **change}))) == status, change


def test_workspace_sizes(mok):
    size = mok.mok_i8_experts_workspace_bytes
    rows = 1024 * 8 + 127 * 64
    assert size(1024, 512, 256, 64, 8) >= rows * (512 + 4 * 256 + 256 + 2 * 512)
    assert 0 < size(0, 512, 256, 64, 8) <= size(1, 512, 256, 64, 8) < size(1024, 512, 256, 64, 8)
    for bad in ((4, 511, 256, 64, 8), (4, 512, 250, 64, 8), (4, 512, 256, 513, 8), (4, 512, 256, 4, 5), (-1, 512, 256, 4, 2)):
        assert size(*bad) == 0
    with pytest.raises(mok.MokError):
        mok.alloc_i8_workspace(4, 511, 256, 64, 8)


def test_entry_points_want_tensors_on_a_gpu(mok):
    import torch
    x = torch.zeros(4, 32)
    w = mok.I8Weights(torch.zeros(8, 32, dtype=torch.int8), torch.zeros(8))
    for call in (lambda: mok.mok_gate(x, 2), lambda: mok.mok_i8_quantize(x), lambda: mok.mok_i8_linear(x, w)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    for call in (lambda: mok.mok_gate(x), lambda: mok.mok_gate(x, 2, 3, bias=None), lambda: mok.mok_i8_linear(x, w, nothing=1),
                 lambda: mok.mok_i8_linear([1.0], w)):
        with pytest.raises(TypeError):
            call()

"""8-bit operands without a GPU: storage arithmetic, refusals of the C entry points (fake addresses, never dereferenced) and of the
native functions, and the reference the GPU tests compare with."""
import ctypes
import inspect

import numpy as np
import pytest
import torch

import fp8_util as fu
from paper_1905_10759_b200 import build

build.build_lib()

from paper_1905_10759_b200 import hbmm  # noqa: E402


def test_signatures():
    want = {
        "fp8_quantize": "(x, out, stream=None)", "fp8_gemm": "(A, W, C, stream=None)", "fp8_input_grad": "(GY, W, GX, stream=None)",
        "fp8_weight_grad": "(gy, X, GW, base=None, stream=None)", "fp8_binarize_backward": "(X, gy, beta, gx=None, stream=None)",
    }
    assert {n: str(inspect.signature(getattr(hbmm, n))) for n in want} == want


def test_storage():
    assert hbmm.fp8_operand_bytes(3, 300) == (3 * 304, 3 * 4 * 4, 304, 4)
    assert hbmm.fp8_operand_bytes(300, 1000, 128) == (300 * 1008, 3 * 8 * 4, 1008, 8)
    assert hbmm.fp8_operand_bytes(1, 1) == (16, 16, 16, 4)
    for args, status in (((0, 5), hbmm.ERR_INVALID_ARG), ((5, 0), hbmm.ERR_INVALID_ARG), ((5, 5, 64), hbmm.ERR_UNSUPPORTED),
                         ((5, 1 << 31), hbmm.ERR_UNSUPPORTED)):
        with pytest.raises(hbmm.HbmmError) as e:
            hbmm.fp8_operand_bytes(*args)
        assert e.value.status == status
    op = hbmm.alloc_fp8_operand(200, 300, 128, device="cpu")
    assert op.rows == 200 and tuple(op.codes.shape) == (200, 304) and tuple(op.scales.shape) == (2, 4)


def desc(rows=8, K=256, block_rows=1, codes=0x1000, scales=0x2000, ld_codes=256, ld_scales=4):
    return hbmm.hbmm_fp8_operand(rows, K, codes, ld_codes, scales, ld_scales, block_rows, 0)


BAD_OPERANDS = [
    (dict(rows=0), hbmm.ERR_INVALID_ARG), (dict(K=0), hbmm.ERR_INVALID_ARG), (dict(codes=None), hbmm.ERR_INVALID_ARG),
    (dict(scales=None), hbmm.ERR_INVALID_ARG), (dict(ld_codes=240), hbmm.ERR_INVALID_ARG), (dict(ld_scales=1), hbmm.ERR_INVALID_ARG),
    (dict(ld_codes=264), hbmm.ERR_ALIGNMENT), (dict(ld_scales=6), hbmm.ERR_ALIGNMENT), (dict(codes=0x1008), hbmm.ERR_ALIGNMENT),
    (dict(scales=0x2004), hbmm.ERR_ALIGNMENT), (dict(block_rows=64), hbmm.ERR_UNSUPPORTED), (dict(rows=1 << 31), hbmm.ERR_UNSUPPORTED),
    (dict(ld_codes=1 << 62), hbmm.ERR_UNSUPPORTED), (dict(ld_scales=1 << 62), hbmm.ERR_UNSUPPORTED),
]


@pytest.mark.parametrize("change,status", BAD_OPERANDS)
def test_operands_are_checked_by_every_entry_point(change, status):
    lib, by = hbmm._lib, ctypes.byref
    C, good, w = ctypes.c_void_p(0x8000), desc(), desc(rows=256, block_rows=128)
    bad, bad_w = desc(**change), desc(**{**dict(rows=256, block_rows=128), **change})
    assert lib.hbmm_fp8_quantize(C, 0, bad.rows, bad.K, 256, by(bad), None) == status
    assert lib.hbmm_fp8_gemm(by(bad), by(w), C, 0, 256, None) == status
    assert lib.hbmm_fp8_gemm(by(good), by(bad_w), C, 0, 256, None) == status
    assert lib.hbmm_fp8_input_grad(by(bad), by(w), C, 0, 256, None) == status
    assert lib.hbmm_fp8_input_grad(by(good), by(bad_w), C, 0, 256, None) == status
    assert lib.hbmm_fp8_weight_grad(C, 1, 64, 64, by(bad), None, 0, C, 256, None) == status
    assert lib.hbmm_fp8_binarize_backward(by(bad), C, 0, 256, 32, C, 256, None) == status
    for f in (lib.hbmm_fp8_gemm, lib.hbmm_fp8_input_grad):
        assert f(None, by(w), C, 0, 256, None) == f(by(good), None, C, 0, 256, None) == hbmm.ERR_INVALID_ARG


def test_refusals():
    lib, by = hbmm._lib, ctypes.byref
    INV, UNS, ALI = hbmm.ERR_INVALID_ARG, hbmm.ERR_UNSUPPORTED, hbmm.ERR_ALIGNMENT
    P = ctypes.c_void_p
    a, w, x = desc(), desc(rows=256, block_rows=128), desc()
    q = lambda p=0x4000, dt=0, rows=8, K=256, ld=256: lib.hbmm_fp8_quantize(P(p), dt, rows, K, ld, by(a), None)  # noqa: E731
    assert q(p=None) == q(dt=2) == q(rows=7) == q(K=255) == q(ld=255) == INV
    assert q(p=0x4002) == ALI
    for f in (lib.hbmm_fp8_gemm, lib.hbmm_fp8_input_grad):
        g = lambda A=a, W=w, p=0x8000, dt=0, ld=256: f(by(A), by(W), P(p), dt, ld, None)  # noqa: E731
        assert g(p=None) == g(dt=5) == g(ld=252) == INV
        assert g(p=0x8004) == g(ld=257) == g(dt=1, ld=260) == ALI
        assert g(A=w) == g(W=a) == UNS                                                    # the other kind of scales
    assert lib.hbmm_fp8_gemm(by(desc(K=250)), by(w), P(0x8000), 0, 256, None) == INV      # K differs
    assert lib.hbmm_fp8_input_grad(by(desc(K=250)), by(w), P(0x8000), 0, 256, None) == INV
    wg = lambda p=0x4000, dt=1, N=64, ldg=64, X=x, b=0, ldb=0, gw=0x8000, ldw=256: lib.hbmm_fp8_weight_grad(  # noqa: E731
        P(p), dt, N, ldg, by(X), P(b) if b else None, ldb, P(gw), ldw, None)
    assert wg(p=None) == wg(N=0) == wg(dt=3) == wg(ldg=56) == wg(gw=None) == wg(ldw=252) == wg(b=0x9000, ldb=128) == INV
    assert wg(b=0x8000, ldb=512) == INV                                                   # the gradient itself, another pitch
    assert wg(dt=0) == wg(X=desc(rows=8, block_rows=128)) == wg(ldg=1 << 62) == wg(ldw=1 << 61) == UNS
    assert wg(p=0x4008) == wg(ldg=68) == wg(gw=0x8008) == wg(ldw=258) == wg(b=0x9004, ldb=256) == wg(b=0x9000, ldb=257) == ALI
    bb = lambda X=x, p=0x4000, dt=0, ldg=256, beta=32, o=0x8000, ldo=256: lib.hbmm_fp8_binarize_backward(  # noqa: E731
        by(X), P(p), dt, ldg, beta, P(o), ldo, None)
    assert bb(p=None) == bb(o=None) == bb(dt=2) == bb(ldg=255) == bb(ldo=255) == bb(beta=0) == INV
    assert bb(X=desc(block_rows=128)) == UNS
    assert bb(p=0x4002) == bb(o=0x8001, dt=1) == ALI


@pytest.mark.parametrize("call,error,text", [
    (lambda o, w, t: hbmm.fp8_quantize(t, o), ValueError, "device tensor"),
    (lambda o, w, t: hbmm.fp8_quantize(t, (o.codes, o.scales)), TypeError, "Fp8Operand"),
    (lambda o, w, t: hbmm.fp8_quantize(t, hbmm.Fp8Operand(o.codes.float(), o.scales, 256)), ValueError, "float8_e4m3fn"),
    (lambda o, w, t: hbmm.fp8_quantize(t, hbmm.Fp8Operand(o.codes, o.scales.double(), 256)), ValueError, "float32"),
    (lambda o, w, t: hbmm.fp8_quantize(t, hbmm.Fp8Operand(o.codes, o.scales, 300)), ValueError, "smaller"),
    (lambda o, w, t: hbmm.fp8_quantize(t, hbmm.Fp8Operand(o.codes, o.scales[:, :1], 256)), ValueError, "smaller"),
    (lambda o, w, t: hbmm.fp8_quantize(t, hbmm.Fp8Operand(o.codes, o.scales[:3], 256)), ValueError, "smaller"),
    (lambda o, w, t: hbmm.fp8_quantize(t, hbmm.Fp8Operand(o.codes, o.scales, 0)), ValueError, "smaller"),
    (lambda o, w, t: hbmm.fp8_quantize(t, hbmm.Fp8Operand(o.codes, o.scales, 256, 64)), ValueError, "block_rows"),
    (lambda o, w, t: hbmm.fp8_quantize(t, hbmm.Fp8Operand(o.codes.t(), o.scales, 4)), ValueError, "contiguous"),
    (lambda o, w, t: hbmm.fp8_quantize(t, hbmm.Fp8Operand([1], o.scales, 4)), TypeError, "Tensor"),
    (lambda o, w, t: hbmm.fp8_quantize(t, hbmm.Fp8Operand(o.codes, o.scales, "4")), TypeError, "int"),
    (lambda o, w, t: hbmm.fp8_gemm(o, w), TypeError, "missing"),
    (lambda o, w, t: hbmm.fp8_gemm(o, w, t, None, None), TypeError, "positional"),
    (lambda o, w, t: hbmm.fp8_input_grad(o, w, t, out=t), TypeError, "unexpected"),
    (lambda o, w, t: hbmm.fp8_weight_grad(t, o, t), ValueError, "device tensor"),
    (lambda o, w, t: hbmm.fp8_binarize_backward(o, t, 32), ValueError, "device tensor"),
])
def test_native_functions_refuse(call, error, text):
    o, w = hbmm.alloc_fp8_operand(8, 256, device="cpu"), hbmm.alloc_fp8_operand(256, 256, 128, device="cpu")
    with pytest.raises(error, match=text):
        call(o, w, torch.zeros(8, 256))


def test_reference_codes_are_torch_s():
    """The table and the rounding of the reference against torch's e4m3 on every fp16 value up to 448."""
    v = torch.arange(0x10000, dtype=torch.int32).to(torch.int16).view(torch.float16).float()
    v = v[torch.isfinite(v) & (v.abs() <= 448)].numpy()
    codes = fu.encode(v.astype(np.float64))
    want = torch.from_numpy(v).to(torch.float8_e4m3fn)
    assert np.array_equal(fu.decode(codes), want.double().numpy())
    assert np.array_equal(codes[v != 0], want.view(torch.uint8).numpy()[v != 0])


def test_reference_scales():
    """448 = 1.75 * 2^8: the largest magnitude that a power of two still holds, and the next fp32 above it."""
    x = np.zeros((4, 256), dtype=np.float32)
    x[0, 0], x[1, 0] = 448.0 * 2 ** -20, np.nextafter(np.float32(448.0 * 2 ** -20), np.float32(1))
    x[2, 0], x[3, 130] = 1e-45, -3.0e38
    _, s = fu.quantize(x, 1)
    assert s[0, 0] == 2.0 ** -20 and s[1, 0] == 2.0 ** -19 and s[2, 0] == s[0, 1] == 2.0 ** -117
    assert 3.0e38 / s[3, 1] <= 448 < 3.0e38 / s[3, 1] * 2
    _, s = fu.quantize(x, 128)
    assert s.shape == (1, 2) and s[0, 0] == 2.0 ** -19

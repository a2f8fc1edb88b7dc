"""What the header promises of 8-bit operands beyond the quantizer's own: scales of either sign, long contractions."""
import numpy as np
import pytest
import torch

import fp8_util as fu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hb():
    from paper_1905_10759_b200 import hbmm
    assert hbmm.last_device_error() == 0
    yield hbmm
    assert hbmm.last_device_error() == 0


def normal(rows, K, seed):
    return np.random.default_rng(seed).standard_normal((rows, K)).astype(np.float32)


# group lengths of both kernels: trees inside 128 elements (in a lane, over lanes), teams of 4 threads, of a warp, of a CTA
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("scales", ["pow2", "any"])
@pytest.mark.parametrize("rows,K,beta", [(5, 260, 2), (7, 1000, 16), (9, 640, 32), (6, 700, 128), (4, 515, 3), (5, 1000, 48), (3, 3000, 3000)])
def test_binarize_backward_takes_scales_of_either_sign(hb, rows, K, beta, scales, dtype):
    """Group means and the clip go by |code * scale|, the sign by the code's sign bit: the gradient of an operand whose scales are
    negated here and there is that of the operand with their magnitudes, bit for bit, and Eq. 6's."""
    X, _, codes, s = fu.held(normal(rows, K, rows + K), 1, scales)
    negative = np.random.default_rng(K).random(s.shape) < 0.5
    negative[0, 0] = True
    gy = torch.from_numpy(normal(rows, K, K + beta)).to(torch.float32 if dtype == "fp32" else torch.bfloat16)
    plain = hb.fp8_binarize_backward(X, gy.cuda(), beta)
    X.scales[:, :s.shape[1]] *= torch.from_numpy(np.where(negative, -1, 1).astype(np.float32)).cuda()
    got = hb.fp8_binarize_backward(X, gy.cuda(), beta)
    ref, mag = fu.binarize_backward(codes, np.where(negative, -s, s), gy.double().numpy(), beta)
    # sums of n terms, whatever their order, a mean and a product: at most n + 4 roundings on the terms' magnitudes
    bound = (min(beta, K) + 4) * fu.U * mag + 1e-30
    bound = bound + (fu.BF16 * (np.abs(ref) + bound) if dtype == "bf16" else 0)
    assert (np.abs(got.double().cpu().numpy() - ref) <= bound).all()
    assert torch.equal(got, plain)


def values(op):
    return (op.codes.view(torch.float8_e4m3fn)[:, :op.K].double() * op.scales.double().repeat_interleave(op.block_rows, 0)[:op.rows]
            .repeat_interleave(128, 1)[:, :op.K])


@pytest.mark.parametrize("signs", ["positive", "any"])
@pytest.mark.parametrize("sizes", ["one", "spread"])
@pytest.mark.parametrize("out_type", ["fp32", "bf16"])
@pytest.mark.parametrize("kind,M,N,K", [
    ("gemm", 512, 512, 8192), ("gemm", 512, 512, 16384), ("gemm", 300, 520, 20000), ("gemm", 2600, 2304, 8192), ("gemm", 2600, 2304, 16384),
    ("input_grad", 300, 16384, 520), ("input_grad", 2600, 8192, 2304),
])
def test_sums_of_long_contractions_do_not_pile_up_truncations(hb, kind, M, N, K, out_type, sizes, signs):
    """Power-of-two scales: the tensor cores' sums truncate, always towards zero, which shows where nothing cancels and where groups
    differ in size.  Tiles that are shared along the contraction and tiles that are not.
    By element: 32 products and the sum so far lose less than 2^-25 of the largest each (33 u / 2), their sum at most a step (2 u), so
    18.5 u of sum |a w| per 32 elements; a rounding per run and one more for the last.  By norm 4e-6, as the weight gradient: 64
    instructions a run that lose half a step (u) of a sum growing to its end each, 32 u = 1.9e-6 on average, and as much again for
    the cut terms of groups that are small beside the sum.  bf16: runs four times as long, 1.6e-5, beside half a step of the result."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(M + N + K)
    L = K if kind == "gemm" else N

    def operand(rows, cols, block_rows, spread_rows, spread_cols):
        x = torch.randn(rows, cols, generator=gen, device="cuda")
        x = x.abs() if signs == "positive" else x
        if sizes == "spread":
            e = torch.randint(-12, 13, (-(-rows // spread_rows), -(-cols // spread_cols)), generator=gen, device="cuda").float()
            x *= torch.exp2(e).repeat_interleave(spread_rows, 0)[:rows].repeat_interleave(spread_cols, 1)[:, :cols]
        return hb.fp8_quantize(x, hb.alloc_fp8_operand(rows, cols, block_rows))
    A = operand(M, L, 1, M, 128)
    W = operand(N, K, 128, 128, 128)
    out = torch.empty(M, N if kind == "gemm" else K, dtype=torch.float32 if out_type == "fp32" else torch.bfloat16, device="cuda")
    (hb.fp8_gemm if kind == "gemm" else hb.fp8_input_grad)(A, W, out)
    a, w = values(A), values(W)
    w = w.t() if kind == "gemm" else w
    ref, F = a @ w, a.abs() @ w.abs()
    err = (out.double() - ref).abs()
    bound = (18.5 * -(-L // 32) + -(-L // 128) + 1) * fu.U * F
    rounding = fu.BF16 if out_type == "bf16" else 0.0
    assert (err <= bound + rounding * (ref.abs() + bound)).all()
    far = (err - rounding * ref.abs()).clamp(min=0)            # beyond half a step of the result: what the sum itself is off
    assert far.norm() <= (4e-6 if out_type == "fp32" else 1.6e-5) * ref.norm(), float(far.norm() / ref.norm())


@pytest.mark.parametrize("M", [1, 40])
def test_the_largest_numbers(hb, M):
    """Above 1.9375 * 2^127 an element rounds to a code times scale of 2^128: the products take code and scale apart and give its
    multiple; the weight gradient, which forms it, is infinite there and nowhere else."""
    x = torch.ones(M, 256, device="cuda")
    x[:, 3] = 3.4e38
    X = hb.fp8_quantize(x, hb.alloc_fp8_operand(M, 256))
    w = torch.zeros(24, 256, device="cuda")
    w[:, 3] = torch.arange(24, device="cuda") * 2.0 ** -100
    W = hb.fp8_quantize(w, hb.alloc_fp8_operand(24, 256, 128))
    y = hb.fp8_gemm(X, W, torch.empty(M, 24, device="cuda"))
    assert torch.equal(y.double(), (values(W)[:, 3] * 2.0 ** 128).expand(M, 24))          # of the weights as their codes hold them
    gw = hb.fp8_weight_grad(torch.ones(M, 24, dtype=torch.bfloat16, device="cuda"), X, torch.empty(24, 256, device="cuda"))
    want = torch.full((24, 256), float(M), device="cuda")
    want[:, :128] = 0.0                                    # ones beside 2^128: below the smallest code of its scale
    want[:, 3] = float("inf")
    assert torch.equal(gw, want)


@pytest.mark.parametrize("M", [3, 40, 300])
@pytest.mark.parametrize("scale", [float("nan"), float("inf"), 0.0, 2.0 ** -130, -2.0, 3.0])
def test_a_scale_matters_to_its_group_alone(hb, M, scale):
    """One group's scale in A, one block's in W: every other element of the product is what it was with ordinary ones, every
    element of theirs is the definition's, NaN and infinity included."""
    rng = np.random.default_rng(M)
    A, a, ca, sa = fu.held(rng.integers(1, 9, (M, 700)).astype(np.float32), 1)
    W, w, cw, sw = fu.held(rng.integers(1, 9, (260, 700)).astype(np.float32), 128)
    plain = hb.fp8_gemm(A, W, torch.empty(M, 260, device="cuda")).cpu().numpy()
    A.scales[M // 2, 4] = scale
    W.scales[1, 2] = scale
    got = hb.fp8_gemm(A, W, torch.empty(M, 260, device="cuda")).cpu().numpy()
    sa[M // 2, 4] = sw[1, 2] = np.float32(scale)
    with np.errstate(all="ignore"):
        ref = fu.values(ca, sa, 1) @ fu.values(cw, sw, 128).T
    same = np.ones_like(plain, dtype=bool)
    same[M // 2] = False
    same[:, 128:256] = False
    assert np.array_equal(got[same], plain[same])
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isinf(got), np.isinf(ref))
    fin = np.isfinite(ref)
    assert np.allclose(got[fin], ref[fin], rtol=1e-6, atol=0)

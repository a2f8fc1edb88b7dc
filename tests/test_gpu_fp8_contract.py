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

"""The failure path of the 8-bit kernels' bounded waits: as test_zy_wait_expiry.py, with the waits of the products (codes 400 +) and of
the weight gradient (500 +) on barriers that guard nothing.  Collected late, so that a word left set cannot fail unrelated tests."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hb():
    from paper_1905_10759_b200 import hbmm
    assert hbmm.last_device_error() == 0
    yield hbmm
    hbmm.debug_set_wait_limit(0)
    hbmm.clear_device_error()
    assert hbmm.last_device_error() == 0


def step(hb):
    """A product, an input gradient and a weight gradient of small whole numbers, exact in every format."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    M, N, K = 300, 264, 640
    x, w, g = (torch.randint(-4, 5, s, generator=gen, device="cuda").float() for s in ((M, K), (N, K), (M, N)))
    X, G = (hb.fp8_quantize(t, hb.alloc_fp8_operand(*t.shape)) for t in (x, g))
    W = hb.fp8_quantize(w, hb.alloc_fp8_operand(N, K, 128))
    y, gx, gw = torch.empty(M, N, device="cuda"), torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda")
    hb.fp8_gemm(X, W, y), hb.fp8_input_grad(G, W, gx), hb.fp8_weight_grad(g.bfloat16(), X, gw)
    for got, want in ((y, x.double() @ w.double().t()), (gx, g.double() @ w.double()), (gw, g.double().t() @ x.double())):
        assert torch.equal(got.double(), want)


@pytest.mark.parametrize("family,other", [(400, 500), (500, 400)])
def test_a_wait_that_runs_out_is_reported_then_cleared(hb, family, other):
    hb.debug_set_wait_limit(300)
    hb.debug_expire_wait_of(family)
    torch.cuda.synchronize()                       # the kernel returned by itself
    code = hb._i32(0)
    assert hb._lib.hbmm_last_device_error(code) == hb.ERR_TIMEOUT and code.value == family + 9
    hb.debug_expire_wait_of(family)                # sticky
    assert hb.last_device_error() == family + 9
    hb.debug_set_wait_limit(0)                     # no real kernel runs under a lowered limit
    step(hb)                                       # calls behind it do their work and leave the word as it is
    assert hb.last_device_error() == family + 9
    hb.debug_set_wait_limit(300)
    hb.clear_device_error()
    assert hb._lib.hbmm_last_device_error(code) == hb.OK and code.value == 0
    hb.debug_expire_wait_of(other)                 # a word of its own
    assert hb.last_device_error() == other + 9
    hb.clear_device_error()
    hb.debug_set_wait_limit(0)                     # back to the default limit
    step(hb)
    assert hb.last_device_error() == 0


def test_the_limit_in_force_is_each_family_s_own_copy_of_the_same(hb):
    """With the limit raised again the wait takes longer: the hook reaches both kernel files."""
    def took(family):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        hb.debug_expire_wait_of(family)
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b)
    for family in (400, 500):
        hb.debug_set_wait_limit(10)
        took(family)
        short = min(took(family) for _ in range(3))
        hb.debug_set_wait_limit(10000)
        long = took(family)
        assert long > 5 * short, (family, short, long)
    hb.debug_set_wait_limit(0)
    hb.clear_device_error()

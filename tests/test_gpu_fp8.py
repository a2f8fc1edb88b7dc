"""8-bit operands on the GPU, through the public functions, against the reference of fp8_util in 64 bits."""
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


def normal(rows, K, seed, outliers=True):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, K)).astype(np.float32)
    return x * np.where(rng.random(K) < 0.02, 20, 1).astype(np.float32) if outliers else x


# ------------------------------------------------------------------------------------------------------- quantize
SPECIAL = np.array([0.0, -0.0, 1e-45, -1e-45, 1e-38, -3e-39, 448.0, 448.00003, -1e30, 3.4e38, -3.4e38, np.inf, -np.inf, np.nan, 1.0, -1.0,
                    2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -10, -2.0 ** -30, 2.0 ** -117 * 448], dtype=np.float32)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,K,pad,offset", [
    (1, 1, 0, 0), (1, 4096, 0, 0), (3, 127, 0, 0), (5, 128, 8, 0), (2, 129, 0, 0), (130, 260, 4, 0), (257, 1023, 1, 1), (7, 1025, 3, 3),
    (128, 512, 0, 0), (40, 640, 8, 8), (300, 77, 0, 5),
])
def test_quantize(hb, rows, K, pad, offset, dtype, block_rows):
    """Bit for bit: the only rounding is the conversion's.  Padded rows, starts off any vector boundary, special values."""
    x = normal(rows, K, rows + K)
    x[rows // 2] *= np.float32(2.0) ** np.random.default_rng(K).integers(-60, 60)
    x[rows // 3, : min(K, len(SPECIAL))] = SPECIAL[:K]
    x[rows - 1] = np.where(np.arange(K) < 128, -0.0, x[rows - 1])          # a group of nothing but negative zeros
    buf = torch.full((rows * (K + pad) + offset,), 7e37, dtype=torch.float32)
    t = buf[offset:].view(rows, K + pad)
    t[:, :K] = torch.from_numpy(x)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    dev = buf.to(dt).cuda()[offset:].view(rows, K + pad)[:, :K]
    codes, s = fu.quantize(dev.float().cpu().numpy(), block_rows)
    op = hb.alloc_fp8_operand(rows, K, block_rows)
    op.codes.view(torch.uint8).fill_(0x55)
    op.scales.fill_(-1.0)
    assert hb.fp8_quantize(dev, op) is op
    got, gs = op.codes.view(torch.uint8).cpu().numpy(), op.scales.cpu().numpy()
    assert np.array_equal(gs[:, : s.shape[1]], s.astype(np.float32))
    nan = (codes & 0x7F) == 0x7F
    assert np.array_equal((got[:, :K] & 0x7F) == 0x7F, nan)
    assert np.array_equal(got[:, :K][~nan], codes[~nan])
    assert (got[:, K:] == 0x55).all() and (gs[:, s.shape[1]:] == -1).all()


def test_quantize_into_uint8_codes(hb):
    x = torch.from_numpy(normal(5, 300, 3)).cuda()
    a, b = hb.alloc_fp8_operand(5, 300), hb.alloc_fp8_operand(5, 300)
    b.codes = b.codes.view(torch.uint8)
    hb.fp8_quantize(x, a), hb.fp8_quantize(x, b)
    assert torch.equal(a.codes.view(torch.uint8)[:, :300], b.codes[:, :300])


# ------------------------------------------------------------------------------------------------------- products
def product_bound(F, ref, G, out):
    """A group's 128 products (exact in fp32) summed by the tensor core, each addition at most one fp32 step off (truncated: 2 u),
    the two scales multiplied and applied (2 u), G groups added (u each); F = sum |a| |w|.  bf16: half a step more of the result."""
    e = (2 * 128 + 2 + G) * fu.U * F
    return e + (fu.BF16 * (np.abs(ref) + e) if out == "bf16" else 0.0)


PRODUCTS = [(1, 1, 1), (1, 16, 16), (1, 1000, 4096), (2, 130, 257), (3, 4096, 300), (8, 72, 1111), (9, 200, 384), (16, 128, 128), (17, 64, 128),
            (31, 1000, 500), (33, 300, 640), (64, 129, 1000), (100, 520, 2100), (127, 256, 130), (128, 128, 1024), (129, 257, 384), (256, 1000, 4096),
            (257, 513, 129), (300, 520, 1111), (700, 384, 640), (1025, 136, 72), (1, 4096, 9216), (513, 2304, 16)]


@pytest.mark.parametrize("M,N,K", PRODUCTS)
@pytest.mark.parametrize("out,scales", [("fp32", "pow2"), ("bf16", "any")])
def test_gemm(hb, M, N, K, out, scales):
    A, a, _, _ = fu.held(normal(M, K, M + K), 1, scales, pad=16)
    W, w, _, _ = fu.held(normal(N, K, N + K + 1, False), 128, scales)
    C, clean = fu.framed(M, N, torch.float32 if out == "fp32" else torch.bfloat16, 8)
    assert hb.fp8_gemm(A, W, C) is C
    ref, F = a @ w.T, np.abs(a) @ np.abs(w).T
    err = np.abs(C.double().cpu().numpy() - ref)
    assert (err <= product_bound(F, ref, -(-K // 128), out)).all(), err.max()
    assert clean()


@pytest.mark.parametrize("M,N,K", PRODUCTS)
@pytest.mark.parametrize("out,scales", [("fp32", "pow2"), ("bf16", "any")])
def test_input_grad(hb, M, N, K, out, scales):
    G, g, _, _ = fu.held(normal(M, N, M + N) * 1e-3, 1, scales)
    W, w, _, _ = fu.held(normal(N, K, N + K + 2, False), 128, scales, pad=32)
    GX, clean = fu.framed(M, K, torch.float32 if out == "fp32" else torch.bfloat16, 8)
    assert hb.fp8_input_grad(G, W, GX) is GX
    ref, F = g @ w, np.abs(g) @ np.abs(w)
    err = np.abs(GX.double().cpu().numpy() - ref)
    assert (err <= product_bound(F, ref, -(-N // 128), out)).all(), err.max()
    assert clean()


@pytest.mark.parametrize("M,N,K", [(1, 8, 1), (1, 1000, 4096), (2, 136, 257), (5, 64, 128), (63, 128, 300), (64, 256, 256), (65, 264, 1000),
                                   (256, 1000, 4096), (300, 520, 1111), (513, 8, 640), (1000, 72, 130), (2500, 256, 384), (4097, 40, 72)])
@pytest.mark.parametrize("base", ["none", "other", "itself"])
def test_weight_grad(hb, M, N, K, base):
    X, x, _, _ = fu.held(normal(M, K, M + K), 1, pad=16)
    gy = torch.from_numpy(normal(M, N, M + N + 3) * 1e-2).to(torch.bfloat16)
    gyd = torch.full((M, N + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    gyd[:, :N] = gy.cuda()
    g = gy.double().numpy()
    GW, clean = fu.framed(N, K, torch.float32, 4)
    b, ref = None, g.T @ x
    if base != "none":
        b0 = torch.from_numpy(normal(N, K, N + K, False)).cuda()
        if base == "itself":
            GW.copy_(b0)
            b = GW
        else:
            b = torch.full((N, -(-K // 4) * 4 + 8), float("nan"), device="cuda")[:, :K]
            b.copy_(b0)
        ref = ref + b0.double().cpu().numpy()
    assert hb.fp8_weight_grad(gyd[:, :N], X, GW, base=b) is GW
    # products of bf16 numbers are exact in fp32; M additions at most a step (2 u) off each, one more for the base
    bound = (2 * M + 2) * fu.U * (np.abs(g).T @ np.abs(x)) + fu.U * np.abs(ref) + 1e-38
    err = np.abs(GW.double().cpu().numpy() - ref)
    assert (err <= bound).all(), (err / bound).max()
    assert clean()
    if base == "other":
        assert torch.equal(b, b0)


@pytest.mark.parametrize("M,N,K,base", [(300, 2600, 2300, True), (8300, 2304, 2310, False), (16500, 2200, 2600, True)])
def test_weight_grad_of_many_tiles(hb, M, N, K, base):
    """More tiles than the machine holds at once, rows and groups of their own magnitude, and more rows than one accumulator takes."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(M)
    x = torch.randn(M, K, generator=gen, device="cuda") * torch.exp2(torch.randint(-8, 8, (M, 1), generator=gen, device="cuda").float())
    x *= torch.exp2(torch.randint(-6, 6, (1, -(-K // 128)), generator=gen, device="cuda").float()).repeat_interleave(128, 1)[:, :K]
    gy = (torch.randn(M, N, generator=gen, device="cuda") * torch.exp2(torch.randint(-8, 8, (1, N), generator=gen, device="cuda").float())).bfloat16()
    X = hb.fp8_quantize(x, hb.alloc_fp8_operand(M, K))
    xv, g = on_device((X,)), gy.double()
    GW, clean = fu.framed(N, K, torch.float32, 4)
    b = torch.randn(N, -(-K // 4) * 4, generator=gen, device="cuda")[:, :K] if base else None
    hb.fp8_weight_grad(gy, X, GW, base=b)
    ref = g.t() @ xv
    bound = (2 * M + 2) * fu.U * (g.abs().t() @ xv.abs())
    if base:
        ref += b.double()
    bound += 2 * fu.U * ref.abs() * (M // 8192 + 1)
    assert ((GW.double() - ref).abs() <= bound).all()
    # far inside that bound where nothing cancels: the sums' errors do not pile up row by row
    assert (GW.double() - ref).norm() <= 4e-6 * ref.norm()
    assert clean()
    again = torch.full((N, -(-K // 4) * 4), float("nan"), device="cuda")[:, :K]
    assert torch.equal(hb.fp8_weight_grad(gy, X, again, base=b), GW)


@pytest.mark.parametrize("M,N,K", [(8192, 2304, 2304), (3000, 1024, 1024), (256, 4096, 2304)])
def test_weight_grad_again_and_again(hb, M, N, K):
    """The same bits every time, with the operands in L2 and with other data in their place."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N)
    X = hb.fp8_quantize(torch.randn(M, K, generator=gen, device="cuda"), hb.alloc_fp8_operand(M, K))
    gy = torch.randn(M, N, generator=gen, device="cuda").bfloat16()
    first = hb.fp8_weight_grad(gy, X, torch.empty(N, K, device="cuda"))
    ref = gy.double().t() @ on_device((X,))
    assert (first.double() - ref).norm() <= 2e-6 * ref.norm()      # 512 rows' truncated sums: 32 instructions of a step each at most
    spoil = torch.empty(1 << 26, device="cuda")
    for i in range(60):
        if i % 3 == 0:
            spoil.fill_(float("nan"))
        GW = torch.full((N, K), float("nan"), device="cuda")
        if i % 2:
            GW.zero_()
        assert torch.equal(hb.fp8_weight_grad(gy, X, GW, base=GW if i % 2 else None), first), i


def test_weight_grad_rounds_other_scales_to_bf16(hb):
    """Scales that are no powers of two: X^ is the bf16 number next to code times scale."""
    X, x, _, _ = fu.held(normal(200, 300, 5), 1, "any")
    x = torch.from_numpy(x).float().to(torch.bfloat16).double().numpy()
    gy = torch.from_numpy(normal(200, 64, 6)).to(torch.bfloat16)
    g = gy.double().numpy()
    GW = torch.empty(64, 300, device="cuda")
    hb.fp8_weight_grad(gy.cuda(), X, GW)
    # code * scale is rounded to fp32 before it is rounded to bf16: next to a bf16 midpoint the two roundings may end a step apart
    bound = (2 * 200 + 2) * fu.U * (np.abs(g).T @ np.abs(x)) + 2 * fu.U * 2 ** 16 * (np.abs(g).max(axis=0)[:, None] * np.abs(x).max(axis=0)[None])
    assert (np.abs(GW.double().cpu().numpy() - g.T @ x) <= bound).all()


def on_device(held):
    """An operand's values in 64 bits on the device, from its codes and scales by torch's own conversions."""
    op = held[0]
    return op.codes.view(torch.float8_e4m3fn)[:, :op.K].double() * op.scales.double().repeat_interleave(op.block_rows, 0)[:op.rows].repeat_interleave(128, 1)[:, :op.K]


@pytest.mark.parametrize("kind", ["gemm", "input_grad"])
@pytest.mark.parametrize("M,N,K,scales", [(2600, 2300, 640, "pow2"), (5000, 2050, 130, "pow2"), (2600, 2300, 640, "any"), (2600, 2300, 640, "mixed"),
                                          (1300, 4100, 2500, "mixed"), (2100, 2100, 1100, "pow2")])
def test_products_of_many_tiles(hb, M, N, K, scales, kind):
    """More tiles than the machine holds at once, every row, column block and group of its own magnitude: a scale, a partial sum or
    a staged row of another tile shows.  mixed: some groups' scales are powers of two and some are not."""
    rng = np.random.default_rng(M + N)
    n_a, rows_w, cols_w = (K, N, K) if kind == "gemm" else (N, N, K)

    def spreads(rows, cols, per_row, per_col):
        e = rng.integers(-12, 12, (-(-rows // per_row), 1)).repeat(per_row, 0)[:rows] + rng.integers(-6, 6, (1, -(-cols // per_col))).repeat(per_col, 1)[:, :cols]
        return np.exp2(e).astype(np.float32)
    A = fu.held(normal(M, n_a, M + 1, False) * spreads(M, n_a, 1, 128), 1)
    W = fu.held(normal(rows_w, cols_w, N + 2, False) * spreads(rows_w, cols_w, 128, 128), 128)
    for op, br in ((A[0], 1), (W[0], 128)):
        s = op.scales
        if scales != "pow2":
            f = torch.from_numpy(rng.uniform(1.0, 1.99, tuple(s.shape)).astype(np.float32)).cuda()
            if scales == "mixed":                              # whole runs of groups, and single entries of others
                keep = torch.from_numpy(rng.random((1, s.shape[1])) < 0.6).cuda() | (torch.from_numpy(rng.random(tuple(s.shape)) < 0.998).cuda())
                f = torch.where(keep, 1.0, f)
            s.mul_(f)
    a, w = on_device(A), on_device(W)
    out, clean = fu.framed(M, N if kind == "gemm" else K, torch.float32, 8)
    (hb.fp8_gemm if kind == "gemm" else hb.fp8_input_grad)(A[0], W[0], out)
    w = w.t() if kind == "gemm" else w
    ref, F = a @ w, a.abs() @ w.abs()
    assert ((out.double() - ref).abs() <= product_bound(F, ref, -(-n_a // 128), "fp32")).all()
    assert clean()


@pytest.mark.parametrize("M,N,K,scales", [(256, 256, 640, "any"), (200, 500, 1500, "any"), (300, 1000, 4096, "any"), (300, 1000, 4096, "pow2"),
                                          (20, 136, 9216, "any"), (700, 700, 10000, "pow2")])
def test_products_of_few_tiles_again_and_again(hb, M, N, K, scales):
    """Tiles that several pairs share (and one accumulator after another along a long K): the same bits every time, whatever ran
    before."""
    A, a, _, _ = fu.held(normal(M, K, M + K), 1, scales)
    W, w, _, _ = fu.held(normal(N, K, N + K, False), 128, scales)
    first = hb.fp8_gemm(A, W, torch.empty(M, -(-N // 4) * 4, device="cuda")[:, :N])
    ref, F = a @ w.T, np.abs(a) @ np.abs(w).T
    assert (np.abs(first.double().cpu().numpy() - ref) <= product_bound(F, ref, -(-K // 128), "fp32")).all()
    spoil = torch.empty(1 << 26, device="cuda")
    for i in range(30):
        if i % 3 == 0:
            spoil.fill_(float("nan"))
        C = torch.full((M, -(-N // 4) * 4), float("nan"), device="cuda")[:, :N]
        assert torch.equal(hb.fp8_gemm(A, W, C), first), i


def test_a_nan_stays_in_its_row_and_column(hb):
    a, w = normal(150, 300, 11), normal(260, 300, 12, False)
    a[77, 200], w[130, 299] = np.nan, np.inf
    A, W = fu.held(a, 1)[0], fu.held(w, 128)[0]
    C = torch.empty(150, 264, device="cuda")[:, :260]
    bad = torch.isnan(hb.fp8_gemm(A, W, C))
    want = torch.zeros_like(bad)
    want[77], want[:, 130] = True, True
    assert torch.equal(bad, want)
    G = fu.held(np.where(np.arange(260) == 130, 0, 1) * normal(150, 260, 13), 1)[0]
    GX = torch.empty(150, 304, device="cuda")[:, :300]
    bad = torch.isnan(hb.fp8_input_grad(G, W, GX))             # 0 * NaN in column 299, nowhere else
    want = torch.zeros_like(bad)
    want[:, 299] = True
    assert torch.equal(bad, want)
    GW = torch.empty(64, 300, device="cuda")
    bad = torch.isnan(hb.fp8_weight_grad(torch.ones(150, 64, dtype=torch.bfloat16, device="cuda"), A, GW))
    want = torch.zeros_like(bad)
    want[:, 200] = True
    assert torch.equal(bad, want)


def test_extreme_scales(hb):
    """Groups of the largest and the smallest numbers: x / s and code * s stay exact, the products finite."""
    x = normal(130, 384, 21, False)
    x[:, :128] *= 1e37
    x[:, 128:256] *= 1e-36
    A, a, _, _ = fu.held(x, 1)
    W, w, _, _ = fu.held(normal(140, 384, 22, False) * 1e-3, 128)
    C = hb.fp8_gemm(A, W, torch.empty(130, 140, device="cuda"))
    ref, F = a @ w.T, np.abs(a) @ np.abs(w).T
    assert (np.abs(C.double().cpu().numpy() - ref) <= product_bound(F, ref, 3, "fp32")).all()
    gy = torch.full((130, 8), 0.5, dtype=torch.bfloat16, device="cuda")
    GW = hb.fp8_weight_grad(gy, A, torch.empty(8, 384, device="cuda"))
    ref = 0.5 * np.ones((8, 130)) @ a
    assert (np.abs(GW.double().cpu().numpy() - ref) <= (2 * 130 + 3) * fu.U * 0.5 * np.abs(a).sum(axis=0) + 1e-44).all()


# ------------------------------------------------------------------------------------------------- binarize backward
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,K,beta,pad", [
    (1, 1, 1, 0), (9, 131, 1, 0), (9, 131, 2, 0), (5, 260, 4, 4), (3, 388, 8, 1), (7, 1000, 16, 0), (33, 512, 32, 8), (5, 777, 64, 0), (9, 640, 128, 0),
    (3, 100, 128, 4), (4, 300, 300, 0), (4, 300, 5000, 0), (5, 1000, 3, 0), (5, 1000, 48, 8), (2, 4000, 1500, 0), (6, 900, 256, 3), (1, 9216, 9216, 0),
])
def test_binarize_backward(hb, rows, K, beta, pad, dtype):
    x = normal(rows, K, rows + K)
    x[0, : min(K, 5)] = [1.0, -1.0, 0.0, -0.0, -1e-30][:K]      # the last keeps its sign in a zero code
    X, _, codes, s = fu.held(x, 1, pad=16)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    gy = torch.from_numpy(normal(rows, K, K + beta, False)).to(dt)
    gd = torch.full((rows, K + pad), float("nan"), dtype=dt, device="cuda")
    gd[:, :K] = gy.cuda()
    ref, mag = fu.binarize_backward(codes, s, gy.double().numpy(), min(beta, K))
    n = min(beta, K)
    tree = int(np.ceil(np.log2(max(n, 2)))) + int(np.ceil(n / 4)) + 8   # additions in a row at most: a lane's run, then trees
    bound = (tree + 4) * fu.U * mag + 1e-30
    bound = bound + (fu.BF16 * (np.abs(ref) + bound) if dtype == "bf16" else 0)
    out = torch.full((rows + 1, K + pad), float("nan"), dtype=dt, device="cuda")
    got = hb.fp8_binarize_backward(X, gd[:, :K], beta, out[:rows, :K])
    assert (np.abs(got.double().cpu().numpy() - ref) <= bound).all()
    assert torch.isnan(out[:, K:]).all() and torch.isnan(out[rows:]).all()
    assert torch.equal(hb.fp8_binarize_backward(X, gd[:, :K], beta), got)          # allocated by the call


def test_binarize_backward_is_the_fp32_one_where_nothing_was_rounded(hb):
    """x of e4m3 numbers: the checkpoint loses nothing, so the gradient is the one from x itself."""
    x = fu.decode(np.random.default_rng(3).integers(0, 127, (64, 640)).astype(np.uint8)) * np.where(np.arange(640) % 3, 1, -1)
    x = torch.from_numpy(np.clip(x, -1.5, 1.5)).float().cuda()
    gy = torch.from_numpy(normal(64, 640, 4)).cuda()
    X = hb.fp8_quantize(x, hb.alloc_fp8_operand(64, 640))
    assert torch.equal(hb.fp8_binarize_backward(X, gy, 32), hb.binarize_backward(x, gy, 32))


# ------------------------------------------------------------------------------------------------- used together
def layer(hb, M, N, K, seed):
    """One layer's step as a program runs it: both quantizations, the product, both gradients, the gradient through the binarizer."""
    d = {"x": torch.from_numpy(normal(M, K, seed)).cuda(), "w": torch.from_numpy(normal(N, K, seed + 1, False) * K ** -0.5).cuda(),
         "gy": torch.from_numpy(normal(M, N, seed + 2, False) * 1e-2).to(torch.bfloat16).cuda(),
         "X": hb.alloc_fp8_operand(M, K), "W": hb.alloc_fp8_operand(N, K, 128), "G": hb.alloc_fp8_operand(M, N),
         "y": torch.empty(M, N, dtype=torch.bfloat16, device="cuda"), "gx": torch.empty(M, K, device="cuda"),
         "gw": torch.zeros(N, K, device="cuda"), "gb": torch.empty(M, K, device="cuda")}

    def step(stream=None):
        hb.fp8_quantize(d["x"], d["X"], stream=stream)
        hb.fp8_quantize(d["w"], d["W"], stream=stream)
        hb.fp8_gemm(d["X"], d["W"], d["y"], stream=stream)
        hb.fp8_quantize(d["gy"], d["G"], stream=stream)
        hb.fp8_input_grad(d["G"], d["W"], d["gx"], stream=stream)
        hb.fp8_weight_grad(d["gy"], d["X"], d["gw"], base=d["gw"], stream=stream)
        hb.fp8_binarize_backward(d["X"], d["gx"], 32, d["gb"], stream=stream)
    return d, step


def check_layer(d, before):
    x, w, gy = (d[n].double().cpu().numpy() for n in ("x", "w", "gy"))
    cx, sx = fu.quantize(x, 1)
    xv, wv, gv = fu.values(cx, sx, 1), fu.values(*fu.quantize(w, 128), 128), fu.values(*fu.quantize(gy, 1), 1)
    groups = lambda n: -(-n // 128)  # noqa: E731
    y = xv @ wv.T
    assert (np.abs(d["y"].double().cpu().numpy() - y) <= product_bound(np.abs(xv) @ np.abs(wv).T, y, groups(w.shape[1]), "bf16")).all()
    gx = gv @ wv
    e = product_bound(np.abs(gv) @ np.abs(wv), gx, groups(w.shape[0]), "fp32")
    assert (np.abs(d["gx"].double().cpu().numpy() - gx) <= e).all()
    gw = gy.T @ xv + before
    assert (np.abs(d["gw"].double().cpu().numpy() - gw) <= (2 * x.shape[0] + 2) * fu.U * (np.abs(gy).T @ np.abs(xv)) + fu.U * np.abs(gw)).all()
    gb, mag = fu.binarize_backward(cx, sx, d["gx"].double().cpu().numpy(), 32)
    assert (np.abs(d["gb"].double().cpu().numpy() - gb) <= 20 * fu.U * mag + 1e-30).all()


@pytest.mark.parametrize("M,N,K", [(1, 136, 300), (200, 264, 520), (64, 1000, 256)])
def test_layer_step(hb, M, N, K):
    d, step = layer(hb, M, N, K, M + N)
    step()
    check_layer(d, 0.0)
    first = d["gw"].clone()
    step()                                               # the gradient of a second batch on top of the first
    check_layer(d, first.double().cpu().numpy())


def test_layer_step_on_streams_and_in_graphs(hb):
    """Two steps on streams of their own at once, and two captured ones replayed with other inputs, give what one alone gives."""
    sizes = [(200, 264, 520), (130, 400, 384)]
    alone = []
    for i, s in enumerate(sizes):
        d, step = layer(hb, *s, 50 + i)
        step()
        alone.append(d)
    torch.cuda.synchronize()
    names = ("y", "gx", "gw", "gb")
    both = [layer(hb, *s, 50 + i) for i, s in enumerate(sizes)]
    streams = [torch.cuda.Stream() for _ in sizes]
    torch.cuda.synchronize()
    for (d, step), st in zip(both, streams):
        step(st)
    torch.cuda.synchronize()
    for (d, _), a in zip(both, alone):
        assert all(torch.equal(d[n], a[n]) for n in names)
    graphs = []
    for i, s in enumerate(sizes):
        d, step = layer(hb, *s, 70 + i)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append((d, g))
    for (d, g), (src, _), st in zip(graphs, both, streams):
        for n in ("x", "w", "gy"):
            d[n].copy_(src[n])
        d["gw"].zero_()
    torch.cuda.synchronize()
    for (d, g), st in zip(graphs, streams):
        with torch.cuda.stream(st):
            g.replay()
    torch.cuda.synchronize()
    for (d, _), a in zip(graphs, alone):
        assert all(torch.equal(d[n], a[n]) for n in names)


def test_weight_gradient_is_the_derivative(hb):
    """Loss <Y, R>: its difference along a direction of W is <GW, direction>; the product is linear in W^, so a difference of any
    length is the derivative but for rounding."""
    M, N, K = 40, 64, 256
    X, x, _, _ = fu.held(normal(M, K, 1), 1)
    R = torch.from_numpy(normal(M, N, 2, False)).to(torch.bfloat16)
    r = R.double().numpy()
    GW = hb.fp8_weight_grad(R.cuda(), X, torch.empty(N, K, device="cuda")).double().cpu().numpy()
    Y, F, w = [], [], []
    for seed in (3, 4):
        W, v, _, _ = fu.held(normal(N, K, seed, False), 128)
        Y.append(hb.fp8_gemm(X, W, torch.empty(M, N, device="cuda")).double().cpu().numpy())
        F.append((np.abs(x) @ np.abs(v).T * np.abs(r)).sum())
        w.append(v)
    along = ((w[1] - w[0]) * GW).sum()
    bound = (2 * 128 + 4) * fu.U * (F[0] + F[1]) + (2 * M + 3) * fu.U * (np.abs(w[1] - w[0]) * (np.abs(r).T @ np.abs(x))).sum()
    assert abs((Y[1] * r).sum() - (Y[0] * r).sum() - along) <= bound


def test_input_gradient_is_the_derivative(hb):
    M, N, K = 30, 200, 260
    W, w, _, _ = fu.held(normal(N, K, 1, False), 128)
    G, g, _, _ = fu.held(normal(M, N, 2, False), 1)
    GX = hb.fp8_input_grad(G, W, torch.empty(M, K, device="cuda")).double().cpu().numpy()
    Y, F, x = [], 0.0, []
    for seed in (3, 4):
        X, v, _, _ = fu.held(normal(M, K, seed), 1)
        Y.append(hb.fp8_gemm(X, W, torch.empty(M, N, device="cuda")).double().cpu().numpy())
        F += (np.abs(v) @ np.abs(w).T * np.abs(g)).sum()
        x.append(v)
    along = ((x[1] - x[0]) * GX).sum()
    bound = (2 * 128 + 5) * fu.U * F + (2 * 128 + 4) * fu.U * (np.abs(x[1] - x[0]) * (np.abs(g) @ np.abs(w))).sum()
    assert abs(((Y[1] - Y[0]) * g).sum() - along) <= bound


def test_refusals_on_the_device(hb):
    x = torch.zeros(8, 256, device="cuda")
    X, W = hb.fp8_quantize(x, hb.alloc_fp8_operand(8, 256)), hb.fp8_quantize(torch.zeros(64, 256, device="cuda"), hb.alloc_fp8_operand(64, 256, 128))
    for call, error in [
        (lambda: hb.fp8_quantize(x[:, :255], X), ValueError), (lambda: hb.fp8_quantize(x.double(), X), TypeError),
        (lambda: hb.fp8_quantize(x.t(), X), ValueError),
        (lambda: hb.fp8_gemm(X, W, x), ValueError), (lambda: hb.fp8_gemm(W, X, torch.zeros(64, 8, device="cuda")), hb.HbmmError),
        (lambda: hb.fp8_gemm(X, W, torch.zeros(8, 65, device="cuda")[:, 1:]), hb.HbmmError),
        (lambda: hb.fp8_gemm(X, W, torch.zeros(8, 64, dtype=torch.float16, device="cuda")), TypeError),
        (lambda: hb.fp8_gemm(X, W, torch.zeros(8, 64)), ValueError),
        (lambda: hb.fp8_input_grad(X, W, x), hb.HbmmError),
        (lambda: hb.fp8_weight_grad(torch.zeros(8, 64, device="cuda"), X, torch.zeros(64, 256, device="cuda")), hb.HbmmError),
        (lambda: hb.fp8_weight_grad(torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda"), X, torch.zeros(64, 256, device="cuda").bfloat16()), ValueError),
        (lambda: hb.fp8_weight_grad(torch.zeros(7, 64, dtype=torch.bfloat16, device="cuda"), X, torch.zeros(64, 256, device="cuda")), ValueError),
        (lambda: hb.fp8_binarize_backward(X, x, 0), hb.HbmmError), (lambda: hb.fp8_binarize_backward(X, x, 32, x.bfloat16()), ValueError),
        (lambda: hb.fp8_binarize_backward(W, torch.zeros(64, 256, device="cuda"), 32), hb.HbmmError),
    ]:
        with pytest.raises(error):
            call()

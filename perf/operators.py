"""The 8-bit linear layer of training and serving, as operators to be timed.

A tensor in 8 bits is a matrix of e4m3 codes with one fp32 scale for each group of 128 consecutive elements of a row
(activations, gradients: ``block_rows`` 1) or each block of 128 x 128 elements (weights: ``block_rows`` 128).  The layer

* quantizes its activations (``quantize``), which then serve twice: the product reads them, and they are the checkpoint
  that the backward pass reads in place of the activations themselves,
* forms Y = X^ W^T (``product``), for one token up to long batches,
* backwards, GX = GY^ W^ (``input_grad``) from the quantized gradient, GW = GY^T X^ (``weight_grad``) from the checkpoint,
  and, where the activations were binarized, the gradient through the binarizer (``binarize_backward``) from it too.

Scales written by the quantizer are powers of two; the products take any.
"""
import math

import torch

own = False

GROUP = 128        # elements per scale
TOP = 448.0        # largest e4m3 value


# --------------------------------------------------------------------------------------------------------------
# Cases
# --------------------------------------------------------------------------------------------------------------
def _quantize(rows, K, x, block_rows):
    return {"op": "quantize", "rows": rows, "K": K, "x": x, "block_rows": block_rows}


def _product(M, N, K, out, scales="pow2"):
    return {"op": "product", "M": M, "N": N, "K": K, "out": out, "scales": scales}


def _input_grad(M, N, K, out, scales="pow2"):
    return {"op": "input_grad", "M": M, "N": N, "K": K, "out": out, "scales": scales}


def _weight_grad(M, N, K, accumulate):
    return {"op": "weight_grad", "M": M, "N": N, "K": K, "accumulate": accumulate}


def _binarize_backward(rows, K, beta, g):
    return {"op": "binarize_backward", "rows": rows, "K": K, "beta": beta, "g": g}


def listed():
    return [
        # a long batch of activations on its way into a large layer, and into the checkpoint
        dict(_quantize(8192, 8192, "bf16", 1), name="quantize_rows_8192"),
        # the first fully connected layer's weights, quantized again after each optimiser step
        dict(_quantize(4096, 9216, "fp32", 128), name="quantize_blocks_fc"),
        # one token through the last layer of the fully connected stack: latency
        dict(_product(1, 1000, 4096, "fp32"), name="product_b1_last"),
        # one token through its first layer: weights read once
        dict(_product(1, 4096, 9216, "bf16"), name="product_b1_first"),
        # a batch of no round size, weights and scales quantized elsewhere
        dict(_product(333, 4096, 9216, "bf16", "fp32"), name="product_b333"),
        # the largest square product of the configurations
        dict(_product(8192, 8192, 8192, "bf16"), name="product_8192"),
        # backward of the last layer on a batch: ragged contraction
        dict(_input_grad(256, 1000, 4096, "bf16"), name="input_grad_b256"),
        # backward of a square layer on a long batch
        dict(_input_grad(8192, 4096, 4096, "bf16"), name="input_grad_4096"),
        # first layer on a batch, added to the gradient of the batches before: output traffic
        dict(_weight_grad(256, 4096, 9216, 1), name="weight_grad_b256"),
        # square layer, long batch: tensor cores
        dict(_weight_grad(8192, 4096, 4096, 0), name="weight_grad_4096"),
        # a small layer's activations at one of the paper's group sizes, rows of no round length
        dict(_binarize_backward(333, 1000, 16, "fp32"), name="binarize_bwd_ragged"),
        # a large layer's activations, gradients in bf16
        dict(_binarize_backward(8192, 8192, 32, "bf16"), name="binarize_bwd_8192"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A width: a multiple of 128 for a third of the cases, of 8 for another, anything otherwise."""
    v = _log_int(rng, lo, hi)
    step = rng.choice((128, 8, 1))
    return max(lo, v // step * step)


def draw(rng):
    op = rng.choice(("quantize", "product", "product", "input_grad", "weight_grad", "binarize_backward"))
    rows = _log_int(rng, 1, 8192)
    if op == "quantize":
        block_rows = rng.choice((1, 128))
        rows = rows if block_rows == 1 else _size(rng, 16, 8192)
        return _quantize(rows, _size(rng, 16, 8192), rng.choice(("bf16", "fp32")), block_rows)
    if op == "binarize_backward":
        K = _size(rng, 16, 8192)
        return _binarize_backward(rows, K, rng.choice((2, 4, 8, 16, 32, 64, 128, K)), rng.choice(("bf16", "fp32")))
    while True:
        M, N, K = rows, _size(rng, 16, 8192), _size(rng, 16, 9216)
        if M * N * K <= 8192 ** 3:
            break
        rows = _log_int(rng, 1, 8192)
    if op == "weight_grad":
        return _weight_grad(M, -(-N // 8) * 8, K, rng.choice((0, 1)))       # rows of the bf16 gradient start on 16 bytes
    return (_product if op == "product" else _input_grad)(M, N, K, rng.choice(("bf16", "fp32")), rng.choice(("pow2", "fp32")))


# --------------------------------------------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------------------------------------------
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _round_up(v, step):
    return -(-v // step) * step


def _groups(n):
    return -(-n // GROUP)


def _activations(gen, rows, K):
    """N(0, 1) as a normalisation leaves it, a few channels much larger, as such layers have them."""
    x = torch.randn(rows, K, generator=gen, device="cuda")
    wide = torch.rand(K, generator=gen, device="cuda") < 0.01
    return x * torch.where(wide, 20.0, 1.0)


def _gradients(gen, rows, N):
    """Small, each row of its own size."""
    size = torch.exp(torch.randn(rows, 1, generator=gen, device="cuda"))
    return torch.randn(rows, N, generator=gen, device="cuda") * size * 1e-3


def _weights(gen, N, K):
    return torch.randn(N, K, generator=gen, device="cuda") * math.sqrt(2.0 / K)


def _held(x, block_rows, scales):
    """`x` as a program holds it in 8 bits: codes in rows of whole 16 bytes, scales in rows of whole float4."""
    rows, K = x.shape
    codes, s = _quantized(x, block_rows, scales)
    c = torch.zeros(rows, _round_up(K, 16), dtype=torch.float8_e4m3fn, device="cuda")
    c[:, :K] = codes
    t = torch.zeros(s.shape[0], _round_up(s.shape[1], 4), device="cuda")
    t[:, :s.shape[1]] = s
    return c, t


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    st = {"case": case}
    if op == "quantize":
        rows, K, br = case["rows"], case["K"], case["block_rows"]
        x = _activations(gen, rows, K) if br == 1 else _weights(gen, rows, K)
        st["x"] = x.to(TYPES[case["x"]])
        st["codes"] = torch.empty(rows, _round_up(K, 16), dtype=torch.float8_e4m3fn, device="cuda")
        st["scales"] = torch.empty(-(-rows // br), _round_up(_groups(K), 4), device="cuda")
        return st
    if op == "binarize_backward":
        rows, K = case["rows"], case["K"]
        st["x"] = _held(_activations(gen, rows, K), 1, "pow2")
        st["gy"] = _gradients(gen, rows, K).to(TYPES[case["g"]])
        st["gx"] = torch.empty_like(st["gy"])
        return st
    M, N, K = case["M"], case["N"], case["K"]
    if op == "product":
        st["a"] = _held(_activations(gen, M, K), 1, case["scales"])
        st["w"] = _held(_weights(gen, N, K), 128, case["scales"])
        st["out"] = torch.empty(M, _round_up(N, 8), dtype=TYPES[case["out"]], device="cuda")
    elif op == "input_grad":
        st["gy"] = _held(_gradients(gen, M, N), 1, case["scales"])
        st["w"] = _held(_weights(gen, N, K), 128, case["scales"])
        st["out"] = torch.empty(M, _round_up(K, 8), dtype=TYPES[case["out"]], device="cuda")
    else:
        st["gy"] = _gradients(gen, M, N).to(torch.bfloat16)
        st["x"] = _held(_activations(gen, M, K), 1, "pow2")
        st["gw"] = torch.empty(N, _round_up(K, 4), device="cuda")
        # what the batches before left; a training step may have it in the very buffer that it adds to
        st["before"] = _gradients(gen, N, _round_up(K, 4)) if case["accumulate"] else None
    return st


# --------------------------------------------------------------------------------------------------------------
# Plain forms
# --------------------------------------------------------------------------------------------------------------
def _tiles(x, block_rows):
    """[rows, K] -> [row blocks, block_rows, groups, 128], zeros behind the edges."""
    rows, K = x.shape
    pad = (0, _round_up(K, GROUP) - K, 0, _round_up(rows, block_rows) - rows)
    return torch.nn.functional.pad(x, pad).view(-1, block_rows, _groups(K), GROUP)


def _quantized(x, block_rows, scales="pow2"):
    """Codes and scales of `x`.  pow2: the smallest power of two that brings the largest magnitude to 448 or less, at least
    2^-117; fp32: the magnitude over 448, as other programs write them."""
    rows, K = x.shape
    x = x.float()
    finite = torch.isfinite(x)
    amax = _tiles(torch.where(finite, x, 0.0).abs(), block_rows).amax(dim=(1, 3))
    if scales == "pow2":
        m, e = torch.frexp(amax)                                   # amax = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
        e = (e - 9 + (m > 0.875).to(e.dtype)).clamp(min=-117)
        s = torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), 2.0 ** -117)
    else:
        s = amax.clamp(min=1e-30) / TOP
    v = x / _spread(s, block_rows, rows, K)
    return torch.where(finite, v, float("nan")).to(torch.float8_e4m3fn), s


def _spread(s, block_rows, rows, K):
    """One scale per element."""
    return s.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(GROUP, 1)[:, :K]


def _values(held, block_rows, K):
    codes, s = held
    return codes[:, :K].float() * _spread(s[:, :_groups(K)], block_rows, codes.shape[0], K)


def _binarize_backward_plain(held, gy, beta):
    rows, K = gy.shape
    x, g = _values(held, 1, K), gy.float()
    sign = torch.where(torch.signbit(held[0][:, :K].float()), -1.0, 1.0)
    n = -(-K // beta)
    length = torch.full((n, 1), float(beta), device=gy.device)
    length[-1] = K - (n - 1) * beta

    def mean(v):
        v = torch.nn.functional.pad(v, (0, n * beta - K)).view(rows, n, beta).sum(2, keepdim=True) / length
        return v.expand(rows, n, beta).reshape(rows, n * beta)[:, :K]

    gx = sign * mean(g * sign) + torch.where(x.abs() <= 1, mean(x.abs()) * g, 0.0)
    return gx.to(gy.dtype)


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_1905_10759_b200 import hbmm
        if op == "quantize":
            K = case["K"]
            q = hbmm.fp8_quantize(state["x"], hbmm.Fp8Operand(state["codes"], state["scales"], K, case["block_rows"]))
            return q.codes[:, :K], q.scales[:, :_groups(K)]
        if op == "product":
            K, N = case["K"], case["N"]
            return hbmm.fp8_gemm(hbmm.Fp8Operand(*state["a"], K, 1), hbmm.Fp8Operand(*state["w"], K, 128), state["out"][:, :N])
        if op == "input_grad":
            K, N = case["K"], case["N"]
            return hbmm.fp8_input_grad(hbmm.Fp8Operand(*state["gy"], N, 1), hbmm.Fp8Operand(*state["w"], K, 128), state["out"][:, :K])
        if op == "weight_grad":
            K, before = case["K"], state["before"]
            return hbmm.fp8_weight_grad(state["gy"], hbmm.Fp8Operand(*state["x"], K, 1), state["gw"][:, :K],
                                        base=None if before is None else before[:, :K])
        return hbmm.fp8_binarize_backward(hbmm.Fp8Operand(*state["x"], case["K"], 1), state["gy"], case["beta"], state["gx"])
    if op == "quantize":
        return _quantized(state["x"], case["block_rows"])
    if op == "product":
        a, w = _values(state["a"], 1, case["K"]), _values(state["w"], 128, case["K"])
        return (a @ w.t()).to(TYPES[case["out"]])
    if op == "input_grad":
        g, w = _values(state["gy"], 1, case["N"]), _values(state["w"], 128, case["K"])
        return (g @ w).to(TYPES[case["out"]])
    if op == "weight_grad":
        gw = state["gy"].float().t() @ _values(state["x"], 1, case["K"])
        return state["before"][:, :case["K"]] + gw if case["accumulate"] else gw
    return _binarize_backward_plain(state["x"], state["gy"], case["beta"])


def work(case):
    op = case["op"]
    if op == "quantize":
        rows, K = case["rows"], case["K"]
        size = 4 if case["x"] == "fp32" else 2
        return {"bytes": rows * K * (size + 1) + 4 * -(-rows // case["block_rows"]) * _groups(K), "flops": 3 * rows * K}
    if op == "binarize_backward":
        rows, K = case["rows"], case["K"]
        size = 4 if case["g"] == "fp32" else 2
        return {"bytes": rows * K * (1 + 2 * size) + 4 * rows * _groups(K), "flops": 8 * rows * K}
    M, N, K = case["M"], case["N"], case["K"]
    flops = 2 * M * N * K
    if op == "weight_grad":
        out = N * K * 4
        return {"bytes": 2 * M * N + M * K + 4 * M * _groups(K) + out * (2 if case["accumulate"] else 1), "flops": flops}
    size = 4 if case["out"] == "fp32" else 2
    inner, outer = (K, N) if op == "product" else (N, K)
    return {"bytes": M * inner + N * K + 4 * M * _groups(inner) + 4 * _groups(N) * _groups(K) + size * M * outer, "flops": flops}


# --------------------------------------------------------------------------------------------------------------
# From the definitions, in 64 bits
# --------------------------------------------------------------------------------------------------------------
def _exact_values(held, block_rows, K):
    codes, s = held
    at_row = torch.arange(codes.shape[0], device="cuda") // block_rows
    at_col = torch.arange(K, device="cuda") // GROUP
    return codes[:, :K].double() * s.double()[at_row][:, at_col]


def _exact_codes(x, block_rows):
    rows, K = x.shape
    x = x.double()
    R, G = -(-rows // block_rows), _groups(K)
    at_row = torch.arange(rows, device="cuda") // block_rows
    at_col = torch.arange(K, device="cuda") // GROUP
    amax = torch.zeros(rows, G, dtype=torch.float64, device="cuda").scatter_reduce(1, at_col.expand(rows, K), x.abs(), "amax")
    amax = torch.zeros(R, G, dtype=torch.float64, device="cuda").scatter_reduce(0, at_row[:, None].expand(rows, G), amax, "amax")
    e = torch.ceil(torch.log2(amax.clamp(min=1e-60) / TOP))
    e = torch.where(torch.exp2(e - 1) * TOP >= amax, e - 1, e)         # the logarithm next to a power of two
    e = torch.where(torch.exp2(e) * TOP < amax, e + 1, e).clamp(min=-117)
    s = torch.exp2(e)
    v = x / s[at_row][:, at_col]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -40))).clamp(min=-6) - 3)
    return torch.round(v / step) * step, s                             # ties to even, as e4m3's last bit


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        return _exact_codes(st["x"], case["block_rows"])
    if op == "product":
        return _exact_values(st["a"], 1, case["K"]) @ _exact_values(st["w"], 128, case["K"]).t()
    if op == "input_grad":
        return _exact_values(st["gy"], 1, case["N"]) @ _exact_values(st["w"], 128, case["K"])
    if op == "weight_grad":
        gw = st["gy"].double().t() @ _exact_values(st["x"], 1, case["K"])
        return gw + st["before"][:, :case["K"]].double() if case["accumulate"] else gw
    K, beta = case["K"], case["beta"]
    x, g = _exact_values(st["x"], 1, K), st["gy"].double()
    sign = torch.where(torch.signbit(st["x"][0][:, :K].double()), -1.0, 1.0)
    at = torch.arange(K, device="cuda") // beta
    n = int(at[-1]) + 1
    size = torch.zeros(n, dtype=torch.float64, device="cuda").index_add(0, at, torch.ones(K, dtype=torch.float64, device="cuda"))
    zero = torch.zeros(x.shape[0], n, dtype=torch.float64, device="cuda")
    delta, back = (zero.index_add(1, at, v) / size for v in (x.abs(), g * sign))
    return sign * back[:, at] + (x.abs() <= 1) * delta[:, at] * g

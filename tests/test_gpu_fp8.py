"""GPU tests of the layers in 8-bit floating point: rows to e4m3, products, the gated block and its gradients.

Plain implementations in 64 bits on the same e4m3 numbers.  Tolerances, with F32 = 2^-23 (a sum of n numbers in fp32, in any order and
with truncation, is off by at most n F32 of the sum of their absolute values) and u = half a step of the 16-bit type:

* a product's sum: 128 terms in a block, ceil(K / 128) blocks, three roundings of each block's scaling, bias and residual:
  (128 + ceil(K / 128) + 5) F32 of the sum of absolute values; then one rounding of y (in fp16 at least 2^-25, half its smallest step);
* the gated block: the errors of gate and up reach the result through silu (slope below 1.1) and the product; the logistic function is off by
  the fast exponential's (2 + 1.5 |gate|) F32 (two units in the last place, and the rounding of gate / ln 2) and two roundings, the products add
  three: (6 + 1.5 |gate|) F32 of the result.  Below 2^-126 it counts as zero;
* its gradients: d_up = d silu(gate) (slope below 1.1), d_gate = d up silu'(gate) (slope below 0.5, |silu'| below 1.1), where
  silu' = p + gate p (1 - p) is formed as p (1 + gate (1 - p)): each of its two terms is off by the logistic's error, 1 - p by F32 absolute;
* e4m3 results: nearest to result / scale, so within half a step (2^-4 of the number, 2^-10 of the scale among the smallest) of the fp32
  result, and F32 for each of the scale's and the quotient's roundings.
"""
import math

import pytest
import torch

from paper_2511_19438_b200 import workloads as wl

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2511_19438_b200 import build as libbuild
    libbuild.build()
    from paper_2511_19438_b200 import binding as B
    from paper_2511_19438_b200 import harness as H

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SMALLEST = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}      # half a step of the smallest numbers (bfloat16: 2^-126 counts as zero)
F32 = 2.0 ** -23
DTYPES = [torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def ws():
    return H.WorkspaceHolder()


def gen(*parts):
    return torch.Generator(device="cuda").manual_seed(wl.seed_for("fp8", *parts))


def blocks(n):
    return -(-n // 128)


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def rows(M, K, dtype, *seed):
    g = gen("rows", M, K, str(dtype), *seed)
    x = normal(g, M, K) * torch.exp(normal(g, K) * 0.5)
    return x.to(dtype)


def layer(N, K, *seed, transpose=False):
    """Bytes of every finite e4m3 number alike, block scales over two binades."""
    g = gen("layer", N, K, *seed)
    b = torch.randint(0, 254, (N, K), generator=g, device="cuda")
    b = torch.where(b >= 127, b + 1, b).to(torch.uint8)      # without the two NaNs, 0x7f and 0xff
    s = torch.exp2(2 * torch.rand((blocks(N), blocks(K)), generator=g, device="cuda")) / (K ** 0.5 * 128)
    return H.fp8_linear(b.view(torch.float8_e4m3fn), s, transpose=transpose)


def spread(q, s):
    """float64 of e4m3 rows."""
    return q.double() * s.double().repeat_interleave(128, 1)[:, :q.shape[1]]


def weights(D):
    return D.weight.double() * D.scales.double().repeat_interleave(128, 0)[:D.N].repeat_interleave(128, 1)[:, :D.K]


def quantize(x):
    """(e4m3, fp32 scales) by the definition: both quotients in 32 bits, nearest even."""
    M, K = x.shape
    t = torch.zeros((M, blocks(K) * 128), dtype=torch.float32, device=x.device)
    t[:, :K] = x.float()
    t = t.view(M, -1, 128)
    top = t.abs().amax(2)
    s = (top / torch.full_like(top, 448.0)).clamp(min=2.0 ** -126)
    return (t / s.unsqueeze(2)).to(torch.float8_e4m3fn).view(M, -1)[:, :K].contiguous(), s


def bits(t):
    return t.view(torch.uint8)


# ----------------------------------------------------------------------------------------------------------- rows to e4m3
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K", [(1, 16), (1, 128), (3, 144), (1, 4096), (17, 2064), (5, 11008), (301, 272), (2000, 1024)])
def test_quantize(M, K, dtype):
    x = rows(M, K, dtype)
    q, s = H.fp8_quantize(x)
    qw, sw = quantize(x)
    assert torch.equal(s, sw) and torch.equal(bits(q), bits(qw))


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_every_16_bit_number(dtype):
    """Each finite one in a block of its own neighbours, and with the largest number of 128 others."""
    every = torch.arange(65536, device="cuda").to(torch.int16).view(dtype)
    every = every[every.isfinite()]
    every = every[every.float().abs() >= 2.0 ** -126]
    x = every[:every.numel() // 128 * 128].view(-1, 128).contiguous()
    for t in (x, x[torch.randperm(x.numel(), generator=gen("mix"), device="cuda").view(-1, 128) // 128, torch.arange(128, device="cuda")].contiguous()):
        q, s = H.fp8_quantize(t)
        qw, sw = quantize(t)
        assert torch.equal(s, sw) and torch.equal(bits(q), bits(qw))


def test_quantize_zeros_tiny_and_not_finite():
    x = rows(6, 384, torch.bfloat16, "special")
    x[0] = 0
    x[1, 128:256] = 0
    x[2, 5] = float("inf")
    x[3, 300] = float("nan")
    x[4] = 2.0 ** -130                      # counts as zero
    x[5, :128] = 2.0 ** -126
    x[5, 128:256] = 3e38
    q, s = H.fp8_quantize(x)
    v = spread(q, s)
    assert (v[0] == 0).all() and (s[0] == 2.0 ** -126).all() and (v[1, 128:256] == 0).all() and (v[4] == 0).all()
    assert v[2, :128].isnan().all() and v[2, 128:].isfinite().all()
    assert v[3, 256:].isnan().all() and v[3, :256].isfinite().all()
    assert (v[5, :128] == 2.0 ** -126).all()
    assert ((v[5, 128:256] - x[5, 128:256].double()).abs() <= F32 * 3e38).all()


def test_quantize_leaves_what_is_behind():
    x = rows(9, 272, torch.float16, "behind")
    q = torch.full((11, 272), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((11, 3), -1.0, device="cuda")
    B.check(B.gptq_fp8_quantize(x, q, s, 9, 272, 0), "quantize")
    assert (q[9:] == 0x55).all() and (s[9:] == -1).all() and (s[:9] > 0).all()


@pytest.mark.parametrize("N,K", [(16, 16), (128, 128), (144, 272), (1040, 2064), (256, 4096)])
def test_transpose(N, K):
    D = layer(N, K, "transpose", transpose=True)
    assert torch.equal(bits(D.transposed.weight), bits(D.weight).t()) and torch.equal(D.transposed.scales, D.scales.t())


# --------------------------------------------------------------------------------------------------------------- products
def check_gemm(y, x64, D, bias=None, residual=None):
    w = weights(D)
    want, most = x64 @ w.t(), x64.abs() @ w.abs().t()
    for t in (bias, residual):
        if t is not None:
            want, most = want + t.double(), most + t.double().abs()
    tol = (128 + blocks(D.K) + 5) * F32 * most + U[y.dtype] * want.abs() + SMALLEST[y.dtype]
    err = (y.double() - want).abs()
    assert (err <= tol).all(), (err / tol).max().item()


SHAPES = [(1, 8, 16), (1, 128, 128), (1, 4096, 4096), (2, 24, 144), (3, 136, 2064), (5, 1000, 1024), (8, 4096, 11008), (16, 640, 512),
          (17, 640, 528), (31, 256, 4096), (33, 520, 4112), (64, 1152, 1280), (65, 384, 512), (100, 2048, 2048), (128, 264, 640), (129, 256, 272),
          (255, 392, 384), (300, 1000, 2064), (513, 1032, 272), (1000, 2304, 512), (2100, 4352, 256)]


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm(ws, M, N, K, x8):
    for dtype in DTYPES if M * N * K < 1 << 30 else DTYPES[M % 2:][:1]:
        x, D = rows(M, K, dtype), layer(N, K)
        H.ensure_for_fp8(ws, M, K)
        q, s = quantize(x)
        y = H.gemm_fp8(q, D, x_scales=s, dtype=dtype) if x8 else H.gemm_fp8(x, D)
        check_gemm(y, spread(q, s), D)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [1, 7, 16, 20, 40, 128, 200, 700])
@pytest.mark.parametrize("which", ["bias", "residual", "both"])
def test_gemm_bias_residual(ws, M, which, dtype):
    N, K = 1160, 912
    x, D = rows(M, K, dtype), layer(N, K)
    H.ensure_for_fp8(ws, M, K)
    g = gen("extras", M)
    bias = normal(g, N).to(dtype) if which != "residual" else None
    residual = (3 * normal(g, M, N)).to(dtype) if which != "bias" else None
    y = H.gemm_fp8(x, D, bias, residual)
    check_gemm(y, spread(*quantize(x)), D, bias, residual)
    if residual is not None:      # y may be the residual
        inplace = residual.clone()
        H.gemm_fp8(x, D, bias, inplace, y=inplace)
        assert torch.equal(inplace, y)


@pytest.mark.parametrize("M", [1, 5, 16, 18, 40, 70, 130, 300])
def test_results_behind_the_last_row_stay(ws, M):
    N, K, F = 264, 528, 256
    x, D, G = rows(M, K, torch.float16), layer(N, K), layer(2 * F, K, "g")
    H.ensure_for_fp8(ws, M, K)
    y = torch.full((M + 40, N), 7.0, dtype=torch.float16, device="cuda")
    B.check(B.gptq_gemm_fp8(x, None, D.weight, D.scales, None, None, y, M, N, K, 0), "gemm")
    assert (y[M:] == 7).all()
    q, s = torch.full((M + 40, F), 0x55, dtype=torch.uint8, device="cuda"), torch.full((M + 40, 2), -1.0, device="cuda")
    B.check(B.gptq_gemm_fp8_silu_mul(x, None, G.weight, G.scales, q, s, M, F, K, 0), "gated")
    assert (q[M:] == 0x55).all() and (s[M:] == -1).all() and (s[:M] > 0).all()
    h = torch.full((M + 40, F), 7.0, dtype=torch.float16, device="cuda")
    B.check(B.gptq_gemm_fp8_silu_mul(x, None, G.weight, G.scales, h, None, M, F, K, 0), "gated")
    assert (h[M:] == 7).all()
    q, s = torch.full((M + 40, 2 * F), 0x55, dtype=torch.uint8, device="cuda"), torch.full((M + 40, 4), -1.0, device="cuda")
    d = rows(M, F, torch.float16, "d")
    B.check(B.gptq_gemm_fp8_silu_mul_backward(x, None, G.weight, G.scales, d, q, s, M, F, K, 0), "backward")
    assert (q[M:] == 0x55).all() and (s[M:] == -1).all() and (s[:M] > 0).all()


@pytest.mark.parametrize("M", [1, 4, 20, 40, 200])
def test_a_row_does_not_depend_on_the_others(ws, M):
    """Rows of zeros, infinities and NaN beside ordinary ones; a row's result is its own."""
    N, K = 520, 1040
    x, D = rows(M, K, torch.bfloat16, "own"), layer(N, K)
    H.ensure_for_fp8(ws, M + 3, K)
    want = H.gemm_fp8(x, D)
    odd = torch.zeros((3, K), dtype=x.dtype, device="cuda")
    odd[1, 7], odd[2, 1039] = float("inf"), float("nan")
    y = H.gemm_fp8(torch.cat([odd, x]), D)
    assert (y[0] == 0).all() and y[1:3].isnan().all()
    check_gemm(y[3:], spread(*quantize(x)), D)
    check_gemm(want, spread(*quantize(x)), D)


def test_weights_that_are_nan(ws):
    """A column of the result that reaches a NaN weight, and no other."""
    for M in (1, 9, 40, 140):
        D = layer(264, 256, "nan")
        bits(D.weight)[100, 77] = 0x7f
        y = H.gemm_fp8(*quantize(rows(M, 256, torch.float16))[:1], D, x_scales=quantize(rows(M, 256, torch.float16))[1])
        assert y[:, 100].isnan().all() and y[:, :100].isfinite().all() and y[:, 101:].isfinite().all()


def test_large_and_small_scales(ws):
    """Blocks of very different size in one sum, far from fp16's range in between."""
    for M in (2, 30, 150):
        N, K = 256, 512
        x, D = rows(M, K, torch.bfloat16, "scales"), layer(N, K)
        x[:, :128] *= 1e20
        x[:, 128:256] *= 1e-20
        D.scales[:, 0] *= 1e-19
        D.scales[:, 1] *= 1e19
        H.ensure_for_fp8(ws, M, K)
        check_gemm(H.gemm_fp8(x, D), spread(*quantize(x)), D)


def test_more_than_4_gib(ws):
    """Byte offsets beyond 32 bits in x, in y and among the rows that are quantised."""
    free = torch.cuda.mem_get_info()[0]
    if free < 40 << 30:
        pytest.skip("needs 40 GB")
    K, N, M = 8192, 16, 540000
    D = layer(N, K, "far")
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    tail = rows(200, K, torch.bfloat16, "far")
    x[-200:] = tail
    q, s = H.fp8_quantize(x)
    del x
    qw, sw = quantize(tail)
    assert torch.equal(bits(q[-200:]), bits(qw)) and torch.equal(s[-200:], sw) and (bits(q[:1000]) == 0).all()
    y = H.gemm_fp8(q, D, x_scales=s, dtype=torch.bfloat16)
    check_gemm(y[-200:], spread(qw, sw), D)
    assert (y[:1000] == 0).all()
    del q, s, y
    K, N, M = 128, 8192, 300000
    D, x = layer(N, K, "far"), rows(300, K, torch.float16, "far")
    q, s = quantize(x)
    y = H.gemm_fp8(q.repeat(1000, 1), D, x_scales=s.repeat(1000, 1))
    check_gemm(y[-300:], spread(q, s), D)
    assert torch.equal(y[:300], y[-300:])


# -------------------------------------------------------------------------------------------------------- the gated block
class Block:
    """gate, up, the result and its gradients of e4m3 rows in 64 bits, with the bounds of their errors."""

    def __init__(self, x64, D, d=None):
        F, w = D.N // 2, weights(D)
        y, e = x64 @ w.t(), (128 + blocks(D.K) + 5) * F32 * (x64.abs() @ w.abs().t())
        g, u, eg, eu = y[:, :F], y[:, F:], e[:, :F], e[:, F:]
        p = 1 / (1 + torch.exp(-g))
        rel = (6 + 1.5 * g.abs()) * F32
        tiny = 2.0 ** -126 * (1 + g.abs()) * (1 + u.abs())
        self.h, self.eh = g * p * u, 1.1 * u.abs() * eg + (g * p).abs() * eu + 1.1 * eg * eu + rel * (g * p * u).abs() + tiny
        if d is not None:
            d = d.double()
            slope = p * (1 + g * (1 - p))
            self.dg, self.du = d * u * slope, d * g * p
            self.edg = d.abs() * (1.1 * eu + (0.5 * eg + rel * (p + (g * p * (1 - p)).abs()) + F32 * p * (1 + g.abs())) * (u.abs() + eu) + tiny)
            self.edu = d.abs() * (1.1 * eg + rel * (g * p).abs() + tiny)


def check_16(t, want, e):
    tol = e * (1 + U[t.dtype]) + U[t.dtype] * want.abs() + SMALLEST[t.dtype]
    err = (t.double() - want).abs()
    assert (err <= tol).all(), (err / tol).max().item()


def check_8(q, s, want, e):
    M, F = want.shape
    top, etop = want.abs().view(M, -1, 128).amax(2), e.view(M, -1, 128).amax(2)
    assert ((s.double() - (top / 448).clamp(min=2.0 ** -126)).abs() <= etop / 448 + 2 * F32 * s.double()).all()
    per = s.double().repeat_interleave(128, 1)
    value = torch.maximum(want.abs() + e, q.double().abs() * per)
    tol = e + torch.maximum(2.0 ** -4 * value, 2.0 ** -10 * per) + 3 * F32 * value
    # the largest of a block may fall between 448 and the next number there would be: it is 448 times the scale but for the roundings
    err = (spread(q, s) - want).abs()
    assert (err <= tol).all(), (err / tol).max().item()
    # and it is the nearest number where the fp32 result is well inside a step
    exact = want / per
    mid = (exact.float().to(torch.float8_e4m3fn).double() == (exact * (1 + 1e-4)).float().to(torch.float8_e4m3fn).double()) & (
        exact.float().to(torch.float8_e4m3fn).double() == (exact * (1 - 1e-4)).float().to(torch.float8_e4m3fn).double())
    mid &= (e + 2 * etop.repeat_interleave(128, 1)) / per <= 5e-5 * exact.abs()
    assert torch.equal(q.double()[mid], exact[mid].float().to(torch.float8_e4m3fn).double())


GATED = [(1, 128, 16), (1, 1408, 2048), (2, 128, 128), (7, 384, 272), (16, 512, 1040), (19, 256, 512), (33, 1408, 2048), (64, 256, 4096), (66, 384, 144),
         (128, 128, 1024), (130, 256, 272), (300, 640, 528), (1030, 1280, 256)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,F,K", GATED)
def test_gated(ws, M, F, K, dtype):
    x, D = rows(M, K, dtype), layer(2 * F, K, "gated")
    H.ensure_for_fp8(ws, M, K)
    q, s = quantize(x)
    want = Block(spread(q, s), D)
    h = H.gemm_fp8_silu_mul(x, D)
    check_16(h, want.h, want.eh)
    assert torch.equal(H.gemm_fp8_silu_mul(q, D, x_scales=s, dtype=dtype), h)
    h8, hs = H.gemm_fp8_silu_mul(x, D, quantized=True)
    check_8(h8, hs, want.h, want.eh)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,F,K", GATED)
def test_gated_backward(ws, M, F, K, dtype):
    x, D = rows(M, K, dtype), layer(2 * F, K, "gated")
    d = (0.01 * normal(gen("d", M, F), M, F)).to(dtype)
    H.ensure_for_fp8(ws, M, K)
    q, s = quantize(x)
    want = Block(spread(q, s), D, d)
    dgu = H.gemm_fp8_silu_mul_backward(x, D, d, quantized=False)
    check_16(dgu[:, :F], want.dg, want.edg)
    check_16(dgu[:, F:], want.du, want.edu)
    assert torch.equal(H.gemm_fp8_silu_mul_backward(q, D, d, x_scales=s, quantized=False), dgu)
    d8, ds = H.gemm_fp8_silu_mul_backward(x, D, d)
    check_8(d8[:, :F], ds[:, :F // 128], want.dg, want.edg)
    check_8(d8[:, F:], ds[:, F // 128:], want.du, want.edu)


def test_gated_far_gates(ws):
    """Gates of either sign far beyond the exponential's range, zeros, infinities: what the formula gives."""
    for M in (3, 40, 150):
        F, K = 128, 128
        D = layer(2 * F, K, "far")
        x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
        x[0] = rows(1, K, torch.bfloat16, "far") * 3000
        x[1] = -x[0]
        H.ensure_for_fp8(ws, M, K)
        d = torch.ones((M, F), dtype=torch.bfloat16, device="cuda")
        want = Block(spread(*quantize(x)), D, d)
        assert want.h.abs().max() > 1e4 and (want.h[0] * want.h[1] >= 0).all()      # silu(g) u silu(-g) (-u)
        check_16(H.gemm_fp8_silu_mul(x, D), want.h, want.eh)
        dgu = H.gemm_fp8_silu_mul_backward(x, D, d, quantized=False)
        check_16(dgu[:, :F], want.dg, want.edg)
        check_16(dgu[:, F:], want.du, want.edu)
        q, s = H.gemm_fp8_silu_mul(x, D, quantized=True)
        assert (spread(q, s)[2:] == 0).all() and (s[2:] == 2.0 ** -126).all()
        x[2, 3] = float("nan")
        q, s = H.gemm_fp8_silu_mul(x, D, quantized=True)
        assert spread(q, s)[2].isnan().all() and spread(q, s)[:2].isfinite().all()


def loss(x64, D, d):
    F = D.N // 2
    y = x64 @ weights(D).t()
    g, u = y[:, :F], y[:, F:]
    return (d.double() * g / (1 + torch.exp(-g)) * u).sum(1)


@pytest.mark.parametrize("M", [4, 50, 140])
def test_gradient_of_x(ws, M):
    """Against the formula, and against differences of the block's result in 64 bits."""
    F, K, dtype = 256, 400, torch.bfloat16
    x, D = rows(M, K, dtype, "dx"), layer(2 * F, K, "dx", transpose=True)
    d = (0.1 * normal(gen("ddx", M), M, F)).to(dtype)
    q, s = quantize(x)
    x64 = spread(q, s)
    d8, ds = H.gemm_fp8_silu_mul_backward(q, D, d, x_scales=s)
    dx = H.gemm_fp8(d8, D.transposed, x_scales=ds, dtype=dtype)
    check_gemm(dx, spread(d8, ds), D.transposed)
    # rounding to e4m3 moves an element of d_gate_up by 2^-4 of itself at most (2^-10 of its scale), dx by that times the weights
    want, w = Block(x64, D, d), weights(D)
    full = torch.cat([want.dg, want.du], 1)
    e = torch.cat([want.edg, want.edu], 1) + torch.maximum(2.0 ** -4 * full.abs(), 2.0 ** -10 * ds.double().repeat_interleave(128, 1)) * 1.001
    tol = e @ w.abs() + (133 + blocks(2 * F)) * F32 * (spread(d8, ds).abs() @ w.abs()) + U[dtype] * (full @ w).abs() * 1.1
    assert ((dx.double() - full @ w).abs() <= tol).all()
    for k in range(3):
        v = normal(gen("v", M, k), M, K).double()
        h = 1e-5
        slope = (loss(x64 + h * v, D, d) - loss(x64 - h * v, D, d)) / (2 * h)
        assert ((full @ w * v).sum(1) - slope).abs().max() <= 1e-6 * (full.abs() @ w.abs() * v.abs()).sum(1).max()
        assert (((dx.double() * v).sum(1) - slope).abs() <= (tol * v.abs()).sum(1) + 1e-6 * (full.abs() @ w.abs() * v.abs()).sum(1)).all()


# --------------------------------------------------------------------------------------------------------------- together
def step(x, d_y, gate_up, down):
    return H.mlp_fp8(x, gate_up, down, residual=x), H.mlp_fp8_backward(x, gate_up, down, d_y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [1, 12, 33, 160])
def test_together_eager_stream_and_graph(ws, M, dtype):
    K, F = 528, 384
    gate_up, down = layer(2 * F, K, "up", transpose=True), layer(K, F, "down", transpose=True)
    H.ensure_for_fp8(ws, 160, K)
    x, d_y = rows(M, K, dtype, "step"), rows(M, K, dtype, "back")
    y, dx = step(x, d_y, gate_up, down)
    h8, hs = H.gemm_fp8_silu_mul(x, gate_up, quantized=True)
    check_gemm(y, spread(h8, hs), down, residual=x)
    d_h = H.gemm_fp8(d_y, down.transposed)
    check_gemm(d_h, spread(*quantize(d_y)), down.transposed)
    d8, ds = H.gemm_fp8_silu_mul_backward(x, gate_up, d_h)
    check_gemm(dx, spread(d8, ds), gate_up.transposed)
    for got, want in zip(step(x, d_y, gate_up, down), (y, dx)):
        assert torch.equal(got, want)          # the same bits again
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = step(x, d_y, gate_up, down)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(again[0], y) and torch.equal(again[1], dx)
    graph, static, static_d = torch.cuda.CUDAGraph(), x.clone(), d_y.clone()
    with torch.cuda.graph(graph):
        out = step(static, static_d, gate_up, down)
    for seed in ("first", "second"):
        x2, d2 = rows(M, K, dtype, seed), rows(M, K, dtype, seed, "d")
        want = step(x2, d2, gate_up, down)
        static.copy_(x2)
        static_d.copy_(d2)
        for _ in range(3):
            graph.replay()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    assert B.gptq_check_status() == B.GPTQ_OK


@pytest.mark.parametrize("M", [2, 24, 150])
def test_two_streams_with_scratch_of_their_own(ws, M):
    K, F = 1024, 512
    gate_up, down = layer(2 * F, K, "up2", transpose=True), layer(K, F, "down2", transpose=True)
    x, d_y = rows(M, K, torch.float16, "two"), rows(M, K, torch.float16, "two-d")
    H.ensure_for_fp8(ws, M, K)
    want = step(x, d_y, gate_up, down)
    graphs = []
    for _ in range(2):
        mine, g = H.WorkspaceHolder(), torch.cuda.CUDAGraph()
        H.ensure_for_fp8(mine, M, K)
        with torch.cuda.graph(g):
            outs = [step(x, d_y, gate_up, down) for _ in range(3)]
        graphs.append((g, mine, outs))
    side = [torch.cuda.Stream() for _ in range(2)]
    for s in side:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for (g, _mine, _outs), s in zip(graphs, side):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for _g, _mine, outs in graphs:
        for y, dx in outs:
            assert torch.equal(y, want[0]) and torch.equal(dx, want[1])
    ws.ensure(1)
    assert B.gptq_check_status() == B.GPTQ_OK


@pytest.mark.parametrize("M", [1, 9, 40, 300])
def test_repeats_bit_for_bit(ws, M):
    K, F = 2048, 1024
    gate_up, down = layer(2 * F, K, "rep", transpose=True), layer(K, F, "rep", transpose=True)
    x, d_y = rows(M, K, torch.bfloat16, "rep"), rows(M, K, torch.bfloat16, "rep-d")
    H.ensure_for_fp8(ws, M, K)
    want = step(x, d_y, gate_up, down)
    for _ in range(100):
        for got in [step(x, d_y, gate_up, down) for _ in range(3)]:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_beside_a_4_bit_layer(ws):
    """An e4m3 feed-forward block behind a GPTQ projection, one stream, nothing waited for in between."""
    K, F, M = 512, 256, 10
    proj = H.upload_and_repack(wl.make_linear(K, K, seed=5))
    gate_up, down = layer(2 * F, K, "mix"), layer(K, F, "mix")
    H.ensure_for_fp8(ws, M, K)
    x = rows(M, K, torch.float16, "mix")
    o = H.gemm_bias_residual(x, proj, None, x)
    want = H.mlp_fp8(o, gate_up, down, residual=o).clone()
    torch.cuda.synchronize()
    for _ in range(50):
        o2 = H.gemm_bias_residual(x, proj, None, x)
        y = H.mlp_fp8(o2, gate_up, down, residual=o2)
        z = H.gemm(y, proj)
        assert torch.equal(y, want) and z.shape == (M, K)


def test_needs_its_workspace():
    x, D = rows(3, 256, torch.float16), layer(256, 256)
    q, s = quantize(x)
    B.check(B.gptq_set_workspace(None, 0), "set_workspace")
    with pytest.raises(B.GptqError) as e:
        H.gemm_fp8(x, D)
    assert e.value.status == B.GPTQ_ERR_WORKSPACE
    check_gemm(H.gemm_fp8(q, D, x_scales=s), spread(q, s), D)      # e4m3 rows need none
    small = torch.empty(B.gptq_fp8_workspace_bytes(3, 256) - 1, dtype=torch.uint8, device="cuda")
    B.check(B.gptq_set_workspace(small, small.numel()), "set_workspace")
    with pytest.raises(B.GptqError):
        H.gemm_fp8(x, D)
    B.check(B.gptq_set_workspace(None, 0), "set_workspace")


def test_harness_refuses_what_does_not_fit(ws):
    x, D = rows(3, 256, torch.float16), layer(256, 256)
    q, s = quantize(x)
    H.ensure_for_fp8(ws, 3, 256)
    for bad in (lambda: H.gemm_fp8(x.float(), D), lambda: H.gemm_fp8(x[:, :128], D), lambda: H.gemm_fp8(x.t().contiguous().t(), D),
                lambda: H.gemm_fp8(q, D), lambda: H.gemm_fp8(q, D, x_scales=s[:, :1]), lambda: H.gemm_fp8(x, D, residual=x[:, :8]),
                lambda: H.gemm_fp8(x, D, bias=x[0].bfloat16()), lambda: H.fp8_linear(D.weight, D.scales[:1]),
                lambda: H.gemm_fp8_silu_mul_backward(x, D, x), lambda: H.mlp_fp8_backward(x, D, D, x)):
        with pytest.raises(ValueError):
            bad()

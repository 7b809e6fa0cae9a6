"""GPU tests of the e4m3 products on CTA pairs (the kernel of long prompts), and of what the fused epilogues round to.

The sizes are ones that the rule gives to that kernel on 148 SMs; each test asks gptq_plan_fp8, so that a new rule cannot take them away
unnoticed.  Plain implementations in 64 bits and the tolerances are those of test_gpu_fp8.
"""
import pytest
import torch

from . import test_gpu_fp8 as T
from .test_gpu_fp8 import DTYPES, F32, U, Block, bits, check_16, check_8, check_gemm, gen, layer, normal, quantize, rows, spread, weights, ws  # noqa: F401

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2511_19438_b200 import binding as B
    from paper_2511_19438_b200 import harness as H


def on_pairs(M, N, K, gated=False):
    st, p = B.gptq_plan_fp8(M, N, K, gated, torch.cuda.get_device_properties(0).multi_processor_count)
    B.check(st, "gptq_plan_fp8")
    assert p.kernel == 7, (M, N, K, gated)


# one block of K and less, 2, 4, 5, 6, 8, 9 and 33 blocks (scales come four blocks at a time, the ring has four stages, the epilogue's input is asked for in
# front of the fifth block), ragged ones on every axis, more tiles than pairs of CTAs
SHAPES = [(2100, 4352, 16), (1300, 4360, 128), (1300, 4360, 144), (1300, 4360, 512), (1300, 4360, 640), (1300, 4360, 656), (1290, 3848, 1024), (1100, 4104, 1040),
          (700, 8200, 4112)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_bias_residual(ws, M, N, K, dtype):  # noqa: F811
    on_pairs(M, N, K)
    x, D = rows(M, K, dtype, "pairs"), layer(N, K, "pairs")
    H.ensure_for_fp8(ws, M, K)
    g = gen("pairs", M, N)
    bias, residual = normal(g, N).to(dtype), (3 * normal(g, M, N)).to(dtype)
    q, s = quantize(x)
    x64 = spread(q, s)
    for b, r in ((None, None), (bias, None), (None, residual), (bias, residual)):
        y = H.gemm_fp8(x, D, b, r)
        check_gemm(y, x64, D, b, r)
        assert torch.equal(H.gemm_fp8(q, D, b, r, x_scales=s, dtype=dtype), y)
        if r is not None:      # y may be the residual
            inplace = r.clone()
            H.gemm_fp8(x, D, b, inplace, y=inplace)
            assert torch.equal(inplace, y)


def check_nearest(q, s, want, e, least=0.7):
    """The e4m3 results are the nearest numbers to result / scale, wherever an error of e and one rounding of the quotient cannot decide."""
    per = s.double().repeat_interleave(128, 1)

    def e4m3(v):
        return (v / per).clamp(-448.0, 448.0).float().to(torch.float8_e4m3fn).double()

    slack = e + 2 * F32 * want.abs()
    low, high = e4m3(want - slack), e4m3(want + slack)
    sure = low == high
    assert torch.equal(q.double()[sure], low[sure])
    assert sure.double().mean() >= least, sure.double().mean().item()
    assert ((low <= q.double()) & (q.double() <= high)).all()


GATED = [(1300, 4096, 16), (1300, 2048, 128), (1300, 2304, 528), (1300, 2048, 656), (2100, 1408, 1040), (1300, 2048, 1024), (65, 11008, 4096)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,F,K", GATED)
def test_gated_and_backward(ws, M, F, K, dtype):  # noqa: F811
    on_pairs(M, 2 * F, K, True)
    x, D = rows(M, K, dtype, "pairs"), layer(2 * F, K, "pairs")
    d = (0.01 * normal(gen("pairs", "d", M, F), M, F)).to(dtype)
    H.ensure_for_fp8(ws, M, K)
    q, s = quantize(x)
    want = Block(spread(q, s), D, d)
    h = H.gemm_fp8_silu_mul(x, D)
    check_16(h, want.h, want.eh)
    assert torch.equal(H.gemm_fp8_silu_mul(q, D, x_scales=s, dtype=dtype), h)
    h8, hs = H.gemm_fp8_silu_mul(x, D, quantized=True)
    check_8(h8, hs, want.h, want.eh)
    check_nearest(h8, hs, want.h, want.eh)
    dgu = H.gemm_fp8_silu_mul_backward(x, D, d, quantized=False)
    check_16(dgu[:, :F], want.dg, want.edg)
    check_16(dgu[:, F:], want.du, want.edu)
    d8, ds = H.gemm_fp8_silu_mul_backward(q, D, d, x_scales=s)
    for part, cols, w, e in (("gate", slice(0, F), want.dg, want.edg), ("up", slice(F, 2 * F), want.du, want.edu)):
        sc = ds[:, cols.start // 128:cols.stop // 128]
        check_8(d8[:, cols], sc, w, e)
        check_nearest(d8[:, cols], sc, w, e)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,F,K", T.GATED)
def test_few_rows_round_to_the_nearest(ws, M, F, K, dtype):  # noqa: F811
    x, D = rows(M, K, dtype), layer(2 * F, K, "gated")
    d = (0.01 * normal(gen("d", M, F), M, F)).to(dtype)
    H.ensure_for_fp8(ws, M, K)
    want = Block(spread(*quantize(x)), D, d)
    check_nearest(*H.gemm_fp8_silu_mul(x, D, quantized=True), want.h, want.eh)
    d8, ds = H.gemm_fp8_silu_mul_backward(x, D, d)
    check_nearest(d8[:, :F], ds[:, :F // 128], want.dg, want.edg)
    check_nearest(d8[:, F:], ds[:, F // 128:], want.du, want.edu)


def test_results_behind_the_last_row_stay(ws):  # noqa: F811
    M, N, K, F = 1300, 4360, 656, 2048
    on_pairs(M, N, K)
    on_pairs(M, 2 * F, K, True)
    x, D, G, d = rows(M, K, torch.float16), layer(N, K), layer(2 * F, K, "g"), rows(M, F, torch.float16, "d")
    H.ensure_for_fp8(ws, M, K)
    y = torch.full((M + 256, N), 7.0, dtype=torch.float16, device="cuda")
    for residual in (None, y):
        B.check(B.gptq_gemm_fp8(x, None, D.weight, D.scales, None, residual, y, M, N, K, 0), "gemm")
        assert (y[M:] == 7).all() and y[:M].isfinite().all()
    for cols, backward in ((F, False), (2 * F, True)):
        q, s = torch.full((M + 256, cols), 0x55, dtype=torch.uint8, device="cuda"), torch.full((M + 256, cols // 128), -1.0, device="cuda")
        h = torch.full((M + 256, cols), 7.0, dtype=torch.float16, device="cuda")
        for out, scales in ((q, s), (h, None)):
            B.check(B.gptq_gemm_fp8_silu_mul_backward(x, None, G.weight, G.scales, d, out, scales, M, F, K, 0) if backward else
                    B.gptq_gemm_fp8_silu_mul(x, None, G.weight, G.scales, out, scales, M, F, K, 0), "gated")
        assert (q[M:] == 0x55).all() and (s[M:] == -1).all() and (s[:M] > 0).all() and (h[M:] == 7).all()


def test_rows_and_columns_that_are_odd(ws):  # noqa: F811
    """Rows of zeros, infinities and NaN beside ordinary ones, a NaN weight, in several tiles; everything else is its own."""
    M, N, K = 1300, 4360, 656
    on_pairs(M, N, K)
    x, D = rows(M, K, torch.bfloat16, "odd"), layer(N, K, "odd")
    H.ensure_for_fp8(ws, M, K)
    zero, bad = [0, 255, 700, 1299], [3, 131, 640, 1281]
    x[zero] = 0
    x[bad[:2], 655], x[bad[2:], 300] = float("inf"), float("nan")
    y = H.gemm_fp8(x, D)
    assert (y[zero] == 0).all() and y[bad].isnan().all()
    fine = torch.ones(M, dtype=torch.bool, device="cuda")
    fine[bad] = False
    check_gemm(y[fine], spread(*quantize(x))[fine], D)
    columns = [100, 2047, 4359]
    bits(D.weight)[columns, 77] = 0x7f
    y = H.gemm_fp8(x, D)
    keep = torch.ones(N, dtype=torch.bool, device="cuda")
    keep[columns] = False
    assert y[:, columns].isnan().all() and y[fine][:, keep].isfinite().all()
    # the gated block: the maximum of a block of 128 goes over two warps, a NaN of either takes the block and no more
    F = 2048
    on_pairs(M, 2 * F, K, True)
    x, G = rows(M, K, torch.bfloat16, "odd2"), layer(2 * F, K, "odd2")
    for column in (5, 128 + 100, F + 256 + 3):      # gate's, gate's, up's
        bits(G.weight)[column, 0] = 0x7f
    q, s = H.gemm_fp8_silu_mul(x, G, quantized=True)
    v = spread(q, s)
    assert v[:, :384].isnan().all() and v[:, 384:].isfinite().all()


def test_large_and_small_scales(ws):  # noqa: F811
    M, N, K = 1300, 4360, 656
    on_pairs(M, N, K)
    x, D = rows(M, K, torch.bfloat16, "scales"), layer(N, K)
    x[:, :128] *= 1e20
    x[:, 512:] *= 1e-20
    D.scales[:, 0] *= 1e-19
    D.scales[:, 4:] *= 1e19
    H.ensure_for_fp8(ws, M, K)
    check_gemm(H.gemm_fp8(x, D), spread(*quantize(x)), D)


def test_gradient_of_x(ws):  # noqa: F811
    """Both products of the way back on pairs, against the formula, and against differences of the block's result in 64 bits."""
    M, F, K, dtype = 2600, 1152, 2064, torch.bfloat16
    on_pairs(M, 2 * F, K, True)
    on_pairs(M, K, 2 * F)
    x, D = rows(M, K, dtype, "dx"), layer(2 * F, K, "dx", transpose=True)
    d = (0.1 * normal(gen("ddx", M), M, F)).to(dtype)
    q, s = quantize(x)
    x64 = spread(q, s)
    d8, ds = H.gemm_fp8_silu_mul_backward(q, D, d, x_scales=s)
    dx = H.gemm_fp8(d8, D.transposed, x_scales=ds, dtype=dtype)
    check_gemm(dx, spread(d8, ds), D.transposed)
    want, w = Block(x64, D, d), weights(D)
    full = torch.cat([want.dg, want.du], 1)
    # rounding to e4m3 as in test_gpu_fp8.test_gradient_of_x
    e = torch.cat([want.edg, want.edu], 1) + torch.maximum(2.0 ** -4 * full.abs(), 2.0 ** -10 * ds.double().repeat_interleave(128, 1)) * 1.001
    tol = e @ w.abs() + (133 + T.blocks(2 * F)) * F32 * (spread(d8, ds).abs() @ w.abs()) + U[dtype] * (full @ w).abs() * 1.1
    assert ((dx.double() - full @ w).abs() <= tol).all()
    v, h = normal(gen("v", M), M, K).double(), 1e-5
    slope = (T.loss(x64 + h * v, D, d) - T.loss(x64 - h * v, D, d)) / (2 * h)
    most = (full.abs() @ w.abs() * v.abs()).sum(1)
    assert ((full @ w * v).sum(1) - slope).abs().max() <= 1e-6 * most.max()
    assert (((dx.double() * v).sum(1) - slope).abs() <= (tol * v.abs()).sum(1) + 1e-6 * most).all()


@pytest.fixture(scope="module")
def block():
    """A feed-forward block whose five products are all on pairs."""
    M, F, K = 2600, 1152, 2304
    for shape in ((M, 2 * F, K, True), (M, K, F), (M, F, K), (M, K, 2 * F)):
        on_pairs(*shape)
    return layer(2 * F, K, "up", transpose=True), layer(K, F, "down", transpose=True), M, K


@pytest.mark.parametrize("dtype", DTYPES)
def test_together_repeats_stream_and_graph(ws, block, dtype):  # noqa: F811
    gate_up, down, M, K = block
    H.ensure_for_fp8(ws, M, K)
    x, d_y = rows(M, K, dtype, "step"), rows(M, K, dtype, "back")
    y, dx = T.step(x, d_y, gate_up, down)
    h8, hs = H.gemm_fp8_silu_mul(x, gate_up, quantized=True)
    check_gemm(y, spread(h8, hs), down, residual=x)
    d_h = H.gemm_fp8(d_y, down.transposed)
    check_gemm(d_h, spread(*quantize(d_y)), down.transposed)
    d8, ds = H.gemm_fp8_silu_mul_backward(x, gate_up, d_h)
    check_gemm(dx, spread(d8, ds), gate_up.transposed)
    for _ in range(100):
        got = T.step(x, d_y, gate_up, down)
        assert torch.equal(got[0], y) and torch.equal(got[1], dx)      # the same bits again
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = T.step(x, d_y, gate_up, down)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(again[0], y) and torch.equal(again[1], dx)
    graph, static, static_d = torch.cuda.CUDAGraph(), x.clone(), d_y.clone()
    with torch.cuda.graph(graph):
        out = T.step(static, static_d, gate_up, down)
    for seed in ("first", "second"):
        x2, d2 = rows(M, K, dtype, seed), rows(M, K, dtype, seed, "d")
        want = T.step(x2, d2, gate_up, down)
        static.copy_(x2)
        static_d.copy_(d2)
        for _ in range(3):
            graph.replay()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    assert B.gptq_check_status() == B.GPTQ_OK


def test_two_streams_with_scratch_of_their_own(ws, block):  # noqa: F811
    """Two captured graphs that run at the same time beside one another."""
    gate_up, down, M, K = block
    x, d_y = rows(M, K, torch.float16, "two"), rows(M, K, torch.float16, "two-d")
    H.ensure_for_fp8(ws, M, K)
    want = T.step(x, d_y, gate_up, down)
    graphs = []
    for _ in range(2):
        mine, g = H.WorkspaceHolder(), torch.cuda.CUDAGraph()
        H.ensure_for_fp8(mine, M, K)
        with torch.cuda.graph(g):
            outs = [T.step(x, d_y, gate_up, down) for _ in range(3)]
        graphs.append((g, mine, outs))
    side = [torch.cuda.Stream() for _ in range(2)]
    for s in side:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for (g, _mine, _outs), s in zip(graphs, side):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for _g, _mine, outs in graphs:
        for y, dx in outs:
            assert torch.equal(y, want[0]) and torch.equal(dx, want[1])
    H.ensure_for_fp8(ws, M, K)
    assert B.gptq_check_status() == B.GPTQ_OK

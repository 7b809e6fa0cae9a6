"""GPU tests of the layers in 8-bit floating point: waits that give up, streams, the logistic function."""
import pytest
import torch

from . import test_gpu_fp8 as T
from .test_gpu_fp8 import layer, quantize, rows, spread, weights, ws  # noqa: F401

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2511_19438_b200 import build as libbuild
    libbuild.build()
    from paper_2511_19438_b200 import binding as B
    from paper_2511_19438_b200 import harness as H


@pytest.mark.parametrize("ctas", [1, 2, 4, 8])
def test_a_wait_that_gave_up_keeps_the_whole_cluster_from_storing(ctas):
    """Each CTA of the few-row kernel adds parts of all of its cluster: if one has none, no row is stored."""
    assert B.gptq_check_status() == B.GPTQ_OK
    for who in (-1, 0, ctas - 1):
        stored = torch.zeros(ctas, dtype=torch.int32, device="cuda")
        B.check(B.gptq_selftest_give_up(ctas, who, 200, stored), "selftest launch")      # 200 microseconds
        assert B.gptq_check_status() == (B.GPTQ_OK if who < 0 else B.GPTQ_ERR_TIMEOUT)
        assert (stored == (1 if who < 0 else 0)).all()
    assert B.gptq_check_status() == B.GPTQ_OK


@pytest.mark.parametrize("handle", [False, True])
def test_the_block_on_a_stream_that_is_not_the_current_one(ws, handle):  # noqa: F811
    """What it allocates for itself stays its own until its kernels have read it, whatever the current stream allocates behind the call."""
    M, K, F = 64, 1024, 2048
    gate_up, down = layer(2 * F, K, "up", transpose=True), layer(K, F, "down", transpose=True)
    x, d_y = rows(M, K, torch.bfloat16, "stream"), rows(M, K, torch.bfloat16, "stream-d")
    H.ensure_for_fp8(ws, M, K)
    want = T.step(x, d_y, gate_up, down)
    side = torch.cuda.Stream()
    given = side.cuda_stream if handle else side
    for _ in range(3):
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)      # the block's kernels start some ms behind what follows on the current stream
        y = H.mlp_fp8(x, gate_up, down, residual=x, stream=given)
        dx = H.mlp_fp8_backward(x, gate_up, down, d_y, stream=given)
        taken = [torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda") for shape in ((M, F), (M, F // 32), (M, 2 * F), (M, 2 * F // 32), (M, 2 * K))
                 for _ in range(3)]
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1])
        del taken


def test_a_new_layer_on_another_stream(ws):  # noqa: F811
    """The transposed layer is whole when fp8_linear returns, even if its stream was busy."""
    M, N, K = 16, 4096, 2048
    D = layer(N, K, "late")
    d = rows(M, N, torch.bfloat16, "late")
    q, s = quantize(d)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    L = H.fp8_linear(D.weight, D.scales, transpose=True)
    dx = H.gemm_fp8(q, L.transposed, x_scales=s, dtype=torch.bfloat16, stream=side)
    torch.cuda.synchronize()
    T.check_gemm(dx, spread(q, s), L.transposed)
    assert torch.equal(weights(L.transposed), weights(D).t())


@pytest.mark.parametrize("M", [3, 40, 1300])
def test_arguments_side_by_side(ws, M):  # noqa: F811
    """Inputs and results without a gap between them are not refused, and none is written over."""
    F, K, dtype = 2048, 512, torch.float16
    D, x, d = layer(2 * F, K, "beside"), rows(M, K, dtype, "beside"), rows(M, F, dtype, "beside-d")
    q, s = quantize(x)
    want = H.gemm_fp8_silu_mul_backward(q, D, d, x_scales=s)
    parts = [(M * K, q), (M * 2 * F, None), (4 * M * (K // 128), s), (4 * M * (2 * F // 128), None), (2 * M * F, d)]
    assert all(n % 16 == 0 for n, _ in parts)
    one = torch.full((sum(n for n, _ in parts),), 0x55, dtype=torch.uint8, device="cuda")
    views = one.split([n for n, _ in parts])
    for v, (_, t) in zip(views, parts):
        if t is not None:
            v.copy_(t.reshape(-1).view(torch.uint8))
    qv, out, sv, outs, dv = views
    B.check(B.gptq_gemm_fp8_silu_mul_backward(qv, sv, D.weight, D.scales, dv, out, outs, M, F, K, 0), "backward")
    assert torch.equal(out, want[0].reshape(-1).view(torch.uint8)) and torch.equal(outs, want[1].reshape(-1).view(torch.uint8))
    for v, (_, t) in zip(views, parts):
        assert t is None or torch.equal(v, t.reshape(-1).view(torch.uint8))


def test_the_longest_row():
    """One row of the last multiple of 16 below 2^31."""
    K = (1 << 31) - 16
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    x = torch.zeros((1, K), dtype=torch.float16, device="cuda")
    head, tail = rows(1, 4096, torch.float16, "head"), rows(1, 4080, torch.float16, "tail")
    x[:, :4096], x[:, -4080:] = head, tail
    q, s = H.fp8_quantize(x)
    assert s.shape == (1, 1 << 24)
    for got, scales, part in ((q[:, :4096], s[:, :32], head), (q[:, -4080:], s[:, -32:], tail)):
        want = quantize(part)
        assert torch.equal(scales, want[1]) and torch.equal(got.contiguous().view(torch.uint8), want[0].view(torch.uint8))
    assert (s[:, 32:-32] == 2.0 ** -126).all()


@pytest.mark.parametrize("M", [1, 20, 300])
def test_the_error_of_the_logistic_function(M):
    """Gates of any fp32 value and up = 1, formed without an error: weights of one at the first column, a block's gate is its scale.  All of a
    block's results are alike, so that its scale times 448 shows the fp32 result (one rounding): off by (6 + 1.5 |gate|) 2^-23 of itself at most.
    Gradients of d = 1: d_up as the result, d_gate = p (1 + gate (1 - p)) by each term's share and 1 - p by 2^-23."""
    n, K, F32 = 1024, 16, 2.0 ** -23
    F = 128 * n
    gates = 160 * torch.rand(n, generator=T.gen("gates"), device="cuda") - 80
    gates[:64] = torch.linspace(-20, 20, 64, device="cuda")
    w = torch.zeros((2 * F, K), device="cuda")
    w[:, 0] = 1
    D = H.fp8_linear(w.to(torch.float8_e4m3fn), torch.cat([gates, torch.ones_like(gates)])[:, None].contiguous())
    x = torch.zeros((M, K), device="cuda")
    x[:, 0] = 1
    x, s = x.to(torch.float8_e4m3fn), torch.ones((M, 1), device="cuda")
    g = gates.double()
    p = 1 / (1 + torch.exp(-g))
    rel = (6 + 1.5 * g.abs()) * F32
    _, hs = H.gemm_fp8_silu_mul(x, D, x_scales=s, quantized=True)
    assert ((448 * hs.double() - (g * p).abs()).abs() <= (rel + F32) * (g * p).abs()).all()
    _, ds = H.gemm_fp8_silu_mul_backward(x, D, torch.ones((M, F), dtype=torch.float16, device="cuda"), x_scales=s)
    slope = p * (1 + g * (1 - p))
    e = rel * (p + (g * p * (1 - p)).abs()) + F32 * p * (1 + g.abs())
    assert ((448 * ds[:, :n].double() - slope.abs()).abs() <= e + F32 * slope.abs()).all()
    assert ((448 * ds[:, n:].double() - (g * p).abs()).abs() <= (rel + F32) * (g * p).abs()).all()

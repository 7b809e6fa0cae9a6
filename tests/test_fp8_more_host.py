"""Layers in 8-bit floating point, what needs no GPU: waits, refusals, the harness's streams and devices, sizes, the quotient."""
import ctypes
import ctypes.util
import itertools
import os
import re

import numpy as np
import pytest
import torch

from paper_2511_19438_b200 import build as libbuild

libbuild.build()
from paper_2511_19438_b200 import binding as B  # noqa: E402
from paper_2511_19438_b200 import harness as H  # noqa: E402


def test_no_uniform_branch_on_a_lane_s_own_try():
    """mbarrier.try_wait answers each lane for itself: a branch that promises one answer for the warp (bra.uni) may not hang on it."""
    for f in sorted(os.listdir(libbuild.CSRC)):
        with open(os.path.join(libbuild.CSRC, f)) as h:
            for asm in re.findall(r"asm\s+volatile\s*\((.*?)\);", h.read(), re.S):
                assert not ("try_wait" in asm and "bra.uni" in asm), f


# ------------------------------------------------------------------------------------------------ which kernel takes a call
PAIRS = [(1300, 4360, 656, 0), (1290, 3848, 1024, 0), (1100, 4104, 1040, 0), (4096, 12288, 4096, 0), (1300, 2 * 2048, 656, 1), (2100, 2 * 1408, 1040, 1),
         (1300, 2 * 2048, 1024, 1), (65, 2 * 11008, 4096, 1)]
FEW = [(1, 8, 16, 0), (128, 4096, 4096, 0), (300, 1000, 2064, 0), (512, 4096, 4096, 0), (1, 2 * 128, 16, 1), (64, 2 * 11008, 4096, 1), (512, 2 * 2048, 4096, 1)]


def test_plan_says_which_kernel():
    for shapes, kernel in ((FEW, 6), (PAIRS, 7)):
        for M, N, K, gated in shapes:
            st, p = B.gptq_plan_fp8(M, N, K, gated, 148)
            assert st == B.GPTQ_OK and p.kernel == kernel, (M, N, K, gated, p.kernel)
            assert 1 <= p.ctas and p.ctas % p.cluster_size == 0 and p.smem_bytes <= 227 * 1024
            assert p.workspace_bytes == B.gptq_fp8_workspace_bytes(M, K)
            tiles = -(-M // p.m_tile) * -(-N // (256 if gated or kernel == 7 else 128))
            assert p.items == tiles * -(-K // 128)
            assert p.ctas == tiles * p.cluster_size if kernel == 6 else p.ctas == min(148, 2 * tiles)


def test_plan_refusals():
    assert B._lib.gptq_plan_fp8(4, 256, 256, 0, 148, None) == B.GPTQ_ERR_NULL
    for bad in ((0, 256, 256, 0, 148), (4, 4, 256, 0, 148), (4, 256, 24, 0, 148), (4, 256, 256, 0, 0), (4, 264, 256, 1, 148), (4, 128, 256, 1, 148)):
        assert B.gptq_plan_fp8(*bad)[0] == B.GPTQ_ERR_SHAPE, bad
    for M, N, K, gated in FEW + PAIRS:      # any number of SMs, one too
        for sms in (1, 2, 3, 20, 1000):
            assert B.gptq_plan_fp8(M, N, K, gated, sms)[0] == B.GPTQ_OK


def test_selftest_refusals():
    for bad in ((0, 0, 200), (3, 0, 200), (16, 0, 200), (4, 4, 200), (4, 0, 0), (4, 0, 1000001)):
        assert B.gptq_selftest_give_up(*bad, 4096, stream=0) == B.GPTQ_ERR_SHAPE, bad
    assert B.gptq_selftest_give_up(4, 0, 200, None, stream=0) == B.GPTQ_ERR_NULL


# ------------------------------------------------------------------------------------------------ the harness, on stand-ins for the GPU's calls
@pytest.fixture
def calls(monkeypatch):
    """The library's calls and torch's streams replaced by a list of what happened."""
    log, inside = [], []

    class Stream:
        cuda_stream = 77

        def __init__(self, *a, **kw):
            pass

        def synchronize(self):
            log.append("synchronize")

    class Under:
        def __init__(self, stream):
            pass

        def __enter__(self):
            inside.append(1)

        def __exit__(self, *a):
            inside.pop()

    empty = torch.empty

    def record_empty(*a, **kw):
        t = empty(*a, **kw)
        log.append(("empty", t.data_ptr(), bool(inside)))
        return t

    for name in ("gptq_fp8_quantize", "gptq_fp8_transpose", "gptq_gemm_fp8", "gptq_gemm_fp8_silu_mul", "gptq_gemm_fp8_silu_mul_backward"):
        monkeypatch.setattr(B, name, lambda *a, name=name: log.append(name) or B.GPTQ_OK)
    monkeypatch.setattr(torch, "empty", record_empty)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", Under)
    monkeypatch.setattr(torch.cuda, "current_stream", Stream)
    monkeypatch.setattr(H, "_expect_here", lambda *a: None, raising=False)
    return log


def layer(N, K):
    return H.DeviceFp8Linear(K, N, torch.zeros((N, K), dtype=torch.uint8).view(torch.float8_e4m3fn), torch.ones((-(-N // 128), -(-K // 128))))


@pytest.mark.parametrize("stream", ["object", 77, None])
def test_what_the_block_allocates_for_itself_belongs_to_its_stream(calls, stream):
    """Memory that the caller never sees is freed when the call returns: on another stream than its own it could be given away while it is read."""
    given = torch.cuda.Stream() if stream == "object" else stream
    gate_up, down = layer(512, 256), layer(256, 256)
    gate_up.transposed, down.transposed = layer(256, 512), layer(256, 256)
    x = torch.zeros((4, 256), dtype=torch.float16)
    for run, own in ((lambda: H.mlp_fp8(x, gate_up, down, stream=given), 2), (lambda: H.mlp_fp8_backward(x, gate_up, down, x, stream=given), 3)):
        calls.clear()
        out = run()
        made = [c for c in calls if c[0] == "empty"]
        assert len(made) == own + 1
        for _, address, under in made:
            assert under == (given is not None and address != out.data_ptr())


def test_a_layer_is_laid_out_when_it_is_returned(calls):
    """Products read weights before earlier kernels have ended, and may run on any stream."""
    D = layer(256, 128)
    H.fp8_linear(D.weight, D.scales)
    assert calls == []
    H.fp8_linear(D.weight, D.scales, transpose=True)
    assert [c for c in calls if c[0] != "empty"] == ["gptq_fp8_transpose", "synchronize"]


def test_tensors_elsewhere_are_refused(monkeypatch):
    """Any one of them on another device than the current one: the kernel would be given an address of that device."""
    for name in ("gptq_fp8_quantize", "gptq_fp8_transpose", "gptq_gemm_fp8", "gptq_gemm_fp8_silu_mul", "gptq_gemm_fp8_silu_mul_backward"):
        monkeypatch.setattr(B, name, lambda *a: B.GPTQ_OK)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    monkeypatch.setattr(H, "_here", lambda: torch.device("cpu"))      # as if the CPU were the current device
    D, x = layer(256, 256), torch.zeros((4, 256), dtype=torch.float16)
    x8, s = x.to(torch.float8_e4m3fn), torch.ones((4, 2))
    runs = {
        "linear": (lambda weight, scales: H.fp8_linear(weight, scales), dict(weight=D.weight, scales=D.scales)),
        "quantize": (lambda x: H.fp8_quantize(x), dict(x=x)),
        "gemm": (lambda x, xs, w, ws, b, r, y: H.gemm_fp8(x, H.DeviceFp8Linear(256, 256, w, ws), b, r, y, x_scales=xs),
                 dict(x=x8, xs=s, w=D.weight, ws=D.scales, b=x[0].clone(), r=x, y=x.clone())),
        "gated": (lambda x, xs, w, ws: H.gemm_fp8_silu_mul(x, H.DeviceFp8Linear(256, 256, w, ws), x_scales=xs),
                  dict(x=x8, xs=s, w=D.weight, ws=D.scales)),
        "backward": (lambda x, xs, w, ws, d: H.gemm_fp8_silu_mul_backward(x, H.DeviceFp8Linear(256, 256, w, ws), d, x_scales=xs),
                     dict(x=x8, xs=s, w=D.weight, ws=D.scales, d=x[:, :128].contiguous())),
    }
    for name, (run, tensors) in runs.items():
        run(**tensors)
        for t in tensors:
            with pytest.raises(ValueError, match="meta"):
                run(**{**tensors, t: tensors[t].to("meta")})


def test_a_gated_layer_has_as_many_rows_of_up_as_of_gate(calls):
    """An odd row at the end would have been left out without a word."""
    x, d = torch.zeros((4, 256), dtype=torch.float16), torch.zeros((4, 128), dtype=torch.float16)
    for N in (257, 264, 128, 384):
        with pytest.raises(ValueError, match="rows"):
            H.gemm_fp8_silu_mul(x, layer(N, 256))
        with pytest.raises(ValueError, match="rows"):
            H.gemm_fp8_silu_mul_backward(x, layer(N, 256), torch.zeros((4, N // 2), dtype=torch.float16))
    H.gemm_fp8_silu_mul(x, layer(256, 256))
    H.gemm_fp8_silu_mul_backward(x, layer(256, 256), d)


# ------------------------------------------------------------------------------------------------ results over inputs
A, GAP = 1 << 20, 1 << 20      # addresses that are never followed
M, N, K = 8, 512, 256


def overlapping(fn, sizes, results, allowed, numbers):
    """Each result laid over the first, the last and all bytes of each other argument: refused, unless `allowed`; then beside it: not refused
    for that."""
    at = {n: A + GAP * i for i, n in enumerate(sizes)}
    for r in results:
        for n in sizes:
            if n == r or sizes[n] == 0 or sizes[r] == 0:
                continue
            first, last = at[n] - (sizes[r] - 1) // 16 * 16, at[n] + (sizes[n] - 1) // 16 * 16
            for place in {first, last, at[n]}:
                if (r, n) in allowed and place == at[n]:
                    continue
                assert fn(*[None if sizes[k] == 0 else place if k == r else v for k, v in at.items()], *numbers, stream=0) == B.GPTQ_ERR_LAYOUT, (r, n)


def test_refused_overlaps():
    q = {"x": M * K * 2, "q": M * K, "s": M * 2 * 4}
    overlapping(B.gptq_fp8_quantize, q, ("q", "s"), (), (M, K, 0))
    overlapping(B.gptq_fp8_transpose, {"w": N * K, "s": 4 * 2 * 4, "wo": N * K, "so": 4 * 2 * 4}, ("wo", "so"), (), (N, K))
    for x8 in (False, True):
        x = {"x": M * K * (1 if x8 else 2), "xs": M * 2 * 4 if x8 else 0, "w": N * K, "ws": 4 * 2 * 4}
        overlapping(B.gptq_gemm_fp8, {**x, "bias": 2 * N, "residual": 2 * M * N, "y": 2 * M * N}, ("y",), (("y", "residual"),), (M, N, K, 0))
        for out8 in (False, True):
            def outs(columns):
                return {"out": M * columns * (1 if out8 else 2), "outs": M * (columns // 128) * 4 if out8 else 0}
            overlapping(B.gptq_gemm_fp8_silu_mul, {**x, **outs(N // 2)}, ("out", "outs"), (), (M, N // 2, K, 0))
            overlapping(B.gptq_gemm_fp8_silu_mul_backward, {**x, "d": M * N // 2 * 2, **outs(N)}, ("out", "outs"), (), (M, N // 2, K, 0))


def test_the_longest_rows():
    """K up to the last multiple of 16 below 2^31."""
    K = (1 << 31) - 16
    assert B.gptq_fp8_workspace_bytes(1, K) == (1 << 31) + 4 * (1 << 24)      # (e4m3 rows end on 256 bytes)
    assert B.gptq_fp8_workspace_bytes(3, K - 128) == 3 * (K - 128) + (-3 * (K - 128) % 256) + 3 * 4 * ((1 << 24) - 1)
    for shape in ((1, 8, K), (1, (1 << 31) - 8, 16), (1300, (1 << 31) - 8, 16)):
        st, p = B.gptq_plan_fp8(*shape, 0, 148)
        assert st == B.GPTQ_OK and p.items >= 1 << 23 and p.ctas >= 1


# ------------------------------------------------------------------------------------------------ the quotient of the e4m3 results
def test_the_quotient_decides_as_the_nearest_number_does():
    """q + (v - q s) y, q = v y, y = 1 / s rounded, is within 2^-46 of v / s before its last rounding: the e4m3 number can differ from that of the
    correctly rounded quotient only where v / s is that near b, the middle of two fp32 numbers of which one is a middle t of e4m3 numbers (five bits).  With
    s = S 2^a and v = V 2^c (24 bits each) and b = B 2^e, B = 2^20 T +- 1, that is |V 2^j - S B| <= 8, j = 24 or 25: every such pair."""
    fmaf = ctypes.CDLL(ctypes.util.find_library("m")).fmaf
    fmaf.restype, fmaf.argtypes = ctypes.c_float, [ctypes.c_float] * 3
    f = np.float32
    pairs, got, want = 0, [], []
    for T in range(16, 33):
        for sign in (1, -1):
            B_ = (T << 20) + sign
            if not 1 << 24 < B_ < 1 << 25:
                continue
            for n in range(-9, 10):
                for S in ((k << 20) - sign * n for k in range(8, 17)):
                    for j in (24, 25):
                        V, rest = divmod(S * B_ + n, 1 << j)
                        if rest or not (1 << 23 <= S < 1 << 24 and 1 << 23 <= V < 1 << 24):
                            continue
                        pairs += 1
                        s = np.ldexp(f(S), -23)
                        for e in range(-20, 9):      # from beside zero to beyond the largest number
                            v = np.ldexp(f(V), e - 23)
                            y = f(1) / s
                            q = v * y
                            got.append(fmaf(fmaf(-q, s, v), y, q))
                            want.append(v / s)
    assert pairs == 205
    got, want = (torch.tensor(np.array(a, dtype=f)).clamp(max=448.0).to(torch.float8_e4m3fn).view(torch.uint8) for a in (got, want))
    assert torch.equal(got, want)


# ------------------------------------------------------------------------------------------------ tensor memory of an SM
SM_BYTES, CTA_BYTES = 228 * 1024, 1024      # shared memory of an SM, and what each CTA takes of it beside its own


def fp8_residents():
    """(bytes, columns) of each instance of the e4m3 kernels."""
    out = set()
    for gated in (0, 1):
        for M in (1, 16, 20, 32, 40, 64, 100, 128, 3000):
            st, p = B.gptq_plan_fp8(M, 22016, 4096, gated, 148)
            assert st == B.GPTQ_OK
            name = p.kernel_name.decode()
            if p.kernel == 6:
                kind, rows = (int(v) for v in re.findall(r"\d+", name.split("<")[1]))
                columns = (1 + kind) * rows * (4 if (1 + kind) * rows <= 128 else 2)      # accumulators of a block of K each
                out.add((name, p.smem_bytes, max(32, columns)))
            else:
                out.add((name, p.smem_bytes, 512))
    assert len(out) >= 8
    return out


def test_e4m3_kernels_never_wait_for_tensor_memory_beside_another_kernel():
    """A CTA that waits for columns holds its cluster up, whose other CTAs may hold columns that the first one's neighbour's cluster waits for: kernels on one
    SM together must fit into its 512 columns.  The 4-bit kernels take at least these bytes: for all columns more than half of an SM's, for 256 more than a
    third, for 128 more than a quarter."""
    others = [("all columns", 227 * 1024 // 2 + 512, 512), ("two per SM", 227 * 1024 // 3 + 512, 256), ("three per SM", 227 * 1024 // 4 + 512, 128)]
    mine = sorted(fp8_residents())
    for first in mine:
        for n in range(1, 4):
            for rest in itertools.combinations_with_replacement(mine + others, n):
                together = (first, *rest)
                if sum(b + CTA_BYTES for _, b, _ in together) <= SM_BYTES:
                    assert sum(c for _, _, c in together) <= 512, together


def test_rows_of_16_bits_give_results_of_their_own_type(calls):
    """Another type that was asked for was passed over without a word."""
    x, D = torch.zeros((4, 256), dtype=torch.float16), layer(256, 256)
    for fn in (H.gemm_fp8, H.gemm_fp8_silu_mul):
        with pytest.raises(ValueError, match="bfloat16"):
            fn(x, D, dtype=torch.bfloat16)
        assert fn(x, D, dtype=torch.float16).dtype == fn(x, D).dtype == torch.float16
        x8, s = x.to(torch.float8_e4m3fn), torch.ones((4, 2))
        assert fn(x8, D, x_scales=s).dtype == torch.float16 and fn(x8, D, x_scales=s, dtype=torch.bfloat16).dtype == torch.bfloat16

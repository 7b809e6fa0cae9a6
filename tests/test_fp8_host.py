"""Argument checks of the layers in 8-bit floating point: no GPU needed, nothing is launched."""
import pytest

from paper_2511_19438_b200 import build as libbuild

libbuild.build()
from paper_2511_19438_b200 import binding as B  # noqa: E402

A16 = 0x1000  # a fake, 16-byte aligned "device address"; validation never dereferences it


def caller(fn, pointers, sizes, fmt=0):
    def call(**kw):
        p = {n: A16 + 16 * i for i, n in enumerate(pointers)}
        s = dict(sizes)
        f = kw.pop("fmt", fmt)
        for n, v in kw.items():
            (p if n in p else s)[n] = v
        return fn(*p.values(), *s.values(), f, stream=0)
    return call


CALLS = {
    "quantize": (B.gptq_fp8_quantize, ["x", "q", "s"], dict(M=4, K=256), ()),
    "gemm": (B.gptq_gemm_fp8, ["x", "xs", "w", "ws", "bias", "residual", "y"], dict(M=4, N=256, K=256), ("xs", "bias", "residual")),
    "gated": (B.gptq_gemm_fp8_silu_mul, ["x", "xs", "w", "ws", "y", "ys"], dict(M=4, F=128, K=256), ("xs", "ys")),
    "backward": (B.gptq_gemm_fp8_silu_mul_backward, ["x", "xs", "w", "ws", "d", "y", "ys"], dict(M=4, F=128, K=256), ("xs", "ys")),
}


@pytest.mark.parametrize("name", CALLS)
def test_refusals(name):
    fn, pointers, sizes, optional = CALLS[name]
    call = caller(fn, pointers, sizes)
    for p in pointers:
        if p not in optional:
            assert call(**{p: None}) == B.GPTQ_ERR_NULL, p
        assert call(**{p: A16 + 8}) == B.GPTQ_ERR_ALIGN, p
    for bad in (dict(M=0), dict(M=-1), dict(K=0), dict(K=8), dict(K=264), dict(K=-16)):
        assert call(**bad) == B.GPTQ_ERR_SHAPE, bad
    for fmt in (-1, 1, 2, 8, B.GPTQ_FORMAT_BF16 | 1):
        assert call(fmt=fmt) == B.GPTQ_ERR_LAYOUT, fmt


def test_refused_widths():
    gemm = caller(*CALLS["gemm"][:3])
    for N in (0, 4, 7, 12, -8):
        assert gemm(N=N) == B.GPTQ_ERR_SHAPE, N
    for name in ("gated", "backward"):
        call = caller(*CALLS[name][:3])
        for F in (0, 64, 100, 192, -128, 1 << 30):
            assert call(F=F) == B.GPTQ_ERR_SHAPE, (name, F)


def test_refused_overlaps():
    assert caller(*CALLS["quantize"][:3])(q=A16) == B.GPTQ_ERR_LAYOUT
    for name in ("gemm", "gated", "backward"):
        call = caller(*CALLS[name][:3])
        assert call(y=A16) == B.GPTQ_ERR_LAYOUT, name
    assert caller(*CALLS["backward"][:3])(d=A16 + 16 * 5) == B.GPTQ_ERR_LAYOUT      # d_gate_up = d_out


def test_transpose_refusals():
    def call(w=A16, s=A16 + 16, wo=A16 + 32, so=A16 + 48, N=256, K=256):
        return B.gptq_fp8_transpose(w, s, wo, so, N, K, stream=0)

    for p in ("w", "s", "wo", "so"):
        assert call(**{p: None}) == B.GPTQ_ERR_NULL
        assert call(**{p: A16 + 4}) == B.GPTQ_ERR_ALIGN
    for bad in (dict(N=0), dict(N=8), dict(N=24), dict(K=0), dict(K=40), dict(N=-16)):
        assert call(**bad) == B.GPTQ_ERR_SHAPE, bad
    assert call(wo=A16) == B.GPTQ_ERR_LAYOUT
    assert call(so=A16 + 16) == B.GPTQ_ERR_LAYOUT


def test_workspace_sizes():
    # e4m3 rows, then a scale for each block of 128
    assert B.gptq_fp8_workspace_bytes(1, 16) == 256 + 4
    assert B.gptq_fp8_workspace_bytes(3, 4096) == 3 * 4096 + 3 * 32 * 4
    assert B.gptq_fp8_workspace_bytes(5, 4112) >= 5 * 4112 + 5 * 33 * 4
    assert B.gptq_fp8_workspace_bytes(1 << 20, 1 << 16) == (1 << 36) + (1 << 31)
    need = [B.gptq_fp8_workspace_bytes(m, 2064) for m in range(1, 3000)]
    assert need == sorted(need)
    for bad in ((0, 256), (4, 0), (4, 8), (4, 264), (-1, 256)):
        assert B.gptq_fp8_workspace_bytes(*bad) == 0

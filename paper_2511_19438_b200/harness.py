"""Device-side plumbing for tests and the benchmark: uploads a synthetic layer,
runs the one-time repack through the C ABI, keeps the workspace registered.

torch is used only to own device memory and streams; every computation is a
call into libgptq_b200.so through ``binding``.
"""
from __future__ import annotations

import contextlib
from dataclasses import dataclass

import numpy as np
import torch

from . import binding as B
from .workloads import QuantLinear


@dataclass
class DeviceLinear:
    """A layer resident on the GPU: canonical buffers (optional) and the tiled ones."""
    K: int
    N: int
    group_size: int
    act_order: bool
    qweight_t: torch.Tensor      # tiled
    qzeros_t: torch.Tensor
    scales_t: torch.Tensor
    perm: torch.Tensor | None    # int32[K], original index of sorted row i
    canonical: tuple | None      # (qweight, qzeros, scales, g_idx) device tensors, if kept


def to_device(a: np.ndarray, device="cuda") -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(a)).to(device)


def upload_and_repack(L: QuantLinear, keep_canonical: bool = False, device="cuda", gate_up: bool = False,
                      scales_bf16_bits: np.ndarray | None = None) -> DeviceLinear:
    """``scales_bf16_bits`` (uint16 [G, N]) replaces the layer's fp16 scales by bfloat16 ones and marks the tiled
    layer as a bfloat16 layer (to be used with :func:`gemm_bf16`)."""
    qw = to_device(L.qweight, device)
    qz = to_device(L.qzeros, device)
    if scales_bf16_bits is not None:
        assert scales_bf16_bits.dtype == np.uint16 and scales_bf16_bits.shape == (L.K // L.group_size, L.N)
        sc = to_device(scales_bf16_bits.view(np.int16), device).view(torch.bfloat16)
    else:
        sc = to_device(L.scales, device)
    gi = to_device(L.g_idx, device) if L.act_order else None
    qw_t = torch.empty(B.gptq_repack_bytes(0, L.N, L.K, L.group_size, L.act_order), dtype=torch.uint8, device=device)
    qz_t = torch.empty(B.gptq_repack_bytes(1, L.N, L.K, L.group_size, L.act_order), dtype=torch.uint8, device=device)
    sc_t = torch.empty(B.gptq_repack_bytes(2, L.N, L.K, L.group_size, L.act_order), dtype=torch.uint8, device=device)
    perm = torch.empty(L.K, dtype=torch.int32, device=device) if L.act_order else None
    fmt = (B.GPTQ_FORMAT_ZEROS_MINUS_ONE if L.zeros_minus_one else 0) | (B.GPTQ_FORMAT_GATE_UP if gate_up else 0)
    fmt |= B.GPTQ_FORMAT_BF16 if scales_bf16_bits is not None else 0
    B.check(B.gptq_repack_format(qw, qz, sc, gi, qw_t, qz_t, sc_t, perm, L.N, L.K, L.group_size, L.act_order, fmt),
            "gptq_repack_format")
    torch.cuda.current_stream().synchronize()
    canonical = (qw, qz, sc, gi) if keep_canonical else None
    return DeviceLinear(L.K, L.N, L.group_size, L.act_order, qw_t, qz_t, sc_t, perm, canonical)


class WorkspaceHolder:
    """Owns one device scratch buffer and keeps it registered with the library."""

    def __init__(self, device="cuda"):
        self.device = device
        self.buf = None

    def ensure(self, nbytes: int) -> None:
        if nbytes <= 0:
            return
        if self.buf is None or self.buf.numel() < nbytes:
            torch.cuda.synchronize()
            self.buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        # registering is idempotent and cheap (a host-side pointer swap)
        B.check(B.gptq_set_workspace(self.buf, self.buf.numel()), "gptq_set_workspace")

    def ensure_for(self, M: int, D: DeviceLinear) -> None:
        self.ensure(B.gptq_workspace_bytes(M, D.N, D.K, D.group_size, D.act_order))


def gemm(x: torch.Tensor, D: DeviceLinear, y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y = x . dequant(W) through gptq_gemm (x fp16 [M, K] on the device)."""
    M = x.shape[0]
    if y is None:
        y = torch.empty((M, D.N), dtype=torch.float16, device=x.device)
    B.check(B.gptq_gemm(x, D.qweight_t, D.qzeros_t, D.scales_t, D.perm, y, M, D.N, D.K, D.group_size,
                        D.act_order, stream), "gptq_gemm")
    return y


def bf16_from_bits(bits: np.ndarray, device="cuda") -> torch.Tensor:
    """uint16 bit patterns -> a bfloat16 tensor on the device (no conversion: the same 16 bits)."""
    return to_device(np.ascontiguousarray(bits).view(np.int16), device).view(torch.bfloat16)


def bits_of_bf16(t: torch.Tensor) -> np.ndarray:
    """A bfloat16 tensor -> its bit patterns as a numpy uint16 array."""
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def gemm_bf16(x: torch.Tensor, D: DeviceLinear, y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y = x . dequant(W) through gptq_gemm_bf16 (x bfloat16 [M, K] on the device, D repacked with bfloat16 scales)."""
    assert x.dtype == torch.bfloat16
    M = x.shape[0]
    if y is None:
        y = torch.empty((M, D.N), dtype=torch.bfloat16, device=x.device)
    B.check(B.gptq_gemm_bf16(x, D.qweight_t, D.qzeros_t, D.scales_t, D.perm, y, M, D.N, D.K, D.group_size,
                             D.act_order, stream), "gptq_gemm_bf16")
    return y


def gemm_silu_mul(x: torch.Tensor, D: DeviceLinear, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """out[M, N / 2] = silu(gate) * up through gptq_gemm_silu_mul (D repacked with gate_up=True)."""
    M = x.shape[0]
    if out is None:
        out = torch.empty((M, D.N // 2), dtype=torch.float16, device=x.device)
    B.check(B.gptq_gemm_silu_mul(x, D.qweight_t, D.qzeros_t, D.scales_t, D.perm, out, M, D.N, D.K, D.group_size,
                                 D.act_order, stream), "gptq_gemm_silu_mul")
    return out


def gemm_bias_residual(x: torch.Tensor, D: DeviceLinear, bias: torch.Tensor | None, residual: torch.Tensor | None,
                       y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y = x . dequant(W) + bias + residual through gptq_gemm_bias_residual (y may be the residual buffer)."""
    M = x.shape[0]
    if y is None:
        y = torch.empty((M, D.N), dtype=torch.float16, device=x.device)
    B.check(B.gptq_gemm_bias_residual(x, D.qweight_t, D.qzeros_t, D.scales_t, D.perm, bias, residual, y, M, D.N, D.K,
                                      D.group_size, D.act_order, stream), "gptq_gemm_bias_residual")
    return y


def invert_perm(perm: torch.Tensor) -> torch.Tensor:
    """inverse[perm[i]] = i through gptq_invert_perm."""
    inv = torch.empty_like(perm)
    B.check(B.gptq_invert_perm(perm, inv, perm.numel()), "gptq_invert_perm")
    return inv


def gemm_silu_mul_scatter(x: torch.Tensor, D: DeviceLinear, out_index: torch.Tensor, out: torch.Tensor | None = None,
                          stream=None) -> torch.Tensor:
    """gemm_silu_mul whose output column i lands at column out_index[i]."""
    M = x.shape[0]
    if out is None:
        out = torch.empty((M, D.N // 2), dtype=torch.float16, device=x.device)
    B.check(B.gptq_gemm_silu_mul_scatter(x, D.qweight_t, D.qzeros_t, D.scales_t, D.perm, out_index, out, M, D.N, D.K,
                                         D.group_size, D.act_order, stream), "gptq_gemm_silu_mul_scatter")
    return out


def gemm_presorted(x_sorted: torch.Tensor, D: DeviceLinear, y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """gptq_gemm of an act-order layer whose input already is in the layer's sorted row order (no gather)."""
    M = x_sorted.shape[0]
    if y is None:
        y = torch.empty((M, D.N), dtype=torch.float16, device=x_sorted.device)
    B.check(B.gptq_gemm(x_sorted, D.qweight_t, D.qzeros_t, D.scales_t, None, y, M, D.N, D.K, D.group_size,
                        B.GPTQ_ACT_ORDER_PRESORTED, stream), "gptq_gemm (pre-sorted)")
    return y


# ---- 8-bit layers (stored as two stacked 4-bit planes) ----------------------------------------------------------------

def upload_and_repack_w8(L: QuantLinear, keep_canonical: bool = False, device="cuda") -> DeviceLinear:
    """Uploads a canonical 8-bit layer (qweight int32[K/4, N], qzeros int32[G, N/4]) and repacks it with gptq_repack_w8.
    The returned DeviceLinear keeps the checkpoint's K and group size; ``perm`` is int32[2 K]."""
    qw, qz, sc = to_device(L.qweight, device), to_device(L.qzeros, device), to_device(L.scales, device)
    gi = to_device(L.g_idx, device) if L.act_order else None
    outs = [torch.empty(B.gptq_repack_w8_bytes(w, L.N, L.K, L.group_size), dtype=torch.uint8, device=device) for w in range(3)]
    perm = torch.empty(2 * L.K, dtype=torch.int32, device=device)
    nscratch = B.gptq_repack_w8_scratch_bytes(L.N, L.K, L.group_size)
    scratch = torch.empty(nscratch, dtype=torch.uint8, device=device)
    fmt = B.GPTQ_FORMAT_ZEROS_MINUS_ONE if L.zeros_minus_one else 0
    B.check(B.gptq_repack_w8(qw, qz, sc, gi, outs[0], outs[1], outs[2], perm, scratch, nscratch, L.N, L.K, L.group_size,
                             L.act_order, fmt), "gptq_repack_w8")
    torch.cuda.current_stream().synchronize()
    canonical = (qw, qz, sc, gi) if keep_canonical else None
    return DeviceLinear(L.K, L.N, L.group_size, L.act_order, outs[0], outs[1], outs[2], perm, canonical)


def gemm_w8(x: torch.Tensor, D: DeviceLinear, y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y = x . dequant(W8) through gptq_gemm_w8 (the workspace must hold the gathered activations, see ensure_for_w8)."""
    M = x.shape[0]
    if y is None:
        y = torch.empty((M, D.N), dtype=torch.float16, device=x.device)
    B.check(B.gptq_gemm_w8(x, D.qweight_t, D.qzeros_t, D.scales_t, D.perm, y, M, D.N, D.K, D.group_size, stream), "gptq_gemm_w8")
    return y


def ensure_for_w8(ws: "WorkspaceHolder", M: int, D: DeviceLinear) -> None:
    ws.ensure(B.gptq_workspace_bytes(M, D.N, 2 * D.K, D.group_size, 1))


# ---- 2- and 3-bit layers (widened to a 4-bit layer by the repack) -----------------------------------------------------

def upload_and_repack_bits(L: QuantLinear, bits: int, keep_canonical: bool = False, device="cuda") -> DeviceLinear:
    """Uploads a canonical 2- or 3-bit layer and repacks it with gptq_repack_bits; the result is an ordinary tiled 4-bit
    layer for :func:`gemm`."""
    qw, qz, sc = to_device(L.qweight, device), to_device(L.qzeros, device), to_device(L.scales, device)
    gi = to_device(L.g_idx, device) if L.act_order else None
    outs = [torch.empty(B.gptq_repack_bytes(w, L.N, L.K, L.group_size, L.act_order), dtype=torch.uint8, device=device)
            for w in range(3)]
    perm = torch.empty(L.K, dtype=torch.int32, device=device) if L.act_order else None
    nscratch = B.gptq_repack_bits_scratch_bytes(bits, L.N, L.K, L.group_size)
    scratch = torch.empty(nscratch, dtype=torch.uint8, device=device)
    fmt = B.GPTQ_FORMAT_ZEROS_MINUS_ONE if L.zeros_minus_one else 0
    B.check(B.gptq_repack_bits(bits, qw, qz, sc, gi, outs[0], outs[1], outs[2], perm, scratch, nscratch, L.N, L.K,
                               L.group_size, L.act_order, fmt), "gptq_repack_bits")
    torch.cuda.current_stream().synchronize()
    canonical = (qw, qz, sc, gi) if keep_canonical else None
    return DeviceLinear(L.K, L.N, L.group_size, L.act_order, outs[0], outs[1], outs[2], perm, canonical)


# ---- rows that choose their weights: routed experts, low-rank adapters -------------------------------------------------

@dataclass
class DeviceExperts:
    """The experts' layers of one kind (all gate_up or all down) behind one another, tiled."""
    K: int
    N: int
    group_size: int
    act_order: bool
    count: int
    qweight_t: torch.Tensor      # uint8 [count, bytes]
    qzeros_t: torch.Tensor
    scales_t: torch.Tensor
    perm: torch.Tensor | None    # int32 [count, K]
    index: torch.Tensor | None   # its inverse: where row k of the checkpoint sits


def upload_experts(layers: list[QuantLinear], gate_up: bool = False, scales_bf16_bits: list[np.ndarray] | None = None,
                   device="cuda") -> DeviceExperts:
    """Repacks every layer and puts the tiled buffers behind one another, as gptq_moe_mlp takes them."""
    D = [upload_and_repack(L, device=device, gate_up=gate_up, scales_bf16_bits=None if scales_bf16_bits is None else scales_bf16_bits[e])
         for e, L in enumerate(layers)]
    act = D[0].act_order
    return DeviceExperts(D[0].K, D[0].N, D[0].group_size, act, len(D), torch.stack([d.qweight_t for d in D]),
                         torch.stack([d.qzeros_t for d in D]), torch.stack([d.scales_t for d in D]),
                         torch.stack([d.perm for d in D]) if act else None,
                         torch.stack([invert_perm(d.perm) for d in D]) if act else None)


def _expect(name: str, t: torch.Tensor | None, dtype: torch.dtype, shape: tuple) -> None:
    """The kernels take addresses: a tensor of another type, shape or layout would be read as if it had these."""
    if t is not None and (t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous()):
        raise ValueError(f"{name}: contiguous {dtype} {list(shape)} expected, got {t.dtype} {list(t.shape)}, strides {list(t.stride())}")


_LOGITS_TYPE = {torch.float32: B.GPTQ_LOGITS_F32, torch.float16: B.GPTQ_LOGITS_F16, torch.bfloat16: B.GPTQ_LOGITS_BF16}


def moe_route(logits: torch.Tensor, top_k: int, renormalize: bool = True, stream=None) -> tuple[torch.Tensor, torch.Tensor]:
    """(expert ids int32 [M, top_k], weights fp32 [M, top_k]) of router logits [M, E] through gptq_moe_route."""
    M, E = logits.shape
    if logits.dtype not in _LOGITS_TYPE:
        raise ValueError(f"logits: float32, float16 or bfloat16 expected, got {logits.dtype}")
    _expect("logits", logits, logits.dtype, (M, E))
    ids = torch.empty((M, top_k), dtype=torch.int32, device=logits.device)
    weights = torch.empty((M, top_k), dtype=torch.float32, device=logits.device)
    B.check(B.gptq_moe_route(logits, ids, weights, M, E, top_k, _LOGITS_TYPE[logits.dtype], renormalize, stream), "gptq_moe_route")
    return ids, weights


def moe_mlp(x: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor, gate_up: DeviceExperts, down: DeviceExperts,
            residual: torch.Tensor | None = None, y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """A mixture-of-experts MLP through gptq_moe_mlp or, for bfloat16 x, gptq_moe_mlp_bf16 (workspace: ensure_for_moe)."""
    M, K = x.shape
    up, dn = gate_up, down
    if (up.K, up.N, up.count, min(up.group_size, 128), bool(up.act_order)) != (dn.N, 2 * dn.K, dn.count, min(dn.group_size, 128), bool(dn.act_order)):
        raise ValueError(f"gate_up [{up.K}, {up.N}] x {up.count}, groups of {up.group_size}, act-order {up.act_order} and down [{dn.K}, {dn.N}] x "
                         f"{dn.count}, groups of {dn.group_size}, act-order {dn.act_order} are not one layer's experts")
    if y is None:
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
    act = torch.bfloat16 if x.dtype == torch.bfloat16 else torch.float16
    _expect("x", x, act, (M, gate_up.K))
    _expect("ids", ids, torch.int32, (M, ids.shape[-1]))
    _expect("weights", weights, torch.float32, tuple(ids.shape))
    _expect("residual", residual, act, (M, K))
    _expect("y", y, act, (M, K))
    fn = B.gptq_moe_mlp_bf16 if x.dtype == torch.bfloat16 else B.gptq_moe_mlp
    B.check(fn(x, ids, weights, gate_up.qweight_t, gate_up.qzeros_t, gate_up.scales_t, gate_up.perm, down.qweight_t, down.qzeros_t,
               down.scales_t, down.index, residual, y, M, K, down.K, gate_up.count, ids.shape[1], min(gate_up.group_size, 128),
               gate_up.act_order, stream), fn.__name__)
    return y


def ensure_for_moe(ws: "WorkspaceHolder", M: int, gate_up: DeviceExperts, top_k: int) -> None:
    ws.ensure(B.gptq_moe_workspace_bytes(M, gate_up.K, gate_up.N // 2, top_k, gate_up.act_order))


def gemm_lora(x: torch.Tensor, D: DeviceLinear, lora_a: torch.Tensor, lora_b: torch.Tensor, adapter_ids: torch.Tensor,
              adapter_scales: torch.Tensor | None = None, y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y = x . dequant(W) + scale (x A^T) B^T with each row's adapter, through gptq_gemm_lora or, for bfloat16 x,
    gptq_gemm_lora_bf16 (workspace: ensure_for_lora)."""
    M = x.shape[0]
    if y is None:
        y = torch.empty((M, D.N), dtype=x.dtype, device=x.device)
    act = torch.bfloat16 if x.dtype == torch.bfloat16 else torch.float16
    adapters, rank = lora_a.shape[0], lora_a.shape[1]
    _expect("x", x, act, (M, D.K))
    _expect("lora_a", lora_a, act, (adapters, rank, D.K))
    _expect("lora_b", lora_b, act, (adapters, D.N, rank))
    _expect("adapter_ids", adapter_ids, torch.int32, (M,))
    _expect("adapter_scales", adapter_scales, torch.float32, (adapters,))
    _expect("y", y, act, (M, D.N))
    fn = B.gptq_gemm_lora_bf16 if x.dtype == torch.bfloat16 else B.gptq_gemm_lora
    B.check(fn(x, D.qweight_t, D.qzeros_t, D.scales_t, D.perm, lora_a, lora_b, adapter_ids, adapter_scales, y, M, D.N, D.K,
               D.group_size, D.act_order, lora_a.shape[1], lora_a.shape[0], stream), fn.__name__)
    return y


def ensure_for_lora(ws: "WorkspaceHolder", M: int, D: DeviceLinear, rank: int) -> None:
    ws.ensure(B.gptq_lora_workspace_bytes(M, D.N, D.K, D.group_size, D.act_order, rank))


# ---- layers in 8-bit floating point -------------------------------------------------------------------------------------

@dataclass
class DeviceFp8Linear:
    """An e4m3 layer as checkpoints hold it, and its transpose where gradients are wanted."""
    K: int
    N: int
    weight: torch.Tensor         # float8_e4m3fn [N, K]
    scales: torch.Tensor         # float32 [ceil(N / 128), ceil(K / 128)]
    transposed: "DeviceFp8Linear | None" = None


def _blocks(n: int) -> int:
    return -(-n // 128)


def _here() -> torch.device:
    return torch.device("cuda", torch.cuda.current_device())


def _expect_here(*tensors: torch.Tensor | None) -> None:
    """The kernels run on the current device, with the addresses that they are given."""
    here = _here()
    for t in tensors:
        if t is not None and t.device != here:
            raise ValueError(f"a tensor on {t.device}, the current device is {here}")


def fp8_linear(weight: torch.Tensor, scales: torch.Tensor, transpose: bool = False) -> DeviceFp8Linear:
    """A layer whose tensors are on the GPU; ``transpose``: laid out the other way round too (gptq_fp8_transpose)."""
    N, K = weight.shape
    _expect("weight", weight, torch.float8_e4m3fn, (N, K))
    _expect("scales", scales, torch.float32, (_blocks(N), _blocks(K)))
    _expect_here(weight, scales)
    D = DeviceFp8Linear(K, N, weight, scales)
    if transpose:
        T = DeviceFp8Linear(N, K, torch.empty((K, N), dtype=weight.dtype, device=weight.device),
                            torch.empty((_blocks(K), _blocks(N)), dtype=scales.dtype, device=scales.device))
        B.check(B.gptq_fp8_transpose(weight, scales, T.weight, T.scales, N, K), "gptq_fp8_transpose")
        torch.cuda.current_stream().synchronize()      # products on any stream, which do not wait for weights, may follow
        D.transposed = T
    return D


def ensure_for_fp8(ws: "WorkspaceHolder", M: int, K: int) -> None:
    """Scratch for calls that bring [M, K] in 16 bits."""
    ws.ensure(B.gptq_fp8_workspace_bytes(M, K))


def _format_of(dtype: torch.dtype) -> int:
    if dtype not in (torch.float16, torch.bfloat16):
        raise ValueError(f"float16 or bfloat16 expected, got {dtype}")
    return B.GPTQ_FORMAT_BF16 if dtype == torch.bfloat16 else 0


def _result_dtype(x: torch.Tensor, x_scales: torch.Tensor | None, dtype: torch.dtype | None) -> torch.dtype:
    if x_scales is None and dtype not in (None, x.dtype):
        raise ValueError(f"the result of {x.dtype} rows is {x.dtype}, not {dtype}")
    return x.dtype if x_scales is None else dtype or torch.float16


def _expect_rows(x: torch.Tensor, x_scales: torch.Tensor | None, dtype: torch.dtype, D: DeviceFp8Linear) -> int:
    M = x.shape[0]
    _expect("x", x, dtype if x_scales is None else torch.float8_e4m3fn, (M, D.K))
    _expect("x_scales", x_scales, torch.float32, (M, _blocks(D.K)))
    _expect_here(x, x_scales, D.weight, D.scales)
    return M


def _gated_columns(D: DeviceFp8Linear) -> int:
    if D.N % 256:
        raise ValueError(f"gate's rows, then as many of up's, a multiple of 128 each, expected, got {D.N} rows")
    return D.N // 2


def _rows_fp8(M: int, N: int, device) -> tuple[torch.Tensor, torch.Tensor]:
    return (torch.empty((M, N), dtype=torch.float8_e4m3fn, device=device), torch.empty((M, _blocks(N)), dtype=torch.float32, device=device))


def fp8_quantize(x: torch.Tensor, stream=None) -> tuple[torch.Tensor, torch.Tensor]:
    """(e4m3 [M, K], fp32 scales [M, ceil(K / 128)]) of 16-bit rows through gptq_fp8_quantize."""
    M, K = x.shape
    _expect("x", x, x.dtype, (M, K))
    _expect_here(x)
    q, s = _rows_fp8(M, K, x.device)
    B.check(B.gptq_fp8_quantize(x, q, s, M, K, _format_of(x.dtype), stream), "gptq_fp8_quantize")
    return q, s


def gemm_fp8(x: torch.Tensor, D: DeviceFp8Linear, bias: torch.Tensor | None = None, residual: torch.Tensor | None = None,
             y: torch.Tensor | None = None, x_scales: torch.Tensor | None = None, dtype: torch.dtype | None = None,
             stream=None) -> torch.Tensor:
    """y = x w^T + bias + residual through gptq_gemm_fp8: x 16-bit (workspace: ensure_for_fp8), or e4m3 with ``x_scales`` and the
    ``dtype`` of the result."""
    dtype = _result_dtype(x, x_scales, dtype)
    fmt = _format_of(dtype)
    M = _expect_rows(x, x_scales, dtype, D)
    if y is None:
        y = torch.empty((M, D.N), dtype=dtype, device=x.device)
    _expect("bias", bias, dtype, (D.N,))
    _expect("residual", residual, dtype, (M, D.N))
    _expect("y", y, dtype, (M, D.N))
    _expect_here(bias, residual, y)
    B.check(B.gptq_gemm_fp8(x, x_scales, D.weight, D.scales, bias, residual, y, M, D.N, D.K, fmt, stream), "gptq_gemm_fp8")
    return y


def gemm_fp8_silu_mul(x: torch.Tensor, D: DeviceFp8Linear, x_scales: torch.Tensor | None = None, quantized: bool = False,
                      dtype: torch.dtype | None = None, stream=None):
    """silu(gate) * up [M, N / 2] through gptq_gemm_fp8_silu_mul, D's rows = gate's, then up's: 16-bit, or (``quantized``) e4m3 and
    its scales."""
    dtype = _result_dtype(x, x_scales, dtype)
    fmt = _format_of(dtype)
    M, F = _expect_rows(x, x_scales, dtype, D), _gated_columns(D)
    out, s = _rows_fp8(M, F, x.device) if quantized else (torch.empty((M, F), dtype=dtype, device=x.device), None)
    B.check(B.gptq_gemm_fp8_silu_mul(x, x_scales, D.weight, D.scales, out, s, M, F, D.K, fmt, stream), "gptq_gemm_fp8_silu_mul")
    return (out, s) if quantized else out


def gemm_fp8_silu_mul_backward(x: torch.Tensor, D: DeviceFp8Linear, d_out: torch.Tensor, x_scales: torch.Tensor | None = None,
                               quantized: bool = True, stream=None):
    """The gradients [M, N] of gate's and up's columns through gptq_gemm_fp8_silu_mul_backward: e4m3 and scales, or 16-bit."""
    fmt = _format_of(d_out.dtype)
    M, F = _expect_rows(x, x_scales, d_out.dtype, D), _gated_columns(D)
    _expect("d_out", d_out, d_out.dtype, (M, F))
    _expect_here(d_out)
    out, s = _rows_fp8(M, D.N, x.device) if quantized else (torch.empty((M, D.N), dtype=d_out.dtype, device=x.device), None)
    B.check(B.gptq_gemm_fp8_silu_mul_backward(x, x_scales, D.weight, D.scales, d_out, out, s, M, F, D.K, fmt, stream),
            "gptq_gemm_fp8_silu_mul_backward")
    return (out, s) if quantized else out


def _memory_of(stream, device):
    """What is allocated inside and freed before the call returns is used again on ``stream`` only, behind the kernels that read it."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(B._stream(stream), device=device))


def mlp_fp8(x: torch.Tensor, gate_up: DeviceFp8Linear, down: DeviceFp8Linear, residual: torch.Tensor | None = None,
            y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """A gated feed-forward block, y = down(silu(gate) * up) + residual, the activation in 8 bits between the layers
    (workspace: ensure_for_fp8 of x)."""
    if y is None:
        y = torch.empty((x.shape[0], down.N), dtype=x.dtype, device=x.device)
    with _memory_of(stream, x.device):
        h, s = gemm_fp8_silu_mul(x, gate_up, quantized=True, stream=stream)
        return gemm_fp8(h, down, residual=residual, y=y, x_scales=s, dtype=x.dtype, stream=stream)


def mlp_fp8_backward(x: torch.Tensor, gate_up: DeviceFp8Linear, down: DeviceFp8Linear, d_y: torch.Tensor, stream=None) -> torch.Tensor:
    """The gradient of mlp_fp8's x without the residual's share (layers with their transposes; workspace: ensure_for_fp8 of d_y
    and of x)."""
    if gate_up.transposed is None or down.transposed is None:
        raise ValueError("gate_up and down are needed the other way round too: fp8_linear(..., transpose=True)")
    dx = torch.empty((x.shape[0], gate_up.K), dtype=x.dtype, device=x.device)
    with _memory_of(stream, x.device):
        d_h = gemm_fp8(d_y, down.transposed, stream=stream)
        d_gate_up, s = gemm_fp8_silu_mul_backward(x, gate_up, d_h, stream=stream)
        return gemm_fp8(d_gate_up, gate_up.transposed, y=dx, x_scales=s, dtype=x.dtype, stream=stream)

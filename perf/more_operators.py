"""Timed cases of the layers held in 8-bit floating point, next to the quantised 4-bit and 8-bit integer ones.

Every operand is e4m3 (1 sign, 4 exponent, 3 fraction bits) with fp32 scales: activations and gradients have one for each 128
columns of a row, weights [N, K] one for each 128 x 128 block.  Kinds of case (``kind``):

* ``quantize``  rows of 16-bit numbers to e4m3 and their scales (``gptq_fp8_quantize``).
* ``gemm``      y = x W^T, with bias and residual where ``extras`` (``gptq_gemm_fp8``).
* ``gated``     silu(x Wg^T) * (x Wu^T), the first half of a gated feed-forward block (``gptq_gemm_fp8_silu_mul``).
* ``grad``      the way back through it: the gradients of both projections' outputs, and of x
                (``gptq_gemm_fp8_silu_mul_backward``, then ``gptq_gemm_fp8`` with the layer laid out the other way round).

``x8``: x arrives as e4m3 with its scales; otherwise as 16-bit numbers, which the call turns into these.  ``out8``: the result
is wanted as e4m3 with its scales, as the next product takes it; otherwise in 16 bits.
"""
from __future__ import annotations

import torch

own = False

E4M3_MAX, SCALE_MIN, BLOCK = 448.0, 2.0 ** -126, 128
_DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
_workspace = None


def _quantize(name, M, K, **kw):
    return {"name": name, "kind": "quantize", "M": M, "K": K, "dtype": "fp16", **kw}


def _gemm(name, M, K, N, **kw):
    return {"name": name, "kind": "gemm", "M": M, "K": K, "N": N, "dtype": "fp16", "x8": False, "extras": False, **kw}


def _gated(name, M, K, F, **kw):
    return {"name": name, "kind": "gated", "M": M, "K": K, "F": F, "dtype": "fp16", "x8": False, "out8": False, **kw}


def _grad(name, M, K, F, **kw):
    return {"name": name, "kind": "grad", "M": M, "K": K, "F": F, "dtype": "fp16", **kw}


def listed():
    return [
        # a decode batch's activations in front of a layer; those of a long prompt in front of the 7B down projection
        _quantize("quantize_m16", 16, 4096),
        _quantize("quantize_m4096_bf16", 4096, 11008, dtype="bf16"),
        # token generation for one user, a small projection
        _gemm("gemm_m1", 1, 4096, 4096),
        # a handful of users, a long K, bias and residual joined
        _gemm("gemm_m7_bf16", 7, 11008, 4096, dtype="bf16", extras=True),
        # a decode batch on the merged query, key and value projection, x already in 8 bits
        _gemm("gemm_m48", 48, 4096, 12288, x8=True),
        # a short prompt, a layer whose last blocks are ragged on both axes
        _gemm("gemm_m300_ragged_bf16", 300, 2064, 1000, dtype="bf16"),
        # a long prompt
        _gemm("gemm_m4096", 4096, 4096, 12288, x8=True),
        # the feed-forward block of the 7B model for one user
        _gated("gated_m1", 1, 4096, 11008),
        # an odd decode batch on a small block, the result in 8 bits for the down projection
        _gated("gated_m33_bf16", 33, 2048, 1408, dtype="bf16", out8=True),
        # a prompt
        _gated("gated_m2048_bf16", 2048, 4096, 11008, dtype="bf16", x8=True, out8=True),
        # training of adapters on frozen layers: a few rows of a small block, a batch on the 7B block
        _grad("grad_m20", 20, 4096, 2048),
        _grad("grad_m1024_bf16", 1024, 4096, 11008, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["quantize", "gemm", "gemm", "gemm", "gated", "gated", "grad"])
    dtype = rng.choice(["fp16", "bf16"])
    M = _log_int(rng, 1, 4096)
    step = rng.choice([16, 128, 128])      # every third layer has ragged blocks
    K = step * _log_int(rng, 512 // step, 11008 // step)
    if kind == "quantize":
        c = _quantize("", M, K, dtype=dtype)
    elif kind == "gemm":
        step = rng.choice([8, 128, 128])
        c = _gemm("", M, K, step * _log_int(rng, 512 // step, 22016 // step), dtype=dtype, x8=rng.random() < 0.5,
                  extras=rng.random() < 0.3)
    elif kind == "gated":
        c = _gated("", M, K, 128 * _log_int(rng, 4, 86), dtype=dtype, x8=rng.random() < 0.5, out8=rng.random() < 0.5)
    else:
        c = _grad("", M, K, 128 * _log_int(rng, 4, 86), dtype=dtype)
    del c["name"]
    most = {m: max(work(k)[m] for k in listed()) for m in ("bytes", "flops")}
    while any(work(c)[m] > most[m] for m in most):
        c["M"] = max(1, c["M"] * 3 // 4)
    return c


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    M, K = case["M"], case["K"]
    x16, x8 = 2 * M * K, M * K + 4 * M * _blocks(K)
    if case["kind"] == "quantize":
        return {"bytes": x16 + x8, "flops": 3 * M * K}
    if case["kind"] == "gemm":
        N = case["N"]
        moved = N * K + 4 * _blocks(N) * _blocks(K) + (x8 if case["x8"] else x16) + 2 * M * N
        return {"bytes": moved + (2 * N + 2 * M * N if case["extras"] else 0), "flops": 2 * M * N * K}
    F = case["F"]
    weights = 2 * F * K + 4 * _blocks(2 * F) * _blocks(K)
    if case["kind"] == "gated":
        out = M * F + 4 * M * _blocks(F) if case["out8"] else 2 * M * F
        return {"bytes": weights + (x8 if case["x8"] else x16) + out, "flops": 4 * M * F * K}
    # x, the gradient of the block's result, both gradients as e4m3, the gradient of x; the layer read both ways round
    return {"bytes": 2 * weights + x8 + 2 * M * F + 2 * M * F + 8 * M * _blocks(F) + x16, "flops": 8 * M * F * K}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _scales_of(t, dims):
    top = t.abs().amax(dims)
    return (top / torch.full_like(top, E4M3_MAX)).clamp(min=SCALE_MIN)      # (by a number torch would multiply by 1 / 448)


def _weights(gen, N, K):
    """A layer [N, K] as checkpoints hold it: e4m3, one fp32 scale for each 128 x 128 block, the last ones ragged."""
    w = torch.zeros((_blocks(N) * BLOCK, _blocks(K) * BLOCK), device="cuda")
    w[:N, :K] = torch.randn((N, K), generator=gen, device="cuda") / K ** 0.5
    w = w.view(_blocks(N), BLOCK, _blocks(K), BLOCK)
    s = _scales_of(w, (1, 3))
    q = (w / s[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(_blocks(N) * BLOCK, -1)[:N, :K].contiguous(), s


def _to_e4m3(x):
    """(e4m3 [M, K], fp32 scales [M, blocks of K]) of rows of numbers, in 32 bits."""
    M, K = x.shape
    t = torch.zeros((M, _blocks(K) * BLOCK), device=x.device)
    t[:, :K] = x
    t = t.view(M, -1, BLOCK)
    s = _scales_of(t, 2)
    return (t / s.unsqueeze(2)).to(torch.float8_e4m3fn).view(M, -1)[:, :K].contiguous(), s


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    M, K, dt = case["M"], case["K"], _DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    # what a norm leaves: channels of different spread, a few of them far out
    spread = torch.exp(0.3 * normal(K)) * torch.where(torch.rand(K, generator=gen, device="cuda") < 0.002, 20.0, 1.0)
    s = {"x": (normal(M, K) * spread).to(dt)}
    if case["kind"] == "gemm":
        s["w"], s["w_scales"] = _weights(gen, case["N"], K)
        s["bias"] = normal(case["N"]).to(dt) if case["extras"] else None
        s["residual"] = (4 * normal(M, case["N"])).to(dt) if case["extras"] else None
    elif case["kind"] != "quantize":
        s["w"], s["w_scales"] = _weights(gen, 2 * case["F"], K)
    if case["kind"] == "grad":
        s["d_out"] = (0.01 * normal(M, case["F"])).to(dt)
    if case.get("x8") or case["kind"] == "grad":
        s["x"], s["x_scales"] = _to_e4m3(s["x"])
    else:
        s["x_scales"] = None
    return s


# ---- what a user's program keeps -------------------------------------------------------------------------------------

def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    M, K, dt = case["M"], case["K"], _DTYPES[case["dtype"]]
    if own:
        # output buffers, the registered scratch; for gradients the frozen layer the other way round, laid out once
        from paper_2511_19438_b200 import binding as B
        from paper_2511_19438_b200 import harness as H

        def empty8(rows, cols):
            return (torch.empty((rows, cols), dtype=torch.float8_e4m3fn, device="cuda"),
                    torch.empty((rows, _blocks(cols)), dtype=torch.float32, device="cuda"))

        global _workspace
        _workspace = _workspace or H.WorkspaceHolder()
        _workspace.ensure(B.gptq_fp8_workspace_bytes(M, K))
        s["format"] = B.GPTQ_FORMAT_BF16 if case["dtype"] == "bf16" else 0
        if case["kind"] == "quantize":
            s["out"], s["out_scales"] = empty8(M, K)
        elif case["kind"] == "gemm":
            s["out"] = torch.empty((M, case["N"]), dtype=dt, device="cuda")
        elif case["kind"] == "gated":
            s["out"], s["out_scales"] = (empty8(M, case["F"]) if case["out8"] else
                                         (torch.empty((M, case["F"]), dtype=dt, device="cuda"), None))
        else:
            s["out"], s["out_scales"] = empty8(M, 2 * case["F"])
            s["dx"] = torch.empty((M, K), dtype=dt, device="cuda")
            s["w_t"], s["w_t_scales"] = empty8(K, 2 * case["F"])
            s["w_t_scales"] = s["w_t_scales"][:_blocks(K)].contiguous()
            B.check(B.gptq_fp8_transpose(s["w"], s["w_scales"], s["w_t"], s["w_t_scales"], 2 * case["F"], K), "gptq_fp8_transpose")
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def _rows(q, s):
    return q.float() * s.repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _layer(q, s):
    return q.float() * s.repeat_interleave(BLOCK, 0)[:q.shape[0]].repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _plain(s):
    case, dt = s["case"], _DTYPES[s["case"]["dtype"]]
    if case["kind"] == "quantize":
        q, scales = _to_e4m3(s["x"])
        return {"x": q, "x_scales": scales}
    x = _rows(*(_to_e4m3(s["x"]) if s["x_scales"] is None else (s["x"], s["x_scales"])))
    y = x @ _layer(s["w"], s["w_scales"]).t()
    if case["kind"] == "gemm":
        if case["extras"]:
            y = y + s["bias"].float() + s["residual"].float()
        return y.to(dt)
    gate, up = y[:, :case["F"]], y[:, case["F"]:]
    p = 1 / (1 + torch.exp(-gate))
    if case["kind"] == "gated":
        h = gate * p * up
        if not case["out8"]:
            return h.to(dt)
        q, scales = _to_e4m3(h)
        return {"h": q, "h_scales": scales}
    d = s["d_out"].float()
    q, scales = _to_e4m3(torch.cat([d * up * p * (1 + gate * (1 - p)), d * gate * p], 1))
    return {"d_gate_up": q, "d_gate_up_scales": scales, "dx": (_rows(q, scales) @ _layer(s["w"], s["w_scales"])).to(dt)}


def run(state):
    s, case = state, state["case"]
    if not own:
        return _plain(s)
    from paper_2511_19438_b200 import binding as B
    M, K = case["M"], case["K"]
    if case["kind"] == "quantize":
        B.check(B.gptq_fp8_quantize(s["x"], s["out"], s["out_scales"], M, K, s["format"]), "gptq_fp8_quantize")
        return {"x": s["out"], "x_scales": s["out_scales"]}
    if case["kind"] == "gemm":
        B.check(B.gptq_gemm_fp8(s["x"], s["x_scales"], s["w"], s["w_scales"], s["bias"], s["residual"], s["out"], M, case["N"], K,
                                s["format"]), "gptq_gemm_fp8")
        return s["out"]
    F = case["F"]
    if case["kind"] == "gated":
        B.check(B.gptq_gemm_fp8_silu_mul(s["x"], s["x_scales"], s["w"], s["w_scales"], s["out"], s["out_scales"], M, F, K,
                                         s["format"]), "gptq_gemm_fp8_silu_mul")
        return {"h": s["out"], "h_scales": s["out_scales"]} if case["out8"] else s["out"]
    B.check(B.gptq_gemm_fp8_silu_mul_backward(s["x"], s["x_scales"], s["w"], s["w_scales"], s["d_out"], s["out"], s["out_scales"],
                                              M, F, K, s["format"]), "gptq_gemm_fp8_silu_mul_backward")
    B.check(B.gptq_gemm_fp8(s["out"], s["out_scales"], s["w_t"], s["w_t_scales"], None, None, s["dx"], M, K, 2 * F, s["format"]),
            "gptq_gemm_fp8")
    return {"d_gate_up": s["out"], "d_gate_up_scales": s["out_scales"], "dx": s["dx"]}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _nearest_e4m3(v):
    """The nearest e4m3 number to each of ``v`` (|v| <= 448), ties to the even one: steps of 1/8 of the power of two below,
    2^-9 in the smallest binade."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=-6) - 3)
    return torch.round(v / step) * step


def _blockwise(v):
    """Rows of float64 as e4m3 numbers and scales, both as float64.  That scales and quotients have 32 bits is part of the
    definition: x / s of 16-bit x often lies next to the middle of two e4m3 numbers, and its 32 bits say on which side."""
    q, scales = torch.empty_like(v), []
    for k in range(0, v.shape[1], BLOCK):
        part = v[:, k:k + BLOCK]
        s = torch.maximum(part.abs().max(1).values / E4M3_MAX, torch.full_like(part[:, 0], SCALE_MIN)).float().double()
        q[:, k:k + BLOCK] = _nearest_e4m3((part / s[:, None]).float().double().clamp(-E4M3_MAX, E4M3_MAX))
        scales.append(s)
    return q, torch.stack(scales, 1)


def _spread(q, scales):
    v = q.to(torch.float64, copy=True)
    for b in range(scales.shape[1]):
        v[:, b * BLOCK:(b + 1) * BLOCK] *= scales[:, b:b + 1].double()
    return v


def _exact_layer(q, scales):
    w = q.double()
    for n in range(scales.shape[0]):
        w[n * BLOCK:(n + 1) * BLOCK] = _spread(w[n * BLOCK:(n + 1) * BLOCK], scales[n:n + 1])
    return w


def exact(case, seed):
    t = _inputs(case, seed)
    x = _blockwise(t["x"].double()) if t["x_scales"] is None else (t["x"], t["x_scales"])
    if case["kind"] == "quantize":
        return {"x": x[0], "x_scales": x[1]}
    w = _exact_layer(t["w"], t["w_scales"])
    y = torch.einsum("mk,nk->mn", _spread(*x), w)
    if case["kind"] == "gemm":
        return y + t["bias"].double() + t["residual"].double() if case["extras"] else y
    g, u = y.split(case["F"], 1)
    e = torch.exp(-g)
    if case["kind"] == "gated":
        h = g / (1 + e) * u
        if not case["out8"]:
            return h
        q, scales = _blockwise(h)
        return {"h": q, "h_scales": scales}
    d = t["d_out"].double()
    q, scales = _blockwise(torch.cat([d * u * (1 + e + g * e) / (1 + e) ** 2, d * g / (1 + e)], 1))
    return {"d_gate_up": q, "d_gate_up_scales": scales, "dx": torch.einsum("mn,nk->mk", _spread(q, scales), w)}

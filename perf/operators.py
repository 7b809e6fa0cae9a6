"""Timed cases of the operators whose rows choose weights of their own, next to quantised 4-bit layers.

Kinds of case (``kind``):

* ``route``  softmax over a row's expert logits, its ``k`` largest, their weights (``gptq_moe_route``).
* ``moe``    a whole mixture-of-experts MLP for a few tokens: the chosen experts' gate/up products, silu(gate) * up, their
             down products, weighted and summed over a token's experts, plus the residual (``gptq_moe_mlp``, ``_bf16``).
* ``lora``   a shared projection with a low-rank adapter per row (``gptq_gemm_lora``, ``_bf16``).

Layers are GPTQ 4-bit: nibbles packed 8 per int32 along K, zero points 8 per int32 along N, one scale per ``group`` rows,
``act`` = act-order checkpoint (row k belongs to group g_idx[k]), ``minus_one`` = zero points stored minus one.
"""
from __future__ import annotations

import torch

own = False

SCALE_FLOOR, SCALE_SIGMA = 0.002, 0.01      # scales are 0.002 + |N(0, 0.01)|, as in this repository's synthetic layers
_DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
_MAX_BYTES, _MAX_FLOPS = 420e6, 34e9        # what the largest listed cases have to read, and to compute
_workspace = None


def _route(name, M, E, k, **kw):
    return {"name": name, "kind": "route", "M": M, "E": E, "k": k, "dtype": "fp32", "renormalize": True, "masked": 0, **kw}


def _moe(name, M, K, F, E, k, **kw):
    return {"name": name, "kind": "moe", "M": M, "K": K, "F": F, "E": E, "k": k, "dtype": "fp16", "group": 128, "act": False,
            "minus_one": False, "padded": 0, **kw}


def _lora(name, M, K, N, rank, adapters, **kw):
    return {"name": name, "kind": "lora", "M": M, "K": K, "N": N, "rank": rank, "adapters": adapters, "dtype": "fp16",
            "group": 128, "act": False, "minus_one": False, "without": 0, "runs": False, **kw}


def listed():
    return [
        # one token's choice among many experts: latency
        _route("route_m1", 1, 64, 8),
        # the prompts of a batch, logits in the model's type, a quarter of the experts closed
        _route("route_m4096", 4096, 128, 8, dtype="bf16", masked=32),
        # token generation for one user: many small experts, and few large ones
        _moe("moe_m1_small", 1, 2048, 768, 64, 8),
        _moe("moe_m1_large", 1, 4096, 11008, 8, 2),
        # an act-order checkpoint, a handful of users
        _moe("moe_m4_act", 4, 4096, 1408, 16, 2, act=True),
        # an odd batch with padding behind it, groups of 64, bfloat16
        _moe("moe_m11_bf16", 11, 2048, 1408, 60, 4, dtype="bf16", group=64, padded=2),
        # a full decode batch: every expert is in use
        _moe("moe_m64", 64, 4096, 2048, 32, 4),
        # token generation for one user with an adapter on a small projection
        _lora("lora_m1", 1, 4096, 4096, 16, 4),
        # a small batch, each request with an adapter of its own
        _lora("lora_m8", 8, 4096, 12288, 16, 32),
        # an odd batch, long K, wide adapters, older zero-point convention; two requests without an adapter
        _lora("lora_m13_bf16", 13, 11008, 4096, 64, 6, dtype="bf16", group=64, minus_one=True, without=2),
        # a large decode batch on an act-order layer, 64 adapters
        _lora("lora_m64_act", 64, 5120, 5120, 32, 64, act=True),
        # packed prompts of five requests
        _lora("lora_prompts_m1000", 1000, 4096, 4096, 16, 5, runs=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["route", "moe", "moe", "moe", "lora", "lora", "lora"])
    if kind == "route":
        E = _log_int(rng, 4, 256)
        c = _route("", _log_int(rng, 1, 4096), E, min(E, _log_int(rng, 1, 16)), dtype=rng.choice(["fp32", "fp16", "bf16"]),
                   renormalize=rng.random() < 0.7, masked=rng.choice([0, 0, E // 4, E - 1]))
    elif kind == "moe":
        E = _log_int(rng, 2, 64)
        c = _moe("", _log_int(rng, 1, 64), 128 * _log_int(rng, 4, 40), 128 * _log_int(rng, 2, 86), E, min(E, _log_int(rng, 1, 8)),
                 dtype=rng.choice(["fp16", "fp16", "bf16"]), group=rng.choice([128, 128, 64, 32]), act=rng.random() < 0.25,
                 minus_one=rng.random() < 0.2)
        c["padded"] = rng.choice([0, 0, c["M"] // 4])
    else:
        M = _log_int(rng, 1, 1000)
        c = _lora("", M, 128 * _log_int(rng, 8, 86), 128 * _log_int(rng, 8, 172), rng.choice([8, 16, 16, 24, 32, 64, 128]),
                  _log_int(rng, 1, 64), dtype=rng.choice(["fp16", "fp16", "bf16"]), group=rng.choice([128, 128, 64, 32]),
                  act=rng.random() < 0.25, minus_one=rng.random() < 0.2, runs=M > 64)
        c["without"] = rng.choice([0, 0, M // 4])
    del c["name"]
    while kind == "moe" and c["E"] > 2 and c["E"] * c["K"] * c["F"] > 8 * 4096 * 11008:      # what a state holds
        c["E"] //= 2
        c["k"] = min(c["k"], c["E"])
    while kind != "route" and (work(c)["bytes"] > _MAX_BYTES or work(c)["flops"] > _MAX_FLOPS):
        for s in ("F", "N"):
            if s in c:
                c[s] = max(128, c[s] // 256 * 128)
        c["M"] = max(1, c["M"] * 3 // 4)
        for s in ("padded", "without"):
            if s in c:
                c[s] = min(c[s], c["M"] // 4)
    return c


def _layer_bytes(K, N, group, act):
    return K * N // 2 + K // group * (2 * N + N // 2) + (4 * K if act else 0)


def work(case):
    M = case["M"]
    if case["kind"] == "route":
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": M * case["E"] * size + 8 * M * case["k"], "flops": 4 * M * case["E"]}
    if case["kind"] == "moe":
        K, F, E, k = case["K"], case["F"], case["E"], case["k"]
        rows = M - case["padded"]
        active = E * (1 - (1 - k / E) ** rows)      # expected number of experts that some token chose
        expert = _layer_bytes(K, 2 * F, case["group"], case["act"]) + _layer_bytes(F, K, case["group"], case["act"])
        return {"bytes": int(active * expert) + 6 * M * K + 8 * M * k, "flops": 6 * rows * k * K * F}
    K, N, r = case["K"], case["N"], case["rank"]
    rows = M - case["without"]
    in_use = min(case["adapters"], rows)
    return {"bytes": _layer_bytes(K, N, case["group"], case["act"]) + 2 * in_use * r * (K + N) + 2 * M * (K + N) + 4 * M,
            "flops": 2 * M * K * N + 2 * rows * r * (K + N)}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _words(gen, *shape):
    return torch.randint(-(1 << 31), 1 << 31, shape, generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)


def _layers(case, gen, count, K, N):
    """``count`` canonical layers [K, N]: uniform packed words, seeded scales, an order of their own each with act-order."""
    group, dt = case["group"], _DTYPES[case["dtype"]]
    G = K // group
    sc = (SCALE_FLOOR + (torch.randn((count, G, N), generator=gen, device="cuda") * SCALE_SIGMA).abs()).to(dt)
    g_idx = (torch.arange(K, device="cuda") // group).to(torch.int32).expand(count, K)
    if case["act"]:
        order = torch.rand((count, K), generator=gen, device="cuda").argsort(dim=1)
        g_idx = (order // group).to(torch.int32)
    return {"qw": _words(gen, count, K // 8, N), "qz": _words(gen, count, G, N // 8), "sc": sc, "g_idx": g_idx.contiguous(),
            "K": K, "N": N}


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    M, dt = case["M"], _DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if case["kind"] == "route":
        logits = (2 * normal(M, case["E"])).to(dt)
        closed = torch.rand(case["E"], generator=gen, device="cuda").argsort()[:case["masked"]]
        logits[:, closed] = -float("inf")
        return {"logits": logits}
    if case["kind"] == "moe":
        K, F, E, k = case["K"], case["F"], case["E"], case["k"]
        p, ids = normal(M, E).softmax(-1).topk(k)
        ids = ids.to(torch.int32)
        if case["padded"]:
            ids[M - case["padded"]:] = -1
        return {"x": normal(M, K).to(dt), "ids": ids, "weights": (p / p.sum(-1, keepdim=True)).contiguous(),
                "residual": (8 * normal(M, K)).to(dt), "gate_up": _layers(case, gen, E, K, 2 * F), "down": _layers(case, gen, E, F, K)}
    K, N, r, n = case["K"], case["N"], case["rank"], case["adapters"]
    rows = M - case["without"]
    ids = torch.arange(rows, device="cuda")
    ids = ids * n // max(rows, 1) if case["runs"] else ids % n      # a request's prompt is a run of rows
    ids = torch.cat([ids, torch.full((case["without"],), -1, device="cuda")])
    if not case["runs"]:
        ids = ids[torch.rand(M, generator=gen, device="cuda").argsort()]
    return {"x": normal(M, K).to(dt), "layer": _layers(case, gen, 1, K, N), "ids": ids.to(torch.int32).contiguous(),
            "a": (normal(n, r, K) / K ** 0.5).to(dt), "b": (0.3 * normal(n, N, r)).to(dt),
            "scales": 0.5 + torch.rand(n, generator=gen, device="cuda")}


# ---- what a user's program keeps -------------------------------------------------------------------------------------

def _tiled(case, layers, gate_up=False):
    """The tiled buffers of ``count`` layers behind one another, as a server lays its checkpoint out once."""
    from paper_2511_19438_b200 import binding as B
    K, N, group, act = layers["K"], layers["N"], case["group"], case["act"]
    count = layers["qw"].shape[0]
    fmt = (B.GPTQ_FORMAT_ZEROS_MINUS_ONE if case["minus_one"] else 0) | (B.GPTQ_FORMAT_GATE_UP if gate_up else 0)
    fmt |= B.GPTQ_FORMAT_BF16 if case["dtype"] == "bf16" else 0
    outs = [torch.empty((count, B.gptq_repack_bytes(w, N, K, group, act)), dtype=torch.uint8, device="cuda") for w in range(3)]
    perm = torch.empty((count, K), dtype=torch.int32, device="cuda") if act else None
    for e in range(count):
        B.check(B.gptq_repack_format(layers["qw"][e], layers["qz"][e], layers["sc"][e], layers["g_idx"][e] if act else None,
                                     *(o[e] for o in outs), perm[e] if act else None, N, K, group, act, fmt), "gptq_repack_format")
    return outs, perm


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    M, dt = case["M"], _DTYPES[case["dtype"]]
    if own:
        # the checkpoint's layers as the kernels stream them, output buffers, the registered scratch
        from paper_2511_19438_b200 import binding as B
        from paper_2511_19438_b200 import harness as H
        global _workspace
        _workspace = _workspace or H.WorkspaceHolder()
        if case["kind"] == "route":
            s["ids_out"] = torch.empty((M, case["k"]), dtype=torch.int32, device="cuda")
            s["weights_out"] = torch.empty((M, case["k"]), dtype=torch.float32, device="cuda")
            s["logits_type"] = {"fp32": B.GPTQ_LOGITS_F32, "fp16": B.GPTQ_LOGITS_F16, "bf16": B.GPTQ_LOGITS_BF16}[case["dtype"]]
        elif case["kind"] == "moe":
            s["gate_up_t"], s["gate_up_perm"] = _tiled(case, s["gate_up"], gate_up=True)
            s["down_t"], perm = _tiled(case, s["down"])
            s["down_index"] = torch.empty_like(perm) if case["act"] else None
            for e in range(case["E"] if case["act"] else 0):
                B.check(B.gptq_invert_perm(perm[e], s["down_index"][e], case["F"]), "gptq_invert_perm")
            s["y"] = torch.empty_like(s["x"])
            _workspace.ensure(B.gptq_moe_workspace_bytes(M, case["K"], case["F"], case["k"], case["act"]))
        else:
            (qw, qz, sc), perm = _tiled(case, s["layer"])
            s["layer_t"], s["perm"] = (qw, qz, sc), perm
            s["y"] = torch.empty((M, case["N"]), dtype=dt, device="cuda")
            _workspace.ensure(B.gptq_lora_workspace_bytes(M, case["N"], case["K"], case["group"], case["act"], case["rank"]))
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def _unpack(words, dim):
    """[..., n, ...] words of eight nibbles along ``dim`` -> [..., 8 n, ...], fp32."""
    shift = torch.arange(0, 32, 4, device=words.device, dtype=torch.int32)
    q = (words.unsqueeze(dim + 1) >> shift.view(-1, *[1] * (words.dim() - 1 - dim))) & 15
    return q.flatten(dim, dim + 1).float()


def _dequant(case, layers, which=None):
    """fp32 [count, K, N] of the layers ``which`` (all of them without it)."""
    qw, qz, sc, g_idx = (layers[n] if which is None else layers[n][which] for n in ("qw", "qz", "sc", "g_idx"))
    z = _unpack(qz, 2) + (1 if case["minus_one"] else 0)
    rows = g_idx.long().unsqueeze(-1).expand(-1, -1, layers["N"])
    return (_unpack(qw, 1) - z.gather(1, rows)) * sc.float().gather(1, rows)


def _plain_route(s):
    case = s["case"]
    logits = s["logits"].float()
    logits = torch.where(logits.isnan(), -float("inf"), logits).clamp(max=torch.finfo(torch.float32).max)
    top, ids = logits.sort(dim=-1, descending=True, stable=True)      # equal logits: the lowest index first
    top, ids = top[:, :case["k"]], ids[:, :case["k"]]
    none = top == -float("inf")
    p = torch.where(logits == -float("inf"), 0.0, torch.exp(logits - logits.amax(-1, keepdim=True)))
    w = torch.where(none, 0.0, p.gather(1, ids))
    total = w.sum(-1, keepdim=True) if case["renormalize"] else p.sum(-1, keepdim=True)
    return {"ids": torch.where(none, -1, ids).to(torch.int32), "weights": torch.where(none, 0.0, w / total)}


def _plain_moe(s):
    case = s["case"]
    M, F, E, k = case["M"], case["F"], case["E"], case["k"]
    x, ids = s["x"].float(), s["ids"].long()
    used = (ids >= 0) & (ids < E)
    w = torch.where(used, s["weights"], 0.0)
    if M * k < E:      # few tokens: the weights of each token's experts
        which = torch.where(used, ids, 0).flatten()
        y = x.repeat_interleave(k, 0).unsqueeze(1) @ _dequant(case, s["gate_up"], which)
        h = y[..., :F] * y[..., :F].sigmoid() * y[..., F:]
        out = ((h @ _dequant(case, s["down"], which)).view(M, k, -1) * w.unsqueeze(-1)).sum(1)
    else:              # many: every token through every expert, weighted with what it gave that expert
        per_expert = torch.zeros((M, E), device=x.device).scatter_add_(1, torch.where(used, ids, 0), w)
        y = x @ _dequant(case, s["gate_up"])
        h = y[..., :F] * y[..., :F].sigmoid() * y[..., F:]
        out = ((h @ _dequant(case, s["down"])) * per_expert.t().unsqueeze(-1)).sum(0)
    return (out + s["residual"].float()).to(s["x"].dtype)


def _plain_lora(s):
    case = s["case"]
    x, ids = s["x"].float(), s["ids"].long()
    used = (ids >= 0) & (ids < case["adapters"])
    which = torch.where(used, ids, 0)
    v = (s["a"][which].float() @ x.unsqueeze(-1)) * torch.where(used, s["scales"][which], 0.0).view(-1, 1, 1)
    delta = torch.where(used.unsqueeze(-1), (s["b"][which].float() @ v).squeeze(-1), 0.0)
    return (x @ _dequant(case, s["layer"])[0] + delta).to(s["x"].dtype)


def run(state):
    s, case = state, state["case"]
    if not own:
        return {"route": _plain_route, "moe": _plain_moe, "lora": _plain_lora}[case["kind"]](s)
    from paper_2511_19438_b200 import binding as B
    M = case["M"]
    if case["kind"] == "route":
        B.check(B.gptq_moe_route(s["logits"], s["ids_out"], s["weights_out"], M, case["E"], case["k"], s["logits_type"],
                                 case["renormalize"]), "gptq_moe_route")
        return {"ids": s["ids_out"], "weights": s["weights_out"]}
    if case["kind"] == "moe":
        call = B.gptq_moe_mlp_bf16 if case["dtype"] == "bf16" else B.gptq_moe_mlp
        B.check(call(s["x"], s["ids"], s["weights"], *s["gate_up_t"], s["gate_up_perm"], *s["down_t"], s["down_index"], s["residual"],
                     s["y"], M, case["K"], case["F"], case["E"], case["k"], case["group"], case["act"]), "gptq_moe_mlp")
        return s["y"]
    call = B.gptq_gemm_lora_bf16 if case["dtype"] == "bf16" else B.gptq_gemm_lora
    B.check(call(s["x"], *s["layer_t"], s["perm"], s["a"], s["b"], s["ids"], s["scales"], s["y"], M, case["N"], case["K"],
                 case["group"], case["act"], case["rank"], case["adapters"]), "gptq_gemm_lora")
    return s["y"]


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _exact_weights(case, layers, e):
    """float64 [K, N] of layer ``e``, row by row of packed words."""
    K, N = layers["K"], layers["N"]
    q = torch.empty((K, N), dtype=torch.float64, device="cuda")
    z = torch.empty((layers["qz"].shape[1], N), dtype=torch.float64, device="cuda")
    for i in range(8):
        q[i::8] = torch.bitwise_and(torch.bitwise_right_shift(layers["qw"][e].long(), 4 * i), 15).double()
        z[:, i::8] = torch.bitwise_and(torch.bitwise_right_shift(layers["qz"][e].long(), 4 * i), 15).double()
    z += float(case["minus_one"])
    g = layers["g_idx"][e].long()
    return (q - z[g]) * layers["sc"][e].double()[g]


def exact(case, seed):
    t = _inputs(case, seed)
    if case["kind"] == "route":
        rows = [[float(v) for v in r] for r in t["logits"].double().tolist()]
        ids, weights = [], []
        for r in rows:
            open_ = [(-v, e) for e, v in enumerate(r) if v == v and v != -float("inf")]
            chosen = sorted(open_)[:case["k"]]
            top = -min(open_)[0] if open_ else 0.0
            e64 = torch.tensor([-v - top for v, _ in chosen], dtype=torch.float64).exp()
            rest = torch.tensor([-v - top for v, _ in open_], dtype=torch.float64).exp().sum()
            pad = case["k"] - len(chosen)
            ids.append([e for _, e in chosen] + [-1] * pad)
            weights.append((e64 / (e64.sum() if case["renormalize"] else rest)).tolist() + [0.0] * pad)
        return {"ids": torch.tensor(ids, dtype=torch.int32).view(len(rows), -1),
                "weights": torch.tensor(weights, dtype=torch.float64).view(len(rows), -1)}
    x = t["x"].double()
    if case["kind"] == "moe":
        F = case["F"]
        out = t["residual"].double()
        for e in range(case["E"]):
            m, j = (t["ids"] == e).nonzero(as_tuple=True)
            if len(m):
                gu = x[m] @ _exact_weights(case, t["gate_up"], e)
                gate, up = gu[:, :F], gu[:, F:]
                part = (gate / (1 + torch.exp(-gate)) * up) @ _exact_weights(case, t["down"], e)
                out.index_add_(0, m, part * t["weights"][m, j].double().unsqueeze(1))
        return out
    out = x @ _exact_weights(case, t["layer"], 0)
    for a in range(case["adapters"]):
        m = (t["ids"] == a).nonzero().squeeze(1)
        if len(m):
            v = x[m] @ t["a"][a].double().t()
            out[m] += float(t["scales"][a]) * (v @ t["b"][a].double().t())
    return out

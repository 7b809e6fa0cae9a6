"""Argument checks of the operators whose rows choose their weights (routing, routed experts, adapters): no GPU needed, nothing
is launched."""
import os
import re

import pytest
import torch

from paper_2511_19438_b200 import build as libbuild

libbuild.build()
from paper_2511_19438_b200 import binding as B  # noqa: E402

A16 = 0x1000  # a fake, 16-byte aligned "device address"; validation never dereferences it


def route(logits=A16, ids=A16, weights=A16, M=4, E=64, k=8, kind=B.GPTQ_LOGITS_F32, renormalize=1):
    return B.gptq_moe_route(logits, ids, weights, M, E, k, kind, renormalize, stream=0)


def test_route_refusals():
    for name in ("logits", "ids", "weights"):
        assert route(**{name: None}) == B.GPTQ_ERR_NULL
        assert route(**{name: A16 + 4}) == B.GPTQ_ERR_ALIGN
    for bad in (dict(M=0), dict(E=0), dict(k=0), dict(k=65), dict(M=-1)):
        assert route(**bad) == B.GPTQ_ERR_SHAPE, bad
    assert route(E=1025) == B.GPTQ_ERR_UNSUPPORTED
    assert route(k=33) == B.GPTQ_ERR_UNSUPPORTED
    for kind in (-1, 3):
        assert route(kind=kind) == B.GPTQ_ERR_LAYOUT


MOE_POINTERS = ["x", "ids", "weights", "gu_qw", "gu_qz", "gu_sc", "gu_perm", "dn_qw", "dn_qz", "dn_sc", "dn_index", "residual", "y"]


@pytest.mark.parametrize("fn", [B.gptq_moe_mlp, B.gptq_moe_mlp_bf16])
def test_moe_refusals(fn):
    def call(**kw):
        p = {n: A16 for n in MOE_POINTERS}
        s = dict(M=2, K=512, F=256, E=8, k=2, group=128, act=1)
        for n, v in kw.items():
            (p if n in p else s)[n] = v
        return fn(*p.values(), *s.values(), stream=0)

    for name in MOE_POINTERS:
        if name != "residual":
            assert call(**{name: None}) == B.GPTQ_ERR_NULL, name
        assert call(**{name: A16 + 8}) == B.GPTQ_ERR_ALIGN, name
    for bad in (dict(M=0), dict(K=516), dict(F=260), dict(F=0), dict(E=0), dict(k=0), dict(k=9), dict(group=0), dict(K=512 + 64),
                dict(group=512)):
        assert call(**bad) == B.GPTQ_ERR_SHAPE, bad
    assert call(act=2) == B.GPTQ_ERR_LAYOUT
    assert call(act=-1) == B.GPTQ_ERR_LAYOUT
    for bad in (dict(group=16), dict(K=192, F=192, group=64), dict(F=192, group=64), dict(E=1025), dict(E=64, k=33)):
        assert call(**bad) == B.GPTQ_ERR_UNSUPPORTED, bad


LORA_POINTERS = ["x", "qw", "qz", "sc", "g_idx", "a", "b", "ids", "scales", "y"]


@pytest.mark.parametrize("fn", [B.gptq_gemm_lora, B.gptq_gemm_lora_bf16])
def test_lora_refusals(fn):
    def call(**kw):
        p = {n: A16 for n in LORA_POINTERS}
        p["y"] += 16
        s = dict(M=2, N=256, K=512, group=128, act=1, rank=16, adapters=4)
        for n, v in kw.items():
            (p if n in p else s)[n] = v
        return fn(*p.values(), *s.values(), stream=0)

    for name in LORA_POINTERS:
        if name != "scales":
            assert call(**{name: None}) == B.GPTQ_ERR_NULL, name
        assert call(**{name: A16 + 8}) == B.GPTQ_ERR_ALIGN, name
    for bad in (dict(M=0), dict(K=516), dict(N=260 + 1), dict(rank=0), dict(adapters=0), dict(group=0)):
        assert call(**bad) == B.GPTQ_ERR_SHAPE, bad
    for bad in (dict(act=3), dict(act=-1), dict(y=A16)):      # (y = x)
        assert call(**bad) == B.GPTQ_ERR_LAYOUT, bad
    for bad in (dict(group=16), dict(N=192), dict(rank=12), dict(rank=264)):
        assert call(**bad) == B.GPTQ_ERR_UNSUPPORTED, bad


def test_workspace_sizes():
    # the activation of every slot in 16 bits; with act-order also each slot's row of x; passes of 64 tokens share it
    assert B.gptq_moe_workspace_bytes(4, 512, 256, 2, 0) == 2 * 8 * 256 * 2        # few tokens: the activation in two parts
    assert B.gptq_moe_workspace_bytes(4, 512, 256, 2, 1) == 2 * 8 * 256 * 2 + 8 * 512 * 2
    assert B.gptq_moe_workspace_bytes(1000, 512, 256, 2, 0) == 128 * 256 * 2
    for act in (0, 1):      # scratch for many tokens does for fewer
        need = [B.gptq_moe_workspace_bytes(m, 512, 256, 2, act) for m in range(1, 200)]
        assert need == sorted(need)
    for bad in ((0, 512, 256, 2), (4, 500, 256, 2), (4, 512, 200, 2), (4, 512, 256, 0), (4, 512, 256, 33)):
        assert B.gptq_moe_workspace_bytes(*bad, 0) == 0
    few, many = B.gptq_lora_workspace_bytes(16, 256, 512, 128, 0, 16), B.gptq_lora_workspace_bytes(17, 256, 512, 128, 0, 16)
    assert few >= 16 * 16 * 4 and many >= 17 * 16 * 4 + 17 * 256 * 2
    assert B.gptq_lora_workspace_bytes(16, 256, 512, 128, 1, 16) == few + 16 * 512 * 2
    assert B.gptq_lora_workspace_bytes(16, 256, 512, 128, 2, 16) == few
    for bad in ((0, 256, 512, 128, 0, 16), (4, 200, 512, 128, 0, 16), (4, 256, 512, 128, 0, 12), (4, 256, 512, 16, 0, 16)):
        assert B.gptq_lora_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("N,K,rank", [(128, 128, 8), (128, 11008, 256), (4096, 4096, 16), (4096, 4096, 64), (4096, 4096, 256), (4096, 11008, 64),
                                      (12288, 4096, 64), (4096, 512 * 128, 40)])
def test_adapter_scratch_for_many_rows_does_for_fewer(N, K, rank, act):
    rows = list(range(1, 2200)) + list(range(2200, 40000, 37))
    need = [B.gptq_lora_workspace_bytes(m, N, K, 128, act, rank) for m in rows]
    falls = [(rows[i], rows[i + 1]) for i in range(len(need) - 1) if need[i] > need[i + 1]]
    assert not falls, falls[:5]
    # v at least once, with more than 8 rows the expansion, with act-order x
    assert all(n >= m * rank * 4 + (2 * m * N if m > 8 else 0) + (2 * m * K if act == 1 else 0) for m, n in zip(rows, need))


def test_a_ring_stage_is_refilled_behind_the_whole_warps_reads():
    """stream_items copies into the stage that was read last.  Scales and zero points in it are read by other lanes than those that copied
    them, so that between a product and the next copy the warp has to meet.  Followed through two turns of the loop in the source."""
    source = os.path.join(os.path.dirname(libbuild.CSRC), "csrc", "gptq_direct.cuh")
    body = re.sub(r"//[^\n]*", "", open(source).read())
    body = body[body.index("stream_items("):body.index("long_sum(")]
    loop = body[body.index("while (x.tag >= 0)"):]
    steps = re.findall(r"multiply_pair<|copy_pair\(\d\)|__syncwarp\(\)", loop) * 2
    assert sum(s.startswith("multiply") for s in steps) == 4 and sum(s.startswith("copy") for s in steps) == 4
    read = False
    for s in steps:
        if s.startswith("multiply"):
            read = True
        elif s.startswith("__syncwarp"):
            read = False
        else:
            assert not read, "a copy stands behind a product without a barrier of the warp between them"


# ---- the harness: what does not fit together is refused before an address goes anywhere

def experts(K, N, group, act=False, count=4):
    from paper_2511_19438_b200 import harness as H
    t = torch.zeros((count, 16), dtype=torch.uint8)
    return H.DeviceExperts(K, N, group, act, count, t, t, t, None, None)


@pytest.fixture
def no_calls(monkeypatch):
    """The binding's functions count instead of launching."""
    calls = []
    for fn in ("gptq_moe_route", "gptq_moe_mlp", "gptq_moe_mlp_bf16", "gptq_gemm_lora", "gptq_gemm_lora_bf16"):
        stand_in = lambda *a, **k: calls.append(a) or B.GPTQ_OK
        stand_in.__name__ = fn
        monkeypatch.setattr(B, fn, stand_in)
    return calls


def test_harness_experts_that_do_not_fit(no_calls):
    from paper_2511_19438_b200 import harness as H
    M, K, F, k = 3, 256, 128, 2
    good = dict(x=torch.zeros((M, K), dtype=torch.float16), ids=torch.zeros((M, k), dtype=torch.int32), weights=torch.zeros((M, k)),
                gate_up=experts(K, 2 * F, 128), down=experts(F, K, 128), residual=torch.zeros((M, K), dtype=torch.float16))
    H.moe_mlp(**good)
    H.moe_mlp(**{**good, "gate_up": experts(K, 2 * F, 256)})      # (tiled as groups of 128)
    assert len(no_calls) == 2
    for bad in (dict(down=experts(F, K, 64)), dict(gate_up=experts(K, 2 * F, 32)), dict(down=experts(2 * F, K, 128)), dict(down=experts(F, 2 * K, 128)),
                dict(down=experts(F, K, 128, count=3)), dict(down=experts(F, K, 128, act=True)), dict(x=torch.zeros((M, 2 * K), dtype=torch.float16)),
                dict(x=torch.zeros((M, K))), dict(x=torch.zeros((K, M), dtype=torch.float16).t()), dict(ids=torch.zeros((M, k), dtype=torch.int64)),
                dict(ids=torch.zeros((k, M), dtype=torch.int32).t()), dict(ids=torch.zeros((M - 1, k), dtype=torch.int32)),
                dict(weights=torch.zeros((M, k), dtype=torch.float16)), dict(weights=torch.zeros((M, k + 1))),
                dict(residual=torch.zeros((M, K), dtype=torch.bfloat16)), dict(y=torch.zeros((M, K))), dict(y=torch.zeros((M, 2 * K), dtype=torch.float16)[:, :K])):
        with pytest.raises(ValueError):
            H.moe_mlp(**{**good, **bad})
    assert len(no_calls) == 2


def test_harness_adapters_and_logits_that_do_not_fit(no_calls):
    from paper_2511_19438_b200 import harness as H
    M, K, N, r, n = 3, 256, 128, 8, 2
    t = torch.zeros(16, dtype=torch.uint8)
    D = H.DeviceLinear(K, N, 128, False, t, t, t, None, None)
    half = lambda *shape: torch.zeros(shape, dtype=torch.float16)
    good = dict(x=half(M, K), D=D, lora_a=half(n, r, K), lora_b=half(n, N, r), adapter_ids=torch.zeros(M, dtype=torch.int32), adapter_scales=torch.ones(n))
    H.gemm_lora(**good)
    H.gemm_lora(**{**good, "adapter_scales": None, "y": half(M, N)})
    H.moe_route(torch.zeros((M, 8)), 2)
    assert len(no_calls) == 3
    for bad in (dict(lora_a=half(n, r, N)), dict(lora_a=torch.zeros((n, r, K))), dict(lora_b=half(n - 1, N, r)), dict(lora_b=half(n, r, N)),
                dict(adapter_ids=torch.zeros(M, dtype=torch.int64)), dict(adapter_ids=torch.zeros(M + 1, dtype=torch.int32)),
                dict(adapter_scales=torch.ones(n, dtype=torch.float16)), dict(adapter_scales=torch.ones(n + 1)), dict(x=half(M, 2 * K)),
                dict(x=half(K, M).t()), dict(x=torch.zeros((M, K), dtype=torch.bfloat16)), dict(y=half(M, N + 8)), dict(y=torch.zeros((M, N)))):
        with pytest.raises(ValueError):
            H.gemm_lora(**{**good, **bad})
    for logits in (torch.zeros((M, 8), dtype=torch.float64), torch.zeros((8, M)).t()):
        with pytest.raises(ValueError):
            H.moe_route(logits, 2)
    assert len(no_calls) == 3

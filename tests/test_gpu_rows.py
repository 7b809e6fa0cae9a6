"""GPU tests of the operators whose rows choose their weights: routing, routed experts, low-rank adapters.

Plain implementations in 64 bits on the oracle's dequantised weights.  Tolerances, with u = half a step of the 16-bit type
(2^-11 fp16, 2^-8 bfloat16):

* a sum of n products in fp32, in any order and with truncation, is off by at most n 2^-23 of the sum of their absolute values;
* experts: each activation h is rounded once, which moves y by at most u sum |w h d|, and y is rounded once, u |y|; the fp32
  errors of gate and up reach h through silu (slope below 1.1) and the product, 2^-18 covers the fast exponential and division.
  All roundings are independent, so the rms error stays below u sqrt(y^2 + sum (w h d)^2) (three times its variance);
* adapters: one rounding of y up to 8 rows; above, the adapters' part is rounded to 16 bits on its way to the fp32 sums, u |part|; above
  16, so is every scaled weight, u sum |x w|, rms u sqrt(sum (x w)^2).
* the experts' products and the fused adapter product form sum (q - z) x of a quantisation group as sum q x - z sum x (bfloat16:
  sum (128 + q) x - (128 + z) sum x).  Each side is at most eight MMAs deep and sums to at most 15 (143) sum |x|, z sum x to 16 (144)
  sum |x|: together at most 31 (287) sum |x|, off by at most 8 2^-23 of that.  `sums` counts it, times the scale.
"""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2511_19438_b200 import workloads as wl

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2511_19438_b200 import build as libbuild
    libbuild.build()
    from paper_2511_19438_b200 import binding as B
    from paper_2511_19438_b200 import harness as H

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
F32 = 2.0 ** -23


def sums(dtype, x, w64):
    """8 2^-23 (31 or 287) sum |x| s.  s is taken from sum |x| |w|, |w| = |q - z| s: for uniform nibbles the mean of |q - z| is 5.3, and
    over the rows of a column (128 and more) its |x|-weighted mean stays above 3."""
    return 8 * F32 * (287 if dtype == torch.bfloat16 else 31) / 3 * (x.double().abs() @ w64.abs())


@pytest.fixture(scope="module")
def ws():
    return H.WorkspaceHolder()


def gen(*parts):
    return torch.Generator(device="cuda").manual_seed(wl.seed_for(*parts))


def layer(K, N, seed, group=128, act=False, minus_one=False, bf16=False):
    """(QuantLinear, bf16 scale bits or None, float64 [K, N] on the GPU)"""
    L = wl.make_linear(K, N, seed=seed, group_size=group, act_order=act)
    L.zeros_minus_one = minus_one
    if bf16:
        bits = wl.make_scales_bf16(K // group, N, seed + 1)
        w = oracle.dequant_f32_bf16(L.qweight, L.qzeros, bits, L.g_idx, group, minus_one)
    else:
        bits, w = None, oracle.dequant_f32(L.qweight, L.qzeros, L.scales, L.g_idx, group, minus_one)
    return L, bits, H.to_device(w).double()


# ---------------------------------------------------------------------------------------------------------------- routing

def plain_route(logits, k, renormalize):
    ids, weights = [], []
    for row in logits.double().cpu().tolist():
        big = float(np.finfo(np.float32).max)
        open_ = sorted((-min(v, big), e) for e, v in enumerate(row) if v == v and v != -math.inf)
        top = -open_[0][0] if open_ else 0.0
        p = [math.exp(-v - top) for v, _ in open_]
        total = math.fsum(p[:k]) if renormalize else math.fsum(p)
        ids.append([e for _, e in open_[:k]] + [-1] * (k - len(open_[:k])))
        weights.append([q / total for q in p[:k]] + [0.0] * (k - len(open_[:k])))
    return np.array(ids), np.array(weights)


def check_route(logits, k, renormalize):
    ids, w = H.moe_route(logits, k, renormalize)
    want_ids, want_w = plain_route(logits, k, renormalize)
    assert np.array_equal(ids.cpu().numpy(), want_ids)
    # exp and the division are good to a few steps of 2^-24 times the exponent; a sum of E terms
    err = np.abs(w.cpu().double().numpy() - want_w)
    assert np.all(err <= 2.0 ** -18 * want_w + 1e-37), err.max()


@pytest.mark.parametrize("M,E,k", [(1, 1, 1), (1, 64, 8), (3, 7, 7), (5, 32, 4), (130, 33, 2), (2, 100, 32), (9, 128, 6), (4, 256, 8),
                                   (3, 500, 10), (2, 1024, 32), (1025, 60, 4)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_route(M, E, k, dtype):
    logits = (3 * torch.randn((M, E), generator=gen("route", M, E), device="cuda")).to(dtype)
    check_route(logits, k, True)
    check_route(logits, k, False)


def test_route_ties_and_closed_experts():
    g = gen("route-ties")
    logits = torch.randint(-2, 3, (40, 50), generator=g, device="cuda").float()        # many ties, -0 among them
    logits[::2] *= -1.0
    check_route(logits, 8, True)
    check_route(logits.half(), 8, False)
    logits[:, 10:] = -math.inf
    logits[3] = -math.inf                                                              # nothing to choose
    logits[4] = math.nan
    logits[5, :7] = math.nan
    logits[6, 4] = math.inf
    logits[7, 4:6] = math.inf
    for k in (1, 8, 12, 32):
        check_route(logits, k, True)
        check_route(logits, k, False)
    tiny = torch.tensor([[1e-42, 2e-42, 0.0, -0.0, -1e-42, 1e-45]], device="cuda").repeat(2, 1)
    check_route(tiny, 6, True)


# ---------------------------------------------------------------------------------------------------------------- experts

class Moe:
    def __init__(self, K, F, E, group=128, act=False, minus_one=False, dtype=torch.float16):
        bf16 = dtype == torch.bfloat16
        up = [layer(K, 2 * F, wl.seed_for("moe-up", K, F, e, group), group, act, minus_one, bf16) for e in range(E)]
        down = [layer(F, K, wl.seed_for("moe-down", K, F, e, group), group, act, minus_one, bf16) for e in range(E)]
        self.K, self.F, self.E, self.dtype = K, F, E, dtype
        self.up64, self.down64 = [l[2] for l in up], [l[2] for l in down]
        self.up = H.upload_experts([l[0] for l in up], gate_up=True, scales_bf16_bits=[l[1] for l in up] if bf16 else None)
        self.down = H.upload_experts([l[0] for l in down], scales_bf16_bits=[l[1] for l in down] if bf16 else None)

    def plain(self, x, ids, weights, residual):
        """(y, bound of the largest errors, bound of the mean square error), float64"""
        u, x = U[self.dtype], x.double()
        M = x.shape[0]
        # h: rounded to 16 bits; up to 16 tokens what that leaves, exact in fp32, is rounded again, to a step u of at most u |h|.
        # Its fp32 value is off by 2^-18 (dh below), which counts beside the second.
        uh = u if M > 16 else u * u
        uh_mean = u if M > 16 else u * u + 2.0 ** -18
        y = torch.zeros((M, self.K), dtype=torch.float64, device="cuda")
        if residual is not None:
            y += residual.double()
        most, square = y.abs() * 4 * F32, torch.zeros_like(y)
        for m in range(M):
            named = {}
            for e, w in zip(ids[m].tolist(), weights[m].tolist()):
                if 0 <= e < self.E:
                    named[e] = named.get(e, 0.0) + w
            for e, w in named.items():
                gu, size = x[m] @ self.up64[e], x[m].abs() @ self.up64[e].abs()
                more = sums(self.dtype, x[m], self.up64[e])
                gate, up = gu[:self.F], gu[self.F:]
                dg, du = self.K * F32 * size[:self.F] + more[:self.F], self.K * F32 * size[self.F:] + more[self.F:]
                silu = gate * torch.sigmoid(gate)
                h = silu * up
                dh = 1.1 * dg * (up.abs() + du) + silu.abs() * du + 2.0 ** -18 * h.abs()
                d = self.down64[e].abs()
                y[m] += w * (h @ self.down64[e])
                most[m] += abs(w) * (((uh + self.F * F32) * h.abs() + 1.01 * dh + 2.0 ** -24) @ d + sums(self.dtype, h, self.down64[e]))
                square[m] += (w * uh_mean) ** 2 * ((h * h) @ (d * d))
        return y, most + u * y.abs(), square + (u * y) ** 2

    def inputs(self, M, k, *seed):
        g = gen("moe-in", M, k, *seed)
        x = torch.randn((M, self.K), generator=g, device="cuda").to(self.dtype)
        p, ids = torch.randn((M, self.E), generator=g, device="cuda").softmax(-1).topk(k)
        residual = (4 * torch.randn((M, self.K), generator=g, device="cuda")).to(self.dtype)
        return x, ids.to(torch.int32), p.contiguous(), residual

    def check(self, ws, x, ids, weights, residual, y=None):
        want, most, square = self.plain(x, ids, weights, residual)
        H.ensure_for_moe(ws, x.shape[0], self.up, ids.shape[1])
        ws.buf.fill_(0xff)                             # NaNs: nothing of an earlier call may be read
        y = H.moe_mlp(x, ids, weights, self.up, self.down, residual, y)
        assert B.gptq_check_status() == B.GPTQ_OK
        err = (y.double() - want).abs()
        assert torch.isfinite(y).all()
        assert (err <= most).all(), f"{int((err > most).sum())} of {err.numel()} beyond the bound, worst {float((err / most).max()):.2f} of it"
        assert float((err * err).mean()) <= float(square.mean()), (float((err * err).mean()), float(square.mean()))
        return y


@pytest.mark.parametrize("M,K,F,E,k", [(1, 128, 128, 2, 1), (1, 512, 256, 8, 2), (2, 256, 384, 4, 4), (5, 384, 128, 16, 3),
                                       (8, 1152, 256, 3, 2), (9, 256, 128, 5, 2), (16, 128, 640, 4, 1), (17, 256, 256, 3, 2),
                                       (33, 128, 256, 2, 1), (64, 256, 128, 4, 3), (65, 128, 128, 3, 2), (130, 256, 128, 6, 2)])
def test_moe(ws, M, K, F, E, k):
    moe = Moe(K, F, E)
    x, ids, w, r = moe.inputs(M, k)
    moe.check(ws, x, ids, w, r)


# the down kernel with 64 columns per cluster: enough columns and items, clusters of 8 (h in one part and in two), 4, 2 and 1
@pytest.mark.parametrize("M,group,dtype", [(5, 128, torch.float16), (16, 64, torch.float16), (17, 128, torch.float16), (20, 64, torch.float16),
                                           (5, 64, torch.bfloat16), (16, 128, torch.bfloat16), (17, 64, torch.bfloat16), (20, 128, torch.bfloat16)])
def test_moe_wide_columns(ws, M, group, dtype):
    moe = Moe(1280, 1024, 8, group, dtype=dtype)
    x, ids, w, r = moe.inputs(M, 2, "wide", group)
    moe.check(ws, x, ids, w, r)


@pytest.mark.parametrize("M", [3, 18])
@pytest.mark.parametrize("K,F", [(2432, 2176), (4864, 1280), (9600, 1280)])
def test_moe_wide_columns_small_clusters(ws, M, K, F):
    moe = Moe(K, F, 2)
    x, ids, w, r = moe.inputs(M, 2, "clusters")
    moe.check(ws, x, ids, w, r)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("group,act,minus_one", [(128, True, False), (64, False, True), (64, True, False), (32, False, False),
                                                 (32, True, True), (256, False, False)])
@pytest.mark.parametrize("M", [1, 11, 40])
def test_moe_formats(ws, M, group, act, minus_one, dtype):
    moe = Moe(256, 512, 4, group, act, minus_one, dtype)
    x, ids, w, r = moe.inputs(M, 2, group, act)
    moe.check(ws, x, ids, w, r)


def test_moe_larger_shapes(ws):
    moe = Moe(2048, 1408, 4)
    for M, k in ((1, 2), (3, 4), (12, 2)):
        x, ids, w, r = moe.inputs(M, k, "large")
        moe.check(ws, x, ids, w, r)


def test_moe_every_token_to_one_expert(ws):
    moe = Moe(256, 256, 5)
    for M in (8, 16, 31, 64):
        x, ids, w, r = moe.inputs(M, 1, "one")
        ids.fill_(3)
        moe.check(ws, x, ids, w, r)


def test_moe_unused_slots_and_padding(ws):
    moe = Moe(256, 256, 6)
    for M in (4, 20):
        x, ids, w, r = moe.inputs(M, 3, "pad")
        ids[0, 1] = -1
        ids[1] = -1
        ids[2, 0] = moe.E
        ids[2, 2] = -2147483648
        ids[M - 1] = 2147483647
        x[1] = math.nan                    # padding rows hold anything
        x[M - 1] = math.inf
        w[1] = math.nan
        w[0, 1] = math.inf
        clean_x, clean_w = x.clone(), w.clone()
        clean_x[1], clean_x[M - 1], clean_w[1], clean_w[0, 1] = 0, 0, 0, 0
        want, most, _ = moe.plain(clean_x, ids, clean_w, r)
        H.ensure_for_moe(ws, M, moe.up, 3)
        y = H.moe_mlp(x, ids, w, moe.up, moe.down, r)
        assert ((y.double() - want).abs() <= most).all()
        assert torch.equal(y[1], r[1]) and torch.equal(y[M - 1], r[M - 1])
        y = H.moe_mlp(x, ids, w, moe.up, moe.down)
        assert torch.equal(y[1], torch.zeros_like(y[1]))
    x, ids, w, r = moe.inputs(7, 2, "none")
    ids.fill_(-1)
    assert torch.equal(H.moe_mlp(x, ids, w, moe.up, moe.down, r), r)
    assert not H.moe_mlp(x, ids, w, moe.up, moe.down).any()


def test_moe_expert_named_twice(ws):
    moe = Moe(256, 128, 4)
    for M in (1, 6, 30):
        x, ids, w, r = moe.inputs(M, 3, "twice")
        ids[:, 2] = ids[:, 0]
        ids[0] = 2
        moe.check(ws, x, ids, w, r)


def test_moe_top_32_of_many_experts(ws):
    moe = Moe(128, 128, 40)
    for M in (1, 64):
        x, ids, w, r = moe.inputs(M, 32, "many")
        moe.check(ws, x, ids, w, r)


def test_moe_slots_beyond_the_table(ws):
    """More slots times experts than the kernels count in a table: one warp sorts them."""
    moe = Moe(128, 128, 150)
    x, ids, w, r = moe.inputs(64, 32, "serial")
    moe.check(ws, x, ids, w, r)


def test_moe_experts_behind_4_gib(ws):
    """Expert buffers longer than 32 bits of bytes; only those in use are ever written."""
    K, F, E, use = 4096, 4096, 520, (3, 517)
    up = [layer(K, 2 * F, wl.seed_for("far", e)) for e in use]
    down = [layer(F, K, wl.seed_for("far-down", e)) for e in use]
    near = Moe.__new__(Moe)
    near.K, near.F, near.E, near.dtype = K, F, 2, torch.float16
    near.up64, near.down64 = [l[2] for l in up], [l[2] for l in down]
    near.up, near.down = H.upload_experts([l[0] for l in up], gate_up=True), H.upload_experts([l[0] for l in down])
    assert near.up.qweight_t.shape[1] * E > 1 << 33 and near.down.qweight_t.shape[1] * E > 1 << 32
    x, ids, w, r = near.inputs(3, 2, "far")
    y = near.check(ws, x, ids, w, r)

    def spread(d):
        out = {n: torch.empty((E, getattr(d, n).shape[1]), dtype=torch.uint8, device="cuda") for n in ("qweight_t", "qzeros_t", "scales_t")}
        for n, t in out.items():
            for i, e in enumerate(use):
                t[e] = getattr(d, n)[i]
        return H.DeviceExperts(d.K, d.N, d.group_size, False, E, out["qweight_t"], out["qzeros_t"], out["scales_t"], None, None)

    far_ids = torch.tensor(use, dtype=torch.int32, device="cuda")[ids.long()]
    assert torch.equal(H.moe_mlp(x, far_ids, w, spread(near.up), spread(near.down), r), y)


def test_moe_buffers_may_be_shared(ws):
    moe = Moe(256, 256, 4)
    for M in (3, 70):
        x, ids, w, r = moe.inputs(M, 2, "alias")
        y = moe.check(ws, x, ids, w, r)
        shared = r.clone()
        assert torch.equal(H.moe_mlp(x, ids, w, moe.up, moe.down, shared, shared), y)
        shared = x.clone()
        assert torch.equal(H.moe_mlp(shared, ids, w, moe.up, moe.down, r, shared), y)


def test_moe_infinite_activations(ws):
    """An infinity in x reaches its own row only, and there as the formula has it."""
    moe = Moe(256, 128, 4)
    x, ids, w, r = moe.inputs(6, 2, "inf")
    want = moe.check(ws, x, ids, w, r)
    x[2, 17] = math.inf
    y = H.moe_mlp(x, ids, w, moe.up, moe.down, r)
    keep = torch.tensor([0, 1, 3, 4, 5], device="cuda")
    assert torch.equal(y[keep], want[keep])
    assert not torch.isfinite(y[2]).any()


def test_moe_refuses_other_layouts(ws):
    moe = Moe(256, 128, 4)
    bf = Moe(256, 128, 4, dtype=torch.bfloat16)
    plain_up = H.upload_experts([wl.make_linear(256, 256, seed=e) for e in range(4)])
    flagged_down = H.upload_experts([wl.make_linear(128, 256, seed=e) for e in range(4)], gate_up=True)
    x, ids, w, r = moe.inputs(5, 2, "layout")
    H.ensure_for_moe(ws, 5, moe.up, 2)
    for up, down in ((plain_up, moe.down), (moe.up, flagged_down), (bf.up, bf.down), (moe.up, bf.down)):
        y = torch.full_like(x, 7.0)
        H.moe_mlp(x, ids, w, up, down, r, y)
        assert B.gptq_check_status() == B.GPTQ_ERR_LAYOUT
        assert torch.equal(y, torch.full_like(x, 7.0))
    assert B.gptq_check_status() == B.GPTQ_OK


def test_moe_needs_its_workspace(ws):
    moe = Moe(128, 128, 2)
    x, ids, w, r = moe.inputs(2, 1, "ws")
    H.ensure_for_moe(ws, 2, moe.up, 1)
    B.check(B.gptq_set_workspace(None, 0), "unregister")
    with pytest.raises(B.GptqError) as e:
        H.moe_mlp(x, ids, w, moe.up, moe.down, r)
    assert e.value.status == B.GPTQ_ERR_WORKSPACE
    B.check(B.gptq_set_workspace(ws.buf, 255), "small")
    with pytest.raises(B.GptqError):
        H.moe_mlp(x, ids, w, moe.up, moe.down, r)
    ws.ensure(1)


# --------------------------------------------------------------------------------------------------------------- adapters

class Lora:
    def __init__(self, K, N, rank, n, group=128, act=False, minus_one=False, dtype=torch.float16):
        self.L, bits, self.w64 = layer(K, N, wl.seed_for("lora", K, N, group, act), group, act, minus_one, dtype == torch.bfloat16)
        self.D = H.upload_and_repack(self.L, scales_bf16_bits=bits)
        self.K, self.N, self.rank, self.n, self.dtype = K, N, rank, n, dtype
        g = gen("lora", K, N, rank, n)
        self.a = (torch.randn((n, rank, K), generator=g, device="cuda") / K ** 0.5).to(dtype)
        self.b = (0.5 * torch.randn((n, N, rank), generator=g, device="cuda")).to(dtype)
        self.scales = 0.25 + torch.rand(n, generator=g, device="cuda")

    def inputs(self, M, *seed):
        g = gen("lora-in", M, *seed)
        x = torch.randn((M, self.K), generator=g, device="cuda").to(self.dtype)
        ids = torch.randint(-1, self.n, (M,), generator=g, device="cuda").to(torch.int32)
        return x, ids

    def plain(self, x, ids, scales):
        u, x = U[self.dtype], x.double()
        y, size, square = x @ self.w64, x.abs() @ self.w64.abs(), (x * x) @ (self.w64 * self.w64)
        part, part_size = torch.zeros_like(y), torch.zeros_like(y)
        for a in range(self.n):
            m = (ids == a).nonzero().squeeze(1)
            A, Bm = self.a[a].double(), self.b[a].double()
            s = 1.0 if scales is None else float(scales[a])
            part[m] = s * ((x[m] @ A.t()) @ Bm.t())
            part_size[m] = abs(s) * ((x[m].abs() @ A.abs().t()) @ Bm.abs().t())
        y = y + part
        most = u * y.abs() + self.K * F32 * size + (self.K + self.rank) * F32 * part_size + sums(self.dtype, x, self.w64)
        mean_square = (u * y) ** 2
        if x.shape[0] > 8:
            most += u * part.abs()
            mean_square += (u * part) ** 2
        if x.shape[0] > 16:
            most += u * size
            mean_square += u * u * square
        return y, 1.01 * most + 2.0 ** -24, mean_square

    def check(self, ws, x, ids, scales, D=None, y=None, stream=None):
        want, most, square = self.plain(x, ids, scales)
        D = D or self.D
        H.ensure_for_lora(ws, x.shape[0], D, self.rank)
        ws.buf.fill_(0xff)
        y = H.gemm_lora(x, D, self.a, self.b, ids, scales, y)
        assert B.gptq_check_status() == B.GPTQ_OK
        assert torch.isfinite(y).all()
        err = (y.double() - want).abs()
        assert (err <= most).all(), f"{int((err > most).sum())} of {err.numel()} beyond the bound, worst {float((err / most).max()):.2f} of it"
        assert float((err * err).mean()) <= float(square.mean()), (float((err * err).mean()), float(square.mean()))
        return y


@pytest.mark.parametrize("M,K,N,rank,n", [(1, 128, 128, 8, 1), (1, 1024, 384, 16, 4), (2, 2048, 256, 64, 3), (7, 512, 640, 24, 7),
                                          (8, 4096, 256, 16, 2), (9, 640, 128, 128, 5), (16, 1152, 384, 40, 16), (17, 512, 256, 16, 3),
                                          (40, 384, 512, 256, 6), (65, 1024, 256, 8, 64), (130, 640, 384, 64, 2), (513, 512, 384, 16, 9)])
def test_lora(ws, M, K, N, rank, n):
    lora = Lora(K, N, rank, n)
    x, ids = lora.inputs(M)
    lora.check(ws, x, ids, lora.scales)
    lora.check(ws, x, ids, None)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("group,act,minus_one", [(128, True, False), (64, False, True), (32, True, False), (256, False, False)])
@pytest.mark.parametrize("M", [1, 5, 13, 30, 200])
def test_lora_formats(ws, M, group, act, minus_one, dtype):
    lora = Lora(512, 384, 16, 4, group, act, minus_one, dtype)
    x, ids = lora.inputs(M, group)
    lora.check(ws, x, ids, lora.scales)


@pytest.mark.parametrize("M,K,N", [(40, 256, 384), (48, 4096, 4480), (150, 384, 256), (20, 512, 128)])
def test_lora_bf16_many_rows(ws, M, K, N):
    """The residual of every matmul kernel for many rows, in bfloat16: K below 512, few panels and a long K, tiles of many rows."""
    lora = Lora(K, N, 16, 3, dtype=torch.bfloat16)
    x, ids = lora.inputs(M, "residual")
    lora.check(ws, x, ids, lora.scales)


def test_lora_infinite_activations(ws):
    """An infinity in x gives what the product gives: infinities of the weights' signs (NaN where q = z), and in its own row only."""
    lora = Lora(512, 256, 16, 3)
    for M in (1, 5, 8):
        x, ids = lora.inputs(M, "inf")
        ids[M - 1] = -1
        want = lora.check(ws, x, ids, lora.scales)
        x[M - 1, 33] = math.inf
        y = H.gemm_lora(x, lora.D, lora.a, lora.b, ids, lora.scales)
        assert torch.equal(y[:M - 1], want[:M - 1])
        row = lora.w64[33]
        assert torch.equal(y[M - 1][row != 0].double(), math.inf * row[row != 0].sign())
        assert y[M - 1][row == 0].isnan().all() and (row == 0).any()


def test_lora_adapter_of_infinities_stays_with_its_rows(ws):
    lora = Lora(512, 256, 16, 4)
    for M in (6, 14, 40, 100):
        x, ids = lora.inputs(M, "bad")
        ids[ids == 2] = 1
        want = lora.check(ws, x, ids, lora.scales)
        rows = torch.arange(M, device="cuda") % 3 == 1
        a, b = lora.a[2].clone(), lora.b[2].clone()
        lora.a[2, :, ::7], lora.b[2] = math.nan, math.inf
        ids[rows] = 2
        y = H.gemm_lora(x, lora.D, lora.a, lora.b, ids, lora.scales)
        lora.a[2], lora.b[2] = a, b
        assert torch.equal(y[~rows], want[~rows])
        assert y[rows].isnan().all()


def test_lora_presorted(ws):
    lora = Lora(512, 256, 16, 3, act=True)
    for M in (4, 33):
        x, ids = lora.inputs(M, "sorted")
        want = lora.check(ws, x, ids, lora.scales)
        order = lora.D.perm.long()
        D = H.DeviceLinear(**{**lora.D.__dict__, "act_order": B.GPTQ_ACT_ORDER_PRESORTED, "perm": None})
        a = lora.a
        lora.a = a[:, :, order].contiguous()
        y = H.gemm_lora(x[:, order].contiguous(), D, lora.a, lora.b, ids, lora.scales)
        lora.a = a
        _, most, _ = lora.plain(x, ids, lora.scales)
        assert ((y.double() - want.double()).abs() <= 2 * most).all()


def test_lora_rows_without_adapter(ws):
    """Rows without an adapter are rows of the plain product; adapters nobody uses are not read."""
    lora = Lora(512, 256, 16, 4)
    lora.a[2] = math.nan
    lora.b[2] = math.inf
    for M in (1, 6, 16, 50):
        x, ids = lora.inputs(M, "none")
        ids[ids == 2] = 1
        ids[0] = 4
        ids[M // 2] = -2147483648
        lora.a[2], lora.b[2] = 0, 0
        lora.check(ws, x, ids, lora.scales)
        lora.a[2], lora.b[2] = math.nan, math.inf
        y = H.gemm_lora(x, lora.D, lora.a, lora.b, ids, lora.scales)
        assert torch.isfinite(y).all()
        ids.fill_(-1)
        lora.a[2], lora.b[2] = 0, 0
        lora.check(ws, x, ids, None)


def test_lora_runs_of_rows(ws):
    """Packed prompts: runs of rows of odd lengths, a run of one row, rows of one adapter in two places."""
    lora = Lora(512, 384, 16, 5)
    ids = torch.cat([torch.full((c,), a, dtype=torch.int32) for a, c in ((2, 37), (0, 1), (-1, 5), (4, 64), (2, 70), (1, 23))]).cuda()
    x, _ = lora.inputs(ids.numel(), "runs")
    lora.check(ws, x, ids, lora.scales)


def test_lora_refuses_other_layouts(ws):
    lora, bf = Lora(256, 256, 8, 2), Lora(256, 256, 8, 2, dtype=torch.bfloat16)
    flagged = H.upload_and_repack(lora.L, gate_up=True)
    for M in (3, 40):
        x, ids = lora.inputs(M, "layout")
        H.ensure_for_lora(ws, M, lora.D, 8)
        for D in (flagged, bf.D):
            y = torch.full((M, 256), 7.0, dtype=torch.float16, device="cuda")
            H.gemm_lora(x, D, lora.a, lora.b, ids, None, y)
            assert B.gptq_check_status() == B.GPTQ_ERR_LAYOUT
            assert (y == 7).all()


# -------------------------------------------------------------------------------------------------------------- together

def block(x, lora, router, moe, k):
    """A projection under adapters, its residual by hand, then the routed MLP with its residual."""
    ids = block.adapter_ids[:x.shape[0]]
    h = (H.gemm_lora(x, lora.D, lora.a, lora.b, ids, lora.scales).float() + x.float()).to(x.dtype)
    experts, weights = H.moe_route(h @ router, k)
    return h, experts, weights, H.moe_mlp(h, experts, weights, moe.up, moe.down, h)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M", [1, 12, 40])
def test_together_eager_stream_and_graph(ws, M, dtype):
    lora, moe, k = Lora(256, 256, 16, 3, dtype=dtype), Moe(256, 384, 8, dtype=dtype), 2
    H.ensure_for_lora(ws, 64, lora.D, 16)
    H.ensure_for_moe(ws, 64, moe.up, k)
    router = (torch.randn((256, 8), generator=gen("router"), device="cuda") / 16).to(dtype)
    x, block.adapter_ids = lora.inputs(M, "block")
    h, experts, weights, y = block(x, lora, router, moe, k)
    want, most, _ = moe.plain(h, experts, weights, h)
    assert ((y.double() - want).abs() <= most).all()
    assert torch.equal(block(x, lora, router, moe, k)[3], y)          # the same bits again
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = block(x, lora, router, moe, k)[3]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(again, y)
    graph = torch.cuda.CUDAGraph()
    static = x.clone()
    with torch.cuda.graph(graph):
        out = block(static, lora, router, moe, k)[3]
    for seed in ("first", "second"):
        x2, _ = lora.inputs(M, seed)
        want2 = block(x2, lora, router, moe, k)[3]
        static.copy_(x2)
        for _ in range(3):
            graph.replay()
        assert torch.equal(out, want2)
    assert B.gptq_check_status() == B.GPTQ_OK


def test_two_streams_with_scratch_of_their_own(ws):
    """Calls that run at the same time, each captured with a workspace of its own registered."""
    moe, lora = Moe(512, 512, 8), Lora(512, 640, 16, 4)
    x, ids, w, r = moe.inputs(9, 2, "streams")
    xl, il = lora.inputs(30, "streams")
    H.ensure_for_moe(ws, 9, moe.up, 2)
    H.ensure_for_lora(ws, 30, lora.D, 16)
    want, want_l = H.moe_mlp(x, ids, w, moe.up, moe.down, r), H.gemm_lora(xl, lora.D, lora.a, lora.b, il, lora.scales)
    graphs, outs = [], []
    for k in range(2):
        mine = H.WorkspaceHolder()
        H.ensure_for_moe(mine, 9, moe.up, 2)
        mine.ensure(max(mine.buf.numel(), B.gptq_lora_workspace_bytes(30, 640, 512, 128, 0, 16)))
        y, yl = torch.empty_like(x), torch.empty_like(want_l)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(3):
                H.moe_mlp(x, ids, w, moe.up, moe.down, r, y)
                H.gemm_lora(xl, lora.D, lora.a, lora.b, il, lora.scales, yl)
        graphs.append((g, mine))
        outs.append((y, yl))
    side = [torch.cuda.Stream() for _ in range(2)]
    for s in side:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for (g, _mine), s in zip(graphs, side):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for y, yl in outs:
        assert torch.equal(y, want) and torch.equal(yl, want_l)
    ws.ensure(1)
    assert B.gptq_check_status() == B.GPTQ_OK


def test_repeats_bit_for_bit(ws):
    moe, lora = Moe(1024, 512, 8), Lora(1024, 512, 16, 4)
    x, ids, w, r = moe.inputs(7, 3, "repeat")
    xl, il = lora.inputs(9, "repeat")
    H.ensure_for_moe(ws, 7, moe.up, 3)
    H.ensure_for_lora(ws, 9, lora.D, 16)
    y, z = H.moe_mlp(x, ids, w, moe.up, moe.down, r), H.gemm_lora(xl, lora.D, lora.a, lora.b, il, lora.scales)
    for _ in range(200):
        ys = [H.moe_mlp(x, ids, w, moe.up, moe.down, r) for _ in range(4)]
        zs = [H.gemm_lora(xl, lora.D, lora.a, lora.b, il, lora.scales) for _ in range(4)]
        assert all(torch.equal(v, y) for v in ys) and all(torch.equal(v, z) for v in zs)


# ------------------------------------------------------------------------------------- values at the ends of their types' ranges

def zero_weights(lora):
    """The shared layer's weights become zero (every nibble its zero point), so that y is the adapters' part alone.  Up to 8 rows it is formed
    as sum q x - z sum x, off by 8 2^-23 (31 or 287) sum |x| s (the head of this file), where `sums` takes s from |w|, here 0: it is added."""
    lora.L.qweight[:], lora.L.qzeros[:] = -0x77777778, -0x77777778
    lora.w64.zero_()
    bits = wl.make_scales_bf16(lora.L.G, lora.N, 5) if lora.dtype == torch.bfloat16 else None
    lora.D = H.upload_and_repack(lora.L, scales_bf16_bits=bits)
    scales = torch.from_numpy(lora.L.scales).cuda() if bits is None else H.bf16_from_bits(bits)
    s64 = scales.double().repeat_interleave(lora.L.group_size, 0)
    plain = lora.plain

    def with_sums(x, ids, scales):
        y, most, square = plain(x, ids, scales)
        if x.shape[0] > 8:
            return y, most, square
        more = 8 * F32 * (287 if lora.dtype == torch.bfloat16 else 31) * (x.double().abs() @ s64)
        return y, most + more, square + more * more

    lora.plain = with_sums


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,rank", [(8, 16), (64, 16), (65, 16), (65, 40), (200, 256)])
def test_lora_large_and_small_inner_sums(ws, M, rank, dtype):
    """v = s x A^T far beyond and far below fp16's range, B the other way round: it is kept in fp32 (lora.plain's bounds; two 16-bit parts
    of v, 2^-22 and 2^-16 of it, are within (K + rank) 2^-23 of the sum of absolute values).  Columns of A of sizes 2^-8 apart."""
    lora = Lora(512, 256, rank, 3, dtype=dtype)
    zero_weights(lora)
    lora.scales = torch.tensor([2.0 ** 20, 1.0, 2.0 ** -20], device="cuda")
    for a, e in enumerate((-10, 0, 8)):
        lora.b[a] = (lora.b[a].float() * 2.0 ** e).to(dtype)
    even = torch.arange(rank, device="cuda") % 2 == 0
    lora.a[:, even] *= 2.0 ** -4
    lora.b[:, :, even] *= 2.0 ** 4
    lora.a[:, ~even] *= 2.0 ** 4
    lora.b[:, :, ~even] *= 2.0 ** -4
    x, ids = lora.inputs(M, "range")
    lora.check(ws, x, ids, lora.scales)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M", [6, 40, 100])
def test_lora_infinities_in_the_adapter(ws, M, dtype):
    """An infinity in B or in v gives what the sum over the rank gives."""
    lora = Lora(512, 256, 16, 3, dtype=dtype)
    x, ids = lora.inputs(M, "infb")
    want = lora.check(ws, x, ids, lora.scales)
    one, two, three = ids == 0, ids == 1, ids == 2
    columns = torch.arange(256, device="cuda") % 5 == 2
    lora.b[1, columns, 3] = math.inf                    # one infinity in some columns of B: that of v's sign
    lora.a[2] = lora.a[2, :1].clone()                   # v infinite, of one sign for the whole rank, and B positive
    lora.b[2] = lora.b[2].abs() + 0.125
    lora.scales[2] = math.inf
    y = H.gemm_lora(x, lora.D, lora.a, lora.b, ids, lora.scales).double()
    assert torch.equal(y[one], want[one].double())
    assert torch.equal(y[two][:, ~columns], want[two][:, ~columns].double())
    v = x.double() @ lora.a[:, 3].double().t()          # [M, adapter]
    assert torch.equal(y[two][:, columns], (math.inf * v[two, 1].sign())[:, None].expand(-1, int(columns.sum())))
    assert torch.equal(y[three], (math.inf * v[three, 2].sign())[:, None].expand(-1, 256))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M", [1, 5, 16])
def test_moe_small_activations(ws, M, dtype):
    """h of about 1e-6, below fp16's normal numbers, under weights that make y ordinary: its two parts still hold it to far less than
    y's rounding (moe.check's mean square: u^2 + 2^-18 of h)."""
    moe = Moe(256, 256, 4, dtype=dtype)
    x, ids, w, _ = moe.inputs(M, 2, "small")
    moe.check(ws, x * 2.0 ** -9, ids, w * 2.0 ** 15, None)


def heavy(count, K, N, positive, group=128):
    """bfloat16 layers whose weights (q - z) s are all positive or all negative: (QuantLinear list, scale bits, float64 weights)."""
    out = []
    for e in range(count):
        q, z = np.full((K, N), 9 if positive else 4, np.uint8), np.full((K // group, N), 6 if positive else 12, np.uint8)
        L = wl.make_linear_from_values(q, z, np.ones((K // group, N), np.float16), group_size=group)
        bits = wl.make_scales_bf16(K // group, N, wl.seed_for("heavy", e, N))
        out.append((L, bits, H.to_device(oracle.dequant_f32_bf16(L.qweight, L.qzeros, bits, L.g_idx, group, False)).double()))
    return [o[0] for o in out], [o[1] for o in out], [o[2] for o in out]


def test_lora_bf16_sums_whose_parts_overflow(ws):
    """x of one sign and 2^114: sum (128 + q) x is beyond fp32's range, sum (q - z) x s is not."""
    lora = Lora(512, 256, 16, 2, dtype=torch.bfloat16)
    for positive in (False, True):
        layers, bits, w64 = heavy(1, 512, 256, positive)
        lora.D, lora.w64 = H.upload_and_repack(layers[0], scales_bf16_bits=bits[0]), w64[0]
        for M in (1, 7):
            x = torch.full((M, 512), 2.0 ** 114, dtype=torch.bfloat16, device="cuda")
            lora.check(ws, x, torch.full((M,), -1, dtype=torch.int32, device="cuda"), None)


def test_moe_bf16_sums_whose_parts_overflow(ws):
    """The same for experts: gates far below zero, h = 0, y = residual; and h of 2^114 into the down layer."""
    moe = Moe.__new__(Moe)
    moe.K, moe.F, moe.E, moe.dtype = 256, 256, 2, torch.bfloat16
    minus, plus = heavy(2, 256, 512, False), heavy(2, 256, 512, True)
    down = heavy(2, 256, 256, True)
    moe.down, moe.down64 = H.upload_experts(down[0], scales_bf16_bits=down[1]), down[2]
    for M in (1, 9, 20):
        ids = (torch.arange(M, device="cuda") % 2).to(torch.int32)[:, None].contiguous()
        w = torch.ones((M, 1), device="cuda")
        moe.up, moe.up64 = H.upload_experts(minus[0], gate_up=True, scales_bf16_bits=minus[1]), minus[2]
        x = torch.full((M, 256), 2.0 ** 114, dtype=torch.bfloat16, device="cuda")
        r = torch.randn((M, 256), generator=gen("overflow", M), device="cuda").to(torch.bfloat16)
        H.ensure_for_moe(ws, M, moe.up, 1)
        assert torch.equal(H.moe_mlp(x, ids, w, moe.up, moe.down, r), r)
        moe.up, moe.up64 = H.upload_experts(plus[0], gate_up=True, scales_bf16_bits=plus[1]), plus[2]
        x = torch.full((M, 256), 2.0 ** 55, dtype=torch.bfloat16, device="cuda")      # gate and up of 2^57 or so
        moe.check(ws, x, ids, w, r)


# ------------------------------------------------------------------------------------------------------------------------ scratch

@pytest.mark.parametrize("K,rank,most", [(4096, 64, 256), (2048, 256, 33)])
def test_lora_scratch_of_the_largest_call(ws, K, rank, most):
    """Scratch of exactly the size that the largest call asks for: every smaller one runs in it, and nothing behind it is written."""
    lora = Lora(K, 128, rank, 2)
    need = B.gptq_lora_workspace_bytes(most, 128, K, 128, 0, rank)
    buf = torch.full((need + 65536,), 0xa5, dtype=torch.uint8, device="cuda")
    try:
        B.check(B.gptq_set_workspace(buf, need), "gptq_set_workspace")
        for M in (1, 8, 9, 32, 33, most - 9, most - 8, most - 1, most):
            if M > most:
                continue
            x, ids = lora.inputs(M, "scratch")
            want, bound, _ = lora.plain(x, ids, lora.scales)
            y = H.gemm_lora(x, lora.D, lora.a, lora.b, ids, lora.scales)
            assert ((y.double() - want).abs() <= bound).all()
        assert (buf[need:] == 0xa5).all()
    finally:
        ws.ensure(1)


def shared_memory_shares(call):
    """(CTAs, dynamic shared memory, share of the SM asked for in percent) of each kernel with dynamic shared memory that `call(stream)` enqueues."""
    from cuda.bindings import driver

    def ok(result):
        assert result[0] == driver.CUresult.CUDA_SUCCESS, result[0]
        return result[1:] if len(result) > 2 else result[1] if len(result) == 2 else None

    stream = torch.cuda.Stream()
    ok(driver.cuStreamBeginCapture(stream.cuda_stream, driver.CUstreamCaptureMode.CU_STREAM_CAPTURE_MODE_RELAXED))
    try:
        call(stream)
    finally:
        graph = ok(driver.cuStreamEndCapture(stream.cuda_stream))
    out = []
    nodes, _ = ok(driver.cuGraphGetNodes(graph, 64))
    for node in nodes:
        if int(node) == 0 or ok(driver.cuGraphNodeGetType(node)) != driver.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL:
            continue
        p = ok(driver.cuGraphKernelNodeGetParams(node))
        share = ok(driver.cuGraphKernelNodeGetAttribute(node, driver.CUlaunchAttributeID.CU_LAUNCH_ATTRIBUTE_PREFERRED_SHARED_MEMORY_CARVEOUT))
        if p.sharedMemBytes:
            out.append((p.gridDimX, p.sharedMemBytes, share.sharedMemCarveout))
    ok(driver.cuGraphDestroy(graph))
    return sorted(out)


def test_a_layers_share_of_the_sm_does_not_depend_on_other_layers(ws):
    """Room for the CTAs that a launch puts on an SM, whatever the launches of the same kernel before it asked for: few columns take one CTA
    per SM with most of its shared memory, more take two with less."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    few, more = Moe(512, 512, 4), Moe(2048, 768, 4)
    lora = Lora(1024, 32 * 2 * sms // 128 * 128 + 256, 16, 2)
    calls = []
    for moe in (few, more):
        x, ids, w, r = moe.inputs(1, 2, "share")
        H.ensure_for_moe(ws, 1, moe.up, 2)
        y = moe.check(ws, x, ids, w, r)
        calls.append(lambda s, a=(x, ids, w, moe.up, moe.down, r, y): H.moe_mlp(*a, stream=s))
    x, ids = lora.inputs(2, "share")
    H.ensure_for_lora(ws, 2, lora.D, 16)
    y = H.gemm_lora(x, lora.D, lora.a, lora.b, ids, None)
    calls.append(lambda s: H.gemm_lora(x, lora.D, lora.a, lora.b, ids, None, y, stream=s))
    seen = [shared_memory_shares(calls[i]) for i in (1, 0, 1, 0, 2)]
    assert seen[0] == seen[2] and seen[1] == seen[3]
    assert len(seen[0]) == len(seen[1]) == 2 and len(seen[4]) == 1
    assert any(ctas <= sms for ctas, _, _ in seen[1])
    for ctas, smem, share in seen[0] + seen[1] + seen[4]:
        on_an_sm = 1 if ctas <= sms else 2
        assert share / 100 * 228 * 1024 >= on_an_sm * (smem + 1024), (ctas, smem, share)
    B.check(B.gptq_check_status(), "gptq_check_status")


# ------------------------------------------------------------------------------------------------------------ sizes, several passes

def test_moe_refuses_other_layouts_before_the_first_pass(ws):
    """A layer of another tiling that only a later pass of 64 tokens names: nothing is stored by the first one either."""
    moe = Moe(256, 128, 4)
    x, ids, w, r = moe.inputs(130, 2, "passes")
    ids[:] = ids % 2
    ids[ids[:, 0] == ids[:, 1], 1] = 1 - ids[ids[:, 0] == ids[:, 1], 0]
    good = moe.check(ws, x, ids, w, r)
    other = Moe(256, 128, 1, dtype=torch.bfloat16)
    for kind in ("up", "down"):
        for row, expert in ((64, 2), (129, 3)):
            stack = getattr(moe, kind)
            mixed = H.DeviceExperts(**{**stack.__dict__, "qzeros_t": stack.qzeros_t.clone()})
            mixed.qzeros_t[expert] = getattr(other, kind).qzeros_t[0]
            pair = (mixed, moe.down) if kind == "up" else (moe.up, mixed)
            assert torch.equal(H.moe_mlp(x, ids, w, *pair, r), good)           # not named: no matter
            assert B.gptq_check_status() == B.GPTQ_OK
            named = ids.clone()
            named[row, 1] = expert
            for shared in (False, True):
                y = x.clone() if shared else torch.full_like(x, 7.0)
                before = y.clone()
                H.moe_mlp(y if shared else x, named, w, *pair, r, y)
                assert B.gptq_check_status() == B.GPTQ_ERR_LAYOUT
                assert torch.equal(y, before)
    assert torch.equal(H.moe_mlp(x, ids, w, moe.up, moe.down, r), good)
    assert B.gptq_check_status() == B.GPTQ_OK


def test_moe_refused_in_a_graph(ws):
    """A captured call of several passes is refused or not as the layers and ids are when it is replayed."""
    moe, other = Moe(256, 128, 3), Moe(256, 128, 1, dtype=torch.bfloat16)
    x, ids, w, r = moe.inputs(70, 2, "replay")
    ids[:] = torch.tensor([0, 1], dtype=torch.int32)
    want = moe.check(ws, x, ids, w, r)
    up = H.DeviceExperts(**{**moe.up.__dict__, "qzeros_t": moe.up.qzeros_t.clone()})
    up.qzeros_t[2] = other.up.qzeros_t[0]
    y = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        H.moe_mlp(x, ids, w, up, moe.down, r, y)
    for bad in (False, True, True, False, True, False):
        ids[69, 0] = 2 if bad else 0
        y.fill_(7.0)
        graph.replay()
        assert B.gptq_check_status() == (B.GPTQ_ERR_LAYOUT if bad else B.GPTQ_OK)
        assert torch.equal(y, torch.full_like(y, 7.0) if bad else want)


def test_lora_more_rows_than_a_grid_is_high(ws):
    """65536 blocks of 32 rows and some: the last rows are computed like the first."""
    lora = Lora(128, 128, 8, 2)
    M = 32 * 65536 + 40
    x, ids = lora.inputs(100, "far")
    far_x, far_ids = torch.zeros((M, 128), dtype=torch.float16, device="cuda"), torch.full((M,), -1, dtype=torch.int32, device="cuda")
    far_x[-100:], far_ids[-100:] = x, ids
    H.ensure_for_lora(ws, M, lora.D, 8)
    y = H.gemm_lora(far_x, lora.D, lora.a, lora.b, far_ids, lora.scales)
    assert B.gptq_check_status() == B.GPTQ_OK
    want, most, _ = lora.plain(x, ids, lora.scales)
    assert ((y[-100:].double() - want).abs() <= most).all()
    assert not y[:-100].any()


def test_route_weights_of_spread_logits():
    """p = exp(l - max): 2^-22 for the exponential (two steps, as CUDA gives for ex2.approx) and 2^-23 for what goes into it, in numerator
    and sum alike, 2^-22 for the division (two steps), 2^-24 for each addition."""
    g = gen("route-spread")
    for E, k in ((8, 8), (64, 32), (1000, 32)):
        logits = (85 * torch.rand((200, E), generator=g, device="cuda") - 40).float()
        for renormalize in (True, False):
            ids, w = H.moe_route(logits, k, renormalize)
            want_ids, want = plain_route(logits, k, renormalize)
            assert np.array_equal(ids.cpu().numpy(), want_ids)
            err = np.abs(w.cpu().double().numpy() - want) / want
            # the sum over all experts: E / 32 additions in a lane and five between lanes
            assert err.max() <= 2 * (2.0 ** -22 + 2.0 ** -23) + 2.0 ** -22 + (k if renormalize else E / 32 + 5) * 2.0 ** -24, (E, renormalize, err.max() * 2 ** 24)


def test_moe_bf16_overflowing_parts_keep_both_parts_of_h(ws):
    """One h of 2^122 in a row: (128 + q) h is beyond fp32's range, and the second of its two 16-bit parts still counts (moe.check's bound
    allows one rounding of y)."""
    moe = Moe.__new__(Moe)
    moe.K, moe.F, moe.E, moe.dtype = 256, 128, 1, torch.bfloat16
    up, bits, _ = heavy(1, 256, 256, True)
    bits[0][:] = 0
    bits[0][:, [5, 128 + 5]] = wl.bf16_bits(np.float32([3 * 2.0 ** -8]))[0]
    moe.up = H.upload_experts(up, gate_up=True, scales_bf16_bits=bits)
    moe.up64 = [H.to_device(oracle.dequant_f32_bf16(up[0].qweight, up[0].qzeros, bits[0], up[0].g_idx, 128, False)).double()]
    down = heavy(1, 128, 256, True)
    moe.down, moe.down64 = H.upload_experts(down[0], scales_bf16_bits=down[1]), down[2]
    for M in (3, 16):
        x = (2.0 ** 58 * (1 + torch.randint(0, 128, (M, 1), generator=gen("parts", M), device="cuda") / 128)).expand(M, 256).to(torch.bfloat16).contiguous()
        moe.check(ws, x, torch.zeros((M, 1), dtype=torch.int32, device="cuda"), torch.ones((M, 1), device="cuda"), None)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M", [65, 144])
def test_moe_several_passes_of_act_order_layers(ws, M, dtype):
    moe = Moe(256, 128, 5, 64, True, True, dtype)
    x, ids, w, r = moe.inputs(M, 3, "passes-act")
    ids[M // 2] = -1
    moe.check(ws, x, ids, w, r)

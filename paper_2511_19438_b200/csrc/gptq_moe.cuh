// Routed experts: the choice of experts for each token, and a whole mixture-of-experts MLP for a few tokens in two kernels.
#pragma once
#include "gptq_common.cuh"
#include "gptq_direct.cuh"
#include "gptq_splitk.cuh"   // silu_mul, cluster barriers, map_to_cluster_rank

namespace gptq {

// ------------------------------------------------------------------------------ routing
// One warp per token; lane l holds the logits of experts l, l + 32, ... as keys whose unsigned order is the order of the
// logits (0: an expert that cannot be chosen).  A pick is two warp-wide reductions: the largest key, then the lowest expert
// that has it.  The weights are exp(l - max) over their sum, or over the sum of all experts, in fp32.
constexpr int kRouteMaxExperts = 1024, kRouteMaxTopK = 32, kRouteWarps = 4;

__device__ __forceinline__ uint32_t logit_bits(const void *logits, int type, size_t i)
{
    if (type == GPTQ_LOGITS_F32) return __ldg(reinterpret_cast<const uint32_t *>(logits) + i);
    const unsigned short v = __ldg(reinterpret_cast<const unsigned short *>(logits) + i);
    return type == GPTQ_LOGITS_BF16 ? (uint32_t)v << 16 : __float_as_uint(__half2float(__ushort_as_half(v)));
}
__device__ __forceinline__ uint32_t logit_key(uint32_t b)
{
    if ((b << 1) == 0) b = 0;                                    // -0 and +0 are equal
    if (b == 0xff800000u || (b << 1) > 0xff000000u) return 0;    // -inf, NaN
    if (b == 0x7f800000u) b = 0x7f7fffffu;                       // +inf: the largest finite number
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

template <int NV>
__global__ void __launch_bounds__(32 * kRouteWarps)
route_kernel(const void *__restrict__ logits, int type, int32_t *__restrict__ ids, float *__restrict__ weights, int M, int E, int k,
             int renormalize)
{
    const int m = blockIdx.x * kRouteWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    pdl_wait();
    pdl_launch_dependents();
    if (m >= M) return;
    uint32_t key[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = lane + 32 * i;
        key[i] = e < E ? logit_key(logit_bits(logits, type, (size_t)m * E + e)) : 0u;
    }
    float top = 0.f, total = 0.f, mine = 0.f;
    int my_id = -1;
    for (int j = 0; j < k; ++j) {
        uint32_t best = key[0];
#pragma unroll
        for (int i = 1; i < NV; ++i) best = max(best, key[i]);
        const uint32_t all = __reduce_max_sync(0xffffffffu, best);
        if (all == 0) break;                                      // nothing left that can be chosen
        if (j == 0) {
            top = key_logit(all);
            if (!renormalize) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (key[i]) sum += __expf(key_logit(key[i]) - top);
#pragma unroll
                for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                total = sum;
            }
        }
        uint32_t at = 0xffffffffu;
#pragma unroll
        for (int i = NV - 1; i >= 0; --i)
            if (key[i] == all) at = lane + 32 * i;
        const uint32_t e = __reduce_min_sync(0xffffffffu, at);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (e == (uint32_t)(lane + 32 * i)) key[i] = 0;
        const float p = __expf(key_logit(all) - top);
        if (renormalize) total += p;
        if (lane == j) { mine = p; my_id = (int)e; }
    }
    if (lane < k) {
        ids[(size_t)m * k + lane] = my_id;
        weights[(size_t)m * k + lane] = my_id >= 0 ? mine / total : 0.f;
    }
}

int launch_route(const void *logits, int type, int32_t *ids, float *weights, int M, int E, int k, int renormalize, cudaStream_t s)
{
    const dim3 grid((unsigned)((M + kRouteWarps - 1) / kRouteWarps));
    const int T = 32 * kRouteWarps;
    if (E <= 32) return launch_dependent(route_kernel<1>, grid, T, 0, 1, s, logits, type, ids, weights, M, E, k, renormalize);
    if (E <= 64) return launch_dependent(route_kernel<2>, grid, T, 0, 1, s, logits, type, ids, weights, M, E, k, renormalize);
    if (E <= 128) return launch_dependent(route_kernel<4>, grid, T, 0, 1, s, logits, type, ids, weights, M, E, k, renormalize);
    if (E <= 256) return launch_dependent(route_kernel<8>, grid, T, 0, 1, s, logits, type, ids, weights, M, E, k, renormalize);
    if (E <= 512) return launch_dependent(route_kernel<16>, grid, T, 0, 1, s, logits, type, ids, weights, M, E, k, renormalize);
    return launch_dependent(route_kernel<32>, grid, T, 0, 1, s, logits, type, ids, weights, M, E, k, renormalize);
}

// ------------------------------------------------------------------------------ the experts' MLP
constexpr int kMoeMaxRows = 64;                 // tokens of one pass
constexpr int kMoeWarps = 8, kMoeThreads = 32 * kMoeWarps;
constexpr int kMoeMaxExperts = 1024, kMoeMaxTopK = 32;

struct MoeArgs {
    const __half *x;          // [M, K]; with act-order [M k, K], each slot's row in its expert's order
    const int32_t *ids;       // [M, k]
    const float *weights;     // [M, k]
    const uint8_t *gu_w, *gu_z, *gu_s, *dn_w, *dn_z, *dn_s;
    size_t gu_w_bytes, gu_z_bytes, gu_s_bytes, dn_w_bytes, dn_z_bytes, dn_s_bytes;    // of one expert
    const int32_t *down_index;      // [E, F] or nullptr
    __half *h;                // [M k, F]
    const __half *residual;   // [M, K] or nullptr
    __half *y;                // [M, K]
    int M, k, E, K, F;
    int x_by_slot;            // rows of x: slots instead of tokens
};

// The slots (m, j) of a batch grouped by expert, in the order of experts and, within one, of slots.  An expert's slots are cut
// into SEGMENTS of at most R, the rows that one sweep over the expert's weights serves.
struct SlotPlan {
    float *weight;       // [P] by slot: the weights that a token gives its expert, summed
    int *counts;         // [E] while it is built
    short *key;          // [P] by slot: its expert, -1 where the slot is not used
    short *slot;         // [P] slots by expert
    short *rank;         // [P] by slot, while it is built
    short *seg_begin;    // [segments + 1] into slot
    short *seg_expert;   // [segments]
};
__host__ __device__ constexpr int slot_plan_bytes(int P, int E) { return (4 * P + 4 * E + 12 * (P + 2) + 15) & ~15; }
__device__ __forceinline__ SlotPlan slot_plan_view(uint8_t *smem, int P, int E)
{
    SlotPlan p;
    p.weight = reinterpret_cast<float *>(smem);
    p.counts = reinterpret_cast<int *>(p.weight + P);
    p.key = reinterpret_cast<short *>(p.counts + E);
    p.slot = p.key + P + 2;
    p.rank = p.slot + P + 2;
    p.seg_begin = p.rank + P + 2;
    p.seg_expert = p.seg_begin + P + 2;
    return p;
}

// By all threads of a block; returns the number of segments.  A slot whose expert a lower slot of the same token names already
// adds its weight there.  `seg_expert` holds the raw ids until the segments are known.
__device__ __forceinline__ int build_slot_plan(const MoeArgs &a, int R, const SlotPlan &p)
{
    __shared__ int s_segments;
    const int P = a.M * a.k, tid = threadIdx.x, lane = tid & 31;
    short *raw = p.seg_expert;
    for (int s = tid; s < P; s += kMoeThreads) {
        const int e = __ldg(a.ids + s);
        raw[s] = (unsigned)e < (unsigned)a.E ? (short)e : (short)-1;
        p.weight[s] = __ldg(a.weights + s);
    }
    for (int e = tid; e < a.E; e += kMoeThreads) p.counts[e] = 0;
    __syncthreads();
    for (int s = tid; s < P; s += kMoeThreads) {
        const int e = raw[s], j = s % a.k;
        bool first = e >= 0;
        for (int i = 1; i <= j; ++i) first &= raw[s - i] != e;
        if (first) {
            float sum = p.weight[s];
            for (int i = s + 1; i < s - j + a.k; ++i)
                if (raw[i] == e) sum += p.weight[i];      // (a slot of its own token, whose weight nobody changes)
            p.weight[s] = sum;
        }
        p.key[s] = first ? (short)e : (short)-1;
    }
    __syncthreads();
    if (tid < 32) {
        for (int base = 0; base < P; base += 32) {
            const int s = base + lane, e = s < P ? p.key[s] : -1;
            const uint32_t same = __match_any_sync(0xffffffffu, e);
            const int before = __popc(same & ((1u << lane) - 1));
            int from = 0;
            if (e >= 0) from = p.counts[e];
            __syncwarp();
            if (e >= 0) {
                p.rank[s] = (short)(from + before);
                if (before == 0) p.counts[e] = from + __popc(same);
            }
            __syncwarp();
        }
        // positions and segments of the experts: a lane takes neighbouring experts, the warp a scan over the lanes
        const int per = (a.E + 31) / 32, e0 = min(lane * per, a.E), e1 = min(e0 + per, a.E);
        int slots = 0, segs = 0;
        for (int e = e0; e < e1; ++e) slots += p.counts[e], segs += (p.counts[e] + R - 1) / R;
        int sum = slots | segs << 16;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        const int total = __shfl_sync(0xffffffffu, sum, 31);
        int pos = (sum & 0xffff) - slots, seg = (sum >> 16) - segs;
        for (int e = e0; e < e1; ++e) {
            const int c = p.counts[e];
            p.counts[e] = pos;
            for (int i = 0; i < c; i += R) {
                p.seg_expert[seg] = (short)e;
                p.seg_begin[seg++] = (short)(pos + i);
            }
            pos += c;
        }
        if (lane == 0) {
            p.seg_begin[total >> 16] = (short)(total & 0xffff);
            s_segments = total >> 16;
        }
    }
    __syncthreads();
    for (int s = tid; s < P; s += kMoeThreads)
        if (p.key[s] >= 0) p.slot[p.counts[p.key[s]] + p.rank[s]] = (short)s;
    __syncthreads();
    return s_segments;
}

// Kernel 1: h[slot] = silu(gate) * up.  A TILE is a segment and 16 gate columns with their 16 up columns; a CTA works through a
// range of neighbouring tiles (their rows of x stay in L1).  The warps share a tile's items along K and meet in shared memory at its
// end; their loads run on into the next tile.
template <int NT, int SUB, bool BF>
__global__ void __launch_bounds__(kMoeThreads, NT <= 2 ? 2 : 1) moe_gate_up_kernel(const MoeArgs a)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const SlotPlan plan = slot_plan_view(smem, a.M * a.k, a.E);
    float *red = reinterpret_cast<float *>(smem + slot_plan_bytes(a.M * a.k, a.E));
    pdl_wait();
    pdl_launch_dependents();
    const int segments = build_slot_plan(a, 8 * NT, plan);
    const int G = a.K / kGroup, per_seg = a.F / 16, T = segments * per_seg;
    const int t0 = (int)((long long)blockIdx.x * T / gridDim.x), t1 = (int)((long long)(blockIdx.x + 1) * T / gridDim.x);

    // ---- loads: tile l_tile, item l_item; a warp starts at another item in every tile, so that all get their share where the
    // items are no multiple of the warps
    int l_tile = t0 - 1, l_item = G, l_seg = 0, l_col = 0;
    uint32_t l_flags = 0;
    UnitPtrs ptrs{};
    const __half *rows[NT];
    auto enter_segment = [&]() {
        const int first = plan.seg_begin[l_seg], count = plan.seg_begin[l_seg + 1] - first;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            rows[t] = nullptr;
            if (8 * t + g < count) {
                const int s = plan.slot[first + 8 * t + g];
                rows[t] = a.x + (size_t)(a.x_by_slot ? s : s / a.k) * a.K + 8 * t4;
            }
        }
    };
    auto advance = [&]() {      // to the next item that is this warp's; l_tile = t1: none
        l_item += kMoeWarps;
        while (l_item >= G) {
            if (++l_tile >= t1) return;
            l_item = (warp + l_tile) & (kMoeWarps - 1);
            const bool start = l_tile == t0;
            if (start || ++l_col == per_seg) {
                l_seg = start ? l_tile / per_seg : l_seg + 1;
                l_col = start ? l_tile - l_seg * per_seg : 0;
                enter_segment();
            }
            const int e = plan.seg_expert[l_seg];
            const uint8_t *zeros = a.gu_z + e * a.gu_z_bytes;
            l_flags = __ldg(&reinterpret_cast<const TiledTrailer *>(zeros + a.gu_z_bytes - kTrailerBytes)->flags);
            ptrs = unit_ptrs<SUB>(a.gu_w + e * a.gu_w_bytes, a.gu_s + e * a.gu_s_bytes, zeros, l_col >> 2, G, l_col & 3, lane);
        }
    };
    constexpr int D = NT == 1 ? 2 : 1;
    DirectRegs<NT, 2, SUB> regs[D];
    uint32_t flags[D] = {};
    int tile_of[D];
    auto load = [&](int d) {
        advance();
        tile_of[d] = l_tile;
        if (l_tile < t1) {
            load_item_weights<NT, 2, 4, SUB>(regs[d], ptrs, l_item);
            load_item_rows<NT, 2, SUB>(regs[d], rows, l_item);
            flags[d] = l_flags;
        }
    };

    // ---- arithmetic
    float acc[2][NT][4] = {};
    int tile = t0;
    auto finish_tile = [&]() {      // sums over the warps, in their order: [buffer][warp][value][lane]
        float *buf = red + (tile & 1) * (kMoeWarps * 8 * NT * 32);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    buf[(warp * (8 * NT) + (u * NT + t) * 4 + i) * 32 + lane] = acc[u][t][i];
                    acc[u][t][i] = 0.f;
                }
        __syncthreads();
        const int seg = tile / per_seg, c16 = tile - seg * per_seg;
        const int first = plan.seg_begin[seg], count = plan.seg_begin[seg + 1] - first;
        for (int o = threadIdx.x; o < NT * 4 * 32; o += kMoeThreads) {
            const int v = o >> 5, t = v >> 2, i = v & 3;            // (lane of o = lane: the block is a multiple of a warp)
            const int r = 8 * t + 2 * t4 + (i & 1);
            if (r >= count) continue;
            float gate = 0.f, up = 0.f;
#pragma unroll
            for (int w = 0; w < kMoeWarps; ++w) {
                gate += buf[(w * (8 * NT) + v) * 32 + lane];
                up += buf[(w * (8 * NT) + 4 * NT + v) * 32 + lane];
            }
            int col = 16 * c16 + g + 8 * (i >> 1);
            if (a.down_index) col = __ldg(a.down_index + (size_t)plan.seg_expert[seg] * a.F + col);
            store_out16<BF>(a.h + (size_t)plan.slot[first + r] * a.F + col, silu_mul(gate, up));
        }
        ++tile;
    };
#pragma unroll
    for (int d = 0; d < D; ++d) load(d);
    for (bool more = true; more;) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            while (tile < tile_of[d] && tile < t1) finish_tile();
            if (tile_of[d] >= t1) { more = false; break; }
            multiply_item<NT, 2, SUB, BF>(regs[d], flags[d] & kFormatZerosMinusOne, acc);
            load(d);
        }
    }
}

// Kernel 2: y = residual + sum over a token's experts of weight * (h Wd).  A cluster of S CTAs takes 32 columns of y; the items
// of all segments, one behind the other, are shared out evenly over its 8 S warps.  A warp that reaches the end of a segment (or
// of its share) adds its sums, weighted, to its own [token][32] tile in shared memory; the tiles are summed in the order of warps
// and ranks, so results are reproducible.
constexpr int kDownCols = 32;
template <int NT, int SUB, bool BF>
__global__ void __launch_bounds__(kMoeThreads, NT <= 2 ? 2 : 1) moe_down_kernel(const MoeArgs a, int S)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int s_bad;
    constexpr int NU = kDownCols / 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const int tile = blockIdx.x / S, rank = blockIdx.x - tile * S;
    const int G = a.F / kGroup, panel = tile / (8 / NU), unit = tile % (8 / NU) * NU;
    pdl_launch_dependents();
    // ids and weights are older than the kernel before this one, which waited for them before it let this one in
    const SlotPlan plan = slot_plan_view(smem, a.M * a.k, a.E);
    float *tiles = reinterpret_cast<float *>(smem + slot_plan_bytes(a.M * a.k, a.E));
    const int cells = a.M * kDownCols;
    float *mine = tiles + warp * cells;
    for (int i = lane; i < cells; i += 32) mine[i] = 0.f;
    if (threadIdx.x == 0) s_bad = 0;
    const int segments = build_slot_plan(a, 8 * NT, plan);
    const int W = kMoeWarps * S, wi = rank * kMoeWarps + warp;
    const int U = segments * G, j0 = (int)((long long)wi * U / W), j1 = (int)((long long)(wi + 1) * U / W), n = j1 - j0;

    // what is loaded next
    int l_seg = 0, l_item = 0;
    UnitPtrs ptrs{};
    uint32_t l_flags = 0;
    const __half *rows[NT];
    auto enter_segment = [&]() {
        const int e = plan.seg_expert[l_seg], first = plan.seg_begin[l_seg], count = plan.seg_begin[l_seg + 1] - first;
        const uint8_t *zeros = a.dn_z + e * a.dn_z_bytes;
        l_flags = __ldg(&reinterpret_cast<const TiledTrailer *>(zeros + a.dn_z_bytes - kTrailerBytes)->flags);
        ptrs = unit_ptrs<SUB>(a.dn_w + e * a.dn_w_bytes, a.dn_s + e * a.dn_s_bytes, zeros, panel, G, unit, lane);
#pragma unroll
        for (int t = 0; t < NT; ++t) rows[t] = 8 * t + g < count ? a.h + (size_t)plan.slot[first + 8 * t + g] * a.F + 8 * t4 : nullptr;
    };
    constexpr int D = NT == 1 ? 2 : 1;
    DirectRegs<NT, NU, SUB> regs[D];
    uint32_t flags[D] = {};
    int seg_of[D], item_of[D];
    auto load_weights = [&](int d) {
        load_item_weights<NT, NU, 1, SUB>(regs[d], ptrs, l_item);
        flags[d] = l_flags;
        seg_of[d] = l_seg;
        item_of[d] = l_item;
    };
    auto next = [&]() {
        if (++l_item == G) {
            l_item = 0;
            if (++l_seg < segments) enter_segment();
        }
    };
    // A layer of the wrong format anywhere: nothing is stored.  Every CTA looks at all experts in use, so that they agree; the
    // trailers are asked for here and looked at behind the main loop.
    uint32_t up_flags = kFormatGateUp | (BF ? kFormatBf16 : 0u), down_flags = BF ? kFormatBf16 : 0u;
    auto trailer_flags = [](const uint8_t *zeros, size_t bytes, int e) {
        return __ldg(&reinterpret_cast<const TiledTrailer *>(zeros + (size_t)(e + 1) * bytes - kTrailerBytes)->flags);
    };
    if ((int)threadIdx.x < segments) {
        up_flags = trailer_flags(a.gu_z, a.gu_z_bytes, plan.seg_expert[threadIdx.x]);
        down_flags = trailer_flags(a.dn_z, a.dn_z_bytes, plan.seg_expert[threadIdx.x]);
    }
    // weights never depend on the kernel before this one, h does
    if (n > 0) {
        l_seg = j0 / G;
        l_item = j0 - l_seg * G;
        enter_segment();
        load_weights(0);
    }
    pdl_wait();
    if (n > 0) {
        load_item_rows<NT, NU, SUB>(regs[0], rows, l_item);
        next();
#pragma unroll
        for (int d = 1; d < D; ++d)
            if (d < n) {
                load_weights(d);
                load_item_rows<NT, NU, SUB>(regs[d], rows, l_item);
                next();
            }
    }
    float acc[NU][NT][4] = {};
    for (int i = 0; i < n; i += D)
#pragma unroll
        for (int d = 0; d < D; ++d)
            if (i + d < n) {
                const int seg = seg_of[d];
                const bool flush = item_of[d] == G - 1 || i + d == n - 1;
                multiply_item<NT, NU, SUB, BF>(regs[d], flags[d] & kFormatZerosMinusOne, acc);
                if (i + d + D < n) {
                    load_weights(d);
                    load_item_rows<NT, NU, SUB>(regs[d], rows, l_item);
                    next();
                }
                if (flush) {
                    const int first = plan.seg_begin[seg], count = plan.seg_begin[seg + 1] - first;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int odd = 0; odd < 2; ++odd) {
                            const int r = 8 * t + 2 * t4 + odd;
                            if (r < count) {
                                const int s = plan.slot[first + r];
                                const float w = plan.weight[s];
                                float *cell = mine + (s / a.k) * kDownCols + g;
#pragma unroll
                                for (int u = 0; u < NU; ++u) {
                                    cell[16 * u] = fmaf(w, acc[u][t][odd], cell[16 * u]);
                                    cell[16 * u + 8] = fmaf(w, acc[u][t][2 + odd], cell[16 * u + 8]);
                                }
                            }
                        }
#pragma unroll
                    for (int u = 0; u < NU; ++u)
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int v = 0; v < 4; ++v) acc[u][t][v] = 0.f;
                    __syncwarp();
                }
            }
    auto fits = [](uint32_t up, uint32_t down) {
        return (up & (kFormatGateUp | kFormatBf16)) == (kFormatGateUp | (BF ? kFormatBf16 : 0u)) &&
               (down & (kFormatGateUp | kFormatBf16)) == (BF ? kFormatBf16 : 0u);
    };
    bool bad = !fits(up_flags, down_flags);
    for (int i = threadIdx.x + kMoeThreads; i < segments; i += kMoeThreads) {
        const int e = plan.seg_expert[i];
        bad |= !fits(trailer_flags(a.gu_z, a.gu_z_bytes, e), trailer_flags(a.dn_z, a.dn_z_bytes, e));
    }
    if (bad) {
        s_bad = 1;
        atomicMax(&g_device_status, (int)kStatusLayoutMismatch);
    }
    __syncthreads();
    const bool ok = s_bad == 0;
    for (int o = threadIdx.x; o < cells; o += kMoeThreads) {
        float v = tiles[o];
#pragma unroll
        for (int w = 1; w < kMoeWarps; ++w) v += tiles[w * cells + o];
        tiles[o] = v;
    }
    auto store = [&](int o, float v) {
        const size_t at = (size_t)(o / kDownCols) * a.K + panel * kPanel + 16 * unit + o % kDownCols;
        if (a.residual) v += out16_to_float<BF>(a.residual[at]);
        store_out16<BF>(a.y + at, v);
    };
    if (S == 1) {
        // (a cell is stored by the thread that summed it)
        if (ok)
            for (int o = threadIdx.x; o < cells; o += kMoeThreads) store(o, tiles[o]);
        return;
    }
    __syncthreads();
    cluster_arrive_release();
    cluster_wait_acquire();
    if (ok) {
        const uint32_t base = smem_u32(tiles);
        for (int o = cells * rank / S + threadIdx.x; o < cells * (rank + 1) / S; o += kMoeThreads) {
            float v = 0.f;
            for (int q = 0; q < S; ++q) {
                float part;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part) : "r"(map_to_cluster_rank(base + 4u * o, (uint32_t)q)) : "memory");
                v += part;
            }
            store(o, v);
        }
    }
    cluster_arrive_release();      // no CTA may leave while its tile is being read
    cluster_wait_acquire();
}

// x_out[s][i] = x[s / k][perm[e][i]], e = ids[s]: each slot's row of x in its expert's sorted order (act-order checkpoints)
__global__ void moe_gather_kernel(const __half *__restrict__ x, const int32_t *__restrict__ ids, const int32_t *__restrict__ perm,
                                  __half *__restrict__ x_out, int P, int k, int E, int K)
{
    pdl_wait();
    pdl_launch_dependents();
    const int i = 4 * (blockIdx.x * blockDim.x + threadIdx.x), s = blockIdx.y;
    if (i >= K) return;
    const int e = __ldg(ids + s);
    if ((unsigned)e >= (unsigned)E) return;
    const int4 c = __ldg(reinterpret_cast<const int4 *>(perm + (size_t)e * K + i));
    const __half *row = x + (size_t)(s / k) * K;
    const __half2 lo = __halves2half2(row[c.x], row[c.y]), hi = __halves2half2(row[c.z], row[c.w]);
    *reinterpret_cast<uint2 *>(x_out + (size_t)s * K + i) = make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
}

int launch_moe_gather(const __half *x, const int32_t *ids, const int32_t *perm, __half *x_out, int P, int k, int E, int K, cudaStream_t s)
{
    return launch_dependent(moe_gather_kernel, dim3((unsigned)((K / 4 + 255) / 256), (unsigned)P), 256, 0, 1, s, x, ids, perm, x_out, P, k, E, K);
}

inline size_t moe_h_bytes(int P, int F) { return ((size_t)P * F * 2 + 255) & ~(size_t)255; }
inline size_t moe_workspace_need(int M, int K, int F, int k, int act_order)
{
    const int P = (M < kMoeMaxRows ? M : kMoeMaxRows) * k;
    return moe_h_bytes(P, F) + (act_order ? (((size_t)P * K * 2 + 255) & ~(size_t)255) : 0);
}

template <int NT, int SUB, bool BF>
static int launch_moe_nt(const MoeArgs &a, int sms, cudaStream_t s)
{
    const int P = a.M * a.k, R = 8 * NT, plan = slot_plan_bytes(P, a.E), slots = 2 * sms;      // two CTAs per SM
    const int experts = a.E < P ? a.E : P;
    const int most = experts + P / R < P ? experts + P / R : P;      // segments: one per expert in use, one more per R slots
    static int configured_up[64] = {}, configured_down[64] = {};
    const int up_smem = plan + 2 * kMoeWarps * 8 * NT * 32 * 4, down_smem = plan + kMoeWarps * a.M * kDownCols * 4;
    int st = ensure_dynamic_smem((const void *)moe_gate_up_kernel<NT, SUB, BF>, configured_up, up_smem);
    if (!st) st = ensure_dynamic_smem((const void *)moe_down_kernel<NT, SUB, BF>, configured_down, down_smem);
    if (st) return st;
    const long long tiles = (long long)most * (a.F / 16);
    st = launch_dependent(moe_gate_up_kernel<NT, SUB, BF>, dim3((unsigned)(tiles < slots ? tiles : slots)), kMoeThreads, (size_t)up_smem, 1, s, a);
    if (st) return st;
    const int down_tiles = a.K / kDownCols;
    int S = 1;
    while (S < 8 && down_tiles * S * 2 <= slots) S *= 2;
    return launch_dependent(moe_down_kernel<NT, SUB, BF>, dim3((unsigned)(down_tiles * S)), kMoeThreads, (size_t)down_smem, S, s, a, S);
}
template <int SUB, bool BF>
static int launch_moe_sub(const MoeArgs &a, int sms, cudaStream_t s)
{
    const char *nt = getenv("MOE_NT");
    const int v = nt ? atoi(nt) : 1;
    if (a.M <= 8 || v == 1) return launch_moe_nt<1, SUB, BF>(a, sms, s);
    return launch_moe_nt<2, SUB, BF>(a, sms, s);
}
int launch_moe(const MoeArgs &a, int group_size, int bf16, int sms, cudaStream_t s)
{
    switch ((bf16 ? 10 : 0) + kGroup / group_size) {
    case 1: return launch_moe_sub<1, false>(a, sms, s);
    case 2: return launch_moe_sub<2, false>(a, sms, s);
    case 4: return launch_moe_sub<4, false>(a, sms, s);
    case 11: return launch_moe_sub<1, true>(a, sms, s);
    case 12: return launch_moe_sub<2, true>(a, sms, s);
    default: return launch_moe_sub<4, true>(a, sms, s);
    }
}

}  // namespace gptq

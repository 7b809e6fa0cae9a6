// Routed experts: the choice of experts for each token, and a whole mixture-of-experts MLP for a few tokens in two kernels.
#pragma once
#include "gptq_common.cuh"
#include "gptq_direct.cuh"
#include "gptq_splitk.cuh"   // silu_mul, cluster barriers, map_to_cluster_rank

namespace gptq {

// ------------------------------------------------------------------------------ routing
// One warp per token; lane l holds the logits of experts l, l + 32, ... as keys whose unsigned order is the order of the
// logits (0: an expert that cannot be chosen).  A pick is two warp-wide reductions: the largest key, then the lowest expert
// that has it.  The weights are exp(l - max) over their sum, or over the sum of all experts, in fp32, to some steps of 2^-24 (a lane forms the
// exponential of its own pick, behind the picks).
// Bound by the chain of 2 k reductions: 4096 tokens, 128 experts in bfloat16, top 8: 4.0 us, 0.2 would be its memory's.
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
// exp(l - top) to a few steps of 2^-24 for every l: of x = l - top and of t = x log2(e) the fast exponential takes only the rounded values, whose
// errors grow with x (100 steps at l = top - 80).  Both errors are known exactly - x's by the two-term sum of two floats, t's by an
// fma and the rest of log2(e) - and enter as the factor 2^r = 1 + r ln 2.
__device__ __forceinline__ float exp_below(float l, float top)
{
    constexpr float kLog2e = 1.44269504f, kLog2eRest = 1.92596299e-8f, kLn2 = 0.693147181f;
    const float x = __fsub_rn(l, top), back = __fadd_rn(x, top);
    const float x_rest = __fsub_rn(__fsub_rn(l, back), __fsub_rn(top, __fsub_rn(back, x)));
    const float t = __fmul_rn(x, kLog2e), r = __fmaf_rn(x_rest, kLog2e, __fmaf_rn(x, kLog2eRest, __fmaf_rn(x, kLog2e, -t)));
    float p;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p) : "f"(t));
    return t > -126.f ? __fmaf_rn(p, r * kLn2, p) : p;
}

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
                    if (key[i]) sum += exp_below(key_logit(key[i]), top);
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
        if (lane == j) { mine = key_logit(all); my_id = (int)e; }
    }
    // a lane's pick: its exponential, and the picks' sum
    const float p = my_id >= 0 ? exp_below(mine, top) : 0.f;
    if (renormalize) {
        total = p;
#pragma unroll
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    }
    if (lane < k) {
        ids[(size_t)m * k + lane] = my_id;
        weights[(size_t)m * k + lane] = my_id >= 0 ? p / total : 0.f;
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
constexpr int kMoeSegRows = 8;                   // rows of a segment (see SlotPlan): the columns of an MMA
constexpr int kMoeWarps = 8, kMoeThreads = 32 * kMoeWarps;
constexpr int kMoeCtasPerSm = 2;
constexpr int kMoeMaxExperts = 1024, kMoeMaxTopK = 32;

struct MoeArgs {
    const __half *x;          // [M, K]; with act-order [M k, K], each slot's row in its expert's order
    const int32_t *ids;       // [M, k]
    const float *weights;     // [M, k]
    const uint8_t *gu_w, *gu_z, *gu_s, *dn_w, *dn_z, *dn_s;
    size_t gu_w_bytes, gu_z_bytes, gu_s_bytes, dn_w_bytes, dn_z_bytes, dn_s_bytes;    // of one expert
    const int32_t *down_index;      // [E, F] or nullptr
    __half *h;                // [parts][M k, F], columns as direct_column has them
    const __half *residual;   // [M, K] or nullptr
    __half *y;                // [M, K]
    int M, k, E, K, F;
    int sms;
    uint32_t one;             // 1 (see prepare_rows)
    int x_by_slot;            // rows of x: slots instead of tokens
    int parts;                // of h: rounded to 16 bits, and with 2 what that left, rounded too (see moe_parts)
    unsigned long long call;  // of a call of several passes: its number, else 0 (see moe_check_kernel)
};

// whether the layers of an expert, by their trailers' flags, are the ones that the kernels are for
template <bool BF>
__device__ __forceinline__ bool moe_layers_fit(uint32_t up, uint32_t down)
{
    return (up & (kFormatGateUp | kFormatBf16)) == (kFormatGateUp | (BF ? kFormatBf16 : 0u)) &&
           (down & (kFormatGateUp | kFormatBf16)) == (BF ? kFormatBf16 : 0u);
}
__device__ __forceinline__ uint32_t trailer_flags(const uint8_t *zeros, size_t bytes, int e)
{
    return __ldg(&reinterpret_cast<const TiledTrailer *>(zeros + (size_t)(e + 1) * bytes - kTrailerBytes)->flags);
}

// A call of several passes is refused as a whole: one block goes over the experts that any of its tokens names before the first pass.  Numbers
// of refused calls stand in a table until the call runs again (a graph's replay) and fits; a call finds its own number or nothing.
// (Two refused calls under way at once whose numbers are kRefusedCalls apart: the one loses its entry, and is refused pass by pass.)
constexpr int kRefusedCalls = 256, kMoeCheckThreads = 1024;
static_assert(kMoeMaxExperts <= kMoeCheckThreads, "a thread per expert");
__device__ unsigned long long g_refused_calls[kRefusedCalls];
template <bool BF>
__global__ void __launch_bounds__(kMoeCheckThreads) moe_check_kernel(const MoeArgs a, long long slots)
{
    __shared__ uint32_t named[kMoeCheckThreads / 32];
    if (threadIdx.x < kMoeCheckThreads / 32) named[threadIdx.x] = 0;
    pdl_wait();
    pdl_launch_dependents();
    __syncthreads();
    auto name = [&](int e) {
        if ((unsigned)e < (unsigned)a.E && !(*(volatile uint32_t *)&named[e >> 5] >> (e & 31) & 1)) atomicOr(&named[e >> 5], 1u << (e & 31));
    };
    for (long long s = 4 * threadIdx.x; s < slots; s += 4 * kMoeCheckThreads) {
        if (s + 4 <= slots) {
            const int4 e = __ldg(reinterpret_cast<const int4 *>(a.ids + s));
            name(e.x), name(e.y), name(e.z), name(e.w);
        } else
            for (long long i = s; i < slots; ++i) name(__ldg(a.ids + i));
    }
    __syncthreads();
    const int e = threadIdx.x;
    const bool bad = e < a.E && (named[e >> 5] >> (e & 31) & 1) &&
                     !moe_layers_fit<BF>(trailer_flags(a.gu_z, a.gu_z_bytes, e), trailer_flags(a.dn_z, a.dn_z_bytes, e));
    if (bad) atomicMax(&g_device_status, (int)kStatusLayoutMismatch);
    const bool refused = __syncthreads_or(bad);
    unsigned long long *entry = &g_refused_calls[a.call % kRefusedCalls];
    if (threadIdx.x == 0) {
        if (refused) *entry = a.call;
        else if (*entry == a.call) *entry = 0;
    }
}

// The slots (m, j) of a batch grouped by expert, in the order of experts and, within one, of slots.  An expert's slots are cut
// into SEGMENTS of at most R, the rows that one sweep over the expert's weights serves.
struct SlotPlan {
    float *weight;       // [P] by slot: the weights that a token gives its expert, summed
    int *counts;         // [E] while it is built: slots, then the first one's position
    short *key;          // [P] by slot: its expert, -1 where the slot is not used
    short *slot;         // [P] slots by expert
    short *rank;         // [P] by slot, while it is built
    short *token;        // [P] by slot
    short *seg_begin;    // [segments + 1] into slot
    short *seg_expert;   // [segments]
};
__host__ __device__ constexpr int slot_plan_room(int P) { return (P + 8) & ~7; }      // of an array by slot or segment, more than P
__host__ __device__ constexpr int slot_plan_bytes(int P, int E) { return 14 * slot_plan_room(P) + ((4 * E + 15) & ~15); }
__device__ __forceinline__ SlotPlan slot_plan_view(uint8_t *smem, int P, int E)
{
    const int room = slot_plan_room(P);
    SlotPlan p;
    p.key = reinterpret_cast<short *>(smem);
    p.slot = p.key + room;
    p.rank = p.slot + room;
    p.token = p.rank;      // (once the ranks are done with)
    p.seg_begin = p.rank + room;
    p.seg_expert = p.seg_begin + room;
    p.weight = reinterpret_cast<float *>(p.seg_expert + room);
    p.counts = reinterpret_cast<int *>(p.weight + room);
    return p;
}

// By all threads of a block; returns the number of segments.  A slot whose expert a lower slot of the same token names already
// adds its weight there.  `seg_expert` holds the raw ids until the segments are known.
constexpr int kSlotTableEntries = 4096;      // (8 KB of the room for sums and ring, not in use yet)
__device__ __forceinline__ int build_slot_plan(const MoeArgs &a, int R, const SlotPlan &p, unsigned short *table)
{
    __shared__ int s_segments;
    const int P = a.M * a.k, tid = threadIdx.x, lane = tid & 31;
    if (P <= 32) {      // a slot per lane of one warp, experts in the order of their first slots
        if (tid < 32) {
            const int j = lane % a.k, id = lane < P ? __ldg(a.ids + lane) : -1;
            float w = lane < P ? __ldg(a.weights + lane) : 0.f;
            const bool named = (unsigned)id < (unsigned)a.E;
            uint32_t same = __match_any_sync(0xffffffffu, named ? id : -1);
            const uint32_t own = (a.k < 32 ? (1u << a.k) - 1 : 0xffffffffu) << (lane - j), before = (1u << lane) - 1;
            const bool used = named && !(same & own & before);
            if (__any_sync(0xffffffffu, named && !used)) {
                const uint32_t more = used ? same & own : 0u;      // (this lane and later ones: the weights in the order of slots)
                float sum = w;
                for (int l = 0; l < 32; ++l) {
                    const float v = __shfl_sync(0xffffffffu, w, l);
                    if (l > lane && (more >> l & 1)) sum += v;
                }
                w = sum;
            }
            same &= __ballot_sync(0xffffffffu, used);
            const int rank = __popc(same & before), c = __popc(same);
            const bool leads = used && rank == 0;
            int sum = leads ? c | (c + R - 1) / R << 16 : 0;
            const int mine = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += v;
            }
            const int total = __shfl_sync(0xffffffffu, sum, 31);
            const int at = __shfl_sync(0xffffffffu, sum - mine, used ? __ffs(same) - 1 : 0);
            if (lane < P) {
                p.weight[lane] = w;
                p.key[lane] = used ? (short)id : (short)-1;
                p.token[lane] = (short)(lane / a.k);
            }
            if (used) {
                p.slot[(at & 0xffff) + rank] = (short)lane;
                if (rank % R == 0) {
                    const int seg = (at >> 16) + rank / R;
                    p.seg_expert[seg] = (short)id;
                    p.seg_begin[seg] = (short)((at & 0xffff) + rank);
                }
            }
            if (lane == 0) {
                p.seg_begin[total >> 16] = (short)(total & 0xffff);
                s_segments = total >> 16;
            }
        }
        __syncthreads();
        return s_segments;
    }
    // Otherwise the slots are taken 32 at a time: what a slot finds of its expert in its own 32, and how many there are in those before.
    // The counts per 32 slots and expert stand in `table`, or, where that is too small, one warp takes the 32s in turn.
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
    const int chunks = (P + 31) / 32;
    if (chunks * a.E <= kSlotTableEntries) {
        __shared__ int s_sums[kMoeThreads / 32];
        for (int i = tid; i < chunks * a.E; i += kMoeThreads) table[i] = 0;
        __syncthreads();
        const int warp = tid >> 5;
        for (int c = warp; c < chunks; c += kMoeThreads / 32) {
            const int s = 32 * c + lane, e = s < P ? p.key[s] : -1;
            const uint32_t same = __match_any_sync(0xffffffffu, e);
            const int before = __popc(same & ((1u << lane) - 1));
            if (e >= 0) {
                p.rank[s] = (short)before;
                if (before == 0) table[c * a.E + e] = (unsigned short)__popc(same);
            }
        }
        __syncthreads();
        // a thread per expert (of neighbouring ones, where there are more): the 32s' counts become positions behind its first slot
        const int per = (a.E + kMoeThreads - 1) / kMoeThreads, e0 = min(tid * per, a.E), e1 = min(e0 + per, a.E);
        int sum = 0;
        for (int e = e0; e < e1; ++e) {
            int n = 0;
            for (int c = 0; c < chunks; ++c) {
                const int here = table[c * a.E + e];
                table[c * a.E + e] = (unsigned short)n;
                n += here;
            }
            p.counts[e] = n;
            sum += n | (n + R - 1) / R << 16;
        }
        const int mine = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) s_sums[warp] = sum;
        __syncthreads();
        int total = 0, at = sum - mine;
#pragma unroll
        for (int w = 0; w < kMoeThreads / 32; ++w) {
            if (w < warp) at += s_sums[w];
            total += s_sums[w];
        }
        int pos = at & 0xffff, seg = at >> 16;
        for (int e = e0; e < e1; ++e) {
            const int n = p.counts[e];
            p.counts[e] = pos;
            for (int i = 0; i < n; i += R) {
                p.seg_expert[seg] = (short)e;
                p.seg_begin[seg++] = (short)(pos + i);
            }
            pos += n;
        }
        if (tid == 0) p.seg_begin[total >> 16] = (short)(total & 0xffff);
        __syncthreads();
        for (int s = tid; s < P; s += kMoeThreads) {
            const int e = p.key[s];
            if (e >= 0) p.slot[p.counts[e] + table[(s >> 5) * a.E + e] + p.rank[s]] = (short)s;
            p.token[s] = (short)(s / a.k);
        }
        __syncthreads();
        return total >> 16;
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
    for (int s = tid; s < P; s += kMoeThreads) {
        if (p.key[s] >= 0) p.slot[p.counts[p.key[s]] + p.rank[s]] = (short)s;
        p.token[s] = (short)(s / a.k);
    }
    __syncthreads();
    return s_segments;
}

// An activation's parts.  With two, 16 bits and the 16 of what they leave, y's rounding is the only one that counts: h is good to 2^-22
// (bfloat16 2^-16).  In fp16 the second part is kept times 2^11, as large as h at most, so that a small h (down to 2^-14; below, to 2^-36)
// loses nothing to the subnormal numbers; the down kernel takes the power out of its sums.  An infinity leaves nothing.
template <bool BF>
__host__ __device__ constexpr float second_part_scale() { return BF ? 1.f : 2048.f; }
template <bool BF>
__device__ __forceinline__ void store_h(const MoeArgs &a, __half *at, float v)
{
    store_out16<BF>(at, v);
    if (a.parts == 1) return;
    const float left = (v - out16_to_float<BF>(*at)) * second_part_scale<BF>();
    store_out16<BF>(at + (size_t)a.M * a.k * a.F, isfinite(left) ? left : 0.f);
}

// Kernel 1: h[slot] = silu(gate) * up.  The work is counted in units of a segment and 16 gate columns (with their 16 up columns); a
// CTA takes a range of neighbouring units, in tiles of two where they are a pair of the panel, else of one.  The warps share a
// tile's items along K; at its end each leaves its sums in shared memory, goes on with the next tile, and adds up its part of them at
// the next tile's end, when all have long arrived.
//
// Bound by instruction issue: 64 rows, 32 experts of 4096 x 2048, top 4: 2.4 instructions per clock and SM at 51 % of the DRAM rate and
// 34 % of the tensor pipe's.  Two CTAs of 8 warps per SM with rings; the whole layer of 64 rows takes 156 us (65 would be its memory's),
// 167 with one CTA of 16 warps per SM.
template <int NU, int SUB, bool BF>
__global__ void __launch_bounds__(kMoeThreads, kMoeCtasPerSm) moe_gate_up_kernel(const MoeArgs a)
{
    extern __shared__ __align__(16) uint8_t smem[];
    constexpr int kValues = 4 * NU;
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const SlotPlan plan = slot_plan_view(smem, a.M * a.k, a.E);
    float *red = reinterpret_cast<float *>(smem + slot_plan_bytes(a.M * a.k, a.E));
    __shared__ __align__(8) uint64_t arrived[2];
    const uint32_t bars = smem_u32(arrived);
    if (threadIdx.x == 0) {
        mbar_init(bars, kMoeWarps);
        mbar_init(bars + 8, kMoeWarps);
    }
    pdl_wait();
    pdl_launch_dependents();
    const int segments = build_slot_plan(a, kMoeSegRows, plan, reinterpret_cast<unsigned short *>(red));
    const int G = a.K / kGroup, per_seg = a.F / 16, T = segments * per_seg;
    // the CTAs of an SM (which they are given out to in turn) take neighbouring ranges: the same rows of x
    int cta = blockIdx.x;
    if (gridDim.x % a.sms == 0) cta = cta % a.sms * (gridDim.x / a.sms) + cta / a.sms;
    const int t0 = share_begin(T, gridDim.x, cta), t1 = share_begin(T, gridDim.x, cta + 1);
    auto width = [&](int unit) { return NU == 4 && (unit & 1) == 0 && unit + 1 < t1 ? 2 : 1; };      // (per_seg is even)

    // ---- what comes next: the tile at unit l_unit, item l_item; a warp starts at another item in every tile, so that all get their
    // share where the items are no multiple of the warps
    int l_unit = t0, l_next = t0, l_item = G, l_seg = 0, l_col = 0, l_turn = warp - 1;
    uint32_t l_flags = 0;
    LanePtrs<SUB> ptrs{};
    const __half *row = nullptr;
    auto row_of = [&](int s) { return a.x + (size_t)(a.x_by_slot ? s : plan.token[s]) * a.K; };
    auto up_flags = [&](int e) { return trailer_flags(a.gu_z, a.gu_z_bytes, e); };
    auto next = [&](DirectItem<SUB> &it) {
        l_item += kMoeWarps;
        while (l_item >= G) {
            if (l_next >= t1) {
                it.tag = -1;
                return;
            }
            const bool start = l_next == t0;
            l_col += l_next - l_unit;
            l_unit = l_next;
            l_next += width(l_unit);
            l_item = ++l_turn & (kMoeWarps - 1);
            if (start || l_col == per_seg) {
                l_seg = start ? l_unit / per_seg : l_seg + 1;
                l_col = start ? l_unit - l_seg * per_seg : 0;
                const int first = plan.seg_begin[l_seg], count = plan.seg_begin[l_seg + 1] - first;
                row = row_of(plan.slot[first + (g < count ? g : 0)]) + 8 * t4;
                l_flags = up_flags(plan.seg_expert[l_seg]);
            }
            const int e = plan.seg_expert[l_seg];
            ptrs = lane_ptrs<true, SUB>(unit_ptrs<SUB>(a.gu_w + e * a.gu_w_bytes, a.gu_s + e * a.gu_s_bytes, a.gu_z + e * a.gu_z_bytes, l_col >> 2, G, l_col & 3), lane);
        }
        set_item<SUB>(it, ptrs, row, l_item, lane);
        it.flags = l_flags;
        it.tag = l_unit;
        it.pairs = l_next - l_unit;
    };

    // ---- the end of a tile
    float acc[NU][4] = {};
    // the tile at hand, the one before it (its segment and column), how many came before
    int unit = t0, seg_at = t0 / per_seg, col_at = t0 - seg_at * per_seg, left = t0, left_seg = 0, left_col = 0, tiles = 0;
    bool again = false;
    auto add_up = [&]() {      // the sums of the tile at `left` over the warps, in their order
        const int done = tiles - 1;
        if (!mbar_wait(bars + 8 * (done & 1), (done >> 1) & 1)) return;
        const int seg = left_seg, c0 = left_col * 16;
        const int first = plan.seg_begin[seg], count = plan.seg_begin[seg + 1] - first;
        const float *buf = red + (done & 1) * (kMoeWarps * kValues * 32);
        for (int o = threadIdx.x; o < width(left) * 128; o += kMoeThreads) {
            const int v = o >> 5, p = v >> 2, i = v & 3;            // (lane of o = lane: the block is a multiple of a warp)
            const int r = 2 * t4 + (i & 1), at = (8 * p + i) * 32 + lane;
            if (r >= count) continue;
            float gate = 0.f, up = 0.f;
#pragma unroll
            for (int w = 0; w < kMoeWarps; ++w) {
                gate += buf[w * (kValues * 32) + at];
                up += buf[w * (kValues * 32) + 128 + at];
            }
            again |= needs_long_sum<BF>(gate) || needs_long_sum<BF>(up);
            int col = c0 + 16 * p + g + 8 * (i >> 1);
            if (a.down_index) col = __ldg(a.down_index + (size_t)plan.seg_expert[seg] * a.F + col);
            store_h<BF>(a, a.h + (size_t)plan.slot[first + r] * a.F + direct_column<BF>(col), silu_mul(gate, up));
        }
    };
    auto finish_tile = [&]() {
        // (no warp still reads this buffer: all have left their sums of the tile before this one, after adding up the one before that)
        if (tiles) add_up();
        float *buf = red + (tiles & 1) * (kMoeWarps * kValues * 32);      // [warp][value][lane]
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                buf[(warp * kValues + 4 * u + i) * 32 + lane] = acc[u][i];
                acc[u][i] = 0.f;
            }
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * (tiles & 1));
        left = unit, left_seg = seg_at, left_col = col_at;
        unit += width(unit);
        col_at += unit - left;
        if (col_at == per_seg) col_at = 0, ++seg_at;
        ++tiles;
    };
    const uint32_t ring = smem_u32(red + 2 * kMoeWarps * kValues * 32) + warp * direct_ring_bytes<NU, SUB>(1);
    stream_items<NU, true, SUB, BF, false>(ring, lane, a.one, acc, next, [] {}, [&](int t) { while (unit < t) finish_tile(); });
    while (unit < t1) finish_tile();
    if (tiles) add_up();
    if (!again) return;
    // a thread goes over its outputs again and forms those that are not finite, as h is where gate or up was not, the long way
    for (unit = t0; unit < t1; unit += width(unit)) {
        const int seg = unit / per_seg, c0 = (unit - seg * per_seg) * 16, e = plan.seg_expert[seg];
        const int first = plan.seg_begin[seg], count = plan.seg_begin[seg + 1] - first;
        const uint8_t *zeros = a.gu_z + e * a.gu_z_bytes;
        const uint32_t z_add = up_flags(e) & kFormatZerosMinusOne;
        for (int o = threadIdx.x; o < width(unit) * 128; o += kMoeThreads) {
            const int v = o >> 5, r = 2 * t4 + (v & 1), c = g + 8 * ((v >> 1) & 1);
            if (r >= count) continue;
            const int s = plan.slot[first + r], col = c0 + 16 * (v >> 2) + c;
            __half *at = a.h + (size_t)s * a.F + direct_column<BF>(a.down_index ? __ldg(a.down_index + (size_t)e * a.F + col) : col);
            const float now = out16_to_float<BF>(*at);
            if (isfinite(now)) continue;
            float sum[2];
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                const UnitPtrs p = unit_ptrs<SUB>(a.gu_w + e * a.gu_w_bytes, a.gu_s + e * a.gu_s_bytes, zeros, col / 64, G, col % 64 / 16 + 4 * half);
                sum[half] = long_sum<BF>(p.w, p.s, p.z, SUB, c, z_add, row_of(s), G, false);
            }
            store_h<BF>(a, at, silu_mul(sum[0], sum[1]));
        }
    }
}

// Kernel 2: y = residual + sum over a token's experts of weight * (h Wd).  A cluster of S CTAs takes 16 NU columns of y; the items
// of all segments, one behind the other, are shared out evenly over its CTAs.  A CTA's part of a segment is what a tile is in
// kernel 1; what its warps leave of it is added up, weighted, in a [token][column] tile in shared memory, part after part, and
// the CTAs' tiles in the order of ranks: the order of all sums is fixed.
// Clusters, because a few tokens leave too few columns for the machine: as many CTAs as fill two per SM, up to 8 to a cluster.  One row,
// 8 experts of 4096 x 11008, top 2: both kernels 40 us, 22 would be their memory's.
template <int NU, int SUB, bool BF>
__global__ void __launch_bounds__(kMoeThreads, kMoeCtasPerSm) moe_down_kernel(const MoeArgs a, int S)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int s_bad;
    __shared__ __align__(8) uint64_t arrived[2];
    constexpr int kCols = 16 * NU, kValues = 4 * NU;
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const int tile = blockIdx.x / S, rank = blockIdx.x - tile * S;
    const int G = a.F / kGroup, panel = tile / (8 / NU), unit = tile % (8 / NU) * NU;
    const uint32_t bars = smem_u32(arrived);
    pdl_launch_dependents();
    const SlotPlan plan = slot_plan_view(smem, a.M * a.k, a.E);
    const int cells = a.M * kCols;
    float *ysum = reinterpret_cast<float *>(smem + slot_plan_bytes(a.M * a.k, a.E));      // [token][column]
    float *recv = ysum + cells;                              // with S > 1: [rank][cell of this CTA's share]
    float *red = recv + (S > 1 ? cells : 0);
    for (int i = threadIdx.x; i < cells; i += kMoeThreads) ysum[i] = 0.f;
    if (threadIdx.x == 0) {
        s_bad = 0;
        mbar_init(bars, kMoeWarps);
        mbar_init(bars + 8, kMoeWarps);
    }
    // ids and weights are older than the kernel before this one, which waited for them before it let this one in
    // with h in two parts a segment is 4 slots: their first parts are columns 0 .. 3 of an MMA, the second ones 4 .. 7
    const int R = kMoeSegRows / a.parts;
    const int segments = build_slot_plan(a, R, plan, reinterpret_cast<unsigned short *>(red));
    if (S > 1) cluster_arrive_release();      // "this CTA has begun": waited for before anything is sent
    const int U = segments * G, u0 = share_begin(U, S, rank), u1 = share_begin(U, S, rank + 1);
    const int seg0 = u0 / G, parts = u1 > u0 ? (u1 - 1) / G - seg0 + 1 : 0;

    // ---- what comes next: part l_part (segment seg0 + l_part), item l_item
    int l_part = -1, l_item = G, l_end = 0;
    uint32_t l_flags = 0;
    LanePtrs<SUB> ptrs{};
    const __half *row = nullptr;
    auto next = [&](DirectItem<SUB> &it) {
        l_item += kMoeWarps;
        while (l_item >= l_end) {
            if (++l_part >= parts) {
                l_end = -1;
                it.tag = -1;
                return;
            }
            const int seg = seg0 + l_part, e = plan.seg_expert[seg], first = plan.seg_begin[seg], count = plan.seg_begin[seg + 1] - first;
            l_item = max(u0 - seg * G, 0) + ((warp + l_part) & (kMoeWarps - 1));
            l_end = min(u1 - seg * G, G);
            l_flags = trailer_flags(a.dn_z, a.dn_z_bytes, e);
            ptrs = lane_ptrs<false, SUB>(unit_ptrs<SUB>(a.dn_w + e * a.dn_w_bytes, a.dn_s + e * a.dn_s_bytes, a.dn_z + e * a.dn_z_bytes, panel, G, unit), lane);
            const int r = g & (R - 1);
            row = a.h + ((size_t)(g >= R ? a.M * a.k : 0) + plan.slot[first + (r < count ? r : 0)]) * a.F + 8 * t4;
        }
        set_item<SUB>(it, ptrs, row, l_item, lane);
        it.flags = l_flags;
        it.tag = l_part;
        it.pairs = NU / 2;
    };
    // A layer of the wrong format anywhere: nothing is stored.  Every CTA looks at all experts in use, so that they agree; the
    // trailers are asked for here and looked at behind the main loop.
    uint32_t up_flags = kFormatGateUp | (BF ? kFormatBf16 : 0u), down_flags = BF ? kFormatBf16 : 0u;
    if ((int)threadIdx.x < segments) {
        up_flags = trailer_flags(a.gu_z, a.gu_z_bytes, plan.seg_expert[threadIdx.x]);
        down_flags = trailer_flags(a.dn_z, a.dn_z_bytes, plan.seg_expert[threadIdx.x]);
    }

    // ---- the end of a part (see kernel 1)
    float acc[NU][4] = {};
    int now = 0;
    auto add_up = [&](int done) {
        if (!mbar_wait(bars + 8 * (done & 1), (done >> 1) & 1)) return;
        const int first = plan.seg_begin[seg0 + done], count = plan.seg_begin[seg0 + done + 1] - first;
        const float *buf = red + (done & 1) * (kMoeWarps * kValues * 32);
#pragma unroll
        for (int o = threadIdx.x; o < kValues * 32; o += kMoeThreads) {
            const int v = o >> 5, u = v >> 2, i = v & 3;
            const int r = 2 * t4 + (i & 1);
            if (r >= count) continue;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < kMoeWarps; ++w) sum += buf[(w * kValues + v) * 32 + lane];
            if (a.parts == 2) {      // column r + 4
                float second = 0.f;
#pragma unroll
                for (int w = 0; w < kMoeWarps; ++w) second += buf[(w * kValues + v) * 32 + lane + 2];
                sum = fmaf(second, 1.f / second_part_scale<BF>(), sum);
            }
            const int s = plan.slot[first + r];
            float *cell = ysum + plan.token[s] * kCols + 16 * u + g + 8 * (i >> 1);
            *cell = fmaf(plan.weight[s], sum, *cell);
        }
    };
    auto finish_part = [&]() {
        if (now) add_up(now - 1);
        float *buf = red + (now & 1) * (kMoeWarps * kValues * 32);      // [warp][value][lane]
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                buf[(warp * kValues + 4 * u + i) * 32 + lane] = acc[u][i];
                acc[u][i] = 0.f;
            }
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * (now & 1));
        ++now;
    };
    const uint32_t ring = smem_u32(red + 2 * kMoeWarps * kValues * 32) + warp * direct_ring_bytes<NU, SUB>(1);
    stream_items<NU, false, SUB, BF, true>(ring, lane, a.one, acc, next, [] { pdl_wait(); }, [&](int p) { while (now < p) finish_part(); });
    while (now < parts) finish_part();
    if (parts) add_up(parts - 1);

    bool bad = !moe_layers_fit<BF>(up_flags, down_flags);
    for (int i = threadIdx.x + kMoeThreads; i < segments; i += kMoeThreads) {
        const int e = plan.seg_expert[i];
        bad |= !moe_layers_fit<BF>(trailer_flags(a.gu_z, a.gu_z_bytes, e), trailer_flags(a.dn_z, a.dn_z_bytes, e));
    }
    if (a.call && threadIdx.x == 0) bad |= *(volatile unsigned long long *)&g_refused_calls[a.call % kRefusedCalls] == a.call;
    if (bad) {
        s_bad = 1;
        atomicMax(&g_device_status, (int)kStatusLayoutMismatch);
    }
    __syncthreads();
    const bool ok = s_bad == 0;
    auto place = [&](int o) { return (size_t)(o / kCols) * a.K + panel * kPanel + 16 * unit + o % kCols; };
    auto store = [&](int o, float v, float residual) {
        const int m = o / kCols, c = o % kCols;
        if (needs_long_sum<BF>(v)) {
            v = 0.f;
#pragma unroll 1
            for (int s = m * a.k; s < (m + 1) * a.k; ++s) {
                const int e = plan.key[s];
                if (e < 0) continue;
                const UnitPtrs p = unit_ptrs<SUB>(a.dn_w + e * a.dn_w_bytes, a.dn_s + e * a.dn_s_bytes, a.dn_z + e * a.dn_z_bytes, panel, G, unit + c / 16);
                const uint32_t z_add = trailer_flags(a.dn_z, a.dn_z_bytes, e) & kFormatZerosMinusOne;
                const __half *h = a.h + (size_t)s * a.F;
                v = fmaf(plan.weight[s], long_sum<BF>(p.w, p.s, p.z, SUB, c % 16, z_add, h, G, true), v);
                // (h's second part: in fp16 an infinity brought us here, which has none that counts)
                if (BF && a.parts == 2) v = fmaf(plan.weight[s], long_sum<BF>(p.w, p.s, p.z, SUB, c % 16, z_add, h + (size_t)a.M * a.k * a.F, G, true), v);
            }
        }
        store_out16<BF>(a.y + place(o), v + residual);
    };
    if (S == 1) {
        if (ok)
            for (int o = threadIdx.x; o < cells; o += kMoeThreads) store(o, ysum[o], a.residual ? out16_to_float<BF>(a.residual[place(o)]) : 0.f);
        return;
    }
    // each CTA finishes a share of the cells: it gets all CTAs' sums of them
    const int share = cells / S, from = rank * share;
    cluster_wait_acquire();
    for (int q = 0; q < S; ++q) {
        const uint32_t to = map_to_cluster_rank(smem_u32(recv + rank * share), (uint32_t)q);
        for (int i = threadIdx.x; i < share; i += kMoeThreads)
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4u * i), "f"(ysum[q * share + i]) : "memory");
    }
    cluster_arrive_release();
    float residual = 0.f;
    if (a.residual && (int)threadIdx.x < share) residual = out16_to_float<BF>(a.residual[place(from + threadIdx.x)]);
    cluster_wait_acquire();      // (nothing reaches into another CTA behind this)
    if (ok)
        for (int i = threadIdx.x; i < share; i += kMoeThreads) {
            float v = 0.f;
            for (int q = 0; q < S; ++q) v += recv[q * share + i];
            if (a.residual && i >= kMoeThreads) residual = out16_to_float<BF>(a.residual[place(from + i)]);
            store(from + i, v, residual);
        }
}

// Bound by latency: one round trip for indexes, one for x.
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

int launch_moe_check(const MoeArgs &a, long long slots, int bf16, cudaStream_t s)
{
    return bf16 ? launch_dependent(moe_check_kernel<true>, dim3(1), kMoeCheckThreads, 0, 1, s, a, slots)
                : launch_dependent(moe_check_kernel<false>, dim3(1), kMoeCheckThreads, 0, 1, s, a, slots);
}
int launch_moe_gather(const __half *x, const int32_t *ids, const int32_t *perm, __half *x_out, int P, int k, int E, int K, cudaStream_t s)
{
    return launch_dependent(moe_gather_kernel, dim3((unsigned)((K / 4 + 255) / 256), (unsigned)P), 256, 0, 1, s, x, ids, perm, x_out, P, k, E, K);
}

// Parts of h for a pass of M tokens.  Rounding h and y to 16 bits gives 1.4 times the error of rounding y alone (one case of four tokens
// came to 1.5).  Where experts have up to four tokens the second part takes columns of the MMAs that would be idle; where they
// have more it costs another sweep over the down layer.  Layers of 32 x 4096 x 2048 top 4 / 64 x 2048 x 768 top 8 / 8 x 4096 x 11008
// top 2, one part -> two, us: 8 tokens 69.3 -> 69.7 / 44.2 -> 44.4 / 108 -> 109; 16 tokens 95.6 -> 98.6 / 52.5 -> 54.0 / 123 -> 135;
// 64 tokens 155 -> 198 / 83 -> 106 / 323 -> 422.
constexpr int kMoeTwoPartRows = 16;
inline int moe_parts(int M) { return M <= kMoeTwoPartRows ? 2 : 1; }
// room for any pass of a call of M tokens, and of one of fewer: who has registered for the largest call has enough
inline size_t moe_h_bytes(int M, int k, int F)
{
    const int two = 2 * (M < kMoeTwoPartRows ? M : kMoeTwoPartRows), one = M < kMoeMaxRows ? M : kMoeMaxRows;
    return ((size_t)(two > one ? two : one) * k * F * 2 + 255) & ~(size_t)255;
}
inline size_t moe_workspace_need(int M, int K, int F, int k, int act_order)
{
    const int P = (M < kMoeMaxRows ? M : kMoeMaxRows) * k;
    return moe_h_bytes(M, k, F) + (act_order ? (((size_t)P * K * 2 + 255) & ~(size_t)255) : 0);
}

constexpr int kHalfSmBytes = 227 * 1024 / 2 - 1024;      // of a CTA that shares its SM with another
template <int NU, int SUB>
static int moe_red_and_ring_bytes() { return 2 * kMoeWarps * 4 * NU * 32 * 4 + direct_ring_bytes<NU, SUB>(kMoeWarps); }

// (From about 1024 slots in a pass on - 64 tokens, top 16 - the slot plan leaves room for one CTA on an SM; the other half of the grid follows it.)
template <int NU, int SUB, bool BF>
static int launch_gate_up(const MoeArgs &a, int most, cudaStream_t s)
{
    static int configured[64] = {};
    const int smem = slot_plan_bytes(a.M * a.k, a.E) + moe_red_and_ring_bytes<NU, SUB>();
    const int st = ensure_dynamic_smem((const void *)moe_gate_up_kernel<NU, SUB, BF>, configured, smem);
    if (st) return st;
    const long long units = (long long)most * (a.F / 16), slots = kMoeCtasPerSm * a.sms;
    return launch_sharing_sm(moe_gate_up_kernel<NU, SUB, BF>, dim3((unsigned)(units < slots ? units : slots)), kMoeThreads, (size_t)smem, 1,
                             kMoeCtasPerSm, s, a);
}
template <int NU, int SUB>
static int moe_down_smem(const MoeArgs &a, int S)
{
    return slot_plan_bytes(a.M * a.k, a.E) + (S > 1 ? 2 : 1) * a.M * 16 * NU * 4 + moe_red_and_ring_bytes<NU, SUB>();
}
template <int NU>
static int moe_down_cluster(const MoeArgs &a)
{
    int S = 1;
    while (S < 8 && a.K / (16 * NU) * S * 2 <= kMoeCtasPerSm * a.sms) S *= 2;
    return S;
}
template <int NU, int SUB, bool BF>
static int launch_down(const MoeArgs &a, cudaStream_t s)
{
    static int configured[64] = {};
    const int tiles = a.K / (16 * NU), S = moe_down_cluster<NU>(a);
    int smem = moe_down_smem<NU, SUB>(a, S);
    // exactly as many CTAs per SM as it takes: with more room clusters pile up on some SMs and leave others empty
    const int per_sm = tiles * S <= a.sms ? 1 : kMoeCtasPerSm;
    const int pad = 227 * 1024 / (per_sm + 1) + 512;
    if (smem < pad) smem = pad;
    const int st = ensure_dynamic_smem((const void *)moe_down_kernel<NU, SUB, BF>, configured, smem);
    if (st) return st;
    return launch_sharing_sm(moe_down_kernel<NU, SUB, BF>, dim3((unsigned)(tiles * S)), kMoeThreads, (size_t)smem, S, per_sm, s, a, S);
}
template <int SUB, bool BF>
static int launch_moe_format(const MoeArgs &a, cudaStream_t s)
{
    const int P = a.M * a.k, R = kMoeSegRows, experts = a.E < P ? a.E : P;
    const int most = experts + P / R < P ? experts + P / R : P;      // segments: one per expert in use, one more per R slots
    constexpr int NU = SUB == 4 ? 2 : 4;
    const int st = launch_gate_up<NU, SUB, BF>(a, most, s);
    if (st) return st;
    // The down kernel: half the columns per cluster where that keeps two CTAs on an SM, where otherwise SMs were left without one (32 of
    // 1024 x 512 top 4: one token 16.7 -> 12.2 us, 16 tokens 35 -> 23), and where a CTA has an item per warp at most, so that the smaller
    // cluster counts for more than x read twice (60 of 2048 x 1408 top 4, one token: 15.8 -> 14.1, 64 of 2048 x 768 top 8: 16.1 -> 15.2).
    // With more to do four units are ahead (32 of 4096 x 2048 top 4, one token: 23.4 against 24.1, 16 tokens 99 against 106).
    const int S = moe_down_cluster<NU>(a);
    const bool narrow = a.K / (16 * NU) * S <= a.sms || (long long)most * (a.F / kGroup) <= (long long)kMoeWarps * S;
    if (NU == 2 || narrow || moe_down_smem<NU, SUB>(a, S) > kHalfSmBytes) return launch_down<2, SUB, BF>(a, s);
    return launch_down<NU, SUB, BF>(a, s);
}
int launch_moe(const MoeArgs &a, int group_size, int bf16, cudaStream_t s)
{
    switch ((bf16 ? 10 : 0) + kGroup / group_size) {
    case 1: return launch_moe_format<1, false>(a, s);
    case 2: return launch_moe_format<2, false>(a, s);
    case 4: return launch_moe_format<4, false>(a, s);
    case 11: return launch_moe_format<1, true>(a, s);
    case 12: return launch_moe_format<2, true>(a, s);
    default: return launch_moe_format<4, true>(a, s);
    }
}

}  // namespace gptq

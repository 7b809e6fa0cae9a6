// Products of e4m3 layers with few token rows (up to a few hundred): HBM-bound, weights on the MMA's rows.
//
// A CTA has 128 weight rows (gated kinds: 128 of gate and the same 128 of up), which are the MMA's rows and the lanes of tensor memory, a tile of
// up to TT token rows, the MMA's columns, and a part of K; S CTAs of a cluster share K.  TMA brings a block of K (16 KB of weights) per
// stage, one thread multiplies it into an accumulator of its own, the drain warps add that, times the scales, to sums in registers.  A
// column's scale comes from shared memory, where a warp of its own puts the products of both scales ahead of time.
// At the end the CTAs of a cluster hand each other the sums of the token rows that each finishes (rank r: r, r + S, ...); a warp
// finishes a whole row of 128 columns: it adds the parts in a fixed order, and has the maximum that e4m3 results need at hand.
// Measured (device, weights from memory): 1 row 4096 x 4096 6.2 us, 16 rows 4096 x 12288 12.0 (4.2 TB/s), 48 rows 13.9, 128 rows 17.0; gated 4096 x 11008 1 row 18.4
// (4.9 TB/s), 64 rows 23.6.  What bounds it: launch, first loads and the exchange (4 us), above 16 rows the drain warps (100 clocks per block of K and 190 per 16 columns).
// Nothing per weight passes through an execution unit: mma.sync has no e4m3 here (it is converted to fp16 first, 283 instructions per 2 KB of weights
// and warp; 1 row 4096 x 4096 7.4 us, gated 4096 x 11008 26).
#pragma once
#include "gptq_fp8.cuh"

namespace gptq {

constexpr int kFp8FewMaxSplit = 8, kFp8FewFirstDrain = 4;
constexpr int kFp8FewInline = 4;      // up to this many rows of 16-bit x become e4m3 in the kernel that multiplies them
__host__ __device__ constexpr int few_parts(int kind) { return kind == kFp8Plain ? 1 : 2; }      // accumulators of 128 weight rows
// four drain warps for every 32 token rows
__host__ __device__ constexpr int few_drain_warps(int TT) { return TT <= 32 ? 4 : TT / 8; }
__host__ __device__ constexpr int few_most_rows(int kind) { return kind == kFp8Plain ? 128 : 64; }
__host__ __device__ constexpr int few_threads(int kind, int TT) { return 32 * (kFp8FewFirstDrain + few_drain_warps(TT)); }
// two CTAs per SM where their sums and half of the shared memory allow: what is resident is more even, and one's start hides behind the other's loads
__host__ __device__ constexpr int few_per_sm(int kind, int TT) { return TT * few_parts(kind) <= 64 ? 2 : 1; }
__host__ __device__ constexpr int few_stage_bytes(int kind, int TT) { return (few_parts(kind) * 128 + TT) * kFp8Block; }
__host__ __device__ constexpr int few_buffers(int kind, int TT) { return TT * few_parts(kind) <= 128 ? 4 : 2; }
__host__ __device__ constexpr int few_columns(int kind, int TT)
{
    int c = 32;
    while (c < few_buffers(kind, TT) * TT * few_parts(kind)) c <<= 1;
    return c;
}
__host__ __device__ constexpr int few_scale_bytes(int kind, int TT) { return 2 * few_buffers(kind, TT) * few_parts(kind) * TT * 4; }
__host__ __device__ constexpr int few_stages(int kind, int TT)
{
    const int room = 227 * 1024 / few_per_sm(kind, TT) - 1024 - 2048 - few_scale_bytes(kind, TT);
    const int n = room / few_stage_bytes(kind, TT);
    return n < 8 ? n : 8;
}
// With 113 KB two CTAs fill an SM's 228 KB (1 KB goes with each), and neither fits beside one of the kernels that take all 512 columns of tensor memory
// (116736 bytes and more).  Such a pair on one SM, of two streams' clusters, each with its columns on one SM and waiting for them on another, would never end.
__host__ __device__ constexpr int few_smem(int kind, int TT)
{
    const int need = 2048 + few_stages(kind, TT) * few_stage_bytes(kind, TT) + few_scale_bytes(kind, TT);
    return need < 113 * 1024 ? 113 * 1024 : need;
}
// the parts of the sums that land in the idle ring: of each of S CTAs, of every S-th token row (S divides TT)
__host__ __device__ constexpr int few_parts_bytes(int kind, int TT) { return TT * few_parts(kind) * 512; }

struct Fp8FewArgs {
    const uint8_t *x16;        // 16-bit x, where the kernel makes e4m3 of it
    int K;
    const float *x_scales, *w_scales;
    const uint16_t *bias, *in;
    void *out;
    float *out_scales;
    int M, N, KB;              // gated kinds: N = 2 F
    int tiles_n, tok, log_S;   // tok: token rows per tile, a multiple of 16; S = 2^log_S
};

__device__ __forceinline__ void umma_f8_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void st_cluster_f32(uint32_t addr, float v)
{
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ void fma2_of(uint64_t &acc, uint32_t lo, uint32_t hi, uint32_t s_lo, uint32_t s_hi)
{
    asm volatile("{\n\t.reg .b64 v, s;\n\tmov.b64 v, {%1, %2};\n\tmov.b64 s, {%3, %4};\n\tfma.rn.f32x2 %0, v, s, %0;\n\t}"
                 : "+l"(acc) : "r"(lo), "r"(hi), "r"(s_lo), "r"(s_hi));
}

// Between the two barriers of a cluster's exchange, one thread of a CTA whose wait gave up: then no CTA of the cluster stores a row, since each
// adds parts of all of them.
__device__ __forceinline__ void few_tell_cluster(uint32_t flag, int S)
{
    for (int p = 0; p < S; ++p) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_cluster_rank(flag, p)), "r"(1u) : "memory");
}

// XQ: x is 16-bit.  Two warps make e4m3 of the rows, a block of K each in turn, write them where TMA would have put them (128-byte rows, 128-byte
// swizzle) and their scales where the scale warp would have; every CTA does so for its part of K.
template <int KIND, bool BF, bool OUT8, int TT, bool XQ>
__global__ void __launch_bounds__(few_threads(KIND, TT), few_per_sm(KIND, TT))
fp8_few_kernel(const Fp8FewArgs a, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map)
{
    extern __shared__ uint8_t smem_raw[];
    constexpr int G = few_parts(KIND), DW = few_drain_warps(TT), GROUPS = DW / 4, COLS = TT / GROUPS, NB = few_buffers(KIND, TT);
    constexpr int NS = few_stages(KIND, TT), kStage = few_stage_bytes(KIND, TT), kW = G * 128 * kFp8Block, kScale = G * TT * 4;
    constexpr uint32_t kCols = few_columns(KIND, TT);
    static_assert(NS >= 2 && COLS % 16 == 0, "");
    static_assert(kCols <= 512 / few_per_sm(KIND, TT) && few_per_sm(KIND, TT) * (few_smem(KIND, TT) + 1024) <= 228 * 1024, "tensor memory and shared memory of an SM");
    static_assert(few_parts_bytes(KIND, TT) <= NS * kStage, "the parts would run over the scales");
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar_full = base, bar_empty = base + 64, bar_dfull = base + 128, bar_dempty = base + 160, tmem_slot = base + 192, flag = base + 196;
    const uint32_t ring = base + 1024, scale_ring = ring + NS * kStage;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int log_S = a.log_S, S = 1 << log_S, rank = blockIdx.x & (S - 1), tile = blockIdx.x >> log_S;
    const int tm = tile / a.tiles_n, tn = tile - tm * a.tiles_n, m0 = tm * a.tok, KB = a.KB, F = a.N / 2;
    const int kb0 = KB * rank >> log_S, nkb = (KB * (rank + 1) >> log_S) - kb0;
    const int rows = min(a.tok, a.M - m0);

    if (threadIdx.x == 0) {
        for (int s = 0; s < NS; ++s) {
            mbar_init(bar_full + 8 * s, 2);      // weights, activations
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int s = 0; s < NB; ++s) {
            mbar_init(bar_dfull + 8 * s, 2);
            mbar_init(bar_dempty + 8 * s, DW);
        }
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(flag), "r"(0u) : "memory");
        fence_barrier_init();
        fence_proxy_async();
    }
    if (warp == 1) {
        tmem_alloc(tmem_slot, kCols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = lds32(tmem_slot);
    pdl_launch_dependents();

    if (warp == 0 || (warp == 3 && !XQ)) {
        // ------------------------------------------------------------------------------------------ TMA (a thread each)
        // A turn of such a loop takes its thread 210 clocks (wait, expect, copy) whatever the copy's size: two threads share the
        // work, and nothing else is in the loops.  Weights do not depend on earlier kernels: they are not waited for.
        if (elect_one()) {
            int s = 0, done = 0;
            uint32_t ph = 1;
            if (warp == 0) {
                tma_prefetch_descriptor(&w_map);
                uint32_t k = (uint32_t)kb0 * kFp8Block;      // (the last step may leave an int)
                for (int i = 0; i < nkb; ++i, k += kFp8Block) {
                    if (i >= NS && !mbar_wait_once(bar_empty + 8 * s, ph)) break;
                    mbar_arrive_expect_tx(bar_full + 8 * s, kW);
#pragma unroll
                    for (int g = 0; g < G; ++g) tma_load_2d(ring + s * kStage + g * 128 * kFp8Block, &w_map, (int)k, g * F + tn * 128, bar_full + 8 * s);
                    done = i + 1;
                    if (++s == NS) s = 0, ph ^= 1;
                }
            } else {
                tma_prefetch_descriptor(&x_map);
                pdl_wait();
                const uint32_t x_bytes = (uint32_t)a.tok * kFp8Block;
                uint32_t k = (uint32_t)kb0 * kFp8Block;
                for (int i = 0; i < nkb; ++i, k += kFp8Block) {
                    if (i >= NS && !mbar_wait_once(bar_empty + 8 * s, ph)) break;
                    mbar_arrive_expect_tx(bar_full + 8 * s, x_bytes);
                    tma_load_2d(ring + s * kStage + kW, &x_map, (int)k, m0, bar_full + 8 * s);
                    done = i + 1;
                    if (++s == NS) s = 0, ph ^= 1;
                }
            }
            // nothing of this thread's may be on its way into the ring when the sums' parts are put there, or when the CTA ends
            for (int j = done < NS ? 0 : done - NS; j < done; ++j) mbar_wait(bar_full + 8 * (j % NS), (uint32_t)(j / NS) & 1);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------------------------------ MMA (one thread)
        if (elect_one()) {
            const uint32_t idesc = umma_idesc_f16(128, a.tok);      // (both operands e4m3: format fields 0)
            int s = 0, d = 0;
            uint32_t ph = 0, dph = 1;
            for (int i = 0; i < nkb; ++i) {
                if (i >= NB && !mbar_wait_once(bar_dempty + 8 * d, dph)) break;
                if (!mbar_wait_once(bar_full + 8 * s, ph)) break;
                tc_fence_after_sync();
                const uint64_t xd = umma_desc_k_major_sw128(ring + s * kStage + kW);
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const uint64_t wd = umma_desc_k_major_sw128(ring + s * kStage + g * 128 * kFp8Block);
#pragma unroll
                    for (int j = 0; j < 4; ++j) umma_f8_ss(tmem + (d * G + g) * TT, wd + 2 * j, xd + 2 * j, idesc, j);
                }
                umma_commit(bar_dfull + 8 * d);
                umma_commit(bar_empty + 8 * s);
                if (++s == NS) s = 0, ph ^= 1;
                if (++d == NB) d = 0, dph ^= 1;
            }
        }
    } else if (XQ && (warp == 2 || warp == 3)) {
        // ------------------------------------------------------------------------------------------ x and its scales
        pdl_wait();
        const float *ws[G];
#pragma unroll
        for (int g = 0; g < G; ++g) ws[g] = a.w_scales + (size_t)(g * (F / kFp8Block) + tn) * KB + kb0;
        uint2 next[kFp8FewInline];      // four numbers of each row
        float w_next[G];
        auto fetch = [&](int i) {
            const uint32_t k = (uint32_t)(kb0 + i) * kFp8Block + 4 * lane;
#pragma unroll
            for (int m = 0; m < kFp8FewInline; ++m)
                next[m] = i < nkb && m < a.M && k < (uint32_t)a.K ? ldg64_behind(a.x16 + ((size_t)m * a.K + k) * 2) : make_uint2(0, 0);
#pragma unroll
            for (int g = 0; g < G; ++g) w_next[g] = i < nkb ? ldgf_behind(ws[g] + i) : 0.0f;
        };
        int s = warp - 2;
        uint32_t ph = 1;
        bool ok = true;
        fetch(warp - 2);
        for (int i = warp - 2; i < nkb && ok; i += 2) {
            uint32_t q[kFp8FewInline];
            float scale[kFp8FewInline], w[G];
#pragma unroll
            for (int m = 0; m < kFp8FewInline; ++m) {
                if (m >= a.M) break;
                const float2 lo = pair_to_float2<BF>(next[m].x), hi = pair_to_float2<BF>(next[m].y);
                scale[m] = fp8_scale(__reduce_max_sync(0xffffffffu, max(max(abs_bits(lo.x), abs_bits(lo.y)), max(abs_bits(hi.x), abs_bits(hi.y)))));
                const Fp8Quotient by(scale[m]);
                q[m] = fp8_four(by(lo.x), by(lo.y), by(hi.x), by(hi.y));
            }
#pragma unroll
            for (int g = 0; g < G; ++g) w[g] = w_next[g];
            fetch(i + 2);
            // the stage is free, and the scales' slot (as below)
            if (i >= NS) ok = mbar_wait_warp(bar_empty + 8 * s, ph);
            if (ok && i >= NB) ok = mbar_wait_warp(bar_dfull + 8 * (i & (NB - 1)), (uint32_t)(i / NB - 1) & 1);
            if (!ok) break;      // (stage and slot may still be read)
            const uint32_t to = ring + s * kStage + kW + (lane & 3) * 4, slot = scale_ring + (i & (2 * NB - 1)) * kScale;
#pragma unroll
            for (int m = 0; m < kFp8FewInline; ++m) {
                if (m >= a.M) break;
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + m * 128 + ((lane >> 2 ^ m) << 4)), "r"(q[m]) : "memory");
                if (lane < G) asm volatile("st.shared.f32 [%0], %1;" ::"r"(slot + (lane * TT + m) * 4), "f"(scale[m] * (lane == 0 ? w[0] : w[G - 1])) : "memory");
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(bar_full + 8 * s);
                mbar_arrive(bar_dfull + 8 * (i & (NB - 1)));
            }
            s += 2;
            if (s >= NS) s -= NS, ph ^= 1;
        }
    } else if (!XQ && warp == 2) {
        // ------------------------------------------------------------------------------------------ scales
        // Block i's go into slot i % (2 NB) once block i - NB is complete: its MMA waited until block i - 2 NB, which had the slot, was drained.
        pdl_wait();
        constexpr int R = (TT + 31) / 32;
        const float *xs[R], *ws[G];
#pragma unroll
        for (int r = 0; r < R; ++r) xs[r] = a.x_scales + (size_t)min(m0 + 32 * r + lane, a.M - 1) * KB + kb0;
#pragma unroll
        for (int g = 0; g < G; ++g) ws[g] = a.w_scales + (size_t)(g * (F / kFp8Block) + tn) * KB + kb0;
        float x[2][R], w[2][G];
        auto fetch = [&](int j, int kb) {
#pragma unroll
            for (int r = 0; r < R; ++r) x[j][r] = kb < nkb ? ldgf_behind(xs[r] + kb) : 0.0f;
#pragma unroll
            for (int g = 0; g < G; ++g) w[j][g] = kb < nkb ? ldgf_behind(ws[g] + kb) : 0.0f;
        };
        fetch(0, 0);
        fetch(1, 1);
        bool ok = true;
        for (int i0 = 0; i0 < nkb && ok; i0 += 2)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int i = i0 + j;
                if (i >= nkb || !ok) break;
                if (i >= NB && !(ok = mbar_wait_warp(bar_dfull + 8 * (i & (NB - 1)), (uint32_t)(i / NB - 1) & 1))) break;      // (the slot may still be read)
                const uint32_t slot = scale_ring + (i & (2 * NB - 1)) * kScale;
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        if (TT >= 32 || lane < TT)
                            asm volatile("st.shared.f32 [%0], %1;" ::"r"(slot + (g * TT + 32 * r + lane) * 4), "f"(x[j][r] * w[j][g]) : "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_dfull + 8 * (i & (NB - 1)));
                fetch(j, i + 2);
            }
    }
    uint64_t acc[G][COLS / 2];
    const int q = warp & 3, group = (warp - kFp8FewFirstDrain) >> 2;
    if (warp >= kFp8FewFirstDrain) {
        // ------------------------------------------------------------------------------------------ drain
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int j = 0; j < COLS / 2; ++j) acc[g][j] = 0;
        pdl_wait();
        const uint32_t from = tmem + ((uint32_t)(32 * q) << 16) + group * COLS;
        const int chunks = min(COLS, a.tok - group * COLS) / 16;      // (may be none)
        bool ok = true;
        for (int i = 0; i < nkb; ++i) {
            const int d = i & (NB - 1);
            if (!(ok = mbar_wait_warp_inline(bar_dfull + 8 * d, (uint32_t)(i / NB) & 1))) break;
            tc_fence_after_sync();
            const uint32_t slot = scale_ring + (i & (2 * NB - 1)) * kScale + group * COLS * 4;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int c = 0; c < COLS / 16; ++c)
                    if (c < chunks) {
                        uint32_t v[16];
                        uint4 s[4];
                        tmem_ld_32x16(from + (d * G + g) * TT + 16 * c, v);
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[j] = lds128(slot + (g * TT + 16 * c + 4 * j) * 4);
                        tmem_wait_ld();
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            fma2_of(acc[g][8 * c + 2 * j], v[4 * j], v[4 * j + 1], s[j].x, s[j].y);
                            fma2_of(acc[g][8 * c + 2 * j + 1], v[4 * j + 2], v[4 * j + 3], s[j].z, s[j].w);
                        }
                    }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_dempty + 8 * d);
        }
        if (!ok && lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(flag), "r"(1u) : "memory");
    }
    // ---- the parts of the sums to the CTAs that finish them: [sender][row / S][part][weight row], over the ring
    __syncwarp();
    if (S > 1) {
        cluster_arrive_release();      // everything that was to land in this CTA's ring has, and has been multiplied
        cluster_wait_acquire();
    } else {
        __syncthreads();
    }
    if (S > 1 && threadIdx.x == 0 && lds32(flag) != 0) few_tell_cluster(flag, S);
    const int mine = TT >> log_S;      // rows per sender (of which those below `rows` are sent)
    if (warp >= kFp8FewFirstDrain) {
#pragma unroll
        for (int j = 0; j < COLS; ++j) {
            const int m = group * COLS + j;
            if (m < rows) {
                const uint32_t at = ring + (((rank * mine + (m >> log_S)) * G) * 128 + 32 * q + lane) * 4;
                const uint32_t to = S > 1 ? map_to_cluster_rank(at, m & (S - 1)) : at;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const float2 f = unpack2(acc[g][j / 2]);
                    const float v = j & 1 ? f.y : f.x;
                    if (S > 1) st_cluster_f32(to + g * 512, v);
                    else asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + g * 512), "f"(v) : "memory");
                }
            }
        }
    }
    if (S > 1) {
        cluster_arrive_release();
        cluster_wait_acquire();
    } else {
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, kCols);
    }
    if (lds32(flag) != 0) return;
    // ---- a warp per row: lane l has columns 4 l .. 4 l + 3 of the 128
    if (warp >= kFp8FewFirstDrain) {
        constexpr int kOuts = KIND == kFp8Backward ? 2 : 1;
        const int c = tn * 128 + 4 * lane;      // column of y, or (gated kinds) of the result
        for (int r = warp - kFp8FewFirstDrain; r * S + rank < rows; r += DW) {
            const size_t m = (size_t)m0 + r * S + rank;
            float v[G][4];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                v[g][0] = v[g][1] = v[g][2] = v[g][3] = 0.0f;
                for (int p = 0; p < S; ++p) {
                    const uint4 e = lds128(ring + (((p * mine + r) * G + g) * 128 + 4 * lane) * 4);
                    v[g][0] += __uint_as_float(e.x), v[g][1] += __uint_as_float(e.y), v[g][2] += __uint_as_float(e.z), v[g][3] += __uint_as_float(e.w);
                }
            }
            auto add = [&](float(&f)[4], const uint16_t *p) {
                const uint2 e = ldg64_behind(p);
                const float2 lo = pair_to_float2<BF>(e.x), hi = pair_to_float2<BF>(e.y);
                f[0] += lo.x, f[1] += lo.y, f[2] += hi.x, f[3] += hi.y;
            };
            auto store16 = [&](const float(&f)[4], size_t at) {
                *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(a.out) + at) =
                    make_uint2(pack_out16<BF>(make_float2(f[0], f[1])), pack_out16<BF>(make_float2(f[2], f[3])));
            };
            if constexpr (KIND == kFp8Plain) {
                if (c >= a.N) continue;      // (N % 8 == 0)
                if (a.bias != nullptr) add(v[0], a.bias + c);
                if (a.in != nullptr) add(v[0], a.in + m * a.N + c);
                store16(v[0], m * a.N + c);
            } else {
                float d[4] = {0.0f, 0.0f, 0.0f, 0.0f}, o[kOuts][4];
                if (KIND == kFp8Backward) add(d, a.in + m * F + c);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float gate = v[0][j], up = v[G - 1][j], p = logistic(gate);
                    if constexpr (KIND == kFp8Gated) {
                        o[0][j] = gate * p * up;
                    } else {
                        o[0][j] = d[j] * up * p * (1.0f + gate * (1.0f - p)), o[kOuts - 1][j] = d[j] * gate * p;
                    }
                }
#pragma unroll
                for (int k = 0; k < kOuts; ++k) {
                    const size_t at = m * (size_t)(kOuts * F) + (size_t)k * F + c;
                    if constexpr (OUT8) {
                        const uint32_t top = __reduce_max_sync(0xffffffffu, max(max(abs_bits(o[k][0]), abs_bits(o[k][1])), max(abs_bits(o[k][2]), abs_bits(o[k][3]))));
                        const float s = fp8_scale(top);
                        const Fp8Quotient by(s);
                        *reinterpret_cast<uint32_t *>(reinterpret_cast<uint8_t *>(a.out) + at) =
                            fp8_four(by(o[k][0]), by(o[k][1]), by(o[k][2]), by(o[k][3]));
                        if (lane == 0) a.out_scales[m * (kOuts * (F / kFp8Block)) + k * (F / kFp8Block) + tn] = s;
                    } else {
                        store16(o[k], at);
                    }
                }
            }
        }
    }
}

// the instance that takes tiles of `tok` token rows
__host__ __device__ constexpr int few_instance(int tok) { return tok <= 16 ? 16 : tok <= 32 ? 32 : tok <= 64 ? 64 : 128; }

struct Fp8FewPlan {
    int tok, tiles_m, tiles_n, log_S;
    int waves, blocks;      // of CTAs; blocks of K of each CTA, at most
};
// Token rows in even tiles of at most 128 (gated kinds 64).  S: CTAs for every SM as long as each has two blocks of K; two per SM where each still has eight.
inline Fp8FewPlan plan_fp8_few(int kind, int M, int N, int K, int sms)
{
    Fp8FewPlan p{};
    p.tiles_m = (M - 1) / few_most_rows(kind) + 1;
    p.tok = (((M - 1) / p.tiles_m + 1) + 15) / 16 * 16;
    p.tiles_n = kind == kFp8Plain ? (N - 1) / 128 + 1 : N / 256;
    const long long room = (long long)sms * few_per_sm(kind, few_instance(p.tok)), tiles = (long long)p.tiles_m * p.tiles_n;
    const int KB = fp8_blocks(K);
    while (2 << p.log_S <= kFp8FewMaxSplit && KB >= 4 << p.log_S &&
           (tiles * (2 << p.log_S) <= sms || (tiles * (2 << p.log_S) <= room && KB >= 16 << p.log_S)))
        ++p.log_S;
    p.waves = (int)(((tiles << p.log_S) + room - 1) / room);
    p.blocks = (KB - 1 >> p.log_S) + 1;
    return p;
}

// Up to a tile of token rows the layer is read once here and the pairs of gptq_fp8.cuh would leave most SMs idle: always this kernel.
// Beyond, the shorter of what both take: ns, fitted to calls of 128 to 1000 rows of K = 512 to 11008 (us, this kernel / pairs, whose wave of tiles takes the
// same however few there are: 4096 x 4096 256 rows 11.8 / 20.3, 512 rows 17.3 / 20.3, 768 rows 33.9 / 20.3; 4096 x 12288 384 rows 35.8 to 37.8 / 36.9; gated 4096 x 2048
// 512 rows 22.3 / 24.2, 4096 x 11008 128 rows 47.3 / 42.8).
inline bool fp8_few_is_shorter(int kind, int M, int N, int K, int sms, const Fp8FewPlan &p)
{
    if (M <= few_most_rows(kind) || sms < 2) return true;
    const long long pairs = sms / 2, waves = (fp8_tiles(kind, M, N) + pairs - 1) / pairs, KB = fp8_blocks(K);
    const bool plain = kind == kFp8Plain;
    return p.waves * (4000 + (plain ? 410ll : 590ll) * p.blocks) < (plain ? 4500 : 6000) + waves * KB * (plain ? 495 : 575);
}

template <int KIND, bool BF, bool OUT8, int TT, bool XQ = false>
int launch_fp8_few_as(const Fp8Call &c, const Fp8FewPlan &p, cudaStream_t s)
{
    static int configured[64];
    auto kernel = fp8_few_kernel<KIND, BF, OUT8, TT, XQ>;
    constexpr int smem = few_smem(KIND, TT);
    int st = ensure_dynamic_smem((const void *)kernel, configured, smem);
    if (st) return st;
    Fp8FewArgs a{};
    a.x_scales = c.x_scales, a.w_scales = c.w_scales, a.bias = (const uint16_t *)c.bias, a.in = (const uint16_t *)c.in, a.out = c.out, a.out_scales = c.out_scales;
    a.M = c.M, a.N = c.N, a.KB = fp8_blocks(c.K), a.tiles_n = p.tiles_n, a.tok = p.tok, a.log_S = p.log_S;
    a.x16 = (const uint8_t *)c.x, a.K = c.K;
    CUtensorMap xm, wm;
    const auto u8 = CU_TENSOR_MAP_DATA_TYPE_UINT8;
    st = make_tensor_map_2d(&wm, u8, c.w, c.K, c.N, c.K, kFp8Block, 128, CU_TENSOR_MAP_SWIZZLE_128B);
    if (!st) {
        if (XQ) xm = wm;      // (not used)
        else st = make_tensor_map_2d(&xm, u8, c.x, c.K, c.M, c.K, kFp8Block, p.tok, CU_TENSOR_MAP_SWIZZLE_128B);
    }
    if (st) return st;
    const long long ctas = (long long)p.tiles_m * p.tiles_n << p.log_S;
    if (ctas > 0x7fffffffll) return GPTQ_ERR_UNSUPPORTED;
    void *args[] = {&a, &xm, &wm};
    return record_cuda_error(fp8_launch((void *)kernel, (int)ctas, few_threads(KIND, TT), smem, 1 << p.log_S, s, args));
}

template <int KIND, bool BF, bool OUT8>
int launch_fp8_few_kind(const Fp8Call &c, const Fp8FewPlan &p, cudaStream_t s)
{
    if (c.x_scales == nullptr) return launch_fp8_few_as<KIND, BF, OUT8, 16, true>(c, p, s);
    if (p.tok <= 16) return launch_fp8_few_as<KIND, BF, OUT8, 16>(c, p, s);
    if (p.tok <= 32) return launch_fp8_few_as<KIND, BF, OUT8, 32>(c, p, s);
    if constexpr (KIND == kFp8Plain)
        if (p.tok > 64) return launch_fp8_few_as<KIND, BF, OUT8, 128>(c, p, s);
    return launch_fp8_few_as<KIND, BF, OUT8, 64>(c, p, s);
}

inline int launch_fp8_any(const Fp8Call &c, cudaStream_t s)
{
    const Fp8FewPlan p = plan_fp8_few(c.kind, c.M, c.N, c.K, c.sms);
    if (!fp8_few_is_shorter(c.kind, c.M, c.N, c.K, c.sms, p)) return launch_fp8(c, s);
    const bool out8 = c.out_scales != nullptr;
    switch (c.kind * 4 + (out8 ? 2 : 0) + (c.bf16 ? 1 : 0)) {
    case 0: return launch_fp8_few_kind<kFp8Plain, false, false>(c, p, s);
    case 1: return launch_fp8_few_kind<kFp8Plain, true, false>(c, p, s);
    case 4: return launch_fp8_few_kind<kFp8Gated, false, false>(c, p, s);
    case 5: return launch_fp8_few_kind<kFp8Gated, true, false>(c, p, s);
    case 6: return launch_fp8_few_kind<kFp8Gated, false, true>(c, p, s);
    case 7: return launch_fp8_few_kind<kFp8Gated, true, true>(c, p, s);
    case 8: return launch_fp8_few_kind<kFp8Backward, false, false>(c, p, s);
    case 9: return launch_fp8_few_kind<kFp8Backward, true, false>(c, p, s);
    case 10: return launch_fp8_few_kind<kFp8Backward, false, true>(c, p, s);
    case 11: return launch_fp8_few_kind<kFp8Backward, true, true>(c, p, s);
    default: return GPTQ_ERR_UNSUPPORTED;
    }
}

}  // namespace gptq

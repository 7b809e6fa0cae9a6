// A shared projection with a low-rank adapter per row: y[m] = x[m] W + scale[a] (x[m] A[a]^T) B[a]^T, a = adapter_ids[m].
//
// v[m] = scale[a] x[m] A[a]^T is formed first, in fp32 (`lora_shrink_kernel`).  Up to 8 rows the product with W and the expansion
// v B^T are one kernel: its weights and x are under way while v is still being formed, the expansion joins the fp32 sums in the epilogue
// and y is rounded once.  Above that `lora_delta_rows_kernel` or `lora_delta_runs_kernel` writes the expansion out (16 bits) and it joins the other matmul kernels' fp32
// sums as their residual.
//
// Both adapter kernels look at eight rows at a time, the eight columns of an MMA, and go through the adapters that these name: one for
// a run of rows of a prompt, up to eight in a decode batch.  A product is formed for all eight rows and kept for those whose adapter
// it is, so that nothing of another row's adapter, whatever it holds, reaches a row.
#pragma once
#include "gptq_common.cuh"
#include "gptq_direct.cuh"

namespace gptq {

constexpr int kLoraMaxRank = 256;
constexpr int kLoraDirectRows = 8;       // rows of the fused kernel
constexpr int kLoraWarps = 8, kLoraThreads = 32 * kLoraWarps;
// Up to here rows are taken to have adapters of their own (a CTA of the shrink kernel per adapter of eight rows, lora_delta_rows_kernel), above
// to come in runs of one (a CTA takes eight rows' adapters in turn, lora_delta_runs_kernel).  The ids would tell, but they are on the device.
// Whole calls in us, own adapters / one adapter, 5120 x 5120, rank 32: 16 rows 17.0 / 14.9 this way and 35.6 / 13.7 the other; 64 rows
// 32.8 / 26.4 and 67.8 / 18.5; 128 rows 47.0 / 35.2 and 72.0 / 22.4; 256 rows 71.6 / 50.0 and 124 / 28.0.  So a short prompt of one adapter and
// a decode batch of more than 64 rows get the slower way: by up to 2.1 (rank 64, 64 rows: 50.7 for 23.7) and 2.7 times (rank 16, 256: 108 for 39.3).
constexpr int kLoraDecodeRows = 64;
constexpr int kLoraSteps = 4;            // 32-column steps of K that a warp of the shrink kernel requests at once

template <int N>
struct Int {
    static constexpr int value = N;
};

struct LoraArgs {
    const __half *x;          // [M, K] as given
    const __half *a, *b;      // [adapters, rank, K], [adapters, N, rank]
    const int32_t *ids;       // [M]
    const float *scales;      // [adapters] or nullptr
    float *v;                 // [k_parts, M, rank]: the sums over parts of K
    int M, N, K, rank, adapters;
    int k_parts;
    int sms;
    uint32_t one;             // 1 (see prepare_rows)
};

// The adapters that eight rows name, from row m0 on: lane l < 8 holds row l's id (-1: none) and the first row of each adapter leads.
struct RowAdapters {
    int id;
    uint32_t leads;
    // the id of the j-th adapter (j < popc(leads)) and the rows that have it
    __device__ __forceinline__ int adapter(int j, uint32_t &rows) const
    {
        uint32_t left = leads;
        for (; j; --j) left &= left - 1;
        const int a = __shfl_sync(0xffffffffu, id, __ffs(left) - 1);
        rows = __ballot_sync(0xffffffffu, id == a);
        return a;
    }
};
__device__ __forceinline__ RowAdapters row_adapters(const LoraArgs &a, int m0, int lane)
{
    RowAdapters r;
    r.id = lane < 8 && m0 + lane < a.M ? __ldg(a.ids + m0 + lane) : -1;
    if ((unsigned)r.id >= (unsigned)a.adapters) r.id = -1;
    const uint32_t same = __match_any_sync(0xffffffffu, r.id);
    r.leads = __ballot_sync(0xffffffffu, r.id >= 0 && (same & ((1u << lane) - 1)) == 0);
    return r;
}

// v of eight rows (blockIdx.x), 16 of an adapter's rank (blockIdx.y) and a part of K: rows of A as the 16-row operand, rows of x as
// the columns, the warps sharing the part's steps of 32 columns.  Bound by one
// round trip to memory (see lora_k_parts).  blockIdx.z: part of K, and which of the adapters.
//
// Slices of blockIdx.z beyond these put rows of x in the sorted row order of an act-order layer, for the matmul: a launch less.
template <bool BF>
__global__ void __launch_bounds__(kLoraThreads, 4) lora_shrink_kernel(const LoraArgs a, int adapters_apart, const int32_t *__restrict__ perm, __half *__restrict__ x_sorted)
{
    __shared__ float red[kLoraWarps][4][32];
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const int m0 = 8 * blockIdx.x, r0 = 16 * blockIdx.y, part = blockIdx.z / adapters_apart;
    pdl_wait();
    pdl_launch_dependents();        // (behind the wait: what x was before this kernel is what the next one may read at once)
    if (part >= a.k_parts) {
        const int slice = (blockIdx.z - adapters_apart * a.k_parts) * gridDim.y + blockIdx.y, slices = (gridDim.z - adapters_apart * a.k_parts) * gridDim.y;
        for (int i = 2 * (slice * kLoraThreads + threadIdx.x); i < a.K; i += 2 * slices * kLoraThreads) {
            const int2 from = __ldg(reinterpret_cast<const int2 *>(perm + i));
            const int rows = min(8, a.M - m0);
            __half2 v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const __half *row = a.x + (size_t)(m0 + min(r, rows - 1)) * a.K;
                v[r] = __halves2half2(row[from.x], row[from.y]);
            }
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r < rows) *reinterpret_cast<__half2 *>(x_sorted + (size_t)(m0 + r) * a.K + i) = v[r];
        }
        return;
    }
    const RowAdapters named = row_adapters(a, m0, lane);
    const int n = __popc(named.leads);
    const int w = part * kLoraWarps + warp, W = a.k_parts * kLoraWarps;
    const int s0 = share_begin(a.K / 32, W, w), s1 = share_begin(a.K / 32, W, w + 1);
    const __half *xr = a.x + (size_t)min(m0 + g, a.M - 1) * a.K + 8 * t4;
    for (int j = blockIdx.z % adapters_apart; j < n; j += adapters_apart) {
        uint32_t rows;
        const int id = named.adapter(j, rows);
        const __half *lo = a.a + ((size_t)id * a.rank + r0 + g) * a.K + 8 * t4, *hi = lo + (size_t)8 * a.K;
        const bool has_hi = r0 + 8 < a.rank;      // the rank is a multiple of 8
        if (!has_hi) hi = lo;
        float acc[4] = {};
        int s = s0;
        auto batch = [&](auto steps) {      // all of a batch's loads before its products
            constexpr int n_steps = decltype(steps)::value;
            uint4 p[n_steps], q[n_steps], v[n_steps];
#pragma unroll
            for (int i = 0; i < n_steps; ++i) {
                p[i] = __ldg(reinterpret_cast<const uint4 *>(lo + 32 * (s + i)));
                q[i] = __ldg(reinterpret_cast<const uint4 *>(hi + 32 * (s + i)));
                v[i] = *reinterpret_cast<const uint4 *>(xr + 32 * (s + i));
            }
#pragma unroll
            for (int i = 0; i < n_steps; ++i) {
                mma16<BF, false>(acc, p[i].x, q[i].x, p[i].y, q[i].y, register_pair(v[i].x, v[i].y));
                mma16<BF, false>(acc, p[i].z, q[i].z, p[i].w, q[i].w, register_pair(v[i].z, v[i].w));
            }
            s += n_steps;
        };
        while (s + kLoraSteps <= s1) batch(Int<kLoraSteps>{});
        if (s + 3 == s1) batch(Int<3>{});
        else if (s + 2 == s1) batch(Int<2>{});
        else if (s + 1 == s1) batch(Int<1>{});
#pragma unroll
        for (int i = 0; i < 4; ++i) red[warp][i][lane] = acc[i];
        __syncthreads();
        if (threadIdx.x < 128) {
            const int i = threadIdx.x >> 5, row = 2 * t4 + (i & 1), r = r0 + g + 8 * (i >> 1);      // (lane of threadIdx.x = lane)
            if ((rows >> row & 1) && r < a.rank) {
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < kLoraWarps; ++k) sum += red[k][i][lane];
                a.v[((size_t)part * a.M + m0 + row) * a.rank + r] = a.scales ? sum * __ldg(a.scales + id) : sum;
            }
        }
        __syncthreads();
    }
}

// v[m][r .. r + 4 NV - 1], summed over the parts of K in their order; a batch of parts is requested before the first is added: a loop
// over as many as there are waits for each in turn (4096 x 4096, rank 16, four parts, one row: 6.8 -> 6.3 us; 1000 rows 42.0 -> 41.1).
constexpr int kLoraPartBatch = 4;
template <int NV>
__device__ __forceinline__ void lora_v(const LoraArgs &a, int m, int r, float4 (&v)[NV])
{
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int p = 0; p < a.k_parts; p += kLoraPartBatch) {
        float4 w[kLoraPartBatch][NV];
#pragma unroll
        for (int b = 0; b < kLoraPartBatch; ++b)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                w[b][i] = p + b < a.k_parts ? *reinterpret_cast<const float4 *>(a.v + ((size_t)(p + b) * a.M + m) * a.rank + r + 4 * i)
                                            : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int b = 0; b < kLoraPartBatch; ++b)
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i].x += w[b][i].x, v[i].y += w[b][i].y, v[i].z += w[b][i].z, v[i].w += w[b][i].w;
    }
}
template <bool BF>
__device__ __forceinline__ uint32_t pack16(float a, float b)
{
    return (uint32_t)float_to_out16<BF>(a) | (uint32_t)float_to_out16<BF>(b) << 16;
}

// delta[m][n] = (v B^T)[m][n], 0 without an adapter.  The ids and B are older than the shrink kernel, which waited for what was before it
// when it let these kernels in: they are read while v is still being formed.
//
// Decode batches, every row with an adapter of its own: a column of B has rank / 8 pieces of 16 bytes; neighbouring lanes read
// neighbouring pieces, multiply them with their 8 values of v, which they keep, and add up.  A warp takes a row and kDeltaSteps times the
// columns that its lanes read at once, all requested before the first is used.  Every row has its own B; 60 % of the issue slots, 19 % of
// the DRAM rate, the stalls waits for loads.  64 rows of 5120 x 5120, rank 32: 33 us with the shrink kernel and the matmul, which alone takes 13.4.
constexpr int kDeltaSteps = 4;
template <bool BF>
__global__ void __launch_bounds__(256, 4) lora_delta_rows_kernel(const LoraArgs a, __half *__restrict__ delta)
{
    pdl_launch_dependents();
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int pieces = a.rank / 8, cols = 32 / pieces;      // (rank up to 256: at least one column)
    const int m = blockIdx.y, n0 = kDeltaSteps * cols * (8 * blockIdx.x + warp), n1 = min(n0 + kDeltaSteps * cols, a.N);
    if (n0 >= a.N) return;
    const int id = __ldg(a.ids + m), c = lane / pieces, piece = lane - c * pieces;
    __half *out = delta + (size_t)m * a.N;
    if ((unsigned)id >= (unsigned)a.adapters) {
        pdl_wait();
        for (int n = n0 + lane; n < n1; n += 32) store_out16<BF>(out + n, 0.f);
        return;
    }
    uint4 p[kDeltaSteps];
    const uint4 *b = reinterpret_cast<const uint4 *>(a.b + ((size_t)id * a.N + n0) * a.rank) + lane;
#pragma unroll
    for (int k = 0; k < kDeltaSteps; ++k)
        p[k] = c < cols && n0 + k * cols + c < n1 ? __ldg(b + k * (cols * pieces)) : make_uint4(0, 0, 0, 0);
    float4 v[2] = {};
    pdl_wait();
    if (c < cols) lora_v(a, m, 8 * piece, v);
    const float4 v0 = v[0], v1 = v[1];
#pragma unroll
    for (int k = 0; k < kDeltaSteps; ++k) {
        const float2 p0 = pair_to_float2<BF>(p[k].x), p1 = pair_to_float2<BF>(p[k].y), p2 = pair_to_float2<BF>(p[k].z), p3 = pair_to_float2<BF>(p[k].w);
        float sum = p0.x * v0.x;
        sum = fmaf(p0.y, v0.y, sum), sum = fmaf(p1.x, v0.z, sum), sum = fmaf(p1.y, v0.w, sum);
        sum = fmaf(p2.x, v1.x, sum), sum = fmaf(p2.y, v1.y, sum), sum = fmaf(p3.x, v1.z, sum), sum = fmaf(p3.y, v1.w, sum);
        float total = sum;
        for (int l = 1; l < pieces; ++l) total += __shfl_down_sync(0xffffffffu, sum, l);
        if (c < cols && n0 + k * cols + c < n1 && piece == 0) store_out16<BF>(out + n0 + k * cols + c, total);
    }
}

// Prompts, runs of rows with one adapter: kDeltaRows rows and 256 columns per CTA, MMAs with the rows' v as the 16-row operand and
// eight rows of B as the columns.  v is taken in two 16-bit parts that the CTA prepares in shared memory, each row times the power of two
// that brings its largest value to 2^14 .. 2^15: hi + lo is then v to 2^-22 (bfloat16 2^-16) wherever v lies in fp32's range (fp16: of values
// below 2^-17 of the row's largest, to 2^-39 of the largest).  The product is as good as fp32's next to the 16 bits of delta; the power is taken
// out of the fp32 sums.  A sum that is not finite is formed again in fp32: an infinity times a part that is 0 is NaN.
// 1000 rows of 4096 x 4096 in five runs, rank 16: 41.6 us with the shrink kernel and the matmul, which alone takes 27
// (41.1 without the powers of two and the test for infinities).
constexpr int kDeltaRows = 32, kDeltaTiles = 4;      // tiles: eight columns each, of a warp
template <bool BF>
__device__ __noinline__ float long_expansion(const LoraArgs &a, int m, int n)
{
    const __half *b = a.b + ((size_t)__ldg(a.ids + m) * a.N + n) * a.rank;
    float sum = 0.f;
    for (int r = 0; r < a.rank; r += 4) {
        float4 v[1];
        lora_v(a, m, r, v);
        const uint2 p = __ldg(reinterpret_cast<const uint2 *>(b + r));
        const float2 lo = pair_to_float2<BF>(p.x), hi = pair_to_float2<BF>(p.y);
        sum = fmaf(hi.y, v[0].w, fmaf(hi.x, v[0].z, fmaf(lo.y, v[0].y, fmaf(lo.x, v[0].x, sum))));
    }
    return sum;
}
template <bool BF>
__global__ void __launch_bounds__(256, 2) lora_delta_runs_kernel(const __grid_constant__ LoraArgs a, __half *__restrict__ delta)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float unscale[kDeltaRows];
    pdl_launch_dependents();
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const int n0 = 8 * kDeltaTiles * (8 * blockIdx.x + warp), m0 = kDeltaRows * (blockIdx.z * gridDim.y + blockIdx.y);
    if (m0 >= a.M) return;      // (the last of several layers of the grid)
    const int count = min(kDeltaRows, a.M - m0);
    const int width = (a.rank + 31) & ~31, pitch = 2 * width * 2 + 16;      // a row: hi, lo, 16 bytes against bank conflicts
    int my_id = lane < count ? __ldg(a.ids + m0 + lane) : -1;               // (a row per lane)
    if ((unsigned)my_id >= (unsigned)a.adapters) my_id = -1;
    const uint32_t same = __match_any_sync(0xffffffffu, my_id);
    uint32_t leads = __ballot_sync(0xffffffffu, my_id >= 0 && (same & ((1u << lane) - 1)) == 0);
    auto load_b = [&](uint4 (&p)[kDeltaTiles], int id, int r) {
#pragma unroll
        for (int t = 0; t < kDeltaTiles; ++t)
            p[t] = r < a.rank && n0 < a.N ? __ldg(reinterpret_cast<const uint4 *>(a.b + ((size_t)id * a.N + n0 + 8 * t + g) * a.rank + r)) : make_uint4(0, 0, 0, 0);
    };
    uint4 p[kDeltaTiles] = {};
    if (leads) load_b(p, __shfl_sync(0xffffffffu, my_id, __ffs(leads) - 1), 8 * t4);      // on its way while v is prepared
    pdl_wait();
    {      // eight lanes prepare a row
        const int row = threadIdx.x >> 3, r0 = 4 * (threadIdx.x & 7);
        const bool named = __shfl_sync(0xffffffffu, my_id, row) >= 0;
        float4 v[kLoraMaxRank / 32];
        int top = 0;      // the largest finite magnitude's bits
#pragma unroll
        for (int i = 0; i < kLoraMaxRank / 32; ++i) {
            if (32 * i >= width) break;
            float4 w[1] = {};
            if (named && r0 + 32 * i < a.rank) lora_v(a, m0 + row, r0 + 32 * i, w);
            v[i] = w[0];
            for (float f : {v[i].x, v[i].y, v[i].z, v[i].w}) {
                const int bits = __float_as_int(f) & 0x7fffffff;
                top = max(top, bits < 0x7f800000 ? bits : 0);
            }
        }
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int e = top ? min(14 + 127 - (top >> 23), 126) : 0;      // -113 .. 126
        const float scale = __int_as_float((127 + e) << 23);
        if ((threadIdx.x & 7) == 0) unscale[row] = __int_as_float((127 - e) << 23);
        auto rest = [](float f, float h) { return isfinite(h) ? f - h : 0.f; };
#pragma unroll
        for (int i = 0; i < kLoraMaxRank / 32; ++i) {
            if (32 * i >= width) break;
            const float4 f = make_float4(v[i].x * scale, v[i].y * scale, v[i].z * scale, v[i].w * scale);
            const uint2 h = make_uint2(pack16<BF>(f.x, f.y), pack16<BF>(f.z, f.w));
            const float2 h0 = pair_to_float2<BF>(h.x), h1 = pair_to_float2<BF>(h.y);
            uint8_t *at = smem + row * pitch + 2 * (r0 + 32 * i);
            *reinterpret_cast<uint2 *>(at) = h;
            *reinterpret_cast<uint2 *>(at + 2 * width) = make_uint2(pack16<BF>(rest(f.x, h0.x), rest(f.y, h0.y)), pack16<BF>(rest(f.z, h1.x), rest(f.w, h1.y)));
        }
    }
    __syncthreads();
    if (n0 >= a.N) return;
    float out[2][kDeltaTiles][4] = {};      // [16 rows][8 columns]: rows g and g + 8, columns 2 t4 and 2 t4 + 1
    const uint32_t vs = smem_u32(smem) + g * pitch + 16 * t4;
    for (bool first = true; leads; leads &= leads - 1, first = false) {
        const int id = __shfl_sync(0xffffffffu, my_id, __ffs(leads) - 1);
        const uint32_t rows = __ballot_sync(0xffffffffu, my_id == id);
        float acc[2][kDeltaTiles][4] = {};
        for (int r = 0; r < width; r += 32) {
            if (!first || r) load_b(p, id, r + 8 * t4);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    const uint4 u = lds128(vs + 16 * m * pitch + part * 2 * width + 2 * r), w = lds128(vs + (16 * m + 8) * pitch + part * 2 * width + 2 * r);
#pragma unroll
                    for (int t = 0; t < kDeltaTiles; ++t) {
                        mma16<BF, false>(acc[m][t], u.x, w.x, u.y, w.y, register_pair(p[t].x, p[t].y));
                        mma16<BF, false>(acc[m][t], u.z, w.z, u.w, w.w, register_pair(p[t].z, p[t].w));
                    }
                }
        }
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int t = 0; t < kDeltaTiles; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (rows >> (16 * m + 8 * (i >> 1) + g) & 1) out[m][t][i] = acc[m][t][i];
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int row = 16 * m + 8 * half + g;
            if (row >= count) continue;
            const float by = unscale[row];
#pragma unroll
            for (int t = 0; t < kDeltaTiles; ++t) {
                const int n = n0 + 8 * t + 2 * t4;
                float lo = out[m][t][2 * half] * by, hi = out[m][t][2 * half + 1] * by;
                if (!isfinite(lo)) lo = long_expansion<BF>(a, m0 + row, n);
                if (!isfinite(hi)) hi = long_expansion<BF>(a, m0 + row, n + 1);
                *reinterpret_cast<uint32_t *>(delta + (size_t)(m0 + row) * a.N + n) = pack16<BF>(lo, hi);
            }
        }
}

// The product with W of up to 8 rows, plus the expansion.  The work is counted in pairs of units, 32 columns; a CTA takes a range of
// neighbouring ones, in tiles of two where they are half a panel, else of one.  As in the routed-expert kernels the warps share a
// tile's items along K, leave their sums and go on, and add up at the next tile's end.  W: 8 warps, two CTAs per SM; where there is no
// more than a pair of units for each SM, 16 warps and one (4096 x 4096, rank 16, one row, with the shrink kernel: 0.3 us
// less, now 6.3).
// 8 rows of 8 adapters, 4096 x 12288: 13.0 us with the shrink kernel, the shared matmul alone 8.5 in the decode kernel.  Neither issue (43 % of
// the slots) nor DRAM (22 %) is full: most of the stalls are waits for loads.
template <int W, int NU, int SUB, bool BF>
__global__ void __launch_bounds__(32 * W, 16 / W)
lora_gemm_kernel(const LoraArgs a, const __half *x, const uint8_t *qweight, const uint8_t *scales, const uint8_t *qzeros,
                 const TiledTrailer *trailer, __half *y)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ __align__(8) uint64_t arrived[2];
    __shared__ int s_ids[8];
    constexpr int kValues = 4 * NU, kThreads = 32 * W;
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const uint32_t bars = smem_u32(arrived);
    if (threadIdx.x == 0) {
        mbar_init(bars, W);
        mbar_init(bars + 8, W);
    }
    const uint32_t flags = __ldg(&trailer->flags);
    const int v_pitch = a.rank + 4;
    float *vs = reinterpret_cast<float *>(smem), *red = vs + 8 * v_pitch;      // [row][rank], [buffer][warp][value][lane]
    // where ranges differ the longer ones come first: the last CTAs may have to wait for the shrink kernel's to leave their SMs
    const int G = a.K / kGroup, each = a.N / 32 / gridDim.x, more = a.N / 32 - each * gridDim.x;
    const int t0 = blockIdx.x * each + min((int)blockIdx.x, more), t1 = t0 + each + ((int)blockIdx.x < more ? 1 : 0);
    auto width = [&](int pair) { return NU == 4 && (pair & 1) == 0 && pair + 1 < t1 ? 2 : 1; };
    // x and the ids are older than the kernel before this one, which waited for them before it let this one in
    if (threadIdx.x < 8) s_ids[threadIdx.x] = (int)threadIdx.x < a.M ? __ldg(a.ids + threadIdx.x) : -1;
    __syncthreads();
    pdl_launch_dependents();
    const __half *row = x + (size_t)min(g, a.M - 1) * a.K + 8 * t4;
    // the rows of B that the epilogue will want, on their way to L2
    for (int i = threadIdx.x; i < a.M * (t1 - t0) * 32; i += kThreads) {
        const int id = s_ids[i % a.M];
        if ((unsigned)id >= (unsigned)a.adapters) continue;
        const __half *p = a.b + ((size_t)id * a.N + 32 * t0 + i / a.M) * a.rank;
        for (int r = 0; r < a.rank; r += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + r));
    }
    int l_pair = t0, l_next = t0, l_item = G, l_turn = warp - 1;
    LanePtrs<SUB> ptrs{};
    auto next = [&](DirectItem<SUB> &it) {
        l_item += W;
        while (l_item >= G) {
            if (l_next >= t1) {
                it.tag = -1;
                return;
            }
            l_pair = l_next;
            l_next += width(l_pair);
            l_item = ++l_turn & (W - 1);
            ptrs = lane_ptrs<false, SUB>(unit_ptrs<SUB>(qweight, scales, qzeros, l_pair >> 2, G, 2 * (l_pair & 3)), lane);
        }
        set_item<SUB>(it, ptrs, row, l_item, lane);
        it.flags = flags;
        it.tag = l_pair;
        it.pairs = l_next - l_pair;
    };
    const bool layout_ok = (flags & kFormatGateUp) == 0 && ((flags & kFormatBf16) != 0) == BF;
    if (!layout_ok && threadIdx.x == 0) atomicMax(&g_device_status, (int)kStatusLayoutMismatch);
    float acc[NU][4] = {};
    int pair = t0, left = t0, tiles = 0;      // the tile at hand, the one before it, how many came before
    auto add_up = [&]() {
        const int done = tiles - 1;
        if (done == 0) {
            // v is there, and y no longer in use by earlier kernels
            pdl_wait();
            for (int i = 4 * threadIdx.x; i < a.M * a.rank; i += 4 * kThreads) {
                const int m = i / a.rank, r = i - m * a.rank;
                float4 v[1];
                lora_v(a, m, r, v);
                *reinterpret_cast<float4 *>(vs + m * v_pitch + r) = v[0];
            }
            __syncthreads();
        }
        if (!mbar_wait(bars + 8 * (done & 1), (done >> 1) & 1)) return;
        const float *buf = red + (done & 1) * (W * kValues * 32);
        for (int o = threadIdx.x; o < width(left) * 256; o += kThreads) {
            const int v = o >> 5, i = v & 3, m = 2 * t4 + (i & 1), n = 32 * left + 16 * (v >> 2) + g + 8 * (i >> 1);
            if (m >= a.M || !layout_ok) continue;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) sum += buf[(w * kValues + v) * 32 + lane];
            if (needs_long_sum<BF>(sum)) {
                const UnitPtrs p = unit_ptrs<SUB>(qweight, scales, qzeros, n / kPanel, G, n % kPanel / 16);
                sum = long_sum<BF>(p.w, p.s, p.z, SUB, n % 16, flags & kFormatZerosMinusOne, x + (size_t)m * a.K, G, false);
            }
            const int id = s_ids[m];
            if ((unsigned)id < (unsigned)a.adapters) {
                const uint4 *b = reinterpret_cast<const uint4 *>(a.b + ((size_t)id * a.N + n) * a.rank);
                float part = 0.f;
                for (int c = 0; c < a.rank / 8; ++c) {
                    const uint4 p = __ldg(b + c);
                    const float4 lo = *reinterpret_cast<const float4 *>(vs + m * v_pitch + 8 * c), hi = *reinterpret_cast<const float4 *>(vs + m * v_pitch + 8 * c + 4);
                    const float2 p0 = pair_to_float2<BF>(p.x), p1 = pair_to_float2<BF>(p.y), p2 = pair_to_float2<BF>(p.z), p3 = pair_to_float2<BF>(p.w);
                    part = fmaf(p0.x, lo.x, part), part = fmaf(p0.y, lo.y, part), part = fmaf(p1.x, lo.z, part), part = fmaf(p1.y, lo.w, part);
                    part = fmaf(p2.x, hi.x, part), part = fmaf(p2.y, hi.y, part), part = fmaf(p3.x, hi.z, part), part = fmaf(p3.y, hi.w, part);
                }
                sum += part;
            }
            store_out16<BF>(y + (size_t)m * a.N + n, sum);
        }
    };
    auto finish_tile = [&]() {
        if (tiles) add_up();
        float *buf = red + (tiles & 1) * (W * kValues * 32);
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                buf[(warp * kValues + 4 * u + i) * 32 + lane] = acc[u][i];
                acc[u][i] = 0.f;
            }
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * (tiles & 1));
        left = pair;
        pair += width(pair);
        ++tiles;
    };
    const uint32_t ring = smem_u32(red + 2 * W * kValues * 32) + warp * direct_ring_bytes<NU, SUB>(1);
    stream_items<NU, false, SUB, BF, false>(ring, lane, a.one, acc, next, [] {}, [&](int t) { while (pair < t) finish_tile(); });
    while (pair < t1) finish_tile();
    if (tiles) add_up();
}

// The parts of K that the shrink kernel sums apart: so many that a warp has one batch of steps - a second one costs a round trip to
// memory - as long as the CTAs are not too many anyway.  Whole calls: 64 rows of 64 adapters of 5120 x 5120 x 32 32.8 us with five parts, 33.9
// with four; 13 rows of 11008 x 4096 x 64 21.8 with eleven, 22.2 with eight, 23.9 with four; one row of 11008 x 4096 x 16, where adding the parts up
// counts for more, 10.4, 10.1 and 9.9.  750 or 4000 CTAs at most make no difference to these.
constexpr int kLoraMaxParts = 12, kLoraMaxCtas = 1500;
inline int lora_k_parts(int M, int K, int rank)
{
    const long long ctas = (long long)((M + 7) / 8) * ((rank + 15) / 16) * (M < 8 ? M : M <= kLoraDecodeRows ? 8 : 1);
    const int steps = kLoraWarps * kLoraSteps, most = kLoraMaxCtas / ctas < 1 ? 1 : kLoraMaxCtas / ctas > kLoraMaxParts ? kLoraMaxParts : (int)(kLoraMaxCtas / ctas);
    const int parts = (K / 32 + steps - 1) / steps;
    return parts < most ? parts : most;
}

// Rows of v over all parts that a call of M rows, or of fewer, writes at most: who has registered for the largest call has enough.  parts x
// rows of m rows is m, or as many parts as K has x m and no more than 1500 / ctas x m, which is at most 1500 per 16 of the rank up to
// kLoraDecodeRows rows and 8 times that above.
inline size_t lora_v_rows(int M, int K, int rank)
{
    const long long ranks = (rank + 15) / 16, all = (long long)M * lora_k_parts(1, K, 16);      // (one row and rank 16: as many as K has)
    const long long most = (M <= kLoraDecodeRows ? kLoraMaxCtas : 8 * kLoraMaxCtas) / ranks, rows = all < most ? all : most;
    return (size_t)(rows > M ? rows : M);
}

// scratch: [x in the sorted order][v][expansion]
struct LoraScratch {
    size_t x_perm, v, delta, total;
};
inline LoraScratch lora_scratch(int M, int N, int K, int rank, int act_order)
{
    auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
    LoraScratch l;
    l.x_perm = 0;
    l.v = act_order == 1 ? up((size_t)M * K * 2) : 0;
    l.delta = l.v + up(lora_v_rows(M, K, rank) * rank * 4);
    l.total = l.delta + (M > kLoraDirectRows ? up((size_t)M * N * 2) : 0);
    return l;
}

// perm, x_sorted: see the kernel; nullptr without
int launch_lora_shrink(const LoraArgs &a, const int32_t *perm, __half *x_sorted, int bf16, cudaStream_t s)
{
    // decode batches: a CTA per adapter of eight rows; prompts: one CTA takes them in turn (mostly there is one)
    const int apart = a.M < 8 ? a.M : a.M <= kLoraDecodeRows ? 8 : 1, ranks = (a.rank + 15) / 16;
    const int per_row = (a.K / 2 + kLoraThreads - 1) / kLoraThreads, slices = perm ? (per_row + ranks - 1) / ranks : 0;
    const dim3 grid((unsigned)((a.M + 7) / 8), (unsigned)ranks, (unsigned)(apart * a.k_parts + slices));
    return bf16 ? launch_dependent(lora_shrink_kernel<true>, grid, kLoraThreads, 0, 1, s, a, apart, perm, x_sorted)
                : launch_dependent(lora_shrink_kernel<false>, grid, kLoraThreads, 0, 1, s, a, apart, perm, x_sorted);
}
int launch_lora_delta(const LoraArgs &a, __half *delta, int bf16, cudaStream_t s)
{
    if (a.M <= kLoraDecodeRows) {
        const int per_cta = 8 * kDeltaSteps * (32 / (a.rank / 8));
        const dim3 grid((unsigned)((a.N + per_cta - 1) / per_cta), (unsigned)a.M);
        return bf16 ? launch_dependent(lora_delta_rows_kernel<true>, grid, 256, 0, 1, s, a, delta)
                    : launch_dependent(lora_delta_rows_kernel<false>, grid, 256, 0, 1, s, a, delta);
    }
    // a grid is 65535 blocks high: more blocks of rows lie in layers
    const int blocks = (a.M - 1) / kDeltaRows + 1, layers = (blocks - 1) / 32768 + 1;
    const dim3 grid((unsigned)((a.N + 255) / 256), (unsigned)((blocks - 1) / layers + 1), (unsigned)layers);
    const size_t smem = (size_t)kDeltaRows * (2 * ((a.rank + 31) & ~31) * 2 + 16);      // at most 33 KB
    return bf16 ? launch_dependent(lora_delta_runs_kernel<true>, grid, 256, smem, 1, s, a, delta)
                : launch_dependent(lora_delta_runs_kernel<false>, grid, 256, smem, 1, s, a, delta);
}

template <int W, int NU, int SUB, bool BF>
static int launch_lora_gemm_warps(const LoraArgs &a, const __half *x, const void *qweight, const void *scales, const void *qzeros,
                                  __half *y, cudaStream_t s)
{
    const TiledTrailer *trailer = reinterpret_cast<const TiledTrailer *>((const uint8_t *)qzeros + tiled_zero_bytes(a.N, a.K, kGroup / SUB));
    const int smem = 8 * (a.rank + 4) * 4 + 2 * W * 4 * NU * 32 * 4 + direct_ring_bytes<NU, SUB>(W);
    static int configured[64] = {};
    const int st = ensure_dynamic_smem((const void *)lora_gemm_kernel<W, NU, SUB, BF>, configured, smem);
    if (st) return st;
    const int pairs = a.N / 32, slots = 16 / W * a.sms;
    return launch_sharing_sm(lora_gemm_kernel<W, NU, SUB, BF>, dim3((unsigned)(pairs < slots ? pairs : slots)), 32 * W, (size_t)smem, 1, 16 / W, s, a, x,
                            (const uint8_t *)qweight, (const uint8_t *)scales, (const uint8_t *)qzeros, trailer, y);
}
template <int SUB, bool BF>
static int launch_lora_gemm_sub(const LoraArgs &a, const __half *x, const void *qweight, const void *scales, const void *qzeros,
                                __half *y, cudaStream_t s)
{
    if (a.N / 32 <= a.sms) return launch_lora_gemm_warps<16, 2, SUB, BF>(a, x, qweight, scales, qzeros, y, s);
    return launch_lora_gemm_warps<8, SUB == 4 ? 2 : 4, SUB, BF>(a, x, qweight, scales, qzeros, y, s);
}
// x: in the row order of the tiled layer
int launch_lora_gemm(const LoraArgs &a, const __half *x, const void *qweight, const void *scales, const void *qzeros, __half *y,
                     int group_size, int bf16, cudaStream_t s)
{
    switch ((bf16 ? 10 : 0) + kGroup / group_size) {
    case 1: return launch_lora_gemm_sub<1, false>(a, x, qweight, scales, qzeros, y, s);
    case 2: return launch_lora_gemm_sub<2, false>(a, x, qweight, scales, qzeros, y, s);
    case 4: return launch_lora_gemm_sub<4, false>(a, x, qweight, scales, qzeros, y, s);
    case 11: return launch_lora_gemm_sub<1, true>(a, x, qweight, scales, qzeros, y, s);
    case 12: return launch_lora_gemm_sub<2, true>(a, x, qweight, scales, qzeros, y, s);
    default: return launch_lora_gemm_sub<4, true>(a, x, qweight, scales, qzeros, y, s);
    }
}

}  // namespace gptq

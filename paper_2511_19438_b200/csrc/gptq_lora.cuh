// A shared projection with a low-rank adapter per row: y[m] = x[m] W + scale[a] (x[m] A[a]^T) B[a]^T, a = adapter_ids[m].
//
// v[m] = scale[a] x[m] A[a]^T is formed first, in fp32, by a small kernel (`lora_shrink_kernel`).  Up to 16 rows the product with
// W and the expansion v B^T are one kernel: its weights and x are under way while v is still being formed, the expansion joins
// the fp32 sums in the epilogue and y is rounded once.  Above that the expansion is written out (16 bits) and joins the tcgen05
// kernels' fp32 sums as their residual.
#pragma once
#include "gptq_common.cuh"
#include "gptq_direct.cuh"

namespace gptq {

constexpr int kLoraMaxRank = 256;
constexpr int kLoraDirectRows = 16;      // rows of the fused kernel
constexpr int kLoraWarps = 8, kLoraThreads = 32 * kLoraWarps;

struct LoraArgs {
    const __half *x;          // [M, K] as given
    const __half *a, *b;      // [adapters, rank, K], [adapters, N, rank]
    const int32_t *ids;       // [M]
    const float *scales;      // [adapters] or nullptr
    float *v;                 // [M, rank]
    int M, N, K, rank, adapters;
};

template <bool BF>
__device__ __forceinline__ float dot8(const uint4 &p, const uint4 &q, float sum)
{
    const uint32_t a[4] = {p.x, p.y, p.z, p.w}, b[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 u = pair_to_float2<BF>(a[i]), w = pair_to_float2<BF>(b[i]);
        sum = fmaf(u.x, w.x, sum);
        sum = fmaf(u.y, w.y, sum);
    }
    return sum;
}

// A warp forms one element of v.
template <bool BF>
__global__ void __launch_bounds__(kLoraThreads) lora_shrink_kernel(const LoraArgs a)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, m = blockIdx.y, r = blockIdx.x * kLoraWarps + warp;
    pdl_wait();
    pdl_launch_dependents();        // (behind the wait: what x was before this kernel is what the next one may read at once)
    const int id = __ldg(a.ids + m);
    if ((unsigned)id >= (unsigned)a.adapters || r >= a.rank) return;
    const uint4 *xr = reinterpret_cast<const uint4 *>(a.x + (size_t)m * a.K);
    const uint4 *ar = reinterpret_cast<const uint4 *>(a.a + ((size_t)id * a.rank + r) * a.K);
    float sum = 0.f;
#pragma unroll 4
    for (int c = lane; c < a.K / 8; c += 32) sum = dot8<BF>(__ldg(xr + c), ldg_stream128(ar + c), sum);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) a.v[(size_t)m * a.rank + r] = a.scales ? sum * __ldg(a.scales + id) : sum;
}

// (v B^T)[m][n]; v is read after the kernel that wrote it has finished
template <bool BF>
__device__ __forceinline__ float lora_expand(const LoraArgs &a, int m, int n)
{
    const int id = __ldg(a.ids + m);
    if ((unsigned)id >= (unsigned)a.adapters) return 0.f;
    const uint4 *b = reinterpret_cast<const uint4 *>(a.b + ((size_t)id * a.N + n) * a.rank);
    const float4 *v = reinterpret_cast<const float4 *>(a.v + (size_t)m * a.rank);
    float sum = 0.f;
    for (int c = 0; c < a.rank / 8; ++c) {
        const uint4 p = __ldg(b + c);
        const float4 lo = v[2 * c], hi = v[2 * c + 1];
        const float2 p0 = pair_to_float2<BF>(p.x), p1 = pair_to_float2<BF>(p.y), p2 = pair_to_float2<BF>(p.z), p3 = pair_to_float2<BF>(p.w);
        sum = fmaf(p0.x, lo.x, sum), sum = fmaf(p0.y, lo.y, sum), sum = fmaf(p1.x, lo.z, sum), sum = fmaf(p1.y, lo.w, sum);
        sum = fmaf(p2.x, hi.x, sum), sum = fmaf(p2.y, hi.y, sum), sum = fmaf(p3.x, hi.z, sum), sum = fmaf(p3.y, hi.w, sum);
    }
    return sum;
}

template <bool BF>
__global__ void __launch_bounds__(256) lora_delta_kernel(const LoraArgs a, __half *__restrict__ delta)
{
    pdl_launch_dependents();
    pdl_wait();
    const int n = blockIdx.x * 256 + threadIdx.x, m = blockIdx.y;
    if (n < a.N) store_out16<BF>(delta + (size_t)m * a.N + n, lora_expand<BF>(a, m, n));
}

// The product with W of up to 8 NT rows, 16 NU columns per CTA, the items along K shared by its warps, plus the expansion.
template <int NT, int NU, int SUB, bool BF>
__global__ void __launch_bounds__(kLoraThreads, NT == 1 ? 2 : 1)
lora_gemm_kernel(const LoraArgs a, const __half *x, const uint8_t *qweight, const uint8_t *scales, const uint8_t *qzeros,
                 const TiledTrailer *trailer, __half *y)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const uint32_t flags = __ldg(&trailer->flags);
    const int G = a.K / kGroup, panel = blockIdx.x / (8 / NU), unit = blockIdx.x % (8 / NU) * NU;
    const UnitPtrs ptrs = unit_ptrs<SUB>(qweight, scales, qzeros, panel, G, unit, lane);
    const __half *rows[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) rows[t] = 8 * t + g < a.M ? x + (size_t)(8 * t + g) * a.K + 8 * t4 : nullptr;
    pdl_launch_dependents();
    float acc[NU][NT][4] = {};
    constexpr int D = 2;
    DirectRegs<NT, NU, SUB> regs[D];
    const int n = (G - warp + kLoraWarps - 1) / kLoraWarps;
    // x is older than the kernel before this one, which waited for it before it let this one in
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (d < n) {
            load_item_weights<NT, NU, 1, SUB>(regs[d], ptrs, warp + d * kLoraWarps);
            load_item_rows<NT, NU, SUB>(regs[d], rows, warp + d * kLoraWarps);
        }
    for (int i = 0; i < n; i += D)
#pragma unroll
        for (int d = 0; d < D; ++d)
            if (i + d < n) {
                multiply_item<NT, NU, SUB, BF>(regs[d], flags & kFormatZerosMinusOne, acc);
                if (i + d + D < n) {
                    load_item_weights<NT, NU, 1, SUB>(regs[d], ptrs, warp + (i + d + D) * kLoraWarps);
                    load_item_rows<NT, NU, SUB>(regs[d], rows, warp + (i + d + D) * kLoraWarps);
                }
            }
    const bool layout_ok = (flags & kFormatGateUp) == 0 && ((flags & kFormatBf16) != 0) == BF;
    if (!layout_ok && threadIdx.x == 0) atomicMax(&g_device_status, (int)kStatusLayoutMismatch);
    float *red = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) red[((warp * NU + u) * (4 * NT) + 4 * t + i) * 32 + lane] = acc[u][t][i];
    __syncthreads();
    pdl_wait();      // v; and y may still be in use by earlier kernels until here
    for (int o = threadIdx.x; o < NU * NT * 4 * 32; o += kLoraThreads) {
        const int v = o >> 5, u = v / (4 * NT), t = v % (4 * NT) / 4, i = v & 3;
        const int m = 8 * t + 2 * t4 + (i & 1), col = panel * kPanel + 16 * (unit + u) + g + 8 * (i >> 1);
        if (m >= a.M || !layout_ok) continue;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kLoraWarps; ++w) sum += red[(w * (NU * NT * 4) + v) * 32 + lane];
        store_out16<BF>(y + (size_t)m * a.N + col, sum + lora_expand<BF>(a, m, col));
    }
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
    l.delta = l.v + up((size_t)M * rank * 4);
    l.total = l.delta + (M > kLoraDirectRows ? up((size_t)M * N * 2) : 0);
    return l;
}

int launch_lora_shrink(const LoraArgs &a, int bf16, cudaStream_t s)
{
    const dim3 grid((unsigned)((a.rank + kLoraWarps - 1) / kLoraWarps), (unsigned)a.M);
    return bf16 ? launch_dependent(lora_shrink_kernel<true>, grid, kLoraThreads, 0, 1, s, a)
                : launch_dependent(lora_shrink_kernel<false>, grid, kLoraThreads, 0, 1, s, a);
}
int launch_lora_delta(const LoraArgs &a, __half *delta, int bf16, cudaStream_t s)
{
    const dim3 grid((unsigned)((a.N + 255) / 256), (unsigned)a.M);
    return bf16 ? launch_dependent(lora_delta_kernel<true>, grid, 256, 0, 1, s, a, delta)
                : launch_dependent(lora_delta_kernel<false>, grid, 256, 0, 1, s, a, delta);
}

template <int NT, int SUB, bool BF>
static int launch_lora_gemm_nt(const LoraArgs &a, const __half *x, const void *qweight, const void *scales, const void *qzeros,
                               __half *y, cudaStream_t s)
{
    const TiledTrailer *trailer = reinterpret_cast<const TiledTrailer *>((const uint8_t *)qzeros + tiled_zero_bytes(a.N, a.K, kGroup / SUB));
    constexpr int NU = NT;
    const int smem = kLoraWarps * NU * NT * 4 * 32 * 4;
    return launch_dependent(lora_gemm_kernel<NT, NU, SUB, BF>, dim3((unsigned)(a.N / (16 * NU))), kLoraThreads, (size_t)smem, 1, s, a, x,
                            (const uint8_t *)qweight, (const uint8_t *)scales, (const uint8_t *)qzeros, trailer, y);
}
template <int SUB, bool BF>
static int launch_lora_gemm_sub(const LoraArgs &a, const __half *x, const void *qweight, const void *scales, const void *qzeros,
                                __half *y, cudaStream_t s)
{
    return a.M <= 8 ? launch_lora_gemm_nt<1, SUB, BF>(a, x, qweight, scales, qzeros, y, s)
                    : launch_lora_gemm_nt<2, SUB, BF>(a, x, qweight, scales, qzeros, y, s);
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

// Layers in 8-bit floating point (e4m3 with a scale for each block of 128): rows to e4m3, products, the gated block and its gradients.
//
//     y[m, n] = sum_kb sx[m, kb] sw[n / 128, kb] sum_{k in block kb} qx[m, k] qw[n, k]
//
// The inner sum is an MMA of e4m3 operands with fp32 accumulators; a scale that changes every 128 of K cannot stay outside the whole
// sum, so each block of K gets an accumulator of its own in tensor memory and the warps that drain it add it, times its scale, to
// sums in registers.
#pragma once
#include "gptq_prefill.cuh"      // tcgen05, cluster and stage helpers
#include "gptq_umma2.cuh"        // CTA pairs

namespace gptq {

constexpr int kFp8Block = 128;                        // columns (and weight rows) per scale
constexpr float kFp8Max = 448.0f, kFp8ScaleMin = 1.17549435e-38f;      // largest e4m3 number; 2^-126
__host__ __device__ inline int fp8_blocks(int n) { return (n - 1) / kFp8Block + 1; }      // (n up to 2^31 - 1)

// ---- rows of numbers to e4m3 -------------------------------------------------------------------------------------------
// s = max(max|v| / 448, 2^-126), q = e4m3(v / s): both divisions to the nearest, since with 16-bit v the quotient lies exactly in the
// middle of two e4m3 numbers often (1 of 128 elements where v / max|v| has few digits), and a last bit would decide.
// `top`: the bits of max|v|, by integer maximum, so that a NaN wins over an infinity and both over numbers.
__device__ __forceinline__ float fp8_scale(uint32_t top)
{
    const float s = __fdiv_rn(__uint_as_float(top), kFp8Max);      // (an infinity or NaN stays one: the whole block becomes NaN)
    return s < kFp8ScaleMin ? kFp8ScaleMin : s;
}
// v / s for many v of one s, to be rounded to e4m3: the correction step of Markstein's division (IBM J. Res. Dev. 34, 1990).  With y the nearest number
// to 1 / s, q = v y is off by 2 * 2^-24 of itself at most, v - q s (one rounding) and y by 2^-24 each: q + (v - q s) y lies within 2^-46 of v / s before its
// own rounding.  It can be another number than the nearest to v / s only if v / s is that near the middle of two, and another e4m3 number
// only if that middle is beside the middle of two e4m3 numbers: 205 pairs of significands come so near, and all give the same (a host test goes through
// them).  Small blocks are scaled first, so that the remainder does not underflow.  (The operator's own division leaves its fast way for zeros: padding
// rows made a gated call of 1000 rows 26 us instead of 16.)
struct Fp8Quotient {
    float s, y;
    bool small;
    __device__ __forceinline__ explicit Fp8Quotient(float scale)
    {
        small = scale < 0x1p-60f;
        s = small ? scale * 0x1p64f : scale;
        y = __frcp_rn(s);
    }
    __device__ __forceinline__ float operator()(float v) const
    {
        if (small) v *= 0x1p64f;
        const float q = v * y;
        return fmaf(fmaf(-q, s, v), y, q);
    }
};
// two numbers to e4m3, nearest even; a in the low byte; NaN becomes NaN, what rounds beyond 448 becomes 448
__device__ __forceinline__ uint32_t fp8_pair(float a, float b)
{
    unsigned short v;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(v) : "f"(b), "f"(a));
    return v;
}
__device__ __forceinline__ uint32_t fp8_four(float a, float b, float c, float d) { return fp8_pair(a, b) | fp8_pair(c, d) << 16; }
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// loads that stay behind the wait for earlier kernels
__device__ __forceinline__ uint4 ldg_behind(const void *p)
{
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint2 ldg64_behind(const void *p)
{
    uint2 v;
    asm volatile("ld.global.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ float ldgf_behind(const float *p)
{
    float v;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p));
    return v;
}
// Eight lanes per block of 128: a lane has numbers 8 l .. 8 l + 7 and 64 + 8 l .., two loads of 16 bytes.  Bound by instruction issue and by
// memory alike: with sixteen lanes per block, maxima of fp32 bits and the operator's own division 4096 x 11008 took 46 us, as it is 24.8 (floor 21);
// more blocks of a group requested together made it slower (two 26.1, four 30.7; 300 x 4096 2.3, 3.4 and 4.6).
constexpr int kFp8QuantThreads = 256, kFp8QuantLanes = 8, kFp8QuantCtasPerSm = 16;
template <bool BF>
__global__ void __launch_bounds__(kFp8QuantThreads) fp8_quantize_kernel(const uint4 *x, uint2 *q, float *scales, int K, int KB, long long blocks)
{
    pdl_launch_dependents();
    pdl_wait();
    constexpr int kPer = kFp8QuantThreads / kFp8QuantLanes, kInWarp = 32 / kFp8QuantLanes;
    const int l = threadIdx.x % kFp8QuantLanes;
    // group h of eight lanes has blocks h, h + groups, ... (row after row); the step as rows and blocks: only the first takes a division
    const long long groups = (long long)gridDim.x * kPer, step_row = groups / KB;
    const int step_kb = (int)(groups - step_row * KB);
    long long b = (long long)blockIdx.x * kPer + threadIdx.x / kFp8QuantLanes, row = b / KB;
    int kb = (int)(b - row * KB);
    // (a warp's groups go on together: the maximum is found by the whole warp)
    for (; b - threadIdx.x / kFp8QuantLanes % kInWarp < blocks; b += groups) {
        const int k = kb * kFp8Block + l * 8;
        const size_t at = ((size_t)row * K + k) / 8;
        uint32_t w[8], top = 0;
        bool in[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            in[h] = b < blocks && k + 64 * h < K;
            const uint4 v = in[h] ? ldg_behind(x + at + 8 * h) : make_uint4(0, 0, 0, 0);
            w[4 * h] = v.x, w[4 * h + 1] = v.y, w[4 * h + 2] = v.z, w[4 * h + 3] = v.w;
        }
        // 16-bit numbers without their signs are ordered as integers, NaN above all
#pragma unroll
        for (int j = 0; j < 8; ++j) top = __vmaxu2(top, w[j] & 0x7fff7fffu);
#pragma unroll
        for (int o = kFp8QuantLanes / 2; o; o >>= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float2 tops = pair_to_float2<BF>(top);
        const float s = fp8_scale(max(__float_as_uint(tops.x), __float_as_uint(tops.y)));
        const Fp8Quotient by(s);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float2 f[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f[j] = pair_to_float2<BF>(w[4 * h + j]);
                f[j] = make_float2(by(f[j].x), by(f[j].y));
            }
            if (in[h]) q[at + 8 * h] = make_uint2(fp8_four(f[0].x, f[0].y, f[1].x, f[1].y), fp8_four(f[2].x, f[2].y, f[3].x, f[3].y));
        }
        if (l == 0 && b < blocks) scales[b] = s;
        row += step_row, kb += step_kb;
        if (kb >= KB) kb -= KB, ++row;
    }
}

// ---- a layer the other way round ---------------------------------------------------------------------------------------
// [N, K] -> [K, N], scales likewise; a tile of 64 x 64 bytes per CTA.  Runs once per layer.
__global__ void __launch_bounds__(256) fp8_transpose_kernel(const uint8_t *w, const float *scales, uint8_t *w_out, float *scales_out, int N, int K)
{
    __shared__ uint8_t tile[64][68];
    const int tiles_k = (K - 1) / 64 + 1;
    const int n0 = (int)(blockIdx.x / tiles_k) * 64, k0 = (int)(blockIdx.x % tiles_k) * 64;
    const int r = threadIdx.x / 4, c = threadIdx.x % 4 * 16;
    if (n0 + r < N && k0 + c < K) {
        const uint4 v = *reinterpret_cast<const uint4 *>(w + (size_t)(n0 + r) * K + k0 + c);
        uint32_t *t = reinterpret_cast<uint32_t *>(&tile[r][c]);
        t[0] = v.x, t[1] = v.y, t[2] = v.z, t[3] = v.w;
    }
    __syncthreads();
    if (k0 + r < K && n0 + c < N) {
        uint32_t v[4];
        for (int j = 0; j < 4; ++j)
            v[j] = tile[c + 4 * j][r] | tile[c + 4 * j + 1][r] << 8 | tile[c + 4 * j + 2][r] << 16 | (uint32_t)tile[c + 4 * j + 3][r] << 24;
        *reinterpret_cast<uint4 *>(w_out + (size_t)(k0 + r) * N + n0 + c) = make_uint4(v[0], v[1], v[2], v[3]);
    }
    if (threadIdx.x == 0 && n0 % kFp8Block == 0 && k0 % kFp8Block == 0)
        scales_out[(size_t)(k0 / kFp8Block) * fp8_blocks(N) + n0 / kFp8Block] = scales[(size_t)(n0 / kFp8Block) * fp8_blocks(K) + k0 / kFp8Block];
}

// ---- many rows: CTA pairs, tiles of 256 token rows x 256 weight rows ------------------------------------------------------
// A persistent pair of CTAs (two SMs) multiplies a tile with tcgen05.mma.cta_group::2: each CTA loads 128 token rows (its lanes of the
// accumulator) and 128 of the 256 weight rows, a block of K (32 KB) per stage.  The accumulator alternates between two halves of tensor
// memory, one block of K each, so that a block is drained while the next is multiplied.  Token rows are the MMA's rows: a thread that
// drains holds one token row, hence one scale per block of K and weight block.  A drain warp has 2 x 64 of the tile's columns; in the gated
// kinds these are gate and up of the same 64 columns, so that the activation needs no exchange but the maximum over two warps.
//   warps 0, 3  TMA of this CTA's halves, weights and activations (a turn of such a loop takes its thread 210 clocks whatever the
//           copy's size); both CTAs' copies complete on the leader's barrier
//   warp 1  the MMAs (the leader's)
//   warp 2  products of scales, two blocks ahead: 128 rows x 2 weight blocks per block of K into a ring of four
//   warps 4 to 11 drain.  The first four give registers to them: 128 sums and 32 columns on their way.
// What bounds it, by stamps of %clock: two accumulators, so that two blocks of K take an MMA (512 clocks), a drain (720) and both ways between the
// MMA thread and the drain warps of two SMs (800): 1000 clocks per block; and the power limit (1.5 to 1.7 GHz in that loop).  4096 x 4096 x 12288: 199 us (2.07
// PFLOP/s) on a cool card to 230 at the power limit.  Tried and slower: accumulators of half a tile, four of them (304 us: the MMAs read their rows twice, and the drain warps wait twice as
// often), 16 drain warps (304: instruction issue), one CTA per tile of 128 x 256 (356; gated kinds the same), results sent during the next tile (255).
constexpr int kFp8TileM = 256, kFp8TileN = 256, kFp8HalfM = 128, kFp8Stages = 4;
constexpr int kFp8FirstDrain = 4, kFp8DrainWarps = 8, kFp8Threads = 32 * (kFp8FirstDrain + kFp8DrainWarps);
constexpr int kFp8LaunchRegs = 168, kFp8FewRegs = 72, kFp8ManyRegs = 216;
static_assert(kFp8FewRegs + 2 * kFp8ManyRegs <= 3 * kFp8LaunchRegs, "three warpgroups share what the CTA was launched with");
constexpr int kFp8HalfBytes = kFp8HalfM * kFp8Block, kFp8StageBytes = 2 * kFp8HalfBytes;
constexpr int kFp8OutBytes = 32 * 128;      // 32 rows of 64 16-bit columns, in and out: two per drain warp
constexpr int kFp8ScaleSlots = 4, kFp8ScaleBytes = 2 * kFp8HalfM * 4;
constexpr int kFp8SmemBytes = 2048 + kFp8Stages * kFp8StageBytes + 2 * kFp8DrainWarps * kFp8OutBytes + kFp8ScaleSlots * kFp8ScaleBytes;
static_assert(kFp8SmemBytes <= 227 * 1024 && 2 * kFp8SmemBytes > 227 * 1024, "one CTA per SM: it takes all tensor memory");

enum Fp8Kind : int { kFp8Plain = 0, kFp8Gated = 1, kFp8Backward = 2 };

struct Fp8Args {
    const float *x_scales, *w_scales;      // [M, KB], [blocks of N, KB]
    const __half *bias;                    // [N] or nullptr
    float *out_scales;                     // gated kinds: the result is e4m3 with these scales; nullptr: 16 bits
    int M, N, K, KB;                       // gated kinds: N = 2 F
    int tiles_m, tiles_n;
};

__device__ __forceinline__ void umma_f8_ss_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// tiled load into this CTA's shared memory that completes on a barrier of either CTA of the pair
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t cluster_bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(cluster_bar)
        : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t src, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(c0), "r"(c1), "r"(src)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void tma_store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// A converged warp's wait in few instructions and without a call: what is live in the drain warps fills the registers, and a call
// would have it stored.  A lane's try is its own, limited in time: the warp goes on once every lane has seen the phase end.
__device__ __forceinline__ bool mbar_wait_warp_inline(uint32_t bar, uint32_t parity)
{
    uint64_t start = 0;
    for (;;) {
#pragma unroll 1
        for (int n = 0; n < 4096; ++n)
            if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
        const uint64_t now = global_timer_ns();
        if (start == 0) start = now;
        if (__any_sync(0xffffffffu, now - start > kWaitLimitNs)) break;
    }
    atomicMax(&g_device_status, (int)kStatusWaitTimeout);
    return false;
}
template <int REGS> __device__ __forceinline__ void setmaxnreg_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS)); }
template <int REGS> __device__ __forceinline__ void setmaxnreg_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS)); }
// Two fp32 multiply-adds in one instruction.  (volatile: lo and hi come from tensor memory and are not there before the wait in front.)
__device__ __forceinline__ void fma2(uint64_t &acc, uint32_t lo, uint32_t hi, uint64_t s)
{
    asm volatile("{\n\t.reg .b64 v;\n\tmov.b64 v, {%1, %2};\n\tfma.rn.f32x2 %0, v, %3, %0;\n\t}" : "+l"(acc) : "r"(lo), "r"(hi), "l"(s));
}
__device__ __forceinline__ uint64_t both(float s)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %1};" : "=l"(v) : "r"(__float_as_uint(s)));
    return v;
}
__device__ __forceinline__ float2 unpack2(uint64_t v)
{
    uint32_t lo, hi;
    asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(v));
    return make_float2(__uint_as_float(lo), __uint_as_float(hi));
}
__device__ __forceinline__ uint64_t pack2(float2 f)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(__float_as_uint(f.x)), "r"(__float_as_uint(f.y)));
    return v;
}
// silu(g) * u; p is the logistic function (0 where it is below 2^-126)
__device__ __forceinline__ float logistic(float g) { return __frcp_rn(1.0f + __expf(-g)); }

// tile number -> (row of tiles, column of tiles): columns outermost within groups of 8 rows of tiles, so that what runs at the same time shares
// both operands in L2
__device__ __forceinline__ void fp8_tile(int t, int tiles_m, int tiles_n, int &tm, int &tn)
{
    constexpr int kRows = 8;
    const int group = t / (kRows * tiles_n), first = group * kRows;
    const int rows = min(kRows, tiles_m - first);
    const int in = t - group * kRows * tiles_n;
    tm = first + in % rows;
    tn = in / rows;
}

// IN: plain products have a residual (gated: nothing, backward: the gradient of the result in its place)
template <int KIND, bool BF, bool OUT8, bool IN>
__global__ void __launch_bounds__(kFp8Threads, 1)
fp8_tiles_kernel(const Fp8Args a, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map,
                 const __grid_constant__ CUtensorMap in_map, const __grid_constant__ CUtensorMap out_map)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    // full (the leader's): both CTAs' copies into a stage have landed; empty (in both): the MMAs that read it have completed; dfull (in
    // both): an accumulator is complete and its scales are written; dempty (the leader's): both CTAs have drained it; in: a drain warp's input
    const uint32_t bar_full = base, bar_empty = base + 64, bar_dfull = base + 128, bar_dempty = base + 160, bar_in = base + 192, tmem_slot = base + 448,
                   bell = base + 512;
    const uint32_t ring = base + 1024, out_stage = ring + kFp8Stages * kFp8StageBytes, scale_ring = out_stage + 2 * kFp8DrainWarps * kFp8OutBytes;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int tiles = a.tiles_m * a.tiles_n, KB = a.KB, F = a.N / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kFp8Stages; ++s) {
            mbar_init(bar_full + 8 * s, 2);      // the leader's threads for weights and activations, each with both CTAs' bytes
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar_dfull + 8 * s, 2);      // the MMAs, the scales
            mbar_init(bar_dempty + 8 * s, 1);
        }
        for (int s = 0; s < 2 * kFp8DrainWarps; ++s) mbar_init(bar_in + 8 * s, 1);
        fence_barrier_init();
        fence_proxy_async();
    }
    if (warp == 1) {
        tmem_alloc_pair(tmem_slot, 512);
        tmem_relinquish_pair();
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_arrive_release();      // both CTAs' barriers exist before anything arrives from the other
    cluster_wait_acquire();
    tc_fence_after_sync();
    const uint32_t tmem = lds32(tmem_slot);
    pdl_launch_dependents();

    if (warp < kFp8FirstDrain) {
      setmaxnreg_dec<kFp8FewRegs>();
      if (warp == 0 || warp == 3) {
        // ------------------------------------------------------------------------------------------ TMA (a thread each)
        // The other CTA's bytes may be counted before the leader expects them: the barrier's phase cannot end without the leader's
        // arrivals.  Weights do not depend on earlier kernels: they are not waited for.
        if (elect_one()) {
            const CUtensorMap *map = warp == 0 ? &w_map : &x_map;
            tma_prefetch_descriptor(map);
            const uint32_t full = map_to_cluster_rank(bar_full, 0), to = ring + (warp == 0 ? kFp8HalfBytes : 0);
            if (warp == 3) pdl_wait();
            int s = 0, done = 0;
            uint32_t ph = 1;
            bool ok = true;
            for (int t = pair; t < tiles && ok; t += pairs) {
                int tm, tn;
                fp8_tile(t, a.tiles_m, a.tiles_n, tm, tn);
                const int row = warp == 3 ? tm * kFp8TileM + rank * kFp8HalfM : KIND == kFp8Plain ? tn * kFp8TileN + rank * kFp8Block : rank * F + tn * kFp8Block;
                for (int kb = 0; kb < KB; ++kb) {
                    if (done >= kFp8Stages && !(ok = mbar_wait_once(bar_empty + 8 * s, ph))) break;
                    if (rank == 0) mbar_arrive_expect_tx(bar_full + 8 * s, 2 * kFp8HalfBytes);
                    tma_load_2d_pair(to + s * kFp8StageBytes, map, kb * kFp8Block, row, full + 8 * s);
                    ++done;
                    if (++s == kFp8Stages) s = 0, ph ^= 1;
                }
            }
            // nothing may be on its way into either shared memory when the CTAs end
            if (rank == 0)
                for (int j = done < kFp8Stages ? 0 : done - kFp8Stages; j < done; ++j) mbar_wait(bar_full + 8 * (j % kFp8Stages), (uint32_t)(j / kFp8Stages) & 1);
        }
      } else if (warp == 1) {
        // ------------------------------------------------------------------------------------------ MMA (one thread of the leader)
        if (rank == 0 && elect_one()) {
            constexpr uint32_t idesc = umma_idesc_f16(kFp8TileM, kFp8TileN);      // (both operands e4m3: format fields 0)
            auto wait = [](uint32_t bar, uint32_t parity) { return mbar_try_wait_cluster(bar, parity) || mbar_wait_cluster(bar, parity); };
            const int blocks = ((tiles - 1 - pair) / pairs + 1) * KB;
            int s = 0;
            uint32_t ph = 0;
            for (int i = 0; i < blocks; ++i) {
                const int d = i & 1;
                if (!wait(bar_full + 8 * s, ph)) break;
                if (i >= 2 && !wait(bar_dempty + 8 * d, (uint32_t)(i / 2 - 1) & 1)) break;
                tc_fence_after_sync();
                const uint64_t xd = umma_desc_k_major_sw128(ring + s * kFp8StageBytes);
                const uint64_t wd = umma_desc_k_major_sw128(ring + s * kFp8StageBytes + kFp8HalfBytes);
#pragma unroll
                for (int j = 0; j < 4; ++j) umma_f8_ss_pair(tmem + d * kFp8TileN, xd + 2 * j, wd + 2 * j, idesc, j);
                umma_commit_pair(bar_dfull + 8 * d, 3);
                umma_commit_pair(bar_empty + 8 * s, 3);
                mbar_arrive_expect_tx(bar_dempty + 8 * d, 2 * 4 * kFp8DrainWarps);
                if (++s == kFp8Stages) s = 0, ph ^= 1;
            }
        }
      } else {
        // ------------------------------------------------------------------------------------------ scales
        // Lane l has rows 4 l .. 4 l + 3.  Block i's go into slot i % 4 once block i - 2 is complete: its MMA waited until block
        // i - 4, which had the slot, was drained.  They count as an arrival for block i's accumulator.
        pdl_wait();
        const int nb_last = fp8_blocks(a.N) - 1, l4 = 4 * lane;
        const bool by_four = (KB & 3) == 0;
        auto four = [&](const float *p, int kb) {
            if (by_four) {
                const uint4 v = ldg_behind(p + kb);
                return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
            }
            return make_float4(ldgf_behind(p + kb), ldgf_behind(p + min(kb + 1, KB - 1)), ldgf_behind(p + min(kb + 2, KB - 1)), ldgf_behind(p + min(kb + 3, KB - 1)));
        };
        float4 x[4], w[2];      // [row], [weight block]: four blocks of K
        auto fetch = [&](int t, int kb) {
            int tm, tn;
            fp8_tile(t, a.tiles_m, a.tiles_n, tm, tn);
            const int row = tm * kFp8TileM + rank * kFp8HalfM + l4;
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = four(a.x_scales + (size_t)min(row + r, a.M - 1) * KB, kb);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                w[h] = four(a.w_scales + (size_t)(KIND == kFp8Plain ? min(2 * tn + h, nb_last) : h * (F / kFp8Block) + tn) * KB, kb);
        };
        int i = 0;
        bool ok = true;
        fetch(pair, 0);
        for (int t = pair; t < tiles && ok; t += pairs)
            for (int kb0 = 0; kb0 < KB && ok; kb0 += 4) {
                float4 p[2][4];      // [weight block][block of K]: the lane's rows
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    p[h][0] = make_float4(x[0].x * w[h].x, x[1].x * w[h].x, x[2].x * w[h].x, x[3].x * w[h].x);
                    p[h][1] = make_float4(x[0].y * w[h].y, x[1].y * w[h].y, x[2].y * w[h].y, x[3].y * w[h].y);
                    p[h][2] = make_float4(x[0].z * w[h].z, x[1].z * w[h].z, x[2].z * w[h].z, x[3].z * w[h].z);
                    p[h][3] = make_float4(x[0].w * w[h].w, x[1].w * w[h].w, x[2].w * w[h].w, x[3].w * w[h].w);
                }
                if (kb0 + 4 < KB) fetch(t, kb0 + 4);
                else if (t + pairs < tiles) fetch(t + pairs, 0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (kb0 + j >= KB || !ok) break;
                    if (i >= 2 && !(ok = mbar_wait_warp(bar_dfull + 8 * (i & 1), (uint32_t)(i / 2 - 1) & 1))) break;      // (the slot may still be read)
                    const uint32_t slot = scale_ring + (i & 3) * kFp8ScaleBytes + 4 * l4;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        sts128(slot + h * kFp8HalfM * 4, make_uint4(__float_as_uint(p[h][j].x), __float_as_uint(p[h][j].y), __float_as_uint(p[h][j].z), __float_as_uint(p[h][j].w)));
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_dfull + 8 * (i & 1));
                    ++i;
                }
            }
      }
    } else {
        // ------------------------------------------------------------------------------------------ drain
        setmaxnreg_inc<kFp8ManyRegs>();
        pdl_wait();
        const int q = warp & 3, cols = 64 * ((warp - kFp8FirstDrain) >> 2);      // lanes 32 q .. of tensor memory; first column of a half
        const uint32_t stage = out_stage + (warp - kFp8FirstDrain) * 2 * kFp8OutBytes, my_in = bar_in + 16 * (warp - kFp8FirstDrain);
        const uint32_t lanes = tmem + ((uint32_t)(32 * q) << 16);
        const uint32_t my_scale = scale_ring + (32 * q + lane) * 4;
        // "drained" to the leader: a store of four bytes that counts on its barrier (a remote arrival would hold the warp up)
        const uint32_t leader_dempty = map_to_cluster_rank(bar_dempty, 0), leader_bell = map_to_cluster_rank(bell + 4 * warp, 0);
        auto drained = [&](uint32_t offset) {
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) st_async_f32(leader_bell, 0.0f, leader_dempty + offset);
        };
        uint32_t at = 0, parity = 0, slot = 0;      // of this block of K: its barriers' offset (0 or 8), their parity, its scales
        int ins = 0;
        // false once a wait has given up: from then on this warp waits for nothing, hands no accumulator back and stores nothing, but meets every barrier of
        // the CTA.  The MMAs end with the accumulators that it has not drained, so that the pair's other warps give up too instead of draining what
        // is not whole.
        bool ok = true;
        for (int t = pair; t < tiles; t += pairs) {
            int tm, tn;
            fp8_tile(t, a.tiles_m, a.tiles_n, tm, tn);
            const int row0 = tm * kFp8TileM + rank * kFp8HalfM + 32 * q, row = row0 + lane;
            const bool live = row0 < a.M;
            // first column of this warp's 64 of half h, in y or (gated kinds) among the F columns of the result
            auto out_col = [&](int h) { return KIND == kFp8Plain ? tn * kFp8TileN + h * 128 + cols : tn * kFp8Block + cols; };
            // the input, requested some blocks into the tile: the last tile's results have left the stages by then
            auto request = [&]() {
                if (live && elect_one()) {
                    tma_store_wait_read();
#pragma unroll
                    for (int h = 0; h < (KIND == kFp8Plain ? 2 : 1); ++h)
                        if (KIND != kFp8Plain || out_col(h) < a.N) {
                            mbar_arrive_expect_tx(my_in + 8 * h, kFp8OutBytes);
                            tma_load_2d(stage + h * kFp8OutBytes, &in_map, out_col(h), row0, my_in + 8 * h);
                        }
                }
                __syncwarp();
            };
            const int request_at = IN ? min(4, KB - 1) : -1;
            uint64_t acc[2][32];
#pragma unroll
            for (int j = 0; j < 64; ++j) acc[j / 32][j % 32] = 0;
            for (int kb = ok ? 0 : KB; kb < KB; ++kb) {
                const uint32_t from = lanes + 32 * at + cols;
                if (IN && kb == request_at) request();
                if (!mbar_wait_warp_inline(bar_dfull + at, parity)) {
                    ok = false;
                    if (IN && live && kb >= request_at)      // no copy into the stages may be on its way when the CTA ends
#pragma unroll 1
                        for (int h = 0; h < (KIND == kFp8Plain ? 2 : 1); ++h)
                            if (KIND != kFp8Plain || out_col(h) < a.N) mbar_wait_warp_inline(my_in + 8 * h, (uint32_t)ins >> h & 1);
                    break;
                }
                tc_fence_after_sync();
                if (live) {
                    uint32_t v[2][16];
                    tmem_ld_32x16(from, v[0]);
                    const uint64_t s0 = both(__uint_as_float(lds32(my_scale + slot)));
                    const uint64_t s1 = both(__uint_as_float(lds32(my_scale + slot + kFp8HalfM * 4)));
#pragma unroll
                    for (int c = 0; c < 8; ++c) {      // the next 16 columns are on their way while these are added
                        tmem_wait_ld();
                        if (c < 7) tmem_ld_32x16(from + (c < 3 ? 0 : 128) + 16 * ((c + 1) & 3), v[(c + 1) & 1]);
                        else drained(at);
#pragma unroll
                        for (int j = 0; j < 8; ++j) fma2(acc[c / 4][8 * (c & 3) + j], v[c & 1][2 * j], v[c & 1][2 * j + 1], c < 4 ? s0 : s1);
                    }
                } else {
                    drained(at);
                }
                parity ^= at >> 3;
                at ^= 8;
                slot = (slot + kFp8ScaleBytes) & (kFp8ScaleSlots * kFp8ScaleBytes - 1);
            }
            if (!live) continue;
            if (!IN) {
                if (elect_one()) tma_store_wait_read();
                __syncwarp();
            }

            // row `lane` of a stage, 16-byte piece c: 128-byte rows, 128-byte swizzle (the tensor maps')
            auto piece = [&](int h, int c) { return stage + h * kFp8OutBytes + lane * 128 + ((c ^ (lane & 7)) << 4); };
            if constexpr (KIND == kFp8Plain) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int col = out_col(h);
                    if (col >= a.N) break;
                    if (IN && ok) ok = mbar_wait_warp_inline(my_in + 8 * h, (uint32_t)ins >> h & 1);
                    if (IN) ins ^= 1 << h;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        float2 f[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) f[j] = unpack2(acc[h][4 * c + j]);
                        auto add = [&](const uint4 b) {
                            const uint32_t bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float2 e = pair_to_float2<BF>(bw[j]);
                                f[j].x += e.x, f[j].y += e.y;
                            }
                        };
                        if (a.bias != nullptr && col + 8 * c < a.N) add(ldg_behind(a.bias + col + 8 * c));      // (N % 8 == 0)
                        if (IN) add(lds128(piece(h, c)));
                        sts128(piece(h, c), make_uint4(pack_out16<BF>(f[0]), pack_out16<BF>(f[1]), pack_out16<BF>(f[2]), pack_out16<BF>(f[3])));
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (ok && elect_one()) tma_store_2d(&out_map, stage + h * kFp8OutBytes, col, row0);
                }
            } else {
                // h = silu(gate) up in the place of gate's sums; backward: the gradients in the places of both
                uint32_t top[2] = {0, 0};
                if constexpr (KIND == kFp8Backward) {
                    if (ok) ok = mbar_wait_warp_inline(my_in, (uint32_t)ins & 1);
                    ins ^= 1;
                }
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t dw[4];
                    if constexpr (KIND == kFp8Backward) {
                        const uint4 b = lds128(piece(0, c));
                        dw[0] = b.x, dw[1] = b.y, dw[2] = b.z, dw[3] = b.w;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 g = unpack2(acc[0][4 * c + j]), u = unpack2(acc[1][4 * c + j]);
                        const float2 p = make_float2(logistic(g.x), logistic(g.y));
                        float2 r;
                        if constexpr (KIND == kFp8Gated) {
                            r = make_float2(g.x * p.x * u.x, g.y * p.y * u.y);
                        } else {
                            const float2 e = pair_to_float2<BF>(dw[j]);
                            r = make_float2(e.x * u.x * p.x * (1.0f + g.x * (1.0f - p.x)), e.y * u.y * p.y * (1.0f + g.y * (1.0f - p.y)));
                            const float2 v = make_float2(e.x * g.x * p.x, e.y * g.y * p.y);
                            acc[1][4 * c + j] = pack2(v);
                            top[1] = max(top[1], max(abs_bits(v.x), abs_bits(v.y)));
                        }
                        acc[0][4 * c + j] = pack2(r);
                        top[0] = max(top[0], max(abs_bits(r.x), abs_bits(r.y)));
                    }
                }
                constexpr int kOuts = KIND == kFp8Backward ? 2 : 1;
                __syncwarp();      // every lane has read its input: the stages are free
                if constexpr (OUT8) {
                    // the two warps that hold a row's 128 columns exchange their maxima (in their stages), and whether they are whole
                    if (!ok) top[0] = ~0u;
                    asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(stage + 8 * lane), "r"(top[0]), "r"(top[1]) : "memory");
                    named_bar_sync(1 + q, 64);
                    const uint2 other = lds64(out_stage + ((warp - kFp8FirstDrain) ^ 4) * 2 * kFp8OutBytes + 8 * lane);
                    named_bar_sync(1 + q, 64);
                    ok = __all_sync(0xffffffffu, ok && (int)other.x >= 0);      // (a vote: what hangs on ok stays the warp's; without it 2 to 5 % slower)
                    top[0] = max(top[0], other.x), top[1] = max(top[1], other.y);
                    const int FB = F / kFp8Block;
#pragma unroll
                    for (int o = 0; o < kOuts; ++o) {
                        const float s = fp8_scale(top[o]);
                        const Fp8Quotient by(s);
                        if (cols == 0 && row < a.M && ok) a.out_scales[(size_t)row * kOuts * FB + o * FB + tn] = s;
                        // 64-byte rows, 64-byte swizzle
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t w[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float2 f0 = unpack2(acc[o][8 * c + 2 * j]), f1 = unpack2(acc[o][8 * c + 2 * j + 1]);
                                w[j] = fp8_four(by(f0.x), by(f0.y), by(f1.x), by(f1.y));
                            }
                            sts128(stage + o * kFp8OutBytes + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4), make_uint4(w[0], w[1], w[2], w[3]));
                        }
                    }
                } else {
#pragma unroll
                    for (int o = 0; o < kOuts; ++o)
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            sts128(piece(o, c), make_uint4(pack_out16<BF>(unpack2(acc[o][4 * c])), pack_out16<BF>(unpack2(acc[o][4 * c + 1])),
                                                           pack_out16<BF>(unpack2(acc[o][4 * c + 2])), pack_out16<BF>(unpack2(acc[o][4 * c + 3]))));
                }
                fence_proxy_async();
                __syncwarp();
                if (ok && elect_one())
#pragma unroll
                    for (int o = 0; o < kOuts; ++o) tma_store_2d(&out_map, stage + o * kFp8OutBytes, o * F + out_col(0), row0);
            }
        }
        if (elect_one()) tma_store_wait();
    }
    // neither CTA may free tensor memory or end while the pair's MMAs, or the other's copies and arrivals, can still touch it
    tc_fence_before_sync();
    __syncthreads();
    cluster_arrive_release();
    cluster_wait_acquire();
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc_pair(tmem, 512);
    }
}

// ---- launches -----------------------------------------------------------------------------------------------------------

inline cudaError_t fp8_launch(void *kernel, int grid, int threads, int smem, int cluster, cudaStream_t s, void **args)
{
    cudaLaunchAttribute attr[3] = {};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cfg.attrs = attr;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)cluster;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        attr[2].id = cudaLaunchAttributeClusterSchedulingPolicyPreference;
        attr[2].val.clusterSchedulingPolicyPreference = cudaClusterSchedulingPolicyLoadBalancing;
        cfg.numAttrs = 3;
    }
    return cudaLaunchKernelExC(&cfg, kernel, args);
}

inline int launch_fp8_quantize(const void *x, void *q, float *scales, int M, int K, int bf16, int sms, cudaStream_t s)
{
    int KB = fp8_blocks(K);
    long long blocks = (long long)M * KB;
    const long long per_cta = kFp8QuantThreads / kFp8QuantLanes, want = (blocks + per_cta - 1) / per_cta;
    const long long most = (long long)kFp8QuantCtasPerSm * sms;
    const int grid = (int)(want < most ? want : most);
    const uint4 *xp = (const uint4 *)x;
    uint2 *qp = (uint2 *)q;
    void *args[] = {&xp, &qp, &scales, &K, &KB, &blocks};
    return record_cuda_error(fp8_launch(bf16 ? (void *)fp8_quantize_kernel<true> : (void *)fp8_quantize_kernel<false>, grid, kFp8QuantThreads, 0, 1, s, args));
}

inline int launch_fp8_transpose(const void *w, const float *scales, void *w_out, float *scales_out, int N, int K, cudaStream_t s)
{
    const long long tiles = (long long)((N - 1) / 64 + 1) * ((K - 1) / 64 + 1);
    if (tiles > 0x7fffffffll) return GPTQ_ERR_UNSUPPORTED;
    fp8_transpose_kernel<<<(unsigned)tiles, 256, 0, s>>>((const uint8_t *)w, scales, (uint8_t *)w_out, scales_out, N, K);
    return record_cuda_error(cudaGetLastError());
}

struct Fp8Call {
    int kind;                    // Fp8Kind
    const void *x;               // e4m3 [M, K]
    const float *x_scales;
    const void *w;               // e4m3 [N, K]
    const float *w_scales;
    const void *bias, *in;       // in: residual [M, N], or the gradient of the result [M, N / 2]
    void *out;
    float *out_scales;
    int M, N, K, bf16, sms;
};

inline long long fp8_tiles(int kind, int M, int N)
{
    return ((long long)(M - 1) / kFp8TileM + 1) * (kind == kFp8Plain ? (N - 1) / kFp8TileN + 1 : N / 2 / kFp8Block);
}

template <int KIND, bool BF, bool OUT8, bool IN = KIND == kFp8Backward>
int launch_fp8_tiles(const Fp8Call &c, cudaStream_t s)
{
    static int configured[64];
    static std::atomic<int> registers{0};
    auto kernel = fp8_tiles_kernel<KIND, BF, OUT8, IN>;
    int st = ensure_dynamic_smem((const void *)kernel, configured, kFp8SmemBytes);
    if (st) return st;
    if (registers.load() == 0) {      // the warps that take registers would wait for ever for what the launch did not bring
        cudaFuncAttributes fa;
        const cudaError_t e = cudaFuncGetAttributes(&fa, (const void *)kernel);
        if (e != cudaSuccess) return record_cuda_error(e);
        registers.store(fa.numRegs);
    }
    if (registers.load() < kFp8LaunchRegs) return GPTQ_ERR_UNSUPPORTED;
    const int F = c.N / 2;
    Fp8Args a{};
    a.x_scales = c.x_scales, a.w_scales = c.w_scales, a.bias = (const __half *)c.bias, a.out_scales = c.out_scales;
    a.M = c.M, a.N = c.N, a.K = c.K, a.KB = fp8_blocks(c.K);
    a.tiles_m = (c.M - 1) / kFp8TileM + 1;
    a.tiles_n = KIND == kFp8Plain ? (c.N - 1) / kFp8TileN + 1 : F / kFp8Block;
    const long long tiles = fp8_tiles(KIND, c.M, c.N);
    if (tiles > 0x3fffffffll) return GPTQ_ERR_UNSUPPORTED;
    CUtensorMap xm, wm, im, om;
    const auto u8 = CU_TENSOR_MAP_DATA_TYPE_UINT8;
    const auto b16 = CU_TENSOR_MAP_DATA_TYPE_UINT16;
    const auto sw128 = CU_TENSOR_MAP_SWIZZLE_128B;
    st = make_tensor_map_2d(&xm, u8, c.x, c.K, c.M, c.K, kFp8Block, kFp8HalfM, sw128);
    if (!st) st = make_tensor_map_2d(&wm, u8, c.w, c.K, c.N, c.K, kFp8Block, kFp8Block, sw128);
    const uint64_t in_cols = KIND == kFp8Plain ? c.N : F, out_cols = KIND == kFp8Gated ? F : c.N;
    if (!st) {
        if (OUT8) st = make_tensor_map_2d(&om, u8, c.out, out_cols, c.M, out_cols, 64, 32, CU_TENSOR_MAP_SWIZZLE_64B);
        else st = make_tensor_map_2d(&om, b16, c.out, out_cols, c.M, out_cols * 2, 64, 32, sw128);
    }
    if (!st) {
        if (c.in) st = make_tensor_map_2d(&im, b16, c.in, in_cols, c.M, in_cols * 2, 64, 32, sw128);
        else im = om;
    }
    if (st) return st;
    void *args[] = {&a, &xm, &wm, &im, &om};
    return record_cuda_error(fp8_launch((void *)kernel, 2 * (int)(tiles < c.sms / 2 ? tiles : c.sms / 2), kFp8Threads, kFp8SmemBytes, 2, s, args));
}

inline int launch_fp8(const Fp8Call &c, cudaStream_t s)
{
    const bool out8 = c.out_scales != nullptr;
    switch (c.kind * 4 + (out8 ? 2 : 0) + (c.bf16 ? 1 : 0)) {
    case 0: return c.in ? launch_fp8_tiles<kFp8Plain, false, false, true>(c, s) : launch_fp8_tiles<kFp8Plain, false, false>(c, s);
    case 1: return c.in ? launch_fp8_tiles<kFp8Plain, true, false, true>(c, s) : launch_fp8_tiles<kFp8Plain, true, false>(c, s);
    case 4: return launch_fp8_tiles<kFp8Gated, false, false>(c, s);
    case 5: return launch_fp8_tiles<kFp8Gated, true, false>(c, s);
    case 6: case 7: return launch_fp8_tiles<kFp8Gated, false, true>(c, s);      // (the type of the result is not the type of anything else)
    case 8: return launch_fp8_tiles<kFp8Backward, false, false>(c, s);
    case 9: return launch_fp8_tiles<kFp8Backward, true, false>(c, s);
    case 10: return launch_fp8_tiles<kFp8Backward, false, true>(c, s);
    case 11: return launch_fp8_tiles<kFp8Backward, true, true>(c, s);
    default: return GPTQ_ERR_UNSUPPORTED;
    }
}

}  // namespace gptq

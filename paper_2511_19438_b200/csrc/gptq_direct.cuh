// Products of few rows with parts of tiled layers, each warp fetching what it multiplies: the common ground of the routed-expert
// kernels (gptq_moe.cuh) and of the projection with adapters (gptq_lora.cuh).
//
// A warp takes NU UNITS (16 columns each) of a panel and some of the panel's 128-row items.  A lane's share of a unit's item
// is two 16-byte chunks (see the layout in gptq_common.cuh), exactly the A fragments of eight mma.m16n8k16; it copies them into a
// ring of its warp's in shared memory with cp.async and reads back what it copied itself (scales and zero points: what its warp did), so that
// no barrier of the CTA stands between memory and the tensor cores, and a warp's next item may lie in any layer, panel and row of K - which is what rows that choose their
// weights need.  The ring holds pairs of units: the rest of the item at hand and the whole next one are on their way.  Activations are
// loaded into registers an item ahead: lane (g, t4) reads 16 bytes of token row g, the B fragments for all of the warp's units.  Up to 8
// rows; a lane without a row reads another one's, whose products land in columns that nobody looks at.
//
// Arithmetic, fp16: a nibble alone in a 16-bit word is the subnormal number q 2^-24, so the MMAs take `w & 0x000f000f` and
// `w & 0x00f000f0` as they are (the second kind, 16 q, into sums of its own).  sum (q - z) x = sum q x - z sum x, and sum x of a
// quantisation group comes from MMAs with a matrix of ones, which all units share.  bfloat16 (subnormals would vanish): 128 + q
// by one more OR, and -(128 + z) sum x.  All in fp32: the error is that of sums of (q + z) |x| (bfloat16: (256 + q + z) |x|), far
// below the rounding of the 16-bit results.  Against subtracting z from each weight this is 5 instead of 9 instructions per eight
// weights; these kernels are bound by instruction issue as much as by memory.
// An infinity in x makes such a difference NaN, whatever the product is, and in bfloat16 sum (128 + q) x can leave fp32's range where the
// product does not (x from 2^110 on): sums that end up so are formed again the long way, in the epilogues.
#pragma once
#include "gptq_common.cuh"

namespace gptq {

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async8_if(bool wanted, uint32_t dst, const void *src)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p cp.async.ca.shared.global [%0], [%1], 8;\n\t}"
                 ::"r"(dst), "l"(src), "r"((uint32_t)wanted) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// activations: written by an earlier kernel of the stream, read after it has finished; in L1 for the next tile and CTA
__device__ __forceinline__ uint4 ldg_rows128(const void *p)
{
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// A stage of the ring, a pair of units of an item: the weights, then for each quantisation group 32 bytes of scales and behind those of both
// units 8 bytes of zero points per unit.
constexpr int kPairW = 4 * kUnitBytes, kPairMeta = 80;
template <int SUB>
__host__ __device__ constexpr int direct_stage_bytes() { return kPairW + SUB * kPairMeta; }
template <int NU, int SUB>
__host__ __device__ constexpr int direct_ring_bytes(int warps) { return warps * (NU / 2 + 2) * direct_stage_bytes<SUB>(); }

// fp16 products take the words of eight rows (four pairs e = 01, 23, 45, 67 of a lane's 16 bytes of x) in the order 01, 45, 23, 67: an
// activation that only these kernels read is stored that way.
template <bool BF>
__host__ __device__ constexpr int direct_column(int c)
{
    return BF ? c : (c & ~6) | (c & 2) << 1 | (c & 4) >> 1;
}

// The warp's units, counted from the first: neighbours, or with GATE_UP a gate unit and its up unit, half a panel further, and so on
template <bool GATE_UP>
__host__ __device__ constexpr int unit_offset(int u)
{
    return GATE_UP ? u % 2 * 4 + u / 2 : u;
}
struct UnitPtrs {
    const uint8_t *w, *s, *z;
};
// a lane's share of a warp's units: 16 bytes of weights per unit and K64 block; 8 bytes of a pair's scales (lanes below 8 SUB) or zero points
// (the next 2 SUB lanes; with SUB = 4, where these are no longer in the warp, the first 8 lanes have both)
template <int SUB>
struct LanePtrs {
    const uint8_t *w, *m, *z;      // (z: SUB = 4 only)
};
// a unit in item 0 of a panel
template <int SUB>
__device__ __forceinline__ UnitPtrs unit_ptrs(const uint8_t *qweight, const uint8_t *scales, const uint8_t *qzeros, int panel, int G, int unit)
{
    const size_t item = (size_t)panel * G;
    return {qweight + item * kItemWBytes + unit * kUnitBytes, scales + item * (SUB * kItemSBytes) + unit * 32, qzeros + item * (SUB * kItemZBytes) + unit * 8};
}
template <bool GATE_UP, int SUB>
__device__ __forceinline__ LanePtrs<SUB> lane_ptrs(const UnitPtrs &p, int lane)
{
    const int zl = SUB == 4 ? lane : lane - 8 * SUB;
    const uint8_t *s = p.s + (lane >> 3) * kItemSBytes + unit_offset<GATE_UP>(lane >> 2 & 1) * 32 + (lane & 3) * 8;
    const uint8_t *z = p.z + (zl >> 1) * kItemZBytes + unit_offset<GATE_UP>(zl & 1) * 8;
    return {p.w + lane * 16, SUB == 4 || lane < 8 * SUB ? s : z, z};
}
// What a warp multiplies next: the item's addresses, the lane's token rows at the item's first column + 8 t4, the layer's
// format flags as loaded (looked at only when the item is multiplied), a number of the caller's
// (not negative), and how many of the warp's pairs of units are wanted (the others' sums stay as they are).
template <int SUB>
struct DirectItem {
    LanePtrs<SUB> p;
    const __half *x;
    uint32_t flags;
    int tag, pairs;
};
template <int SUB>
__device__ __forceinline__ void set_item(DirectItem<SUB> &it, const LanePtrs<SUB> &p, const __half *row, int item, int lane)
{
    it.p.w = p.w + (size_t)item * kItemWBytes;
    it.p.m = p.m + (size_t)item * (SUB == 4 || lane < 8 * SUB ? SUB * kItemSBytes : SUB * kItemZBytes);
    if constexpr (SUB == 4) it.p.z = p.z + (size_t)item * (SUB * kItemZBytes);
    it.x = row + (size_t)item * kGroup;
}

struct DirectRows {
    uint4 x[4];                   // [32-row quarter]
    uint32_t flags;
    int tag, pairs;
};
template <int SUB>
__device__ __forceinline__ void load_rows(DirectRows &r, const DirectItem<SUB> &it)
{
    r.tag = it.tag;
    r.flags = it.flags;
    r.pairs = it.pairs;
    if (it.tag < 0) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) r.x[q] = ldg_rows128(it.x + 32 * q);
}

// a value that the compiler keeps instead of working it out again
__device__ __forceinline__ uint32_t kept(uint32_t v)
{
    asm volatile("mov.b32 %0, %1;" : "=r"(v) : "r"(v));
    return v;
}
__device__ __forceinline__ uint64_t register_pair(uint32_t lo, uint32_t hi)
{
    uint64_t p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "r"(lo), "r"(hi));
    return p;
}
// D = A B (START) or D += A B
template <bool BF, bool START>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint64_t b)
{
#define GPTQ_MMA16(TYPE, D, C, ...)                                                                                           \
    asm("{\n\t.reg .b32 b0, b1;\n\tmov.b64 {b0, b1}, %8;\n\t"                                                                \
        "mma.sync.aligned.m16n8k16.row.col.f32." TYPE "." TYPE ".f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {b0,b1}, " C ";\n\t}"      \
        : D(d[0]), D(d[1]), D(d[2]), D(d[3])                                                                                  \
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "l"(b) __VA_ARGS__)
    if constexpr (START) {
        if constexpr (BF) GPTQ_MMA16("bf16", "=f", "{%9,%9,%9,%9}", , "f"(0.f));
        else GPTQ_MMA16("f16", "=f", "{%9,%9,%9,%9}", , "f"(0.f));
    } else {
        if constexpr (BF) GPTQ_MMA16("bf16", "+f", "{%0,%1,%2,%3}", );
        else GPTQ_MMA16("f16", "+f", "{%0,%1,%2,%3}", );
    }
#undef GPTQ_MMA16
}
template <bool BF>
__device__ __forceinline__ void mma16_from(bool start, float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint64_t b)
{
    if (start) mma16<BF, true>(d, a0, a1, a2, a3, b);
    else mma16<BF, false>(d, a0, a1, a2, a3, b);
}

// What the units of an item share: x as B fragments, in the order of the products below, and its sums over the quantisation groups
// (elements 2 and 3 repeat 0 and 1).
template <int SUB>
struct ItemRows {
    uint64_t xp[4][2];
    float xs[SUB][4];
};
// IN_ORDER: x lies in memory as direct_column has it.  Else its words change places, by multiplications with `one` = 1 that the
// compiler cannot see through: as plain moves they are made anew for every unit (84 moves per item of four units instead of 16).
template <int SUB, bool BF, bool IN_ORDER>
__device__ __forceinline__ void prepare_rows(ItemRows<SUB> &rows, const uint4 (&x)[4], uint32_t one)
{
    constexpr uint32_t ONES = BF ? 0x3f803f80u : 0x3c003c00u;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int sub = q * SUB / 4;
        const uint4 v = x[q];
        if constexpr (BF || IN_ORDER) {
            rows.xp[q][0] = register_pair(v.x, v.y);
            rows.xp[q][1] = register_pair(v.z, v.w);
        } else {
            rows.xp[q][0] = register_pair(v.x * one, v.z * one);
            rows.xp[q][1] = register_pair(v.y * one, v.w * one);
        }
        mma16_from<BF>(q * SUB % 4 == 0, rows.xs[sub], ONES, ONES, ONES, ONES, rows.xp[q][0]);
        mma16<BF, false>(rows.xs[sub], ONES, ONES, ONES, ONES, rows.xp[q][1]);
    }
}

// acc[u][i], u = U0, U0 + 1: column g + 8 (i >> 1) of unit u, token 2 t4 + (i & 1); `stage`: the pair's stage of the ring
template <int U0, int NU, int SUB, bool BF>
__device__ __forceinline__ void multiply_pair(uint32_t stage, int lane, uint32_t flags, const ItemRows<SUB> &rows, float (&acc)[NU][4])
{
    const uint32_t slot = stage + lane * 16, meta = stage + kPairW + (lane >> 2) * 4, zeros = stage + kPairW + 64 + (lane >> 2);
    constexpr uint32_t LO = 0x000f000fu, HI = 0x00f000f0u, MAGIC = 0x43004300u;
    // fp16: sums and -z in units of 2^-24, which the scale makes good.  -z as a float: the nibble, or 16 times it, in the lowest bits of 2^23.
    constexpr float kStep = BF ? 1.f : 5.9604645e-8f;
    const float z_add = (flags & kFormatZerosMinusOne) ? 1.f : 0.f;
    const float c_lo = (8388608.f - (BF ? 128.f : 0.f) - z_add) * kStep, c_hi = (524288.f - (BF ? 128.f : 0.f) - z_add) * kStep;
#pragma unroll
    for (int u = U0; u < U0 + 2; ++u) {
        const uint4 wq[2] = {lds128(slot + (u - U0) * 2 * kUnitBytes), lds128(slot + (u - U0) * 2 * kUnitBytes + kUnitBytes)};
        float lo[4], hi[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int sub = q * SUB / 4;
            const bool start = q * SUB % 4 == 0;    // first quarter of a quantisation group
            const uint32_t a = (q & 1) ? wq[q >> 1].y : wq[q >> 1].x, b = (q & 1) ? wq[q >> 1].w : wq[q >> 1].z;
            if constexpr (BF) {
                const uint32_t a0 = lop3_and_or(a, LO, MAGIC), a1 = lop3_and_or(a >> 4, LO, MAGIC), a2 = lop3_and_or(a >> 8, LO, MAGIC),
                               a3 = lop3_and_or(a >> 12, LO, MAGIC);
                const uint32_t b0 = lop3_and_or(b, LO, MAGIC), b1 = lop3_and_or(b >> 4, LO, MAGIC), b2 = lop3_and_or(b >> 8, LO, MAGIC),
                               b3 = lop3_and_or(b >> 12, LO, MAGIC);
                mma16_from<true>(start, lo, a0, b0, a1, b1, rows.xp[q][0]);
                mma16<true, false>(lo, a2, b2, a3, b3, rows.xp[q][1]);
            } else {
                const uint32_t a8 = a >> 8, b8 = b >> 8;
                mma16_from<false>(start, lo, a & LO, b & LO, a8 & LO, b8 & LO, rows.xp[q][0]);
                mma16_from<false>(start, hi, a & HI, b & HI, a8 & HI, b8 & HI, rows.xp[q][1]);
            }
            if ((q + 1) * SUB % 4 == 0) {           // last quarter of the group
                float2 sf = pair_to_float2<BF>(lds32(meta + sub * kPairMeta + (u - U0) * 32));
                if constexpr (!BF) sf.x *= 16777216.f, sf.y *= 16777216.f;
                const uint32_t zz = lds8(zeros + sub * kPairMeta + (u - U0) * 8);
                const float za = fmaf(__uint_as_float((zz & 15u) | 0x4b000000u), -kStep, c_lo);
                const float zb = fmaf(__uint_as_float((zz & 0xf0u) | 0x4b000000u), -0.0625f * kStep, c_hi);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = lo[i];
                    if constexpr (!BF) v = fmaf(hi[i], 0.0625f, v);
                    v = fmaf(i < 2 ? za : zb, rows.xs[sub][i & 1], v);
                    acc[u][i] = fmaf(i < 2 ? sf.x : sf.y, v, acc[u][i]);
                }
            }
        }
    }
}

// Works through the items that `next` yields (it fills a DirectItem, tag < 0 at the end).  `ready()` is called once, between the first
// requests for weights and the first for activations, `before(tag)` ahead of each item's product.  `ring`: the warp's part of the ring.
// A copy goes to the stage that was read last.  A lane's weights are its own copies, but its scales and zero points are other lanes': the
// warp meets behind each product, so that no lane refills a stage that another one still reads.
template <int NU, bool GATE_UP, int SUB, bool BF, bool IN_ORDER, typename Next, typename Ready, typename Before>
__device__ __forceinline__ void stream_items(uint32_t ring, int lane, uint32_t one, float (&acc)[NU][4], Next next, Ready ready, Before before)
{
    static_assert(NU == 2 || NU == 4, "one or two pairs of units");
    constexpr int NP = NU / 2, kStages = NP + 2;
    constexpr uint32_t kStage = direct_stage_bytes<SUB>(), kEnd = kStages * kStage;
    DirectItem<SUB> it{};
    DirectRows x;
    const int zl = SUB == 4 ? lane : lane - 8 * SUB;
    const uint32_t m_at = kept(kPairW + (SUB == 4 || lane < 8 * SUB ? (lane >> 3) * kPairMeta + (lane & 7) * 8 : (zl >> 1) * kPairMeta + 64 + (zl & 1) * 8));
    const uint32_t w_at = kept(lane * 16);
    const int m_step = kept(GATE_UP ? (SUB == 4 || lane < 8 * SUB ? 32 : 8) : (SUB == 4 || lane < 8 * SUB ? 64 : 16));      // from pair to pair
    uint32_t fill = 0, at = 0;      // offsets into the ring
    auto advance = [&](uint32_t &offset) { offset = offset == kEnd - kStage ? 0 : offset + kStage; };
    auto copy_pair = [&](int pair) {
        if (it.tag >= 0 && pair < it.pairs) {
            const uint32_t to = ring + fill;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint8_t *src = it.p.w + unit_offset<GATE_UP>(2 * pair + u) * kUnitBytes;
                cp_async16(to + w_at + u * 2 * kUnitBytes, src);
                cp_async16(to + w_at + u * 2 * kUnitBytes + kUnitBytes, src + kBlockWBytes);
            }
            cp_async8_if(SUB == 4 || lane < 10 * SUB, to + m_at, it.p.m + pair * m_step);
            if constexpr (SUB == 4) cp_async8_if(lane < 8, to + kPairW + (lane >> 1) * kPairMeta + 64 + (lane & 1) * 8, it.p.z + unit_offset<GATE_UP>(2 * pair) * 8);
        }
        cp_async_commit();
        advance(fill);
    };
    next(it);
#pragma unroll
    for (int p = 0; p < NP; ++p) copy_pair(p);
    const DirectItem<SUB> first = it;
    next(it);
    copy_pair(0);
    ready();
    load_rows<SUB>(x, first);
    while (x.tag >= 0) {
        before(x.tag);
        ItemRows<SUB> rows;
        prepare_rows<SUB, BF, IN_ORDER>(rows, x.x, one);
        const uint32_t flags = x.flags;
        const int pairs = x.pairs;
        load_rows<SUB>(x, it);
        if constexpr (NP == 2) {
            copy_pair(1);
            cp_async_wait<NP + 1>();
            __syncwarp();      // (the scales and zero points are other lanes' copies)
            multiply_pair<0, NU, SUB, BF>(ring + at, lane, flags, rows, acc);
            __syncwarp();
            advance(at);
        }
        next(it);
        copy_pair(0);
        cp_async_wait<NP + 1>();
        __syncwarp();
        if (NP == 1 || pairs == NP) multiply_pair<NU - 2, NU, SUB, BF>(ring + at, lane, flags, rows, acc);
        __syncwarp();
        advance(at);
    }
}

// whether a sum is formed again the long way (fp16 sums do not leave fp32's range: an infinity of x is NaN here)
template <bool BF>
__device__ __forceinline__ bool needs_long_sum(float v)
{
    if constexpr (BF) return !isfinite(v);
    else return v != v;
}
// The sum over n items for one column (0 .. 15) of a unit and one token row, the formula as it stands, for sums that need it (see above).
// w, s, z: the unit's addresses without a lane's share; in_order: the row lies in memory as direct_column has it.
template <bool BF>
__device__ __noinline__ float long_sum(const uint8_t *w, const uint8_t *s, const uint8_t *z, int sub, int col, uint32_t z_add,
                                       const __half *row, int n, bool in_order)
{
    const int g = col & 7, h = col >> 3;
    float sum = 0.f;
    for (int item = 0; item < n; ++item)
        for (int k = 0; k < kGroup; ++k) {
            const int blk = k >> 6, j = (k >> 5) & 1, t4 = (k >> 3) & 3, e = k & 7;
            const size_t grp = (size_t)item * sub + k * sub / kGroup;
            const uint32_t word = *reinterpret_cast<const uint32_t *>(w + (size_t)item * kItemWBytes + blk * kBlockWBytes + (4 * g + t4) * 16 + (j + 2 * h) * 4);
            const uint32_t zb = z[grp * kItemZBytes + g];
            const int q = (int)((word >> (4 * nibble_slot(e))) & 15u) - (int)((h ? zb >> 4 : zb & 15u) + z_add);
            const float sc = out16_to_float<BF>(*reinterpret_cast<const __half *>(s + grp * kItemSBytes + (2 * g + h) * 2));
            sum = fmaf((float)q * sc, out16_to_float<BF>(row[(size_t)item * kGroup + (in_order ? direct_column<BF>(k) : k)]), sum);
        }
    return sum;
}

// n things given out to `parts` in neighbouring ranges, the longer ranges spread evenly: the first of range i
__device__ __forceinline__ int share_begin(int n, int parts, int i) { return (int)((unsigned long long)n * (unsigned)i / (unsigned)parts); }

// A kernel launched as a programmatic dependent, in clusters of `cluster` CTAs.  With per_sm it asks for shared memory for that many CTAs per
// SM; what is left of the SM's 228 KB is L1, in which these kernels keep the rows that they read again and again.  That goes with the launch,
// not with the kernel: other launches of it want another size or number (one token, 64 experts of 2048 x 768 behind a call of 512 x 512:
// 22.0 us with the latter's share, 15.6 with its own).
template <typename... Params, typename... Args>
static int launch_sharing_sm(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, int cluster, int per_sm, cudaStream_t s, Args... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[4];
    int n = 0;
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)cluster;
        attr[n].val.clusterDim.y = 1;
        attr[n++].val.clusterDim.z = 1;
        attr[n].id = cudaLaunchAttributeClusterSchedulingPolicyPreference;      // clusters spread over the SMs
        attr[n++].val.clusterSchedulingPolicyPreference = cudaClusterSchedulingPolicyLoadBalancing;
    }
    if (per_sm) {
        const int percent = (int)((per_sm * (smem + 2048) * 100 + 228 * 1024 - 1) / (228 * 1024));      // (2 KB: static and the system's)
        attr[n].id = cudaLaunchAttributePreferredSharedMemoryCarveout;
        attr[n++].val.sharedMemCarveout = (unsigned)(percent < 100 ? percent : 100);
    }
    cfg.attrs = attr;
    cfg.numAttrs = (unsigned)n;
    return record_cuda_error(cudaLaunchKernelEx(&cfg, kernel, Params(args)...));
}
template <typename... Params, typename... Args>
static int launch_dependent(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t s, Args... args)
{
    return launch_sharing_sm(kernel, grid, threads, smem, cluster, 0, s, args...);
}

}  // namespace gptq

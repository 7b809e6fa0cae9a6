// Products of few rows with parts of tiled layers, weights straight from global memory into the registers of the warp that
// multiplies them: the common ground of the routed-expert kernels (gptq_moe.cuh) and of the projection with adapters
// (gptq_lora.cuh).
//
// A warp takes NU UNITS (16 columns each) of a panel and some of the panel's 128-row items.  A lane's share of a unit's item
// is two 16-byte chunks (see the layout in gptq_common.cuh), exactly the A fragments of eight mma.m16n8k16, so a load of 512
// neighbouring bytes per warp is all there is between memory and the dequantisation: no ring, no barriers, and a warp's work can
// begin in any layer, panel and row of K - which is what rows that choose their weights need.  The activations are read the
// same way: lane (g, t4) reads 16 bytes of token row g, which serve as B fragments for all of the warp's units.  Up to 8 NT
// rows; rows beyond `count` are zeros that no memory is read for.  Loads run kDepth items ahead of the arithmetic.
//
// Arithmetic as in the mma.sync kernels: exact integers q - z times x, fp32 sums per quantisation group, the scale in fp32.
#pragma once
#include "gptq_common.cuh"
#include "gptq_streamk.cuh"

namespace gptq {

// read once, by one SM: not kept in L1
__device__ __forceinline__ uint4 ldg_stream128(const void *p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// activations: written by an earlier kernel of the stream, read after griddepcontrol.wait; neighbouring CTAs of an SM read the
// same rows, so these stay in L1
__device__ __forceinline__ uint4 ldg_rows128(const void *p)
{
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

template <int NT, int NU, int SUB>
struct DirectRegs {
    uint4 w[NU][2];               // [K64 block]
    uint32_t sc[NU][SUB], z[NU][SUB];
    uint4 x[NT][4];               // [32-row quarter]
};

// A warp's units within a panel: addresses of item 0, the lane's share added
struct UnitPtrs {
    const uint8_t *w, *s, *z;
};
template <int SUB>
__device__ __forceinline__ UnitPtrs unit_ptrs(const uint8_t *qweight, const uint8_t *scales, const uint8_t *qzeros, int panel, int G,
                                              int unit, int lane)
{
    const size_t item = (size_t)panel * G;
    const int g = lane >> 2;
    return {qweight + item * kItemWBytes + unit * kUnitBytes + lane * 16, scales + item * (SUB * kItemSBytes) + (16 * unit + 2 * g) * 2,
            qzeros + item * (SUB * kItemZBytes) + 8 * unit + g};
}

// DU: distance of the warp's units (1 neighbours, 4 a gate unit and its up unit)
template <int NT, int NU, int DU, int SUB>
__device__ __forceinline__ void load_item_weights(DirectRegs<NT, NU, SUB> &r, const UnitPtrs &p, int item)
{
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        const uint8_t *w = p.w + (size_t)item * kItemWBytes + u * DU * kUnitBytes;
        r.w[u][0] = ldg_stream128(w);
        r.w[u][1] = ldg_stream128(w + kBlockWBytes);
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) {
            r.sc[u][sub] = __ldg(reinterpret_cast<const uint32_t *>(p.s + (size_t)item * (SUB * kItemSBytes) + sub * kItemSBytes + u * DU * 32));
            r.z[u][sub] = __ldg(p.z + (size_t)item * (SUB * kItemZBytes) + sub * kItemZBytes + u * DU * 8);
        }
    }
}
// rows[t]: the lane's token row of tile t at column 8 * t4 (nullptr: none)
template <int NT, int NU, int SUB>
__device__ __forceinline__ void load_item_rows(DirectRegs<NT, NU, SUB> &r, const __half *const (&rows)[NT], int item)
{
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            r.x[t][q] = rows[t] ? ldg_rows128(rows[t] + (size_t)item * kGroup + 32 * q) : make_uint4(0, 0, 0, 0);
}

// acc[u][t][i]: column g + 8 (i >> 1) of unit u, token 8 t + 2 t4 + (i & 1)
template <int NT, int NU, int SUB, bool BF>
__device__ __forceinline__ void multiply_item(const DirectRegs<NT, NU, SUB> &r, uint32_t z_add, float (&acc)[NU][NT][4])
{
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        float gs[NT][4];
        uint32_t zloA = 0, zhiA = 0, zloB = 0, zhiB = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int sub = q * SUB / 4;
            if (q * SUB % 4 == 0) {                 // first quarter of a quantisation group
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) gs[t][i] = 0.f;
                zero_constants<BF>((r.z[u][sub] & 15u) + z_add, zloA, zhiA);
                zero_constants<BF>((r.z[u][sub] >> 4) + z_add, zloB, zhiB);
            }
            const uint4 wq = r.w[u][q >> 1];
            uint32_t pA[4], pB[4];
            nibble_pairs_minus_zero<BF>((q & 1) ? wq.y : wq.x, zloA, zhiA, pA);
            nibble_pairs_minus_zero<BF>((q & 1) ? wq.w : wq.z, zloB, zhiB, pB);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const uint4 xb = r.x[t][q];
                if constexpr (BF) {
                    mma_m16n8k16_bf16(gs[t], pA[0], pB[0], pA[1], pB[1], xb.x, xb.y);
                    mma_m16n8k16_bf16(gs[t], pA[2], pB[2], pA[3], pB[3], xb.z, xb.w);
                } else {
                    mma_m16n8k16(gs[t], pA[0], pB[0], pA[1], pB[1], xb.x, xb.y);
                    mma_m16n8k16(gs[t], pA[2], pB[2], pA[3], pB[3], xb.z, xb.w);
                }
            }
            if ((q + 1) * SUB % 4 == 0) {           // last quarter of the group
                const float2 sf = pair_to_float2<BF>(r.sc[u][sub]);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    acc[u][t][0] = fmaf(sf.x, gs[t][0], acc[u][t][0]);
                    acc[u][t][1] = fmaf(sf.x, gs[t][1], acc[u][t][1]);
                    acc[u][t][2] = fmaf(sf.y, gs[t][2], acc[u][t][2]);
                    acc[u][t][3] = fmaf(sf.y, gs[t][3], acc[u][t][3]);
                }
            }
        }
    }
}

// a kernel launched as a programmatic dependent, in clusters of `cluster` CTAs
template <typename... Params, typename... Args>
static int launch_dependent(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t s, Args... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return record_cuda_error(cudaLaunchKernelEx(&cfg, kernel, Params(args)...));
}

}  // namespace gptq

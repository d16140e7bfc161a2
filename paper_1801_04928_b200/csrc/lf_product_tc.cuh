// What the matrix products on the 5th-generation tensor cores share (16-bit layers and 8-bit blocks of 128): operand blocks of 128
// rows x 128 bytes in the 128-byte swizzle, barriers with bounded waits, matrix descriptors, the
// persistent schedule of CTA pairs, tensor maps.
#pragma once

#include "lf_ops_internal.h"
#include "lf_ptx.cuh"

namespace {

constexpr int LT_BK = 64;
constexpr int LT_BLOCK_BYTES = 128 * LT_BK * 2;          // 16 KiB: 128 rows (or columns) x 64 contraction steps
constexpr int LT_STAGE_BYTES = 2 * LT_BLOCK_BYTES;
constexpr int LT_STAGES = 6;

struct LtShared {
    unsigned long long full[LT_STAGES];
    unsigned long long empty[LT_STAGES];
    unsigned long long acc_full[2];
    unsigned long long acc_empty[2];
    unsigned long long scaled[8];      // (8-bit blocks: scales of a stage are there ...
    unsigned long long scale_free[8];  //  ... and have been read)
    unsigned tmem_base;
    volatile unsigned abort_flag;
    unsigned prog_it;                  // stage loads this CTA's producer has issued
};
static_assert(sizeof(LtShared) <= 512, "the barrier block must fit into the space reserved for it");

// Bounded wait (acquire at cluster scope: the peer's arrivals count too); false once this CTA has given up.
// CLUSTER = false: an acquire of this CTA's scope, for barriers that order tensor memory and bulk copies only (which have fences of
// their own): several times a stage, the wider scope's fences were half of the time (8-bit products, 8192 x 4096 -> 16384: 1206 us, 600 without).
template <bool CLUSTER = true, typename PARAMS>
__device__ __forceinline__ bool lt_wait(unsigned bar, unsigned parity, const PARAMS& P, LtShared* sh)
{
    auto done = [&]() { return CLUSTER ? lfptx::mbar_try_wait_cluster(bar, parity) : lfptx::mbar_try_wait(bar, parity); };
    if (!CLUSTER && lfptx::mbar_test_wait(bar, parity)) return true;
    if (done()) return true;
    if (sh->abort_flag) return false;
    const unsigned long long t0 = lfptx::globaltimer_ns();
    unsigned spins = 0;
    while (!done()) {
        if ((++spins & 15u) == 0u) {
            if (sh->abort_flag) return false;
            if (lfptx::globaltimer_ns() - t0 > P.budget_ns || (((spins & 1023u) == 0u) && *((volatile unsigned*)P.status) != 0u)) {
                atomicOr(P.status, 2u);          // a wait on a barrier ran out
                sh->abort_flag = 1u;
                return false;
            }
        }
    }
    return true;
}

// Shared-memory matrix descriptors of a 16-bit operand block in the 128-byte swizzle.
// K-major: 128 rows of 64 contraction steps (128 bytes), eight rows per 1024-byte atom (SBO).
// MN-major: 64 rows/columns run along a 128-byte line, eight contraction steps form an atom, the next eight
// follow after 1024 bytes (SBO), the next 64 rows/columns after 8 KiB (LBO).
template <bool MN>
__device__ __forceinline__ unsigned long long lt_desc(unsigned addr)
{
    unsigned long long d = (unsigned long long)((addr & 0x3FFFFu) >> 4);
    d |= (unsigned long long)(MN ? (8192u >> 4) : 1u) << 16;
    d |= (unsigned long long)(1024u >> 4) << 32;
    d |= 1ull << 46;                   // descriptor version of this architecture
    d |= 2ull << 61;                   // 128-byte swizzle
    return d;
}
// bytes from one instruction's operand (16 contraction steps) to the next
template <bool MN>
__device__ __forceinline__ unsigned lt_step(int kk) { return (unsigned)kk * (MN ? 2048u : 32u); }

template <bool PAIR>
__device__ __forceinline__ void lt_commit(unsigned bar)        // PAIR: arrives in both CTAs
{
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((unsigned short)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void lt_arrive_cluster(unsigned cluster_bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// the same where no memory that the generic proxy wrote is handed over (the tcgen05 fences order what is)
__device__ __forceinline__ void lt_arrive_cluster_relaxed(unsigned cluster_bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void lt_complete_tx(unsigned bar, unsigned bytes)
{
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ unsigned lt_ld_cluster_u32(unsigned addr)
{
    unsigned v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 lt_ld_cluster_f4(unsigned addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

// One operand block of a stage: `mn` the first row/column, `k` the first contraction step; `cols` as many as are
// needed of its 128 (of an MN-major block, in boxes of 64; of a K-major one, what the map's box says).
template <bool MN, bool PAIR>
__device__ __forceinline__ void lt_load(unsigned dst, const CUtensorMap* map, unsigned bar, int mn, int k, int cols = 128)
{
    if (MN) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i * 64 >= cols) break;
            if (PAIR) lfptx::tma_load_2d_pair(dst + i * 8192, map, bar, mn + i * 64, k);
            else lfptx::tma_load_2d(dst + i * 8192, map, bar, mn + i * 64, k);
        }
    } else {
        if (PAIR) lfptx::tma_load_2d_pair(dst, map, bar, k, mn);
        else lfptx::tma_load_2d(dst, map, bar, k, mn);
    }
}

// tile of a persistent schedule: bands of 2048 rows, column by column inside a band, so that the
// tiles worked on at one time share both operands in L2
template <typename PARAMS>
__device__ __forceinline__ void lp_tile(int t, const PARAMS& P, int& tm, int& tn)
{
    const int per_band = P.band * P.tiles_n, band = t / per_band, in = t - band * per_band;
    const int rows = min(P.band, P.tiles_m - band * P.band);
    tn = in / rows;
    tm = band * P.band + (in - tn * rows);
}

inline lf_encode_fn lt_encode()
{
    static lf_encode_fn fn = nullptr;
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<lf_encode_fn>(p);
        else
            cudaGetLastError();
    }
    return fn;
}

// row-major [rows][cols] matrix, boxes of `bc` columns x `br` rows in the 128-byte swizzle
inline bool lt_map(CUtensorMap* m, CUtensorMapDataType type, const void* base, int rows, int cols, long long ld, int bc, int br)
{
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * (type == CU_TENSOR_MAP_DATA_TYPE_UINT8 ? 1 : 2)};
    cuuint32_t box[2] = {(cuuint32_t)bc, (cuuint32_t)br};
    cuuint32_t estr[2] = {1, 1};
    return lt_encode()(m, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline void lt_cluster_config(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* at, int grid, int threads, int cluster, size_t smem, cudaStream_t s)
{
    *cfg = cudaLaunchConfig_t{};
    cfg->gridDim = dim3((unsigned)grid);
    cfg->blockDim = dim3((unsigned)threads);
    cfg->dynamicSmemBytes = smem;
    cfg->stream = s;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cluster;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg->attrs = at;
    cfg->numAttrs = 2;
}

}  // namespace

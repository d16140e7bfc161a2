// The dense layer for up to 16 tokens:  y = sigma(x w^T + bias) + residual, z in 8 bits.
// 2 n_in n_out bytes of weights are read for at most 16 multiply-adds each, so the layer is bound by memory and
// the kernel is a stream: every lane loads 128-bit pieces of four weight rows straight into the registers of
// a warp-wide 16 x 8 x 16 product (the order of the contraction is the same permutation for both operands, so
// a lane's eight consecutive values serve as they are), with up to 16 such loads in flight.  A CTA has 32
// output columns -- one 8-bit scale group --, its eight warps split the contraction, and where that
// leaves multiprocessors idle a cluster of CTAs splits it further; partial sums meet in shared memory
// in a fixed order.
#include "lf_ops_internal.h"
#include "lf_ptx.cuh"
#include "lf_rows.cuh"

namespace {

using namespace lfrow;

constexpr int SR_ROWS = 32, SR_WARPS = 8, SR_UNROLL = 4;

template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1, T);
template <>
__device__ __forceinline__ void mma16816(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1, __nv_bfloat16)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1, __half)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 ld_weights(const void* p)     // read once
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// TT: blocks of eight tokens (1 or 2)
template <typename T, int TT>
__global__ void __launch_bounds__(SR_WARPS * 32, 2) k_linear_stream(const lf_product p, int splits)
{
    // [warp][token][column]: 33 words a row keep the lanes of a fragment on different banks
    __shared__ float red[SR_WARPS][TT * 8][SR_ROWS + 1];
    __shared__ float part_sum[TT * 8][SR_ROWS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int part = (int)(blockIdx.x % (unsigned)splits);
    const int n0 = (int)(blockIdx.x / (unsigned)splits) * SR_ROWS;
    const T* w = static_cast<const T*>(p.b);
    const T* x = static_cast<const T*>(p.a);

    const int chunks = (p.K + 31) >> 5, slots = splits * SR_WARPS, slot = part * SR_WARPS + warp;
    const int c0 = (int)((long long)chunks * slot / slots), c1 = (int)((long long)chunks * (slot + 1) / slots);

    const T* wr[4];
    bool wv[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int row = n0 + g + 8 * r;
        wv[r] = row < p.N;
        wr[r] = w + (size_t)(wv[r] ? row : 0) * p.ld_b + 8 * t;
    }
    const T* xr[TT];
    bool xv[TT];
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const int tok = j * 8 + g;
        xv[j] = tok < p.M;
        xr[j] = x + (size_t)(xv[j] ? tok : 0) * p.ld_a + 8 * t;
    }
    float acc[2][TT][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < TT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.f;

    lf_grid_wait();
    lf_grid_release();
    for (int c = c0; c < c1; c += SR_UNROLL) {
        uint4 a[SR_UNROLL][4], b[SR_UNROLL][TT];
#pragma unroll
        for (int u = 0; u < SR_UNROLL; ++u) {
            const int k = (c + u) * 32;
            const bool kv = c + u < c1 && k + 8 * t < p.K;
#pragma unroll
            for (int r = 0; r < 4; ++r) a[u][r] = kv && wv[r] ? ld_weights(wr[r] + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < TT; ++j) b[u][j] = kv && xv[j] ? *reinterpret_cast<const uint4*>(xr[j] + k) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < SR_UNROLL; ++u)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int j = 0; j < TT; ++j) {
                    mma16816(acc[m][j], a[u][2 * m].x, a[u][2 * m + 1].x, a[u][2 * m].y, a[u][2 * m + 1].y, b[u][j].x, b[u][j].y, T());
                    mma16816(acc[m][j], a[u][2 * m].z, a[u][2 * m + 1].z, a[u][2 * m].w, a[u][2 * m + 1].w, b[u][j].z, b[u][j].w, T());
                }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < TT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) red[warp][j * 8 + 2 * t + (i & 1)][m * 16 + g + 8 * (i >> 1)] = acc[m][j][i];
    __syncthreads();
    // a warp takes a token at a time, a lane a column
    for (int tok = warp; tok < TT * 8; tok += SR_WARPS) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < SR_WARPS; ++i) v += red[i][tok][lane];
        part_sum[tok][lane] = v;
    }
    if (splits > 1) lfptx::cluster_sync_all();
    if (part == 0) {
        const int col = n0 + lane;
        for (int tok = warp; tok < TT * 8 && tok < p.M; tok += SR_WARPS) {
            float v = part_sum[tok][lane];
            for (int q = 1; q < splits; ++q) {
                float o;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o) : "r"(lfptx::map_to_cta(lfptx::smem_u32(&part_sum[tok][lane]), (unsigned)q)) : "memory");
                v += o;
            }
            const bool in = col < p.N;
            if (in && p.bias) v += p.bias[col];
            if (p.q) {
                const unsigned b = scale_byte(__reduce_max_sync(0xFFFFFFFFu, in ? abs_bits(v) : 0u));
                if (in) p.q[(size_t)tok * p.N + col] = (unsigned char)(to_e4m3x4(v * inv_scale(b), 0.f, 0.f, 0.f) & 0xFFu);
                if (lane == 0) p.s[(size_t)tok * ((p.N + 31) / 32) + (n0 >> 5)] = (unsigned char)b;
            }
            float two[2] = {v, 0.f};
            act_n<true, 2>(two, p.act);
            v = two[0];
            if (in) {
                if (p.add) v += (float)static_cast<const T*>(p.add)[(size_t)tok * p.ld_add + col];
                static_cast<T*>(p.d)[(size_t)tok * p.ld_d + col] = (T)v;
            }
        }
    }
    if (splits > 1) lfptx::cluster_sync_all();       // the other parts' sums have been read
}

template <typename T>
cudaError_t stream_go(const lf_product& p, int sm_count, cudaStream_t s, int* splits_out)
{
    // Two CTAs per multiprocessor keep enough loads in flight; a part is at least two unrolled steps of a warp.
    const int tiles = (p.N + SR_ROWS - 1) / SR_ROWS, chunks = (p.K + 31) / 32;
    int splits = 1;
    while (splits < 8 && tiles * splits < 2 * sm_count && chunks >= splits * 2 * SR_WARPS * 2 * SR_UNROLL) splits *= 2;
    *splits_out = splits;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    cfg.gridDim = dim3((unsigned)(tiles * splits));
    cfg.blockDim = dim3(SR_WARPS * 32);
    cfg.stream = s;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)splits; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 2;
    if (p.M <= 8) return cudaLaunchKernelEx(&cfg, k_linear_stream<T, 1>, p, splits);
    return cudaLaunchKernelEx(&cfg, k_linear_stream<T, 2>, p, splits);
}

}  // namespace

cudaError_t lfk_linear_stream(const lf_product& p, int sm_count, cudaStream_t s, int* splits)
{
    return p.dtype == LF_BF16 ? stream_go<__nv_bfloat16>(p, sm_count, s, splits) : stream_go<__half>(p, sm_count, s, splits);
}

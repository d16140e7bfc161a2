// Internal declarations of the layer operators (lf_ops handle and the launchers behind it).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "leapfrog.h"

struct lf_ops {
    int device;
    int sm_count;
    int max_pairs;              // CTA pairs of the 256 x 256 tile kernels that are resident at once (0: none)
    int max_pair_splits;        // resident clusters of the split pair kernels
    cudaStream_t stream;
    unsigned char* ws;          // workspace: fixed part first, then the unpacked layer input
    size_t ws_bytes;
    unsigned* counters;         // LF_OPS_COUNTERS words, zero between calls
    unsigned* status_dev;
    unsigned* status_host;
    long long wait_budget_us;
    int withhold;
    int last_cuda_error;
    lf_ops_stats stats;
};

// The fixed part of the workspace holds partial column sums: at most LF_OPS_PARTIAL_ROWS rows of at
// most LF_OPS_MAX_NORM floats (gain gradients), or rows of any width that fit the same bytes (bias gradients).
constexpr int LF_OPS_MAX_NORM = 16384;
constexpr int LF_OPS_PARTIAL_ROWS = 320;
constexpr size_t LF_OPS_FIXED_BYTES = (size_t)LF_OPS_PARTIAL_ROWS * LF_OPS_MAX_NORM * sizeof(float);

constexpr int LF_OPS_MAX_WIDTH = 1 << 24;
constexpr int LF_OPS_COUNTERS = LF_OPS_MAX_WIDTH / 256;      // one per 256 columns of a bias gradient

// (the error is taken back: pending, it would be reported as another call's)
#define LF_OPS_TRY(o, expr)                                     \
    do {                                                        \
        cudaError_t e__ = (expr);                               \
        if (e__ != cudaSuccess) {                               \
            cudaGetLastError();                                 \
            (o)->last_cuda_error = (int)e__;                    \
            return LF_ECUDA;                                    \
        }                                                       \
    } while (0)

// Kernels of the layer operators may be launched while the kernel before them is still running: each waits for it
// (lf_grid_wait) before it touches global memory and lets the next one be launched (lf_grid_release) as
// soon as its own blocks are under way, so that only the set-up overlaps.
#ifdef __CUDACC__
__device__ __forceinline__ void lf_grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void lf_grid_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// in clusters of `cluster` blocks
template <typename... P, typename... A>
cudaError_t lf_launch_clusters(void (*kernel)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t s, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
template <typename... P, typename... A>
cudaError_t lf_launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, A... args)
{
    return lf_launch_clusters(kernel, grid, threads, smem, 1, s, args...);
}
#endif

inline size_t lf_groups(int n) { return ((size_t)n + 31) / 32; }

typedef CUresult (*lf_encode_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// ---- launchers: sizes and pointers are checked by the caller ------------------------------------
int lf_rows_init();                 // opts the kernels in
cudaError_t lfk_rms_norm(const lf_rms_norm_args& a, int sm_count, cudaStream_t s);
cudaError_t lfk_rms_norm_backward(const lf_rms_norm_backward_args& a, float* partial, int sm_count, cudaStream_t s,
                                  int* launches);
cudaError_t lfk_pack8(int dtype, int tokens, int n, const void* x, long long ld, unsigned char* q, unsigned char* s8,
                      int sm_count, cudaStream_t s);
cudaError_t lfk_unpack8(int dtype, int act, int tokens, int n, const unsigned char* q, const unsigned char* s8, void* x,
                        long long ld, int sm_count, cudaStream_t s);
cudaError_t lfk_act_backward(int dtype, int act, int tokens, int n, const void* dy, long long ld_dy,
                             const unsigned char* q, const unsigned char* s8, void* dz, long long ld_dz, int sm_count,
                             cudaStream_t s);
// grad_w's bias gradient (where a.gb) and its input from 8 bits into x (where a.q), in one launch; partial:
// LF_OPS_FIXED_BYTES of scratch, counters: LF_OPS_COUNTERS words that are zero between calls
cudaError_t lfk_grad_w_prepare(const lf_linear_grad_w_args& a, long long ld_dz, void* x, float* partial, unsigned* counters, int sm_count,
                               cudaStream_t s);

// ---- matrix products -----------------------------------------------------------------------------
// What a product is for: which operands are transposed and what its epilogue does.
enum lf_prod { LF_PROD_FORWARD = 0, LF_PROD_GRAD_X = 1, LF_PROD_GRAD_W = 2 };

// D[m][n] = sum_k A[m][k] B[n][k], epilogue on D.
struct lf_product {
    int prod;                   // enum lf_prod
    int dtype;                  // LF_BF16 or LF_F16
    int out_dtype;              // dtype, or LF_F32 (LF_PROD_GRAD_W)
    int act;
    int M, N, K;                // of the product (not of the layer)
    const void* a; long long ld_a;
    const void* b; long long ld_b;
    void* d; long long ld_d;
    const float* bias;          // [N]
    const void* add; long long ld_add;   // residual
    unsigned char *q, *s;       // FORWARD: written; GRAD_X: read
};
int lf_product_tc_init(lf_ops* o);              // opts the kernels in, finds max_pairs
int lf_product_tc(lf_ops* o, const lf_product& p);
// few tokens, forward only
constexpr int LF_STREAM_MAX_TOKENS = 16;
int lf_linear_stream_init();
cudaError_t lfk_linear_stream(const lf_product& p, int sm_count, cudaStream_t s);

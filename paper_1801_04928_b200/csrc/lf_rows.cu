// Row operators of the layer: root-mean-square norm with the residual's addition (both directions),
// the 8-bit form of a matrix, and column sums.  All of them move every element once and are bound
// by memory; a lane always holds eight consecutive columns (one 128-bit access in 16 bits), the
// four lanes of an 8-bit scale group are neighbours.
#include "lf_ops_internal.h"
#include "lf_rows.cuh"

namespace {

using namespace lfrow;

inline int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* red)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if (TPR > 32) {
        __syncthreads();                     // the previous row's partial sums have been read
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < TPR / 32; ++i) v += red[i];
    }
    return v;
}

// ---- h = x + residual, y = h / sqrt(mean h^2 + eps) * gain -------------------------------------------
// A block of TPR threads takes one row at a time, VPT vectors of eight columns per thread: the row stays
// in registers between the sum and the scaling, so x and residual are read once.
template <typename T, int TPR, int VPT>
__global__ void __launch_bounds__(TPR) k_rms_norm(const lf_rms_norm_args a)
{
    __shared__ float red[TPR / 32];
    const int nv = a.n >> 3;
    const size_t gpr = (size_t)((a.n + 31) / 32);
    for (int row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + (size_t)row * a.ld_x;
        vec8<T> xv[VPT], rv[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + threadIdx.x;
            xv[j].zero(); rv[j].zero();
            if (i < nv) {
                xv[j].load(x + 8 * i);
                if (a.residual) rv[j].load(static_cast<const T*>(a.residual) + (size_t)row * a.ld_residual + 8 * i);
            }
        }
        float h[VPT][8], ss = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + threadIdx.x;
            float r[8];
            xv[j].get(h[j]);
            if (a.residual) {
                rv[j].get(r);
#pragma unroll
                for (int k = 0; k < 8; ++k) h[j][k] += r[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) ss = fmaf(h[j][k], h[j][k], ss);
            if (a.h && i < nv) {
                vec8<T> o;
                o.set(h[j]);
                o.store(static_cast<T*>(a.h) + (size_t)row * a.ld_h + 8 * i);
            }
        }
        ss = row_sum<TPR>(ss, red);
        const float rstd = 1.0f / sqrtf(ss / (float)a.n + a.eps);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + threadIdx.x;
            if (i < nv) {
                float g[8];
                vec8<float> gv;
                gv.load(a.gain + 8 * i);
                gv.get(g);
#pragma unroll
                for (int k = 0; k < 8; ++k) h[j][k] = h[j][k] * rstd * g[k];
                if (a.y) {
                    vec8<T> o;
                    o.set(h[j]);
                    o.store(static_cast<T*>(a.y) + (size_t)row * a.ld_y + 8 * i);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) h[j][k] = 0.f;
            }
            if (a.q) {                       // all lanes of a warp take part: j * TPR + 32 w is uniform
                const unsigned b = group_byte(h[j]);
                if (i < nv) {
                    *reinterpret_cast<uint2*>(a.q + (size_t)row * a.n + 8 * i) = quantize8(h[j], b);
                    if ((i & 3) == 0) a.s[(size_t)row * gpr + (i >> 2)] = (unsigned char)b;
                }
            }
        }
    }
}

// ---- dh = r (u - h r mean(u h r)) + dres, partial column sums of dy h r -----------------------------
template <typename T, int TPR, int VPT>
__global__ void __launch_bounds__(TPR) k_rms_norm_backward(const lf_rms_norm_backward_args a, float* partial)
{
    __shared__ float red[TPR / 32], red2[TPR / 32];
    const int nv = a.n >> 3;
    float dg[VPT][8];
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) dg[j][k] = 0.f;
    for (int row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        vec8<T> hv[VPT], yv[VPT], rv[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + threadIdx.x;
            hv[j].zero(); yv[j].zero(); rv[j].zero();
            if (i < nv) {
                hv[j].load(static_cast<const T*>(a.h) + (size_t)row * a.ld_h + 8 * i);
                yv[j].load(static_cast<const T*>(a.dy) + (size_t)row * a.ld_dy + 8 * i);
                if (a.dres) rv[j].load(static_cast<const T*>(a.dres) + (size_t)row * a.ld_dres + 8 * i);
            }
        }
        float ss = 0.f, su = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + threadIdx.x;
            float h[8], y[8], g[8];
            vec8<float> gv;
            gv.zero();
            if (i < nv) gv.load(a.gain + 8 * i);
            gv.get(g);
            hv[j].get(h);
            yv[j].get(y);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                ss = fmaf(h[k], h[k], ss);
                su = fmaf(g[k] * y[k], h[k], su);
            }
        }
        ss = row_sum<TPR>(ss, red);
        su = row_sum<TPR>(su, red2);
        const float r = 1.0f / sqrtf(ss / (float)a.n + a.eps);
        const float c = su * r * r / (float)a.n;         // mean(u h r) r
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + threadIdx.x;
            if (i >= nv) continue;
            float h[8], y[8], g[8], d[8];
            vec8<float> gv;
            gv.load(a.gain + 8 * i);
            gv.get(g);
            hv[j].get(h);
            yv[j].get(y);
            rv[j].get(d);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                dg[j][k] = fmaf(y[k], h[k] * r, dg[j][k]);
                const float t = r * (g[k] * y[k] - h[k] * c);
                d[k] = a.dres ? t + d[k] : t;
            }
            vec8<T> o;
            o.set(d);
            o.store(static_cast<T*>(a.dh) + (size_t)row * a.ld_dh + 8 * i);
        }
    }
    if (partial) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + threadIdx.x;
            if (i < nv) {
                vec8<float> o;
                o.set(dg[j]);
                o.store(partial + (size_t)blockIdx.x * a.n + 8 * i);
            }
        }
    }
}

// out[c] = sum over the rows of partial[rows][n], in row order per thread group, then across groups
__global__ void __launch_bounds__(256) k_sum_rows(const float* partial, int rows, int n, float* out)
{
    __shared__ float red[8][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), g = threadIdx.x >> 5;
    float v = 0.f;
    if (c < n)
        for (int r = g; r < rows; r += 8) v += partial[(size_t)r * n + c];
    red[g][threadIdx.x & 31] = v;
    __syncthreads();
    if (g == 0 && c < n) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t += red[i][threadIdx.x & 31];
        out[c] = t;
    }
}

// column sums of a 16-bit matrix: a block takes 256 columns (a warp all of them, eight per lane) and every
// gridDim.y-th run of rows
template <typename T>
__global__ void __launch_bounds__(256) k_colsum16(const T* x, long long ld, int tokens, int n, float* partial)
{
    __shared__ float red[8][256];
    const int c = blockIdx.x * 256 + (threadIdx.x & 31) * 8, w = threadIdx.x >> 5;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < n) {
#pragma unroll 4
        for (int r = blockIdx.y * 8 + w; r < tokens; r += gridDim.y * 8) {
            vec8<T> xv;
            float f[8];
            xv.load(x + (size_t)r * ld + c);
            xv.get(f);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += f[k];
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) red[w][(threadIdx.x & 31) * 8 + k] = v[k];
    __syncthreads();
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (col < n) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t += red[i][threadIdx.x];
        partial[(size_t)blockIdx.y * n + col] = t;
    }
}

// ---- 8-bit form -------------------------------------------------------------------------------------
// Threads run along the row (blockIdx.x) and take every gridDim.y-th row.
template <typename T>
__global__ void __launch_bounds__(256) k_pack8(const T* x, long long ld, int tokens, int n, unsigned char* q, unsigned char* s)
{
    const int i = blockIdx.x * 256 + threadIdx.x, nv = n >> 3;
    if ((i & ~31) >= nv) return;             // whole warps only: the group maximum is taken across lanes
    const size_t gpr = (size_t)((n + 31) / 32);
    for (int row = blockIdx.y; row < tokens; row += gridDim.y) {
        vec8<T> v;
        v.zero();
        if (i < nv) v.load(x + (size_t)row * ld + 8 * i);
        float f[8];
        v.get(f);
        const unsigned b = group_byte(f);
        if (i < nv) {
            *reinterpret_cast<uint2*>(q + (size_t)row * n + 8 * i) = quantize8(f, b);
            if ((i & 3) == 0) s[(size_t)row * gpr + (i >> 2)] = (unsigned char)b;
        }
    }
}

// GRAD = false: x = sigma(value);  GRAD = true: x = dy * sigma'(value)
template <typename T, bool GRAD>
__global__ void __launch_bounds__(256) k_unpack8(const unsigned char* q, const unsigned char* s, const T* dy,
                                                 long long ld_dy, int tokens, int n, int kind, T* x, long long ld)
{
    constexpr bool FAST = sizeof(T) == 2;
    const int i = blockIdx.x * 256 + threadIdx.x, nv = n >> 3;
    if (i >= nv) return;
    const size_t gpr = (size_t)((n + 31) / 32);
    for (int row = blockIdx.y; row < tokens; row += gridDim.y) {
        float v[8];
        dequantize8(*reinterpret_cast<const uint2*>(q + (size_t)row * n + 8 * i), s[(size_t)row * gpr + (i >> 2)], v);
        vec8<T> o;
        if (GRAD) {
            float d[8];
            o.load(dy + (size_t)row * ld_dy + 8 * i);
            o.get(d);
            prime_n<FAST, 8>(d, v, kind);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = d[k];
        } else {
            act_n<FAST, 8>(v, kind);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = clamp_keep_nan(v[k], max_finite(T()));
        }
        o.set(v);
        o.store(x + (size_t)row * ld + 8 * i);
    }
}

dim3 row_grid(int tokens, int n, int sm_count)
{
    const int bx = ceil_div(n >> 3, 256);
    int by = ceil_div((long long)sm_count * 16, bx);
    if (by > tokens) by = tokens;
    if (by > 65535) by = 65535;
    return dim3((unsigned)bx, (unsigned)by);
}

// Threads per row: four vectors per thread when there are rows enough to fill the device, otherwise
// one, so that a few rows are read by as many threads as they have vectors.
template <template <typename, int, int> class F, typename T, typename... A>
void pick_row_shape(int n, bool many, A&&... args)
{
    const int nv = n >> 3;
    if (many) {
        if (nv <= 32) F<T, 32, 1>::go(args...);
        else if (nv <= 64) F<T, 32, 2>::go(args...);
        else if (nv <= 128) F<T, 32, 4>::go(args...);
        else if (nv <= 256) F<T, 64, 4>::go(args...);
        else if (nv <= 512) F<T, 128, 4>::go(args...);
        else if (nv <= 1024) F<T, 256, 4>::go(args...);
        else F<T, 512, 4>::go(args...);
    } else {
        if (nv <= 32) F<T, 32, 1>::go(args...);
        else if (nv <= 128) F<T, 128, 1>::go(args...);
        else if (nv <= 512) F<T, 512, 1>::go(args...);
        else if (nv <= 1024) F<T, 512, 2>::go(args...);
        else F<T, 512, 4>::go(args...);
    }
}

template <typename T, int TPR, int VPT>
struct norm_go {
    static void go(const lf_rms_norm_args& a, int sm_count, cudaStream_t s)
    {
        const int per_sm = 2048 / TPR < 16 ? 2048 / TPR : 16;
        const int grid = a.tokens < sm_count * per_sm ? a.tokens : sm_count * per_sm;
        k_rms_norm<T, TPR, VPT><<<grid, TPR, 0, s>>>(a);
    }
};
template <typename T, int TPR, int VPT>
struct norm_backward_go {
    static void go(const lf_rms_norm_backward_args& a, float* partial, int sm_count, cudaStream_t s, int* grid_out)
    {
        const int per_sm = 1024 / TPR < 8 ? 1024 / TPR : 8;
        // partial sums: one row per block, within the fixed workspace
        long long most = (long long)(LF_OPS_FIXED_BYTES / sizeof(float)) / a.n;
        if (most > (long long)sm_count * per_sm) most = (long long)sm_count * per_sm;
        const int grid = a.tokens < most ? a.tokens : (int)most;
        k_rms_norm_backward<T, TPR, VPT><<<grid, TPR, 0, s>>>(a, a.dgain ? partial : nullptr);
        *grid_out = grid;
    }
};

}  // namespace

cudaError_t lfk_rms_norm(const lf_rms_norm_args& a, int sm_count, cudaStream_t s)
{
    const bool many = a.tokens >= 2 * sm_count;
    if (a.dtype == LF_F32) pick_row_shape<norm_go, float>(a.n, many, a, sm_count, s);
    else if (a.dtype == LF_BF16) pick_row_shape<norm_go, __nv_bfloat16>(a.n, many, a, sm_count, s);
    else pick_row_shape<norm_go, __half>(a.n, many, a, sm_count, s);
    return cudaGetLastError();
}

cudaError_t lfk_rms_norm_backward(const lf_rms_norm_backward_args& a, float* partial, int sm_count, cudaStream_t s,
                                  int* launches)
{
    const bool many = a.tokens >= 2 * sm_count;
    int grid = 0;
    if (a.dtype == LF_F32) pick_row_shape<norm_backward_go, float>(a.n, many, a, partial, sm_count, s, &grid);
    else if (a.dtype == LF_BF16) pick_row_shape<norm_backward_go, __nv_bfloat16>(a.n, many, a, partial, sm_count, s, &grid);
    else pick_row_shape<norm_backward_go, __half>(a.n, many, a, partial, sm_count, s, &grid);
    *launches = 1;
    if (a.dgain) {
        k_sum_rows<<<ceil_div(a.n, 32), 256, 0, s>>>(partial, grid, a.n, a.dgain);
        *launches = 2;
    }
    return cudaGetLastError();
}

cudaError_t lfk_pack8(int dtype, int tokens, int n, const void* x, long long ld, unsigned char* q, unsigned char* s8,
                      int sm_count, cudaStream_t s)
{
    const dim3 g = row_grid(tokens, n, sm_count);
    if (dtype == LF_F32) k_pack8<float><<<g, 256, 0, s>>>(static_cast<const float*>(x), ld, tokens, n, q, s8);
    else if (dtype == LF_BF16) k_pack8<__nv_bfloat16><<<g, 256, 0, s>>>(static_cast<const __nv_bfloat16*>(x), ld, tokens, n, q, s8);
    else k_pack8<__half><<<g, 256, 0, s>>>(static_cast<const __half*>(x), ld, tokens, n, q, s8);
    return cudaGetLastError();
}

template <bool GRAD>
static cudaError_t unpack_any(int dtype, int act, int tokens, int n, const void* dy, long long ld_dy, const unsigned char* q,
                              const unsigned char* s8, void* x, long long ld, int sm_count, cudaStream_t s)
{
    const dim3 g = row_grid(tokens, n, sm_count);
    if (dtype == LF_F32)
        k_unpack8<float, GRAD><<<g, 256, 0, s>>>(q, s8, static_cast<const float*>(dy), ld_dy, tokens, n, act, static_cast<float*>(x), ld);
    else if (dtype == LF_BF16)
        k_unpack8<__nv_bfloat16, GRAD><<<g, 256, 0, s>>>(q, s8, static_cast<const __nv_bfloat16*>(dy), ld_dy, tokens, n, act,
                                                         static_cast<__nv_bfloat16*>(x), ld);
    else
        k_unpack8<__half, GRAD><<<g, 256, 0, s>>>(q, s8, static_cast<const __half*>(dy), ld_dy, tokens, n, act,
                                                  static_cast<__half*>(x), ld);
    return cudaGetLastError();
}

cudaError_t lfk_unpack8(int dtype, int act, int tokens, int n, const unsigned char* q, const unsigned char* s8, void* x,
                        long long ld, int sm_count, cudaStream_t s)
{
    return unpack_any<false>(dtype, act, tokens, n, nullptr, 0, q, s8, x, ld, sm_count, s);
}

cudaError_t lfk_act_backward(int dtype, int act, int tokens, int n, const void* dy, long long ld_dy,
                             const unsigned char* q, const unsigned char* s8, void* dz, long long ld_dz, int sm_count,
                             cudaStream_t s)
{
    return unpack_any<true>(dtype, act, tokens, n, dy, ld_dy, q, s8, dz, ld_dz, sm_count, s);
}

cudaError_t lfk_colsum16(int dtype, int tokens, int n, const void* x, long long ld, float* out, float* partial,
                         int sm_count, cudaStream_t s, int* launches)
{
    const int bx = ceil_div(n, 256);
    long long by = ceil_div((long long)sm_count * 4, bx);
    const long long most = (long long)(LF_OPS_FIXED_BYTES / sizeof(float)) / n, rows8 = ceil_div(tokens, 8);
    if (by > most) by = most;
    if (by > rows8) by = rows8;
    if (by < 1) by = 1;
    const dim3 g((unsigned)bx, (unsigned)by);
    float* to = by == 1 ? out : partial;
    if (dtype == LF_BF16) k_colsum16<__nv_bfloat16><<<g, 256, 0, s>>>(static_cast<const __nv_bfloat16*>(x), ld, tokens, n, to);
    else k_colsum16<__half><<<g, 256, 0, s>>>(static_cast<const __half*>(x), ld, tokens, n, to);
    *launches += 1;
    if (by > 1) {
        k_sum_rows<<<ceil_div(n, 32), 256, 0, s>>>(partial, (int)by, n, out);
        *launches += 1;
    }
    return cudaGetLastError();
}

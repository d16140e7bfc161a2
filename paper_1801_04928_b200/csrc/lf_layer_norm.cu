// Layer norm with the residual's addition, both directions, and the 8-bit blocks of 128 that products take their
// operands in.  Rows as in the root-mean-square norm: a lane holds eight consecutive columns, a block of 128 columns is 16
// neighbouring lanes.
#include <math_constants.h>

#include "lf_ops_internal.h"
#include "lf_ptx.cuh"
#include "lf_rows.cuh"

namespace {

using namespace lfrow;

// The scale byte (e + 127) of a block of 128: as a group of 32's, but e >= -126, so that 2^e is a normal fp32 number.
__device__ __forceinline__ unsigned block_byte(unsigned amax_bits) { return max(scale_byte(amax_bits), 1u); }

// ---- h = x + residual, y = (h - m) r gain + bias ------------------------------------------------------
// The row stays in registers between its mean, the sum of squares about that mean (which does not cancel, as the mean
// square less the squared mean would) and the result.  Bound by memory: 16384 x 4096 bf16 with residual, h and statistics 90 us, 5.95 TB/s;
// one row of 4096 2.4 us in a row of launches, 3.0 to 3.3 among others.  With 8-bit blocks as well 104 us, those and h alone 83.
template <typename T, int TPR, int VPT>
__global__ void __launch_bounds__(TPR) k_layer_norm(const lf_layer_norm_args a)
{
    __shared__ float red[2][TPR / 32];
    const int nv = a.n >> 3;
    lf_grid_wait();
    lf_grid_release();
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
        float h[VPT][8], sum = 0.f, ss = 0.f;
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
            for (int k = 0; k < 8; ++k) sum += h[j][k];
            if (a.h && i < nv) {
                vec8<T> o;
                o.set(h[j]);
                o.store(static_cast<T*>(a.h) + (size_t)row * a.ld_h + 8 * i);
            }
        }
        const float mean = row_sum<TPR>(sum, red[0]) / (float)a.n;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            if (j * TPR + threadIdx.x < nv) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    h[j][k] -= mean;
                    ss = fmaf(h[j][k], h[j][k], ss);
                }
            }
        }
        ss = row_sum<TPR>(ss, red[1]);
        const float rstd = 1.0f / sqrtf(ss / (float)a.n + a.eps);
        if (a.mean && threadIdx.x == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + threadIdx.x;
            if (i < nv) {
                float g[8], b[8];
                vec8<float> gv;
                gv.load(a.gain + 8 * i);
                gv.get(g);
                gv.zero();
                if (a.bias) gv.load(a.bias + 8 * i);
                gv.get(b);
#pragma unroll
                for (int k = 0; k < 8; ++k) h[j][k] = fmaf(h[j][k] * rstd, g[k], b[k]);
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
                unsigned m = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) m = max(m, abs_bits(h[j][k]));
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
                const unsigned b = block_byte(m);
                if (i < nv) {
                    *reinterpret_cast<uint2*>(a.q + (size_t)row * a.ld_q + 8 * i) = quantize8(h[j], b);
                    if ((i & 15) == 0) a.s[(size_t)(i >> 4) * a.tokens + row] = scale(b);
                }
            }
        }
    }
}

// ---- dh = r (u - mean u - c mean(u c)) + dres, partial column sums of dy c and dy ---------------------
// As k_rms_norm_backward: groups of TPR threads walk down the matrix, the rows ahead are on their way into shared memory
// (cp.async; a thread reads only what it copied itself, so dh may be any of the inputs), both row sums share one
// exchange, the gradients of gain and bias stay in registers and are added at the end, a partial row of 2 n per block.  16384 x 8192 bf16 with
// dres: 204 us, 5.26 TB/s, bound like that kernel by the chain load, sums, barrier, results of the two rows that a multiprocessor overlaps
// (mean and rstd a row ahead: no change); 999 x 1032 fp32 11.3 us, of which the second launch, the sum over 250 blocks, is half.
// ONE: the grid is one cluster, which adds the gradients of gain and bias through distributed shared memory: a launch instead of
// two for up to eight blocks and 4096 columns (one row of 4096: 4.1 us, one of 2344 3.5).
constexpr int NORM_CLUSTER = 8;
template <typename T, int TPR, int VPT, int GROUPS, bool ONE>
__global__ void __launch_bounds__(TPR * GROUPS) k_layer_norm_backward(const lf_layer_norm_backward_args a, float* sums, int depth)
{
    extern __shared__ __align__(16) unsigned char ring[];      // [depth][tensor][VPT][thread] pieces of eight elements
    __shared__ float2 red[2][GROUPS][TPR / 32];
    constexpr int PIECE = 8 * (int)sizeof(T), THREADS = TPR * GROUPS;
    const int nv = a.n >> 3, t = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const int tensors = a.dres ? 3 : 2;
    const unsigned slot_bytes = (unsigned)(tensors * VPT) * THREADS * PIECE;
    auto piece = [&](int slot, int tensor, int j) { return ring + (size_t)slot * slot_bytes + ((size_t)(tensor * VPT + j) * THREADS + threadIdx.x) * PIECE; };
    const int stride = gridDim.x * GROUPS, first = blockIdx.x * GROUPS + g;
    auto fetch = [&](int row, int slot) {
        if (row < a.tokens) {
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int i = j * TPR + t;
                if (i >= nv) continue;
                const T* src[3] = {static_cast<const T*>(a.h) + (size_t)row * a.ld_h, static_cast<const T*>(a.dy) + (size_t)row * a.ld_dy,
                                   static_cast<const T*>(a.dres) + (size_t)row * a.ld_dres};
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    if (k == 2 && tensors < 3) continue;
                    const unsigned dst = (unsigned)__cvta_generic_to_shared(piece(slot, k, j));
#pragma unroll
                    for (int c = 0; c < PIECE / 16; ++c) cp_async16(dst + 16 * c, src[k] + 8 * i + c * (16 / (int)sizeof(T)));
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    lf_grid_wait();
    for (int d = 0; d < depth - 1; ++d) fetch(first + d * stride, d);
    float2 dg[VPT][4], db[VPT][4];
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) dg[j][k] = db[j][k] = f2(0.f);
    const float inv_n = 1.0f / (float)a.n;
    // every group of the block makes the same number of steps: the barrier is the block's
    const int steps = (a.tokens - blockIdx.x * GROUPS + stride - 1) / stride;
    int slot = 0;
    for (int st = 0; st < steps; ++st) {
        const int row = first + st * stride;
        const bool live = row < a.tokens;
        const float mean = live ? a.mean[row] : 0.f, r = live ? a.rstd[row] : 0.f;
        int ahead = slot + depth - 1;
        if (ahead >= depth) ahead -= depth;
        fetch(row + (depth - 1) * stride, ahead);
        // all but the newest depth - 1 groups of copies have landed
        if (depth == 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
        else if (depth == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else if (depth == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        const float2 minus_m = f2(-mean), rr = f2(r);        // c = (h - m) r: the difference first (h r - m r cancels where the mean is larger than the deviation)
        float2 su2 = f2(0.f), sc2 = f2(0.f);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + t;
            if (!live || i >= nv) continue;
            float h[8], y[8], gn[8];
            vec8<T> v;
            vec8<float> gv;
            gv.load(a.gain + 8 * i);
            gv.get(gn);
            v.load(reinterpret_cast<const T*>(piece(slot, 0, j)));
            v.get(h);
            v.load(reinterpret_cast<const T*>(piece(slot, 1, j)));
            v.get(y);
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const float2 u = mul2(make_float2(gn[k], gn[k + 1]), make_float2(y[k], y[k + 1]));
                su2 = add2(su2, u);
                sc2 = fma2(u, mul2(add2(make_float2(h[k], h[k + 1]), minus_m), rr), sc2);
            }
        }
        float su = su2.x + su2.y, sc = sc2.x + sc2.y;
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            su += __shfl_xor_sync(0xFFFFFFFFu, su, o);
            sc += __shfl_xor_sync(0xFFFFFFFFu, sc, o);
        }
        if (TPR > 32) {
            if ((threadIdx.x & 31) == 0) red[st & 1][g][t >> 5] = make_float2(su, sc);
            __syncthreads();
            su = sc = 0.f;
#pragma unroll
            for (int i = 0; i < TPR / 32; ++i) { const float2 p = red[st & 1][g][i]; su += p.x; sc += p.y; }
        }
        const float2 mu = f2(-su * inv_n), mc = f2(-sc * inv_n);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + t;
            if (!live || i >= nv) continue;
            float h[8], y[8], gn[8], d[8];
            vec8<float> gv;
            vec8<T> o;
            gv.load(a.gain + 8 * i);
            gv.get(gn);
            o.load(reinterpret_cast<const T*>(piece(slot, 0, j)));
            o.get(h);
            o.load(reinterpret_cast<const T*>(piece(slot, 1, j)));
            o.get(y);
            if (a.dres) { o.load(reinterpret_cast<const T*>(piece(slot, 2, j))); o.get(d); }
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const float2 yk = make_float2(y[k], y[k + 1]);
                const float2 c = mul2(add2(make_float2(h[k], h[k + 1]), minus_m), rr);
                dg[j][k / 2] = fma2(yk, c, dg[j][k / 2]);
                db[j][k / 2] = add2(yk, db[j][k / 2]);
                const float2 in = fma2(c, mc, fma2(make_float2(gn[k], gn[k + 1]), yk, mu));       // u - mean u - c mean(u c)
                const float2 v = a.dres ? fma2(in, rr, make_float2(d[k], d[k + 1])) : mul2(in, rr);
                d[k] = v.x; d[k + 1] = v.y;
            }
            o.set(d);
            o.store(static_cast<T*>(a.dh) + (size_t)row * a.ld_dh + 8 * i);
        }
        if (++slot == depth) slot = 0;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    lf_grid_release();
    if (!ONE && !sums) return;
    if (GROUPS > 1) {
        // add the groups' sums in group order, the gain's first (each fits the ring, see norm_backward_go::bytes)
        float2* all = reinterpret_cast<float2*>(ring);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) all[(size_t)(j * 4 + k) * THREADS + threadIdx.x] = which ? db[j][k] : dg[j][k];
            __syncthreads();
            if (g == 0) {
#pragma unroll
                for (int j = 0; j < VPT; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int o = 1; o < GROUPS; ++o) {
                            float2& to = which ? db[j][k] : dg[j][k];
                            to = add2(to, all[(size_t)(j * 4 + k) * THREADS + o * TPR + t]);
                        }
            }
        }
        if (!ONE && g > 0) return;
    }
    float* mine = reinterpret_cast<float*>(ring);            // [2][n]
    if (ONE) __syncthreads();
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int i = j * TPR + t;
        if (i >= nv || (ONE && g > 0)) continue;
        float4* to = reinterpret_cast<float4*>((ONE ? mine : sums + (size_t)blockIdx.x * 2 * a.n) + 8 * i);
        to[0] = make_float4(dg[j][0].x, dg[j][0].y, dg[j][1].x, dg[j][1].y);
        to[1] = make_float4(dg[j][2].x, dg[j][2].y, dg[j][3].x, dg[j][3].y);
        to += a.n / 4;
        to[0] = make_float4(db[j][0].x, db[j][0].y, db[j][1].x, db[j][1].y);
        to[1] = make_float4(db[j][2].x, db[j][2].y, db[j][3].x, db[j][3].y);
    }
    if (ONE) {
        // every block adds the blocks' sums of its share of the columns, in block order
        __syncwarp();
        lfptx::cluster_sync_all();
        const unsigned from = lfptx::smem_u32(mine);
        for (int v = (int)blockIdx.x * THREADS + (int)threadIdx.x; v < a.n / 2; v += (int)gridDim.x * THREADS) {
            float4 p[NORM_CLUSTER];
#pragma unroll
            for (unsigned c = 0; c < NORM_CLUSTER; ++c)
                if (c < gridDim.x)
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                 : "=f"(p[c].x), "=f"(p[c].y), "=f"(p[c].z), "=f"(p[c].w) : "r"(lfptx::map_to_cta(from, c) + 16u * (unsigned)v) : "memory");
#pragma unroll
            for (unsigned c = 1; c < NORM_CLUSTER; ++c)
                if (c < gridDim.x) { p[0].x += p[c].x; p[0].y += p[c].y; p[0].z += p[c].z; p[0].w += p[c].w; }
            float* to = v < a.n / 4 ? a.dgain : a.dbias;
            if (to) *reinterpret_cast<float4*>(to + 4 * (v < a.n / 4 ? v : v - a.n / 4)) = p[0];
        }
        __syncwarp();
        lfptx::cluster_sync_all();                              // nobody leaves while its sums are being read
    }
}

template <typename T, int TPR, int VPT>
struct norm_go {
    static cudaError_t go(const lf_layer_norm_args& a, int sm_count, cudaStream_t s)
    {
        const int per_sm = 2048 / TPR < 16 ? 2048 / TPR : 16;
        const int grid = a.tokens < sm_count * per_sm ? a.tokens : sm_count * per_sm;
        return lf_launch(k_layer_norm<T, TPR, VPT>, dim3(grid), TPR, 0, s, a);
    }
};
// A block has about 256 threads: several rows side by side where a row takes fewer.  The ring is as deep as shared
// memory allows with two blocks per multiprocessor, up to four rows.
template <typename T, int TPR, int VPT>
struct norm_backward_go {
    static constexpr int GROUPS = TPR >= 256 ? 1 : 256 / TPR;
    static constexpr size_t slot(bool dres) { return (size_t)(dres ? 3 : 2) * VPT * TPR * GROUPS * 8 * sizeof(T); }
    static int depth(bool dres)
    {
        const size_t most = 110 * 1024;
        int d = 4;
        while (d > 1 && slot(dres) * d > most) --d;
        if (d == 1 && slot(dres) * 2 <= 220 * 1024) d = 2;         // one block per multiprocessor, two rows in flight
        return d;
    }
    // (the groups' sums, 32 bytes per thread and vector, fit one slot: two tensors of 16 bytes at least)
    static constexpr size_t one_bytes(bool dres) { return slot(dres) > (size_t)64 * TPR ? slot(dres) : (size_t)64 * TPR; }      // a row, or 2 n sums
    static cudaError_t go(const lf_layer_norm_backward_args& a, float* partial, int sm_count, cudaStream_t s, int* grid_out)
    {
        const long long blocks = ((long long)a.tokens + GROUPS - 1) / GROUPS;
        if constexpr (VPT == 1) {                                  // (few rows of up to 4096 columns)
            if ((a.dgain || a.dbias) && blocks <= NORM_CLUSTER) {
                int grid = 1;
                while (grid < blocks) grid *= 2;
                *grid_out = 0;
                return lf_launch_clusters(k_layer_norm_backward<T, TPR, VPT, GROUPS, true>, dim3((unsigned)grid), TPR * GROUPS, one_bytes(a.dres), grid, s, a,
                                          (float*)nullptr, 1);     // a row each: a ring of one
            }
        }
        const long long room = (long long)(LF_OPS_FIXED_BYTES / (2 * sizeof(float))) / a.n;
        // (wide rows: a block a multiprocessor, and as many partial rows as the workspace holds; 160 blocks of 4096 x 16384 took two rounds, 221 us)
        long long grid = room >= 2 * sm_count ? 2 * sm_count : room < sm_count ? room : sm_count;
        if (grid > blocks) grid = blocks;
        const int d = depth(a.dres);
        *grid_out = (int)grid;
        return lf_launch(k_layer_norm_backward<T, TPR, VPT, GROUPS, false>, dim3((unsigned)grid), TPR * GROUPS, slot(a.dres) * d, s, a,
                         a.dgain || a.dbias ? partial : nullptr, d);
    }
};
// shared memory is opted for once: it belongs to the kernel and not to a call
template <typename T, int TPR, int VPT>
struct norm_backward_ready {
    typedef norm_backward_go<T, TPR, VPT> shape;
    static cudaError_t go()
    {
        const size_t with = shape::slot(true) * shape::depth(true), without = shape::slot(false) * shape::depth(false);
        cudaError_t e = cudaFuncSetAttribute(k_layer_norm_backward<T, TPR, VPT, shape::GROUPS, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)(with > without ? with : without));
        if constexpr (VPT == 1)
            if (e == cudaSuccess)
                e = cudaFuncSetAttribute(k_layer_norm_backward<T, TPR, VPT, shape::GROUPS, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shape::one_bytes(true));
        return e;
    }
};

// ---- blocks of 128 -----------------------------------------------------------------------------------
// A block of 256 threads takes a tile of 128 x 128 values: a thread has 8 columns of 8 consecutive rows in registers, so
// that the largest magnitudes of rows, columns or the tile are taken, and both forms written, from one read.  Magnitudes are compared as
// integers, 16-bit ones two at a time.  The transposed form is turned in shared memory, in pieces of 8 rows of a column whose
// place is turned by the column, so that neither side meets a bank twice; it is written a piece of 16 bytes at a time, the last one of a row byte
// by byte where it is not full.  Bound by memory: both forms of 8192 x 16384 bf16 104 us, 5.2 TB/s, the transposed one 69, 5.8;
// tiles of 32000 x 4096 (weights, when they change) bf16 82 us in both forms, 58 as it lies, fp32 115 and 94.
template <typename T>
struct magnitudes {                         // of eight columns
    static constexpr int N = sizeof(T) == 2 ? 4 : 8;
    unsigned w[N];
    static __device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return sizeof(T) == 2 ? __vmaxu2(a, b) : max(a, b); }
    __device__ __forceinline__ void of(const vec8<T>& v)
    {
        if constexpr (sizeof(T) == 2) {
            w[0] = v.u.x & 0x7FFF7FFFu; w[1] = v.u.y & 0x7FFF7FFFu; w[2] = v.u.z & 0x7FFF7FFFu; w[3] = v.u.w & 0x7FFF7FFFu;
        } else {
            w[0] = abs_bits(v.a.x); w[1] = abs_bits(v.a.y); w[2] = abs_bits(v.a.z); w[3] = abs_bits(v.a.w);
            w[4] = abs_bits(v.b.x); w[5] = abs_bits(v.b.y); w[6] = abs_bits(v.b.z); w[7] = abs_bits(v.b.w);
        }
    }
    __device__ __forceinline__ void join(const magnitudes& o)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = larger(w[i], o.w[i]);
    }
    __device__ __forceinline__ unsigned largest() const       // still in pairs where they are
    {
        unsigned m = w[0];
#pragma unroll
        for (int i = 1; i < N; ++i) m = larger(m, w[i]);
        return m;
    }
    // fp32 bits of a magnitude, of the larger one of a pair
    static __device__ __forceinline__ unsigned bits(unsigned m)
    {
        if constexpr (sizeof(T) == 2) {
            const float2 f = unpack2(max(m & 0xFFFFu, m >> 16), T());
            return __float_as_uint(f.x);
        } else {
            return m;
        }
    }
};
// column 2 i and 2 i + 1 of eight
template <typename T>
__device__ __forceinline__ float2 columns_of(const vec8<T>& v, int i)
{
    if constexpr (sizeof(T) == 2) {
        return unpack2(i == 0 ? v.u.x : i == 1 ? v.u.y : i == 2 ? v.u.z : v.u.w, T());
    } else {
        return i == 0 ? make_float2(v.a.x, v.a.y) : i == 1 ? make_float2(v.a.z, v.a.w) : i == 2 ? make_float2(v.b.x, v.b.y) : make_float2(v.b.z, v.b.w);
    }
}

// TILES: a scale for the tile; TURN: the transposed form is wanted (without either: k_pack_rows)
template <typename T, bool TILES, bool TURN>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) k_pack_blocks(const lf_pack_blocks_args a)
{
    typedef magnitudes<T> mags;
    __shared__ __align__(16) unsigned col_max[TURN || TILES ? 8 : 1][TURN || TILES ? 16 * mags::N : 1];
    __shared__ __align__(16) unsigned char turned[TURN ? 128 * 128 : 16];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, warp = threadIdx.x >> 5;
    const unsigned nbx = ((unsigned)a.n + 127) / 128, nby = ((unsigned)a.tokens + 127) / 128;
    const unsigned by = blockIdx.x / nbx, bx = blockIdx.x - by * nbx;
    const int col = bx * 128 + tx * 8, row0 = by * 128 + ty * 8;
    const bool in = col < a.n;
    lf_grid_wait();
    lf_grid_release();
    vec8<T> v[8];
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        v[p].zero();
        if (in && row0 + p < a.tokens) v[p].load(static_cast<const T*>(a.x) + (size_t)(row0 + p) * a.ld_x + col);
    }
    unsigned tile = 0;
    if (TILES) {
        mags m, o;
        m.of(v[0]);
#pragma unroll
        for (int p = 1; p < 8; ++p) { o.of(v[p]); m.join(o); }
        const unsigned w = __reduce_max_sync(0xFFFFFFFFu, mags::bits(m.largest()));
        if ((threadIdx.x & 31) == 0) col_max[0][warp] = w;
        __syncthreads();
        unsigned t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, col_max[0][i]);
        tile = block_byte(t);
        if (threadIdx.x == 0) {
            if (a.s) a.s[(size_t)by * nbx + bx] = scale(tile);
            if (a.st) a.st[(size_t)bx * nby + by] = scale(tile);
        }
    }
    if (!TURN || a.q) {
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const int row = row0 + p;
            unsigned b = tile;
            if (!TILES) {
                mags m;
                m.of(v[p]);
                unsigned w = m.largest();
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) w = mags::larger(w, __shfl_xor_sync(0xFFFFFFFFu, w, o));
                b = block_byte(mags::bits(w));
            }
            if (in && row < a.tokens) {
                float f[8];
                v[p].get(f);
                *reinterpret_cast<uint2*>(a.q + (size_t)row * a.ld_q + col) = quantize8(f, b);
                if (!TILES && tx == 0) a.s[(size_t)bx * a.tokens + row] = scale(b);
            }
        }
    }
    if (!TURN) return;
    unsigned cb[8];                          // scale bytes of the eight columns
    if (TILES) {
#pragma unroll
        for (int j = 0; j < 8; ++j) cb[j] = tile;
    } else {
        mags m, o;
        m.of(v[0]);
#pragma unroll
        for (int p = 1; p < 8; ++p) { o.of(v[p]); m.join(o); }
#pragma unroll
        for (int i = 0; i < mags::N; ++i) m.w[i] = mags::larger(m.w[i], __shfl_xor_sync(0xFFFFFFFFu, m.w[i], 16));
        if ((threadIdx.x & 16) == 0) {
#pragma unroll
            for (int i = 0; i < mags::N; i += 4)
                *reinterpret_cast<uint4*>(&col_max[warp][tx * mags::N + i]) = make_uint4(m.w[i], m.w[i + 1], m.w[i + 2], m.w[i + 3]);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < mags::N; ++i) {
            unsigned w = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) w = mags::larger(w, col_max[k][tx * mags::N + i]);
            if (sizeof(T) == 2) {
                cb[2 * i & 7] = block_byte(mags::bits(w & 0xFFFFu));
                cb[(2 * i + 1) & 7] = block_byte(mags::bits(w >> 16));
            } else {
                cb[i] = block_byte(w);
            }
        }
        if (ty == 0 && in) {
            float sc[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) sc[j] = scale(cb[j]);
            vec8<float> to;
            to.set(sc);
            to.store(a.st + (size_t)by * a.n + col);
        }
    }
    // a thread's 8 x 8 values, two columns at a time: rows 0 .. 3 and 4 .. 7 of a column are a word each
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 r = make_float2(inv_scale(cb[2 * i]), inv_scale(cb[2 * i + 1]));
        float2 f[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) f[p] = mul2(columns_of(v[p], i), r);
        unsigned char* to = turned + (tx * 8 + 2 * i) * 128 + ((ty ^ tx) << 3);
        *reinterpret_cast<uint2*>(to) = make_uint2(to_e4m3x4(f[0].x, f[1].x, f[2].x, f[3].x), to_e4m3x4(f[4].x, f[5].x, f[6].x, f[7].x));
        *reinterpret_cast<uint2*>(to + 128) = make_uint2(to_e4m3x4(f[0].y, f[1].y, f[2].y, f[3].y), to_e4m3x4(f[4].y, f[5].y, f[6].y, f[7].y));
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int c = k * 32 + (threadIdx.x >> 3), u = threadIdx.x & 7, turn = c >> 3;
        uint4 w = *reinterpret_cast<const uint4*>(turned + c * 128 + ((u ^ (turn >> 1)) << 4));
        if (turn & 1) w = make_uint4(w.z, w.w, w.x, w.y);
        const int to_row = bx * 128 + c, at = by * 128 + u * 16;
        if (to_row >= a.n || at >= a.tokens) continue;
        unsigned char* to = a.qt + (size_t)to_row * a.ld_qt + at;
        if (at + 16 <= a.tokens) {
            *reinterpret_cast<uint4*>(to) = w;
        } else {
            const unsigned b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 15; ++i)
                if (at + i < a.tokens) to[i] = (unsigned char)(b[i >> 2] >> (8 * (i & 3)));
        }
    }
}

// Rows alone: a thread has eight columns of four rows, one after the other, and no block needs to know another row.  Shallower than the
// tiles above, for few rows (509 x 4096: 2.6 us), and with more loads in flight
// for many (8192 x 16384 bf16 63 us, 6.3 TB/s; as tiles of 8192 x 4096 26 us, now 17).
constexpr int PACK_ROWS = 4;
template <typename T>
__global__ void __launch_bounds__(256) k_pack_rows(const lf_pack_blocks_args a, int lanes_log2)
{
    typedef magnitudes<T> mags;
    const unsigned nv = (unsigned)a.n >> 3, nbx = (nv + 255) / 256, by = blockIdx.x / nbx, bx = blockIdx.x - by * nbx;
    const int lanes = 1 << lanes_log2, i = bx * 256 + (threadIdx.x & (lanes - 1));
    const int row0 = ((int)by * (256 >> lanes_log2) + ((int)threadIdx.x >> lanes_log2)) * PACK_ROWS;
    lf_grid_wait();
    lf_grid_release();
    vec8<T> v[PACK_ROWS];
#pragma unroll
    for (int p = 0; p < PACK_ROWS; ++p) {
        v[p].zero();
        if (i < (int)nv && row0 + p < a.tokens) v[p].load(static_cast<const T*>(a.x) + (size_t)(row0 + p) * a.ld_x + 8 * i);
    }
#pragma unroll
    for (int p = 0; p < PACK_ROWS; ++p) {
        const int row = row0 + p;
        mags m;
        m.of(v[p]);
        unsigned w = m.largest();
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) w = mags::larger(w, __shfl_xor_sync(0xFFFFFFFFu, w, o));
        const unsigned b = block_byte(mags::bits(w));
        if (i < (int)nv && row < a.tokens) {
            float f[8];
            v[p].get(f);
            *reinterpret_cast<uint2*>(a.q + (size_t)row * a.ld_q + 8 * i) = quantize8(f, b);
            if ((i & 15) == 0) a.s[(size_t)(i >> 4) * a.tokens + row] = scale(b);
        }
    }
}

template <typename T>
cudaError_t pack_of(const lf_pack_blocks_args& a, bool tiles, cudaStream_t s)
{
    const dim3 grid((unsigned)ceil_div(a.n, 128) * (unsigned)ceil_div(a.tokens, 128));       // (2^31 tiles would be 35 TB)
    if (tiles) return lf_launch(a.qt ? k_pack_blocks<T, true, true> : k_pack_blocks<T, true, false>, grid, 256, 0, s, a);
    if (a.qt) return lf_launch(k_pack_blocks<T, false, true>, grid, 256, 0, s, a);
    const int pieces = a.n >> 3;
    int log2 = 4;                            // (a block's lanes at least)
    while (log2 < 8 && (1 << log2) < pieces) ++log2;
    const long long blocks = (long long)ceil_div(pieces, 256) * ceil_div(a.tokens, (256 >> log2) * PACK_ROWS);
    return lf_launch(k_pack_rows<T>, dim3((unsigned)blocks), 256, 0, s, a, log2);
}

}  // namespace

int lf_layer_norm_init()
{
    for (int n = 256; n <= LF_OPS_MAX_NORM; n *= 2)                // every shape that pick_row_shape has
        for (int many = 0; many < 2; ++many)
            if (pick_row_shape<norm_backward_ready, float>(n, many != 0) != cudaSuccess ||
                pick_row_shape<norm_backward_ready, __nv_bfloat16>(n, many != 0) != cudaSuccess ||
                pick_row_shape<norm_backward_ready, __half>(n, many != 0) != cudaSuccess)
                return LF_ECUDA;
    return LF_OK;
}

cudaError_t lfk_layer_norm(const lf_layer_norm_args& a, int sm_count, cudaStream_t s)
{
    const bool many = a.tokens >= 2 * sm_count;
    if (a.dtype == LF_F32) return pick_row_shape<norm_go, float>(a.n, many, a, sm_count, s);
    if (a.dtype == LF_BF16) return pick_row_shape<norm_go, __nv_bfloat16>(a.n, many, a, sm_count, s);
    return pick_row_shape<norm_go, __half>(a.n, many, a, sm_count, s);
}

cudaError_t lfk_layer_norm_backward(const lf_layer_norm_backward_args& a, float* partial, int sm_count, cudaStream_t s, int* launches)
{
    const bool many = a.tokens >= 2 * sm_count;
    int grid = 0;
    cudaError_t e;
    if (a.dtype == LF_F32) e = pick_row_shape<norm_backward_go, float>(a.n, many, a, partial, sm_count, s, &grid);
    else if (a.dtype == LF_BF16) e = pick_row_shape<norm_backward_go, __nv_bfloat16>(a.n, many, a, partial, sm_count, s, &grid);
    else e = pick_row_shape<norm_backward_go, __half>(a.n, many, a, partial, sm_count, s, &grid);
    *launches = 1;
    if (e == cudaSuccess && (a.dgain || a.dbias) && grid > 0) {
        e = lfk_sum_rows(partial, grid, 2 * a.n, a.dgain, a.dbias, a.n, s);
        *launches = 2;
    }
    return e;
}

cudaError_t lfk_pack_blocks(const lf_pack_blocks_args& a, bool tiles, cudaStream_t s)
{
    if (a.dtype == LF_F32) return pack_of<float>(a, tiles, s);
    if (a.dtype == LF_BF16) return pack_of<__nv_bfloat16>(a, tiles, s);
    return pack_of<__half>(a, tiles, s);
}

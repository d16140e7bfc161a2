// Row operators of the layer: root-mean-square norm with the residual's addition (both directions),
// the 8-bit form of a matrix, and column sums.  All of them move every element once and are bound
// by memory once there are rows enough; a lane holds 8 or 16 consecutive columns (one 128- or 256-bit access
// in 16 bits), the lanes of an 8-bit scale group are neighbours.  A few rows cost a launch, 2.2 to 2.5 us.
#include "lf_ops_internal.h"
#include "lf_ptx.cuh"
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
// in registers between the sum and the scaling, so x and residual are read once.  With few rows a row has as many
// threads as vectors (one row of 4096: 2.6 us, a launch), with many four vectors per thread, for fewer
// barriers and more loads in flight.  Bound by memory: 16384 x 4096 bf16 with residual, h, y and y in 8 bits 95 to
// 102 us by the card, 6.0 to 6.35 TB/s.
template <typename T, int TPR, int VPT>
__global__ void __launch_bounds__(TPR) k_rms_norm(const lf_rms_norm_args a)
{
    __shared__ float red[TPR / 32];
    const int nv = a.n >> 3;
    const size_t gpr = (size_t)((a.n + 31) / 32);
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
                const unsigned b = group_byte<8>(h[j]);
                if (i < nv) {
                    *reinterpret_cast<uint2*>(a.q + (size_t)row * a.n + 8 * i) = quantize8(h[j], b);
                    if ((i & 3) == 0) a.s[(size_t)row * gpr + (i >> 2)] = (unsigned char)b;
                }
            }
        }
    }
}

// ---- dh = r (u - h r mean(u h r)) + dres, partial column sums of dy h r -----------------------------
// Groups of TPR threads take a row at a time and walk down the matrix.  The rows ahead are on their way into shared
// memory meanwhile (cp.async; a thread copies exactly what it will read itself, so the ring needs no
// barriers, and dh may be h, dy or dres), which keeps the memory busy through the row's two phases: with the row loaded into registers at
// the top of the loop instead, 16384 x 8192 took 283 us, 3.8 TB/s.  Both row sums share one exchange, in
// buffers that alternate, so a row has one barrier.  The gain's gradient stays in registers, eight
// columns per vector; the groups of a block add theirs at the end, one partial row per block.  16384 x 8192 bf16 with
// dres: 194 to 208 us by the card, 5.2 to 5.5 TB/s; what is left is the chain load, sums, barrier, results of a row, of which a
// multiprocessor overlaps two (blocks of 512 threads: 212 us; one block with a ring twice as deep: 265).
__device__ __forceinline__ void cp_async16(unsigned dst, const void* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// ONE: the grid is one cluster, which adds the gain's gradient through distributed shared memory (`sums` is the gradient then,
// else the partial rows): a launch instead of two.  Up to eight blocks and 4096 columns: one row of 4096 and 64 of 248 3.6 us
// instead of 5.7, 8 of 2048 4.5 instead of 5.9; wider rows gain nothing (8 of 8192: 6.2 against 5.7, 6 of 14432: 10.6, 10.9).
constexpr int NORM_CLUSTER = 8;
template <typename T, int TPR, int VPT, int GROUPS, bool ONE>
__global__ void __launch_bounds__(TPR * GROUPS) k_rms_norm_backward(const lf_rms_norm_backward_args a, float* sums, int depth)
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
    float2 dg[VPT][4];                       // packed fp32 throughout: the row's arithmetic is what limits the copies' rate
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) dg[j][k] = f2(0.f);
    // every group of the block makes the same number of steps: the barrier is the block's
    const int steps = (a.tokens - blockIdx.x * GROUPS + stride - 1) / stride;
    int slot = 0;
    for (int st = 0; st < steps; ++st) {
        const int row = first + st * stride;
        int ahead = slot + depth - 1;
        if (ahead >= depth) ahead -= depth;
        fetch(row + (depth - 1) * stride, ahead);
        // all but the newest depth - 1 groups of copies have landed
        if (depth == 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
        else if (depth == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else if (depth == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        const bool live = row < a.tokens;
        vec8<T> hv[VPT], yv[VPT];
        float2 ss2 = f2(0.f), su2 = f2(0.f);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + t;
            hv[j].zero(); yv[j].zero();
            if (!live || i >= nv) continue;
            hv[j].load(reinterpret_cast<const T*>(piece(slot, 0, j)));
            yv[j].load(reinterpret_cast<const T*>(piece(slot, 1, j)));
            float h[8], y[8], gn[8];
            vec8<float> gv;
            gv.load(a.gain + 8 * i);
            gv.get(gn);
            hv[j].get(h);
            yv[j].get(y);
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const float2 hk = make_float2(h[k], h[k + 1]);
                ss2 = fma2(hk, hk, ss2);
                su2 = fma2(mul2(make_float2(gn[k], gn[k + 1]), make_float2(y[k], y[k + 1])), hk, su2);
            }
        }
        float ss = ss2.x + ss2.y, su = su2.x + su2.y;
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
            su += __shfl_xor_sync(0xFFFFFFFFu, su, o);
        }
        if (TPR > 32) {
            if ((threadIdx.x & 31) == 0) red[st & 1][g][t >> 5] = make_float2(ss, su);
            __syncthreads();
            ss = su = 0.f;
#pragma unroll
            for (int i = 0; i < TPR / 32; ++i) { const float2 p = red[st & 1][g][i]; ss += p.x; su += p.y; }
        }
        const float r = 1.0f / sqrtf(ss / (float)a.n + a.eps);
        const float c = su * r * r / (float)a.n;         // mean(u h r) r
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + t;
            if (!live || i >= nv) continue;
            float h[8], y[8], gn[8], d[8];
            vec8<float> gv;
            vec8<T> o;
            gv.load(a.gain + 8 * i);
            gv.get(gn);
            hv[j].get(h);
            yv[j].get(y);
            if (a.dres) { o.load(reinterpret_cast<const T*>(piece(slot, 2, j))); o.get(d); }
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const float2 hk = make_float2(h[k], h[k + 1]), yk = make_float2(y[k], y[k + 1]);
                dg[j][k / 2] = fma2(yk, mul2(hk, f2(r)), dg[j][k / 2]);
                const float2 in = fma2(hk, f2(-c), mul2(make_float2(gn[k], gn[k + 1]), yk));       // u - h r mean(u h r)
                const float2 v = a.dres ? fma2(in, f2(r), make_float2(d[k], d[k + 1])) : mul2(in, f2(r));
                d[k] = v.x; d[k + 1] = v.y;
            }
            o.set(d);
            o.store(static_cast<T*>(a.dh) + (size_t)row * a.ld_dh + 8 * i);
        }
        if (++slot == depth) slot = 0;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    lf_grid_release();
    if (sums) {
        float* mine = reinterpret_cast<float*>(ring);           // (free soon; it holds at least eight floats per thread and vector)
        if (GROUPS > 1) {
            // add the groups' sums in group order
            float2* all = reinterpret_cast<float2*>(ring);
            __syncthreads();
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) all[(size_t)(j * 4 + k) * THREADS + threadIdx.x] = dg[j][k];
            __syncthreads();
            if (!ONE && g > 0) return;
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int o = 1; o < GROUPS; ++o)
                        if (!ONE || g == 0) dg[j][k] = add2(dg[j][k], all[(size_t)(j * 4 + k) * THREADS + o * TPR + t]);
        }
        if (ONE) __syncthreads();
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * TPR + t;
            if (i < nv && (!ONE || g == 0)) {
                float4* to = reinterpret_cast<float4*>((ONE ? mine : sums + (size_t)blockIdx.x * a.n) + 8 * i);
                to[0] = make_float4(dg[j][0].x, dg[j][0].y, dg[j][1].x, dg[j][1].y);
                to[1] = make_float4(dg[j][2].x, dg[j][2].y, dg[j][3].x, dg[j][3].y);
            }
        }
        if (ONE) {
            // every block adds the blocks' sums of its share of the columns, in block order
            __syncwarp();
            lfptx::cluster_sync_all();
            const unsigned from = lfptx::smem_u32(mine);
            for (int v = (int)blockIdx.x * THREADS + (int)threadIdx.x; v < a.n / 4; v += (int)gridDim.x * THREADS) {
                float4 p[NORM_CLUSTER];
#pragma unroll
                for (unsigned c = 0; c < NORM_CLUSTER; ++c)
                    if (c < gridDim.x)
                        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                     : "=f"(p[c].x), "=f"(p[c].y), "=f"(p[c].z), "=f"(p[c].w) : "r"(lfptx::map_to_cta(from, c) + 16u * (unsigned)v) : "memory");
#pragma unroll
                for (unsigned c = 1; c < NORM_CLUSTER; ++c)
                    if (c < gridDim.x) { p[0].x += p[c].x; p[0].y += p[c].y; p[0].z += p[c].z; p[0].w += p[c].w; }
                *reinterpret_cast<float4*>(sums + 4 * v) = p[0];
            }
            __syncwarp();
            lfptx::cluster_sync_all();                          // nobody leaves while its sums are being read
        }
    }
}

// out[c] = sum over the rows of partial[rows][n]: a block has 32 columns and 32 runs of rows, added in a fixed order
__global__ void __launch_bounds__(1024) k_sum_rows(const float* partial, int rows, int n, float* out)
{
    __shared__ float red[32][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), g = threadIdx.x >> 5;
    float v = 0.f;
    lf_grid_wait();
    if (c < n) {
#pragma unroll 8
        for (int r = g; r < rows; r += 32) v += partial[(size_t)r * n + c];
    }
    red[g][threadIdx.x & 31] = v;
    __syncthreads();
    v = red[threadIdx.x & 31][g];            // column g, run (lane)
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if ((threadIdx.x & 31) == 0 && blockIdx.x * 32 + g < n) out[blockIdx.x * 32 + g] = v;
}

// Column sums of a 16-bit matrix: a block takes 256 columns (a warp all of them, eight per lane) and run `by` of n_by
// runs of rows.  The block that finishes a column group last -- a counter per group says which one, and
// goes back to zero -- adds the runs, in their order.
template <typename T>
__device__ __forceinline__ void colsum_block(const T* x, long long ld, int tokens, int n, float* partial, unsigned* counters, float* out,
                                             int bx, int by, int n_by)
{
    __shared__ float red[8][256];
    __shared__ unsigned last;
    const int c = bx * 256 + (threadIdx.x & 31) * 8, w = threadIdx.x >> 5;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < n) {
#pragma unroll 8
        for (int r = by * 8 + w; r < tokens; r += n_by * 8) {
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
    const int col = bx * 256 + threadIdx.x;
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += red[i][threadIdx.x];
    if (n_by == 1) {
        if (col < n) out[col] = t;
        return;
    }
    if (col < n) partial[(size_t)by * n + col] = t;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        const unsigned k = atomicAdd(&counters[bx], 1u);
        last = k == (unsigned)(n_by - 1);
        if (last) counters[bx] = 0u;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (col < n) {
        t = 0.f;
#pragma unroll 8
        for (int i = 0; i < n_by; ++i) t += __ldcg(partial + (size_t)i * n + col);
        out[col] = t;
    }
}

// ---- 8-bit form -------------------------------------------------------------------------------------
// Threads run along the row, W columns each (16 in 256-bit accesses where widths, strides and addresses allow it, else
// 8); a block has 256 / lanes rows side by side, lanes = 2^lanes_log2 >= the row's pieces (at most 256: wider rows take
// several blocks), and walks down the matrix, ROWS_AT_ONCE rows at a time, all loads ahead of the first use.
// 8192 x 16384 bf16: packed in 61 to 64 us (6.4 to 6.7 TB/s), read back in 65 (6.2), as GELU in 73 (5.6: the unit for
// exponentials and reciprocals is 82 % busy), applied to a gradient with GELU' in 112 (6.0).
constexpr int ROWS_AT_ONCE = 4, ROWS_GRAD = 2;       // (two where a second matrix is read: registers)
template <int W> struct bytes_of;                // W e4m3 numbers
template <> struct bytes_of<16> { typedef uint4 type; };
template <> struct bytes_of<8> { typedef uint2 type; };
__device__ __forceinline__ void quantize(const float (&v)[8], unsigned byte, uint2& q) { q = quantize8(v, byte); }
__device__ __forceinline__ void quantize(const float (&v)[16], unsigned byte, uint4& q)
{
    const float r = inv_scale(byte);
    q = make_uint4(to_e4m3x4(v[0] * r, v[1] * r, v[2] * r, v[3] * r), to_e4m3x4(v[4] * r, v[5] * r, v[6] * r, v[7] * r),
                   to_e4m3x4(v[8] * r, v[9] * r, v[10] * r, v[11] * r), to_e4m3x4(v[12] * r, v[13] * r, v[14] * r, v[15] * r));
}
__device__ __forceinline__ void dequantize(uint2 q, unsigned byte, float (&v)[8]) { dequantize8(q, byte, v); }
__device__ __forceinline__ void dequantize(uint4 q, unsigned byte, float (&v)[16])
{
    const float s = scale(byte);
    from_e4m3x4(q.x, s, v[0], v[1], v[2], v[3]);
    from_e4m3x4(q.y, s, v[4], v[5], v[6], v[7]);
    from_e4m3x4(q.z, s, v[8], v[9], v[10], v[11]);
    from_e4m3x4(q.w, s, v[12], v[13], v[14], v[15]);
}

template <typename T, int W>
__global__ void __launch_bounds__(256) k_pack8(const T* x, long long ld, int tokens, int n, unsigned char* q, unsigned char* s, int lanes_log2)
{
    typedef typename bytes_of<W>::type Q;
    const int i = blockIdx.x * 256 + (threadIdx.x & ((1 << lanes_log2) - 1)), nv = n / W;
    const int first = blockIdx.y * (256 >> lanes_log2) + (threadIdx.x >> lanes_log2), stride = gridDim.y * (256 >> lanes_log2);
    const int steps = (tokens - (int)blockIdx.y * (256 >> lanes_log2) + ROWS_AT_ONCE * stride - 1) / (ROWS_AT_ONCE * stride);   // the block's: the group
                                                                                                             // maximum is taken across lanes
    const size_t gpr = (size_t)((n + 31) / 32);
    lf_grid_wait();
    lf_grid_release();
    for (int step = 0; step < steps; ++step) {
        const int row0 = first + step * ROWS_AT_ONCE * stride;
        typename piece_of<T, W>::type v[ROWS_AT_ONCE];
#pragma unroll
        for (int u = 0; u < ROWS_AT_ONCE; ++u) {
            const int row = row0 + u * stride;
            v[u].zero();
            if (i < nv && row < tokens) v[u].load(x + (size_t)row * ld + W * i);
        }
#pragma unroll
        for (int u = 0; u < ROWS_AT_ONCE; ++u) {
            const int row = row0 + u * stride;
            float f[W];
            v[u].get(f);
            const unsigned b = group_byte<W>(f);
            if (i < nv && row < tokens) {
                Q qv;
                quantize(f, b, qv);
                *reinterpret_cast<Q*>(q + (size_t)row * n + W * i) = qv;
                if ((i & (32 / W - 1)) == 0) s[(size_t)row * gpr + i / (32 / W)] = (unsigned char)b;
            }
        }
    }
}

// sigma of a piece of W columns that may lie beyond a type, one element after the other: few groups are like that, and their
// comparisons in the loop below cost it registers and 3 % of its time.  A value beyond fp32 (e = 120) is the largest fp32 number
// to sigma, so that SiLU and GELU of a negative one are 0 and not -infinity * 0; a result beyond T is T's largest number.
template <typename T, int KIND, int W>
__device__ __noinline__ void unpack_saturated(const unsigned char* q, unsigned byte, T* x)
{
#pragma unroll 1
    for (int k = 0; k < W; ++k) {
        float v, none[3];
        from_e4m3x4(q[k], scale(byte), v, none[0], none[1], none[2]);
        v = act2<sizeof(T) == 2, KIND>(f2(clamp_keep_nan(v, max_finite(0.f)))).x;
        x[k] = (T)clamp_keep_nan(v, max_finite(T()));
    }
}

// GRAD = false: x = sigma(value);  GRAD = true: x = dy * sigma'(value)
template <typename T, bool GRAD, int KIND, int W>
__device__ __forceinline__ void unpack_rows(const unsigned char* q, const unsigned char* s, const T* dy, long long ld_dy, int tokens, int n,
                                            T* x, long long ld, int bx, int by, int n_by, int lanes_log2)
{
    typedef typename bytes_of<W>::type Q;
    constexpr bool FAST = sizeof(T) == 2;
    constexpr int ROWS = GRAD ? ROWS_GRAD : ROWS_AT_ONCE;
    const int i = bx * 256 + (threadIdx.x & ((1 << lanes_log2) - 1));
    if (i >= n / W) return;
    const int first = by * (256 >> lanes_log2) + (threadIdx.x >> lanes_log2), stride = n_by * (256 >> lanes_log2);
    const size_t gpr = (size_t)((n + 31) / 32);
    for (int row0 = first; row0 < tokens; row0 += ROWS * stride) {
        Q qv[ROWS];
        unsigned sv[ROWS];
        typename piece_of<T, W>::type dv[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int row = row0 + u * stride;
            if (row < tokens) {
                qv[u] = *reinterpret_cast<const Q*>(q + (size_t)row * n + W * i);
                sv[u] = s[(size_t)row * gpr + i / (32 / W)];
                if (GRAD) dv[u].load(dy + (size_t)row * ld_dy + W * i);
            }
        }
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int row = row0 + u * stride;
            if (row >= tokens) break;
            if (!GRAD && sv[u] >= overflow_byte(T())) {
                unpack_saturated<T, KIND, W>(q + (size_t)row * n + W * i, sv[u], x + (size_t)row * ld + W * i);
                continue;
            }
            float v[W];
            dequantize(qv[u], GRAD ? prime_byte(sv[u]) : sv[u], v);
            typename piece_of<T, W>::type o;
            if (GRAD) {
                float d[W];
                dv[u].get(d);
                prime_all<FAST, W, KIND>(d, v, prime_nan(sv[u]));
                o.set(d);
            } else {
                act_all<FAST, W, KIND>(v);
                o.set(v);
            }
            o.store(x + (size_t)row * ld + W * i);
        }
    }
}
template <typename T, bool GRAD, int W>
__device__ __forceinline__ void unpack_block(const unsigned char* q, const unsigned char* s, const T* dy, long long ld_dy, int tokens, int n,
                                             int kind, T* x, long long ld, int bx, int by, int n_by, int lanes_log2)
{
    switch (kind) {
        case LF_ACT_SIGMOID: unpack_rows<T, GRAD, LF_ACT_SIGMOID, W>(q, s, dy, ld_dy, tokens, n, x, ld, bx, by, n_by, lanes_log2); break;
        case LF_ACT_TANH: unpack_rows<T, GRAD, LF_ACT_TANH, W>(q, s, dy, ld_dy, tokens, n, x, ld, bx, by, n_by, lanes_log2); break;
        case LF_ACT_RELU: unpack_rows<T, GRAD, LF_ACT_RELU, W>(q, s, dy, ld_dy, tokens, n, x, ld, bx, by, n_by, lanes_log2); break;
        case LF_ACT_SILU: unpack_rows<T, GRAD, LF_ACT_SILU, W>(q, s, dy, ld_dy, tokens, n, x, ld, bx, by, n_by, lanes_log2); break;
        case LF_ACT_GELU: unpack_rows<T, GRAD, LF_ACT_GELU, W>(q, s, dy, ld_dy, tokens, n, x, ld, bx, by, n_by, lanes_log2); break;
        default: unpack_rows<T, GRAD, LF_ACT_NONE, W>(q, s, dy, ld_dy, tokens, n, x, ld, bx, by, n_by, lanes_log2); break;
    }
}
template <typename T, bool GRAD, int W>
__global__ void __launch_bounds__(256) k_unpack8(const unsigned char* q, const unsigned char* s, const T* dy,
                                                 long long ld_dy, int tokens, int n, int kind, T* x, long long ld, int lanes_log2)
{
    lf_grid_wait();
    lf_grid_release();
    unpack_block<T, GRAD, W>(q, s, dy, ld_dy, tokens, n, kind, x, ld, blockIdx.x, blockIdx.y, gridDim.y, lanes_log2);
}

// What a weight gradient needs beside its product, in one launch: the column sums of dz (the first sum_x * sum_y
// blocks) and the layer's input unpacked (the others).  sigma(z) is rounded to T here, which the product's operands are: it is the
// number that the layer was given in the forward pass.  The gradient is then 2.8e-4 off the one of an exact sigma (f16, 70 x 520 ->
// 1024) where its own rounding is 2.1e-4, in bf16 (8192 x 16384 -> 4096) 1.9e-3 where that is 1.7e-3.
template <typename T, int W>
__global__ void __launch_bounds__(256) k_grad_w_prepare(const T* dz, long long ld_dz, int tokens, int n_out, float* partial, unsigned* counters,
                                                        float* gb, int sum_x, int sum_y, const unsigned char* q, const unsigned char* s, int n_in,
                                                        int kind, T* x, int unpack_x, int unpack_y, int lanes_log2)
{
    lf_grid_wait();
    lf_grid_release();
    const int b = blockIdx.x, sums = sum_x * sum_y;
    if (b < sums) {
        colsum_block(dz, ld_dz, tokens, n_out, partial, counters, gb, b % sum_x, b / sum_x, sum_y);
    } else {
        const int u = b - sums;
        unpack_block<T, false, W>(q, s, nullptr, 0, tokens, n_in, kind, x, n_in, u % unpack_x, u / unpack_x, unpack_y, lanes_log2);
    }
}

// grid of the row kernels for pieces of w columns, and how many threads share a row
dim3 row_grid(int tokens, int n, int w, int sm_count, int* lanes_log2)
{
    const int pieces = (n + w - 1) / w;
    int log2 = 2;                              // (a scale group's lanes at least)
    while (log2 < 8 && (1 << log2) < pieces) ++log2;
    *lanes_log2 = log2;
    const int bx = ceil_div(pieces, 256), rows = ceil_div(tokens, 256 >> log2);
    int by = ceil_div((long long)sm_count * 16, bx);
    if (by > rows) by = rows;
    if (by > 65535) by = 65535;
    return dim3((unsigned)bx, (unsigned)by);
}
// whether 256-bit accesses fit a matrix of this width, row stride and address (8-bit rows: 128-bit ones)
inline bool wide(int n, long long ld, const void* p) { return (n & 15) == 0 && (ld & 15) == 0 && (reinterpret_cast<uintptr_t>(p) & 31) == 0; }

// Threads per row: four vectors per thread when there are rows enough to fill the device, otherwise
// one, so that a few rows are read by as many threads as they have vectors.
template <template <typename, int, int> class F, typename T, typename... A>
cudaError_t pick_row_shape(int n, bool many, A&&... args)
{
    const int nv = n >> 3;
    if (many) {
        if (nv <= 32) return F<T, 32, 1>::go(args...);
        else if (nv <= 64) return F<T, 32, 2>::go(args...);
        else if (nv <= 128) return F<T, 32, 4>::go(args...);
        else if (nv <= 256) return F<T, 64, 4>::go(args...);
        else if (nv <= 512) return F<T, 128, 4>::go(args...);
        else if (nv <= 1024) return F<T, 256, 4>::go(args...);
        else return F<T, 512, 4>::go(args...);
    } else {
        if (nv <= 32) return F<T, 32, 1>::go(args...);
        else if (nv <= 128) return F<T, 128, 1>::go(args...);
        else if (nv <= 512) return F<T, 512, 1>::go(args...);
        else if (nv <= 1024) return F<T, 512, 2>::go(args...);
        else return F<T, 512, 4>::go(args...);
    }
}

template <typename T, int TPR, int VPT>
struct norm_go {
    static cudaError_t go(const lf_rms_norm_args& a, int sm_count, cudaStream_t s)
    {
        const int per_sm = 2048 / TPR < 16 ? 2048 / TPR : 16;
        const int grid = a.tokens < sm_count * per_sm ? a.tokens : sm_count * per_sm;
        return lf_launch(k_rms_norm<T, TPR, VPT>, dim3(grid), TPR, 0, s, a);
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
    static cudaError_t go(const lf_rms_norm_backward_args& a, float* partial, int sm_count, cudaStream_t s, int* grid_out)
    {
        const long long blocks = ((long long)a.tokens + GROUPS - 1) / GROUPS;
        if constexpr (VPT == 1) {                                  // (few rows of up to 4096 columns)
            if (a.dgain && blocks <= NORM_CLUSTER) {
                int grid = 1;
                while (grid < blocks) grid *= 2;
                *grid_out = 0;
                return lf_launch_clusters(k_rms_norm_backward<T, TPR, VPT, GROUPS, true>, dim3(grid), TPR * GROUPS, slot(a.dres), grid, s, a, a.dgain,
                                          1);                      // a row each: a ring of one
            }
        }
        const int at_most = 2 * sm_count < LF_OPS_PARTIAL_ROWS ? 2 * sm_count : LF_OPS_PARTIAL_ROWS;
        const int grid = blocks < at_most ? (int)blocks : at_most, d = depth(a.dres);
        *grid_out = grid;
        return lf_launch(k_rms_norm_backward<T, TPR, VPT, GROUPS, false>, dim3(grid), TPR * GROUPS, slot(a.dres) * d, s, a, a.dgain ? partial : nullptr, d);
    }
};
// The shared memory that a kernel may be launched with, with dres and without, is set once: it belongs to the
// kernel and not to a call, which another thread's call could take it away from.
template <typename T, int TPR, int VPT>
struct norm_backward_ready {
    typedef norm_backward_go<T, TPR, VPT> shape;
    static cudaError_t go()
    {
        const size_t with = shape::slot(true) * shape::depth(true), without = shape::slot(false) * shape::depth(false);
        cudaError_t e = cudaFuncSetAttribute(k_rms_norm_backward<T, TPR, VPT, shape::GROUPS, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)(with > without ? with : without));
        if constexpr (VPT == 1)
            if (e == cudaSuccess)
                e = cudaFuncSetAttribute(k_rms_norm_backward<T, TPR, VPT, shape::GROUPS, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shape::slot(true));
        return e;
    }
};

}  // namespace

int lf_rows_init()
{
    for (int n = 256; n <= LF_OPS_MAX_NORM; n *= 2)                // every shape that pick_row_shape has
        for (int many = 0; many < 2; ++many)
            if (pick_row_shape<norm_backward_ready, float>(n, many != 0) != cudaSuccess ||
                pick_row_shape<norm_backward_ready, __nv_bfloat16>(n, many != 0) != cudaSuccess ||
                pick_row_shape<norm_backward_ready, __half>(n, many != 0) != cudaSuccess)
                return LF_ECUDA;
    return LF_OK;
}

cudaError_t lfk_rms_norm(const lf_rms_norm_args& a, int sm_count, cudaStream_t s)
{
    const bool many = a.tokens >= 2 * sm_count;
    if (a.dtype == LF_F32) return pick_row_shape<norm_go, float>(a.n, many, a, sm_count, s);
    if (a.dtype == LF_BF16) return pick_row_shape<norm_go, __nv_bfloat16>(a.n, many, a, sm_count, s);
    return pick_row_shape<norm_go, __half>(a.n, many, a, sm_count, s);
}

static cudaError_t sum_rows(const float* partial, int rows, int n, float* out, cudaStream_t s)
{
    return lf_launch(k_sum_rows, dim3((unsigned)ceil_div(n, 32)), 1024, 0, s, partial, rows, n, out);
}

cudaError_t lfk_rms_norm_backward(const lf_rms_norm_backward_args& a, float* partial, int sm_count, cudaStream_t s,
                                  int* launches)
{
    const bool many = a.tokens >= 2 * sm_count;
    int grid = 0;
    cudaError_t e;
    if (a.dtype == LF_F32) e = pick_row_shape<norm_backward_go, float>(a.n, many, a, partial, sm_count, s, &grid);
    else if (a.dtype == LF_BF16) e = pick_row_shape<norm_backward_go, __nv_bfloat16>(a.n, many, a, partial, sm_count, s, &grid);
    else e = pick_row_shape<norm_backward_go, __half>(a.n, many, a, partial, sm_count, s, &grid);
    *launches = 1;
    if (e == cudaSuccess && a.dgain && grid > 0) {
        e = sum_rows(partial, grid, a.n, a.dgain, s);
        *launches = 2;
    }
    return e;
}

template <typename T>
static cudaError_t pack_of(int tokens, int n, const void* x, long long ld, unsigned char* q, unsigned char* s8, int sm_count, cudaStream_t s)
{
    int lanes;
    const int w = wide(n, ld, x) ? 16 : 8;
    const dim3 grid = row_grid(tokens, n, w, sm_count, &lanes);
    return lf_launch(w == 16 ? k_pack8<T, 16> : k_pack8<T, 8>, grid, 256, 0, s, static_cast<const T*>(x), ld, tokens, n, q, s8, lanes);
}
cudaError_t lfk_pack8(int dtype, int tokens, int n, const void* x, long long ld, unsigned char* q, unsigned char* s8,
                      int sm_count, cudaStream_t s)
{
    if (dtype == LF_F32) return pack_of<float>(tokens, n, x, ld, q, s8, sm_count, s);
    if (dtype == LF_BF16) return pack_of<__nv_bfloat16>(tokens, n, x, ld, q, s8, sm_count, s);
    return pack_of<__half>(tokens, n, x, ld, q, s8, sm_count, s);
}

template <typename T, bool GRAD>
static cudaError_t unpack_of(int act, int tokens, int n, const void* dy, long long ld_dy, const unsigned char* q, const unsigned char* s8,
                             void* x, long long ld, int sm_count, cudaStream_t s)
{
    int lanes;
    const int w = wide(n, ld, x) && (!GRAD || wide(n, ld_dy, dy)) ? 16 : 8;
    const dim3 grid = row_grid(tokens, n, w, sm_count, &lanes);
    return lf_launch(w == 16 ? k_unpack8<T, GRAD, 16> : k_unpack8<T, GRAD, 8>, grid, 256, 0, s, q, s8, static_cast<const T*>(dy), ld_dy, tokens, n,
                     act, static_cast<T*>(x), ld, lanes);
}
template <bool GRAD>
static cudaError_t unpack_any(int dtype, int act, int tokens, int n, const void* dy, long long ld_dy, const unsigned char* q,
                              const unsigned char* s8, void* x, long long ld, int sm_count, cudaStream_t s)
{
    if (dtype == LF_F32) return unpack_of<float, GRAD>(act, tokens, n, dy, ld_dy, q, s8, x, ld, sm_count, s);
    if (dtype == LF_BF16) return unpack_of<__nv_bfloat16, GRAD>(act, tokens, n, dy, ld_dy, q, s8, x, ld, sm_count, s);
    return unpack_of<__half, GRAD>(act, tokens, n, dy, ld_dy, q, s8, x, ld, sm_count, s);
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

cudaError_t lfk_grad_w_prepare(const lf_linear_grad_w_args& a, long long ld_dz, void* x, float* partial, unsigned* counters, int sm_count,
                               cudaStream_t s)
{
    int sum_x = 0, sum_y = 0;
    dim3 u(0, 0);
    if (a.gb) {
        sum_x = ceil_div(a.n_out, 256);
        long long by = ceil_div((long long)sm_count * 4, sum_x);
        const long long most = (long long)(LF_OPS_FIXED_BYTES / sizeof(float)) / a.n_out, rows = ceil_div(a.tokens, 128);
        if (by > most) by = most;
        if (by > rows) by = rows;              // at least 16 rows per warp
        sum_y = by < 1 ? 1 : (int)by;
    }
    const bool w16 = wide(a.n_in, a.n_in, x);
    int lanes = 8;
    if (a.q) u = row_grid(a.tokens, a.n_in, w16 ? 16 : 8, sm_count, &lanes);
    const dim3 grid((unsigned)(sum_x * sum_y) + u.x * u.y);
    if (a.dtype == LF_BF16)
        return lf_launch(w16 ? k_grad_w_prepare<__nv_bfloat16, 16> : k_grad_w_prepare<__nv_bfloat16, 8>, grid, 256, 0, s,
                         static_cast<const __nv_bfloat16*>(a.dz), ld_dz, a.tokens, a.n_out, partial, counters, a.gb, sum_x, sum_y, a.q, a.s, a.n_in,
                         a.act, static_cast<__nv_bfloat16*>(x), (int)u.x, (int)u.y, lanes);
    return lf_launch(w16 ? k_grad_w_prepare<__half, 16> : k_grad_w_prepare<__half, 8>, grid, 256, 0, s, static_cast<const __half*>(a.dz), ld_dz,
                     a.tokens, a.n_out, partial, counters, a.gb, sum_x, sum_y, a.q, a.s, a.n_in, a.act, static_cast<__half*>(x), (int)u.x, (int)u.y, lanes);
}

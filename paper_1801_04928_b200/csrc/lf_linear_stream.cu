// The dense layer for up to 16 tokens:  y = sigma(x w^T + bias) + residual, z in 8 bits.
// 2 n_in n_out bytes of weights are read for at most 16 multiply-adds each, so the layer is bound by memory and
// the kernel is a stream: every lane copies 128-bit pieces of four weight rows into a ring of its own in shared
// memory (cp.async: no barriers, no registers) and from there feeds a warp-wide 16 x 8 x 16 product (the order of
// the contraction is the same permutation for both operands, so a lane's eight consecutive values serve as they are).  One persistent block per multiprocessor; its warps
// split the contraction of a tile of up to 32 output columns, and every warp keeps SR_DEPTH - 1 steps
// of loads in flight, on into the next tile.  A tile has as many columns as make the tiles come out even
// over the multiprocessors (4096 columns: 147 blocks of 28; 128 of 32 left a seventh of the memory
// rate unused), or a whole 8-bit scale group where z is kept.  One token, 4096 -> 4096 bf16: 7.3 us with its launch,
// 4.6 TB/s (a plain copy of the weights' bytes: 5.1 us); with the ring in registers 11 us.  16 tokens, 1032 -> 4104: 4.7.
#include "lf_ops_internal.h"
#include "lf_ptx.cuh"
#include "lf_rows.cuh"

namespace {

using namespace lfrow;

constexpr int SR_ROWS = 32, SR_DEPTH = 4;
// The products add into their accumulator by truncation, 1.0e-7 of a sum of one sign per instruction: an accumulator takes
// 512 steps, 1024 instructions, and the fills are added with round-to-nearest.  (LONG: more than one fill, contractions
// beyond 16384 per warp; over 2^20 terms f16 results were 4.2e-4 and 5.6e-4 short without.)
constexpr int SR_FILL = 512;

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
// 16 bytes to shared memory, zeros where there is nothing to copy; CACHE: through L1 (the tokens, which every tile reads)
template <bool CACHE>
__device__ __forceinline__ void copy16(unsigned dst, const void* src, bool valid)
{
    if (CACHE) asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
    else asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}

// TT: blocks of eight tokens (1 or 2)
template <typename T, int TT, int WARPS, bool LONG>
__global__ void __launch_bounds__(WARPS * 32, 1) k_linear_stream(const lf_product p, int rows)
{
    // [tile parity][warp][token][column]: 33 words a row keep the lanes of a fragment on different banks; before
    // it the ring: [step][piece][thread] pieces of 16 bytes, each copied and read by one thread only
    extern __shared__ __align__(16) unsigned char sr_raw[];
    constexpr int PIECES = 4 + TT, THREADS = WARPS * 32;
    auto red = reinterpret_cast<float (*)[WARPS][TT * 8][SR_ROWS + 1]>(sr_raw + (size_t)SR_DEPTH * PIECES * THREADS * 16);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const T* w = static_cast<const T*>(p.b);
    const T* x = static_cast<const T*>(p.a);
    const int tiles = (p.N + rows - 1) / rows;
    const int chunks = (p.K + 31) >> 5;
    const int c0 = chunks * warp / WARPS, c1 = chunks * (warp + 1) / WARPS;
    const unsigned my_ring = lfptx::smem_u32(sr_raw) + threadIdx.x * 16;

    const T* xp[TT];
    bool xv[TT];
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        xv[j] = j * 8 + g < p.M;
        xp[j] = x + (xv[j] ? (size_t)(j * 8 + g) * p.ld_a + 8 * t : 0);
    }
    // the step that is fetched next: 32 contraction steps (c) of a tile
    int f_tile = blockIdx.x, f_c = c0;
    const T* wp[4];
    bool wv[4];
    auto rows_of = [&]() {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int in_tile = g + 8 * r, row = f_tile * rows + in_tile;
            wv[r] = f_tile < tiles && in_tile < rows && row < p.N;
            wp[r] = w + (wv[r] ? (size_t)row * p.ld_b + 8 * t : 0);
        }
    };
    auto fetch = [&](int slot) {
        if (f_tile < tiles && c0 < c1) {
            const int k = f_c * 32;
            const bool kv = k + 8 * t < p.K;
            const unsigned dst = my_ring + (unsigned)(slot * PIECES) * (THREADS * 16);
#pragma unroll
            for (int r = 0; r < 4; ++r) copy16<false>(dst + r * (THREADS * 16), kv && wv[r] ? wp[r] + k : w, kv && wv[r]);
#pragma unroll
            for (int j = 0; j < TT; ++j) copy16<true>(dst + (4 + j) * (THREADS * 16), kv && xv[j] ? xp[j] + k : x, kv && xv[j]);
            if (++f_c == c1) { f_c = c0; f_tile += gridDim.x; rows_of(); }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    rows_of();
    lf_grid_wait();
    lf_grid_release();
#pragma unroll
    for (int d = 0; d < SR_DEPTH - 1; ++d) fetch(d);
    int parity = 0, slot = 0;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, parity ^= 1) {
        float sum[2][TT][4];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < TT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[m][j][i] = 0.f;
        int c = c0;
        do {
            float acc[2][TT][4];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int j = 0; j < TT; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.f;
            for (const int to = LONG ? min(c + SR_FILL, c1) : c1; c < to; ++c) {
                fetch(slot == 0 ? SR_DEPTH - 1 : slot - 1);
                asm volatile("cp.async.wait_group %0;" ::"n"(SR_DEPTH - 1) : "memory");
                const unsigned char* from = sr_raw + (size_t)(slot * PIECES) * (THREADS * 16) + threadIdx.x * 16;
                uint4 a[4], b[TT];
#pragma unroll
                for (int r = 0; r < 4; ++r) a[r] = *reinterpret_cast<const uint4*>(from + r * (THREADS * 16));
#pragma unroll
                for (int j = 0; j < TT; ++j) b[j] = *reinterpret_cast<const uint4*>(from + (4 + j) * (THREADS * 16));
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int j = 0; j < TT; ++j) {
                        mma16816(acc[m][j], a[2 * m].x, a[2 * m + 1].x, a[2 * m].y, a[2 * m + 1].y, b[j].x, b[j].y, T());
                        mma16816(acc[m][j], a[2 * m].z, a[2 * m + 1].z, a[2 * m].w, a[2 * m + 1].w, b[j].z, b[j].w, T());
                    }
                if (++slot == SR_DEPTH) slot = 0;
            }
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int j = 0; j < TT; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[m][j][i] = LONG ? sum[m][j][i] + acc[m][j][i] : acc[m][j][i];
        } while (LONG && c < c1);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < TT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) red[parity][warp][j * 8 + 2 * t + (i & 1)][m * 16 + g + 8 * (i >> 1)] = sum[m][j][i];
        __syncthreads();
        // a warp takes a token at a time, a lane a column; the sums are added in warp order
        const int col = tile * rows + lane;
        for (int tok = warp; tok < TT * 8 && tok < p.M; tok += WARPS) {
            const bool in = lane < rows && col < p.N;
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) v += red[parity][i][tok][lane];
            if (in && p.bias) v += p.bias[col];
            if (p.q) {
                const unsigned by = scale_byte(__reduce_max_sync(0xFFFFFFFFu, in ? abs_bits(v) : 0u));
                if (in) p.q[(size_t)tok * p.N + col] = (unsigned char)(to_e4m3x4(v * inv_scale(by), 0.f, 0.f, 0.f) & 0xFFu);
                if (lane == 0) p.s[(size_t)tok * ((p.N + 31) / 32) + tile] = (unsigned char)by;
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
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// Shared memory for SR_DEPTH steps and the warps' sums: 16 warps with one block of tokens, 12 with two (197 KB each).
template <int TT, int WARPS>
constexpr size_t stream_smem() { return (size_t)SR_DEPTH * (4 + TT) * WARPS * 32 * 16 + sizeof(float) * 2 * WARPS * TT * 8 * (SR_ROWS + 1); }
template <typename T, int TT, int WARPS>
cudaError_t stream_go(const lf_product& p, int sm_count, cudaStream_t s)
{
    int rows = SR_ROWS;
    if (!p.q) {
        const int waves = (p.N + SR_ROWS * sm_count - 1) / (SR_ROWS * sm_count);
        rows = (p.N + sm_count * waves - 1) / (sm_count * waves);
        if (rows < 8) rows = 8;              // a load covers eight rows
    }
    const int tiles = (p.N + rows - 1) / rows;
    return lf_launch((p.K + 31) / 32 > WARPS * SR_FILL ? k_linear_stream<T, TT, WARPS, true> : k_linear_stream<T, TT, WARPS, false>, dim3((unsigned)(tiles < sm_count ? tiles : sm_count)), WARPS * 32, stream_smem<TT, WARPS>(), s, p, rows);
}

}  // namespace

namespace {
template <typename T, int TT, int WARPS>
bool stream_ready()
{
    constexpr int bytes = (int)stream_smem<TT, WARPS>();
    return cudaFuncSetAttribute(k_linear_stream<T, TT, WARPS, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess &&
           cudaFuncSetAttribute(k_linear_stream<T, TT, WARPS, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
}
}  // namespace

int lf_linear_stream_init()
{
    return stream_ready<__nv_bfloat16, 1, 16>() && stream_ready<__half, 1, 16>() && stream_ready<__nv_bfloat16, 2, 12>() && stream_ready<__half, 2, 12>()
               ? LF_OK : LF_ECUDA;
}

cudaError_t lfk_linear_stream(const lf_product& p, int sm_count, cudaStream_t s)
{
    if (p.M <= 8)
        return p.dtype == LF_BF16 ? stream_go<__nv_bfloat16, 1, 16>(p, sm_count, s) : stream_go<__half, 1, 16>(p, sm_count, s);
    return p.dtype == LF_BF16 ? stream_go<__nv_bfloat16, 2, 12>(p, sm_count, s) : stream_go<__half, 2, 12>(p, sm_count, s);
}

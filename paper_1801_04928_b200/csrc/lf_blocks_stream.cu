// Products of 8-bit operands with a scale for each block of 128 of the contraction, for up to 16 rows of a (a token, a
// small batch of them).  n_in n_out bytes of b are read for at most 16 multiply-adds each: bound by memory, a stream like
// k_linear_stream's.  Every lane copies 16-byte pieces of four rows of b into a ring of its own in shared memory
// (cp.async) and feeds warp-wide 16 x 8 x 32 products of e4m3 numbers with them (the order of the contraction is the
// same permutation for both operands).  A step is 64 long, half a block: its sums, exact in fp32 but for the
// tensor core's truncation of four instructions' partial sums, are multiplied by the scales and added in fp32.  One
// persistent block per multiprocessor, whose warps split the contraction of a tile of up to 32 columns.  One row of a:
// 8192 -> 65536 91 us, 5.9 TB/s; 4096 -> 32768 27 us, 4.9, of which about 6 are launch, first loads and the last tile; 4096 -> 4096 5.4.  Warps of
// their own that add the sums, so that no barrier holds the others at a tile's end: no faster, and 16 rows slower.
#include "lf_ops_internal.h"
#include "lf_ptx.cuh"
#include "lf_rows.cuh"

namespace {

using namespace lfrow;

constexpr int BS_ROWS = 32, BS_DEPTH = 4, BS_STEP = 64;
constexpr int BS_PREFETCH = 8192;               // bytes of a row of b

__device__ __forceinline__ void mma16832(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// `valid` of 16 bytes to shared memory, zeros for the others; CACHE: through L1 (a, which every tile reads)
template <bool CACHE>
__device__ __forceinline__ void copy16(unsigned dst, const void* src, int valid)
{
    if (CACHE) asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid) : "memory");
    else asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid) : "memory");
}
template <typename OUT>
__device__ __forceinline__ float as_float(const void* p, size_t at) { return (float)static_cast<const OUT*>(p)[at]; }

// TT: blocks of eight rows of a (1 or 2); B_ROWS: a scale for each row of b; share: warps to a tile
template <typename OUT, int TT, int WARPS, bool B_ROWS>
__global__ void __launch_bounds__(WARPS * 32, 1) k_blocks_stream(const lf_product_blocks_args p, int rows, int share)
{
    // [tile parity][warp][row of a][column]: 33 words keep the lanes of a fragment on different banks; before it the
    // ring: [step][piece][thread] pieces of 16 bytes, each copied and read by one thread only
    extern __shared__ __align__(16) unsigned char bs_raw[];
    constexpr int PIECES = 4 + TT, THREADS = WARPS * 32;
    auto red = reinterpret_cast<float (*)[WARPS][TT * 8][BS_ROWS + 1]>(bs_raw + (size_t)BS_DEPTH * PIECES * THREADS * 16);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int M = p.tokens, N = p.n_out, K = p.n_in;
    const int tiles = (N + rows - 1) / rows, steps = (K + BS_STEP - 1) / BS_STEP, blocks = (K + 127) >> 7;
    const int groups = WARPS / share, group = share == WARPS ? 0 : warp / share, member = warp - group * share;
    const int first = blockIdx.x * groups + group, stride = gridDim.x * groups;
    // (steps are 2^24 at most)
    const int c0 = share == WARPS ? steps * member / WARPS : steps * member / share, c1 = share == WARPS ? steps * (member + 1) / WARPS : steps * (member + 1) / share;
    const unsigned my_ring = lfptx::smem_u32(bs_raw) + threadIdx.x * 16;

    const unsigned char* xp[TT];
    bool xv[TT];
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        xv[j] = j * 8 + g < M;
        xp[j] = p.a + (xv[j] ? (size_t)(j * 8 + g) * p.ld_a + 16 * t : 0);
    }
    // the step that is fetched next
    int f_tile = first, f_c = c0;
    const unsigned char* wp[4];
    bool wv[4];
    auto rows_of = [&]() {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int in_tile = g + 8 * r, row = f_tile * rows + in_tile;
            wv[r] = f_tile < tiles && in_tile < rows && row < N;
            wp[r] = p.b + (wv[r] ? (size_t)row * p.ld_b + 16 * t : 0);
        }
    };
    auto fetch = [&](int slot) {
        if (f_tile < tiles && c0 < c1) {
            const int k = f_c * BS_STEP, kv = min(16, max(0, K - k - 16 * t));     // bytes of this lane's piece that exist
            const unsigned dst = my_ring + (unsigned)(slot * PIECES) * (THREADS * 16);
#pragma unroll
            for (int r = 0; r < 4; ++r) copy16<false>(dst + r * (THREADS * 16), kv && wv[r] ? wp[r] + k : p.b, wv[r] ? kv : 0);
#pragma unroll
            for (int j = 0; j < TT; ++j) copy16<true>(dst + (4 + j) * (THREADS * 16), kv && xv[j] ? xp[j] + k : p.a, xv[j] ? kv : 0);
            if (++f_c == c1) { f_c = c0; f_tile += stride; rows_of(); }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // scales of a block: of the lane's rows of a tile of b, and of its rows of a (columns of the products)
    struct { float w[4], x[TT][2]; } s, s_next;
    auto scales_of = [&](int tile, int block) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = min(tile * rows + g + 8 * r, N - 1);
            s_next.w[r] = B_ROWS ? p.sb[(size_t)block * N + row] : p.sb[(size_t)(row >> 7) * blocks + block];
        }
#pragma unroll
        for (int j = 0; j < TT; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) s_next.x[j][i] = p.sa[(size_t)block * M + min(j * 8 + 2 * t + i, M - 1)];
    };
    rows_of();
    // The first tile of b into L2 while the kernel before this one runs.  What that one still writes there it writes into L2 as
    // well, so nothing is read too early; the tile itself is read after the wait.  (Not where it is the only one: 4096 -> 4096 5.8 us with, 5.5
    // without; 4096 -> 32768 28.1 and 29.6.)
    if (tiles > stride && member == 0 && lane < rows && first * rows + lane < N) {
        const int bytes = min(K & ~15, BS_PREFETCH);
        if (bytes) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p.b + (size_t)(first * rows + lane) * p.ld_b), "r"(bytes) : "memory");
    }
    lf_grid_wait();
    lf_grid_release();
#pragma unroll
    for (int d = 0; d < BS_DEPTH - 1; ++d) fetch(d);
    if (c0 < c1) scales_of(first, c0 >> 1);
    int parity = 0, slot = 0;
    for (int tile = first; tile < tiles; tile += stride, parity ^= 1) {
        float sum[2][TT][4];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < TT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[m][j][i] = 0.f;
        for (int c = c0; c < c1; ++c) {
            if (c == c0 || (c & 1) == 0) {               // a new block: its scales are there, the next one's are sent for
                s = s_next;
                const int next = (c >> 1) + 1;
                if (2 * next < c1) scales_of(tile, next);
                else if (tile + stride < tiles) scales_of(tile + stride, c0 >> 1);
            }
            fetch(slot == 0 ? BS_DEPTH - 1 : slot - 1);
            asm volatile("cp.async.wait_group %0;" ::"n"(BS_DEPTH - 1) : "memory");
            const unsigned char* from = bs_raw + (size_t)(slot * PIECES) * (THREADS * 16) + threadIdx.x * 16;
            uint4 a[4], b[TT];
#pragma unroll
            for (int r = 0; r < 4; ++r) a[r] = *reinterpret_cast<const uint4*>(from + r * (THREADS * 16));
#pragma unroll
            for (int j = 0; j < TT; ++j) b[j] = *reinterpret_cast<const uint4*>(from + (4 + j) * (THREADS * 16));
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int j = 0; j < TT; ++j) {
                    float acc[4] = {0.f, 0.f, 0.f, 0.f};
                    mma16832(acc, a[2 * m].x, a[2 * m + 1].x, a[2 * m].y, a[2 * m + 1].y, b[j].x, b[j].y);
                    mma16832(acc, a[2 * m].z, a[2 * m + 1].z, a[2 * m].w, a[2 * m + 1].w, b[j].z, b[j].w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[m][j][i] = fmaf(s.w[2 * m + (i >> 1)] * s.x[j][i & 1], acc[i], sum[m][j][i]);
                }
            if (++slot == BS_DEPTH) slot = 0;
        }
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < TT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) red[parity][warp][j * 8 + 2 * t + (i & 1)][m * 16 + g + 8 * (i >> 1)] = sum[m][j][i];
        if (share > 1) lfptx::bar_sync(1 + group, share * 32);             // the tile's warps
        else __syncwarp();
        // a warp takes a row of a at a time, a lane a column; the sums are added in warp order
        const int col = tile * rows + lane;
        for (int tok = member; tok < TT * 8 && tok < M; tok += share) {
            if (lane >= rows || col >= N) continue;
            float v = 0.f;
            if (share == WARPS) {
#pragma unroll
                for (int i = 0; i < WARPS; ++i) v += red[parity][i][tok][lane];
            } else {
#pragma unroll 4
                for (int i = group * share; i < (group + 1) * share; ++i) v += red[parity][i][tok][lane];
            }
            if (p.bias) v += p.bias[col];
            if (p.add) v += as_float<OUT>(p.add, (size_t)tok * p.ld_add + col);
            static_cast<OUT*>(p.d)[(size_t)tok * p.ld_d + col] = (OUT)v;
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// nothing to contract: d = bias + add
template <typename OUT>
__global__ void __launch_bounds__(256) k_blocks_empty(const lf_product_blocks_args p)
{
    lf_grid_wait();
    lf_grid_release();
    const long long all = (long long)p.tokens * p.n_out;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
        const long long row = i / p.n_out;
        const int col = (int)(i - row * p.n_out);
        float v = p.bias ? p.bias[col] : 0.f;
        if (p.add) v += as_float<OUT>(p.add, (size_t)row * p.ld_add + col);
        static_cast<OUT*>(p.d)[(size_t)row * p.ld_d + col] = (OUT)v;
    }
}

// Shared memory for the ring and the warps' sums: 16 warps with one block of rows of a, 12 with two (197 KB each).
template <int TT, int WARPS>
constexpr size_t stream_smem() { return (size_t)BS_DEPTH * (4 + TT) * WARPS * 32 * 16 + sizeof(float) * 2 * WARPS * TT * 8 * (BS_ROWS + 1); }

template <typename OUT, int TT, int WARPS>
cudaError_t stream_go(const lf_product_blocks_args& a, int sm_count, cudaStream_t s)
{
    // Warps to a tile: as many as have four steps each, and more where there are too few tiles for the others.  (A tile's end costs
    // its warps a meeting: one row, 968 -> 42800 15.8 us with all 16 to a tile, 13.2 with four; but warps at work on one tile read its rows
    // in longer pieces: one row, 8192 -> 65536 91 us with all 16 to a tile, 109 with one.)
    const int steps = (a.n_in + BS_STEP - 1) / BS_STEP, tiles32 = (a.n_out + BS_ROWS - 1) / BS_ROWS;
    int share = 1;
    while (share < WARPS && (steps / share > 4 || (long long)tiles32 * share < (long long)sm_count * WARPS)) {
        ++share;
        while (WARPS % share) ++share;
    }
    const int groups = sm_count * (WARPS / share);
    const int waves = (a.n_out + BS_ROWS * groups - 1) / (BS_ROWS * groups);
    int rows = (a.n_out + groups * waves - 1) / (groups * waves);              // tiles come out even over the groups
    if (rows < 8) rows = 8;                                                    // a load covers eight rows
    const int tiles = (a.n_out + rows - 1) / rows, blocks = (tiles + WARPS / share - 1) / (WARPS / share);
    return lf_launch(a.b_tiles ? k_blocks_stream<OUT, TT, WARPS, false> : k_blocks_stream<OUT, TT, WARPS, true>,
                     dim3((unsigned)(blocks < sm_count ? blocks : sm_count)), WARPS * 32, stream_smem<TT, WARPS>(), s, a, rows, share);
}
template <typename OUT>
cudaError_t stream_of(const lf_product_blocks_args& a, int sm_count, cudaStream_t s)
{
    if (a.n_in == 0) return lf_launch(k_blocks_empty<OUT>, dim3((unsigned)(sm_count * 8)), 256, 0, s, a);
    return a.tokens <= 8 ? stream_go<OUT, 1, 16>(a, sm_count, s) : stream_go<OUT, 2, 12>(a, sm_count, s);
}
template <typename OUT, int TT, int WARPS>
bool stream_ready()
{
    constexpr int bytes = (int)stream_smem<TT, WARPS>();
    return cudaFuncSetAttribute(k_blocks_stream<OUT, TT, WARPS, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess &&
           cudaFuncSetAttribute(k_blocks_stream<OUT, TT, WARPS, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
}

}  // namespace

int lf_blocks_stream_init()
{
    return stream_ready<float, 1, 16>() && stream_ready<__nv_bfloat16, 1, 16>() && stream_ready<__half, 1, 16>() &&
                   stream_ready<float, 2, 12>() && stream_ready<__nv_bfloat16, 2, 12>() && stream_ready<__half, 2, 12>()
               ? LF_OK : LF_ECUDA;
}

cudaError_t lfk_blocks_stream(const lf_product_blocks_args& a, int sm_count, cudaStream_t s)
{
    if (a.out_dtype == LF_F32) return stream_of<float>(a, sm_count, s);
    if (a.out_dtype == LF_BF16) return stream_of<__nv_bfloat16>(a, sm_count, s);
    return stream_of<__half>(a, sm_count, s);
}

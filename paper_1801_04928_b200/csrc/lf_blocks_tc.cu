// Products of 8-bit operands with a scale for each block of 128 of the contraction, on the 5th-generation tensor cores:
//     D[m][n] = sum_c sa[c][m] sb(c, n) sum_{k in block c} A[m][k] B[n][k] + bias[n] + add[m][n]
// sb(c, n) is one number for 128 columns (tiles of weights) or one for each column (gradients of weights).
// A stage is one block: 128 e4m3 numbers are 128 bytes, a row of an operand block in the 128-byte swizzle, four
// instructions of 32 each.  The products of a block start a new accumulator; the warps that finish the tile take it from tensor
// memory, multiply it by the scales and add it to their own fp32 registers with round-to-nearest, while the tensor cores fill
// the other accumulator with the next block.  So scales are any fp32 numbers and nothing but 128 terms is ever added
// by the tensor core's truncating adder.
//
// Two kernels, chosen by an estimate of each one's time (lb_choose):
//   CTA pairs (k_blocks_pair): tcgen05.mma.cta_group::2, 256 x 256 tiles, persistent.  A CTA's 128 x 256 fp32
//     sums fill half of its registers, which is why tiles are not larger.
//   Split tiles (k_blocks_split): one CTA per 128 x 128 tile and part of the contraction (1, 2, 4 or 8 parts), whose
//     CTAs form a cluster and add their parts through distributed shared memory.
// What bounds them: a block of a 256 x 256 tile takes the tensor cores 512 cycles and its fetch 575 (32 KB a multiprocessor at 57 bytes a
// cycle); the way of an accumulator -- products, barrier, registers, barrier back to the issuer -- is about 1600 and two
// of them are under way, so 820 with one scale for 128 columns.  With column scales two packed operations a pair of sums instead of one
// keep the warps busy for 800 of about 1400.  8192 x 4096 -> 16384 in bf16: 489 us, 2.25 PFLOP/s (the same kernel without scales, one
// accumulator per tile, 393); 4096 x 8192 -> 16384 in fp32 with column scales 691 us, 1.59.  In a loop of seconds
// the power limit lowers the clock and they take 1.25 times as long.  Products of 128 columns at a time, so that an
// accumulator's halves are handed over earlier, were slower (671 us for 503): two multiprocessors multiply 128 columns no faster than 192.
// All waits are bounded; on expiry the status word is raised and the launch drains and ends.
#include "lf_ops_internal.h"
#include "lf_product_tc.cuh"
#include "lf_ptx.cuh"
#include "lf_rows.cuh"

namespace {

using namespace lfrow;

constexpr int LB_BK = 128;                               // a block of the contraction, bytes and numbers
constexpr int LB_STAGES = 6;
constexpr int LB_RING_BYTES = LB_STAGES * LT_STAGE_BYTES;
// Warps: eight finish, one loads, one issues, and where columns have scales of their own one brings them.  Then registers move
// to the two warpgroups that finish, 40 + 2 * 232 = 3 * 168, without them 20 to 30 are spilled in the loop (758 us instead of
// 857 for 4096 x 8192 -> 16384); with one scale for 128 columns 168 do, and 320 threads are faster than 384 (487 against 519 us for 8192 x 4096 -> 16384).
template <bool ROWS> struct lb_warps { static constexpr int threads = 320, finish = 0, load = 8, issue = 9; };
template <> struct lb_warps<true> { static constexpr int threads = 384, finish = 4, load = 0, issue = 1, scales = 2, regs_low = 40, regs_high = 232; };
constexpr int LB_SLOTS = 8;                              // column scales: blocks whose scales lie in shared memory
constexpr int LB_SLOT_BYTES = (128 + 256) * 4;           // of 128 rows and 256 columns
constexpr int LB_EPI_BYTES = 8 * 4096;                   // tiles: 32 rows x 128 bytes per warp that finishes
static_assert(LB_SLOTS * LB_SLOT_BYTES <= LB_EPI_BYTES, "either use of the space fits");
constexpr size_t LB_SMEM = (size_t)LB_RING_BYTES + LB_EPI_BYTES + 1024 + 512;
constexpr int LBS_THREADS = 512, LBS_STAGES = 4, LBS_LD = 132;
constexpr int LBS_TILE_BYTES = 128 * LBS_LD * 4;
constexpr int LBS_SCALE_BYTES = 8 * 2 * (32 + 64) * 4;   // scales of a warp's rows and columns, of two blocks
constexpr size_t LBS_SMEM = (size_t)LBS_STAGES * LT_STAGE_BYTES + LBS_TILE_BYTES + LBS_SCALE_BYTES + 1024 + 512;

struct LbParams {
    int M, N, K;
    int tiles_m, tiles_n, band;
    int stages_per_split;
    unsigned idesc;
    const float *sa, *sb;
    const float* bias;
    const void* add; long long ld_add;
    void* d; long long ld_d;
    int wide_add;                      // 256-bit accesses fit add
    unsigned* status;
    unsigned long long budget_ns;
    int withhold;
};

template <bool PAIR>
__device__ __forceinline__ void lb_mma(unsigned d_tmem, unsigned long long a, unsigned long long b, unsigned idesc, unsigned acc)
{
    if (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// Low word of a K-major operand block's descriptor (lt_desc); the high one is the same for all.  What is added to the
// address, in 16-byte units, cannot leave its 14 bits: shared memory ends below 256 KB.
__device__ __forceinline__ unsigned lb_desc_low(unsigned addr) { return (unsigned)lt_desc<false>(addr); }
// the four instructions of a stage: `a` its first block's descriptor
template <bool PAIR>
__device__ __forceinline__ void lb_products(unsigned d_tmem, unsigned a, unsigned idesc)
{
    const unsigned long long high = lt_desc<false>(0) & 0xFFFFFFFF00000000ull;
#pragma unroll
    for (unsigned kk = 0; kk < 4; ++kk)
        lb_mma<PAIR>(d_tmem, high | (a + 2 * kk), high | (a + (LT_BLOCK_BYTES >> 4) + 2 * kk), idesc, kk > 0 ? 1u : 0u);
}

template <typename OUT> struct half_of { typedef OUT type; };          // type of `add`
template <> struct half_of<float> { typedef __nv_bfloat16 type; };     // (none there)

// acc += s * the COLS columns of an accumulator in t, a row of them per lane
template <int COLS>
__device__ __forceinline__ void lb_scale_add(float* acc, const float* t, float s)
{
#pragma unroll
    for (int i = 0; i < COLS; i += 2) {
        const float2 r = fma2(f2(s), make_float2(t[i], t[i + 1]), make_float2(acc[i], acc[i + 1]));
        acc[i] = r.x; acc[i + 1] = r.y;
    }
}
// Where columns have scales of their own, an accumulator is taken in fragments: a lane has two neighbouring columns, 2 (lane % 4), of
// every eight, of the rows lane / 4 + 0, 8, 16, 24, so that a column's scale serves four rows (a row per lane needed a scale from
// shared memory for every product).  Of 16 columns: [rows 0, 8 | 16, 24][eight columns][row][column].
__device__ __forceinline__ void lb_ld_fragments(unsigned from, float* r)
{
#pragma unroll
    for (int h = 0; h < 2; ++h)
        asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(r[8 * h]), "=f"(r[8 * h + 1]), "=f"(r[8 * h + 2]), "=f"(r[8 * h + 3]), "=f"(r[8 * h + 4]), "=f"(r[8 * h + 5]),
                       "=f"(r[8 * h + 6]), "=f"(r[8 * h + 7]) : "r"(from + ((unsigned)(16 * h) << 16)) : "memory");
}
template <bool FRAGMENTS>
__device__ __forceinline__ void lb_ld(unsigned from, float (&r)[16])
{
    if (FRAGMENTS) lb_ld_fragments(from, r);
    else lfptx::tmem_ld16_async(from, r);
}
// acc += sr[row] * sc[column] * 16 columns in fragments
__device__ __forceinline__ void lb_scale_add(float* acc, const float* t, const float (&sr)[4], const float2* sc)
{
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const float2 s = sc[4 * g];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = 8 * (i >> 1) + 4 * g + 2 * (i & 1);
            const float2 r = fma2(mul2(f2(sr[i]), s), make_float2(t[at], t[at + 1]), make_float2(acc[at], acc[at + 1]));
            acc[at] = r.x; acc[at + 1] = r.y;
        }
    }
}

// ================================================================================================
// CTA pairs
// ================================================================================================
// 32 rows x 128 columns of a tile, a row per lane: bias, residual, and whole lines out through the warp's 32 x 128
// bytes of shared memory.
template <typename OUT>
__device__ __forceinline__ void lb_finish(float (&acc)[128], const LbParams& P, int row0, int col0, unsigned char* blk)
{
    typedef typename half_of<OUT>::type H;
    const int lane = threadIdx.x & 31, row = row0 + lane;
    float4 bias = make_float4(0.f, 0.f, 0.f, 0.f);
    if (P.bias && col0 + 4 * lane < P.N) bias = *reinterpret_cast<const float4*>(P.bias + col0 + 4 * lane);
#pragma unroll
    for (int j = 0; j < 4; ++j) {                                // 32 columns at a time
        const int col = col0 + 32 * j;
        if (j % 2 == 0 && col >= P.N) break;
        float* v = acc + 32 * j;
        if (P.bias) {
#pragma unroll
            for (int g = 0; g < 8; ++g) {                        // lane 8 j + g holds the bias of these four columns
                v[4 * g] += __shfl_sync(0xFFFFFFFFu, bias.x, 8 * j + g);
                v[4 * g + 1] += __shfl_sync(0xFFFFFFFFu, bias.y, 8 * j + g);
                v[4 * g + 2] += __shfl_sync(0xFFFFFFFFu, bias.z, 8 * j + g);
                v[4 * g + 3] += __shfl_sync(0xFFFFFFFFu, bias.w, 8 * j + g);
            }
        }
        if (sizeof(OUT) == 2 && P.add && row < P.M) {
            const H* from = static_cast<const H*>(P.add) + (size_t)row * P.ld_add + col;
            unsigned r[16];
            if (P.wide_add && col + 32 <= P.N) {
                ld256(from, *reinterpret_cast<unsigned(*)[8]>(r));
                ld256(from + 16, *reinterpret_cast<unsigned(*)[8]>(r + 8));
            } else {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    uint4 u = make_uint4(0, 0, 0, 0);
                    if (col + 8 * g < P.N) u = *reinterpret_cast<const uint4*>(from + 8 * g);
                    r[4 * g] = u.x; r[4 * g + 1] = u.y; r[4 * g + 2] = u.z; r[4 * g + 3] = u.w;
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 f = unpack2(r[i], H());
                v[2 * i] += f.x; v[2 * i + 1] += f.y;
            }
        }
        constexpr int PER = sizeof(OUT) == 2 ? 2 : 1;            // blocks of 32 columns per stored line
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float(&w)[8] = *reinterpret_cast<const float(*)[8]>(v + 8 * g);
            // 16-byte units of a 128-byte line, turned by the row so that neither side meets a bank twice
            if (sizeof(OUT) == 2) {
                vec8<H> o;
                o.set(w);
                *reinterpret_cast<uint4*>(blk + lane * 128 + ((((j & 1) * 4 + g) ^ (lane & 7)) << 4)) = o.u;
            } else {
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    *reinterpret_cast<float4*>(blk + lane * 128 + (((g * 2 + u) ^ (lane & 7)) << 4)) = make_float4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
            }
        }
        if (j % PER == PER - 1) {                               // a line of every row is complete: whole lines go out
            __syncwarp();
            constexpr int UC = 16 / (int)sizeof(OUT);           // columns of a 16-byte unit
            const int cu = col - (PER - 1) * 32 + (lane & 7) * UC, r0 = row0 + (lane >> 3);
            const unsigned char* from = blk + (lane >> 3) * 128;
            OUT* to = static_cast<OUT*>(P.d) + (size_t)r0 * P.ld_d + cu;
            const size_t step = (size_t)4 * P.ld_d;
            uint4 u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)                         // row (lane >> 3) + 4 i: its turn alternates
                u[i] = *reinterpret_cast<const uint4*>(from + i * 512 + (((lane & 7) ^ (((lane >> 3) + 4 * i) & 7)) << 4));
            if (cu < P.N) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (r0 + 4 * i < P.M) *reinterpret_cast<uint4*>(to + i * step) = u[i];
            }
            __syncwarp();
        }
    }
}

// The same from fragments: a lane stores two columns at a time, four lanes 32 bytes of a row in fp32.  WHOLE: every row and column exists.
template <typename OUT, bool WHOLE>
__device__ __forceinline__ void lb_finish_fragments(const float (&acc)[128], const LbParams& P, int row0, int col0)
{
    typedef typename half_of<OUT>::type H;
    const int lane = threadIdx.x & 31, c0 = col0 + 2 * (lane & 3), r0 = row0 + (lane >> 2);
    OUT* to[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = static_cast<OUT*>(P.d) + (size_t)(r0 + 8 * i) * P.ld_d + c0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {                               // eight columns at a time
        if (!WHOLE && c0 + 8 * j >= P.N) break;
        float2 bias = f2(0.f);
        if (P.bias) bias = *reinterpret_cast<const float2*>(P.bias + c0 + 8 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = 16 * (j >> 1) + 8 * (i >> 1) + 4 * (j & 1) + 2 * (i & 1);
            if (!WHOLE && r0 + 8 * i >= P.M) continue;
            float2 v = add2(make_float2(acc[at], acc[at + 1]), bias);
            if (sizeof(OUT) == 2) {
                if (P.add) v = add2(v, unpack2(*reinterpret_cast<const unsigned*>(static_cast<const H*>(P.add) + (size_t)(r0 + 8 * i) * P.ld_add + c0 + 8 * j), H()));
                *reinterpret_cast<unsigned*>(to[i] + 8 * j) = pack2(v.x, v.y, H());
            } else {
                *reinterpret_cast<float2*>(to[i] + 8 * j) = v;
            }
        }
    }
}

template <typename OUT, bool ROWS>
__global__ void __launch_bounds__(lb_warps<ROWS>::threads, 1)
k_blocks_pair(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const LbParams P)
{
    typedef lb_warps<ROWS> W;
    extern __shared__ unsigned char lb_smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(lb_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    unsigned char* epi = ring + LB_RING_BYTES;
    float* slots = reinterpret_cast<float*>(epi);
    LtShared* sh = reinterpret_cast<LtShared*>(epi + LB_EPI_BYTES);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned rank = lfptx::cluster_ctarank();
    const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const int n_tiles = P.tiles_m * P.tiles_n;
    const int n_k = (P.K + LB_BK - 1) / LB_BK;

    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
        for (int i = 0; i < LB_STAGES; ++i) {
            lfptx::mbar_init(lfptx::smem_u32(&sh->full[i]), 1);
            lfptx::mbar_init(lfptx::smem_u32(&sh->empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) lfptx::mbar_init(lfptx::smem_u32(&sh->acc_empty[i]), 16);   // eight finishing warps of each CTA
        for (int i = 0; i < LB_SLOTS; ++i) {
            lfptx::mbar_init(lfptx::smem_u32(&sh->scaled[i]), 1);
            lfptx::mbar_init(lfptx::smem_u32(&sh->scale_free[i]), 8);
        }
        sh->abort_flag = 0u;
        sh->prog_it = 0u;
        lfptx::mbar_fence_init();
    }
    if (warp == W::issue) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(lfptx::smem_u32(&sh->tmem_base)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    lfptx::tc_fence_before();
    __syncthreads();
    lfptx::cluster_sync_all();       // the peer's barriers exist before anything can arrive on them
    lfptx::tc_fence_after();
    const unsigned tmem_base = sh->tmem_base;
    lf_grid_wait();                  // (by every thread: the bounded waits below do not count the time until then)
    lf_grid_release();

    if (warp < W::finish || warp >= W::finish + 8) {
      if constexpr (ROWS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(W::regs_low));
      if (warp == W::load) {
        // ------------------------------ TMA producer: this CTA's halves -------------------------
        if (lane == 0) {
            unsigned it = 0;
            bool ok = true;
            for (int t = pair; t < n_tiles && ok; t += n_pairs) {
                int tm, tn;
                lp_tile(t, P, tm, tn);
                const int m0 = (tm * 2 + (int)rank) * 128, n0 = (tn * 2 + (int)rank) * 128;
                for (int ks = 0; ks < n_k; ++ks, ++it) {
                    const unsigned st = it % LB_STAGES, use = it / LB_STAGES;
                    if (use > 0 && !lt_wait<false>(lfptx::smem_u32(&sh->empty[st]), (use - 1) & 1u, P, sh)) { ok = false; break; }
                    const unsigned lbar = lfptx::smem_u32(&sh->full[st]);
                    if (P.withhold && pair == 0 && rank == 1 && it == 0) continue;    // test hook
                    if (rank == 0) lfptx::mbar_arrive_expect_tx(lbar, 2u * LT_STAGE_BYTES);
                    const unsigned bar = lfptx::map_to_cta(lbar, 0);
                    const unsigned dst = lfptx::smem_u32(ring + (size_t)st * LT_STAGE_BYTES);
                    lt_load<false, true>(dst, &map_a, bar, m0, ks * LB_BK);
                    lt_load<false, true>(dst + LT_BLOCK_BYTES, &map_b, bar, n0, ks * LB_BK);
                }
            }
            sh->prog_it = it;
        }
      } else if (warp == W::issue) {
        // ------------------------------ MMA issuer (leader CTA) ---------------------------------
        // One thread, and a stage's products take it little longer than the tensor cores: descriptors are a word counted
        // up, and the next stage's barrier is looked at while this one's products are being issued.
        if (lane == 0 && rank == 0) {
            unsigned it = 0, st = 0, round = 0;      // stages, and accumulators, one for each
            bool ok = true, there = false;
            const unsigned first = lb_desc_low(lfptx::smem_u32(ring)), full0 = lfptx::smem_u32(&sh->full[0]), empty0 = lfptx::smem_u32(&sh->empty[0]);
            for (int t = pair; t < n_tiles && ok; t += n_pairs) {
                for (int ks = 0; ks < n_k; ++ks, ++it) {
                    const unsigned ab = it & 1u, use = it >> 1;
                    if (!there && !lt_wait<false>(full0 + 8u * st, round & 1u, P, sh)) { ok = false; break; }
                    if (use > 0 && !lt_wait<false>(lfptx::smem_u32(&sh->acc_empty[ab]), (use - 1) & 1u, P, sh)) { ok = false; break; }
                    lfptx::tc_fence_after();
                    lb_products<true>(tmem_base + ab * 256u, first + st * (LT_STAGE_BYTES >> 4), P.idesc);
                    // the block's products are done: its stage may be loaded again, its accumulator be read
                    lt_commit<true>(empty0 + 8u * st);
                    if (++st == LB_STAGES) { st = 0; ++round; }
                    there = lfptx::mbar_test_wait(full0 + 8u * st, round & 1u);
                }
            }
        }
      }
      if constexpr (ROWS) if (warp == W::scales) {
        // ------------------------------ scales of this CTA's rows and of all columns, into slots ------
        unsigned it = 0;
        bool ok = true;
        for (int t = pair; t < n_tiles && ok; t += n_pairs) {
            int tm, tn;
            lp_tile(t, P, tm, tn);
            const int m0 = (tm * 2 + (int)rank) * 128, n0 = tn * 256;
            float4 next_a, next_b0, next_b1;            // a block ahead
            auto send_for = [&](int ks) {
                const float *sa = P.sa + (size_t)ks * P.M, *sb = P.sb + (size_t)ks * P.N;
                next_a = make_float4(sa[min(m0 + lane, P.M - 1)], sa[min(m0 + 32 + lane, P.M - 1)], sa[min(m0 + 64 + lane, P.M - 1)], sa[min(m0 + 96 + lane, P.M - 1)]);
                next_b0 = *reinterpret_cast<const float4*>(sb + min(n0 + 4 * lane, P.N - 4));
                next_b1 = *reinterpret_cast<const float4*>(sb + min(n0 + 128 + 4 * lane, P.N - 4));
            };
            send_for(0);
            for (int ks = 0; ks < n_k; ++ks, ++it) {
                const unsigned sl = it % LB_SLOTS, use = it / LB_SLOTS;
                if (use > 0 && !lt_wait<false>(lfptx::smem_u32(&sh->scale_free[sl]), (use - 1) & 1u, P, sh)) { ok = false; break; }
                float* slot = slots + sl * (LB_SLOT_BYTES / 4);
                slot[lane] = next_a.x; slot[32 + lane] = next_a.y; slot[64 + lane] = next_a.z; slot[96 + lane] = next_a.w;
                reinterpret_cast<float4*>(slot + 128)[lane] = next_b0;
                reinterpret_cast<float4*>(slot + 256)[lane] = next_b1;
                __syncwarp();
                if (lane == 0) lfptx::mbar_arrive(lfptx::smem_u32(&sh->scaled[sl]));
                if (ks + 1 < n_k) send_for(ks + 1);
            }
        }
      }
    } else {
        if constexpr (ROWS) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(W::regs_high));
        // ------------------------------ scales and epilogue (eight warps of both CTAs) -----------
        // A warp has one 32-lane quadrant (32 rows) and one half (128 columns, one tile of weights) of the accumulators.
        const int quad = warp & 3, half = (warp - W::finish) >> 2;
        const unsigned leader_acc_empty = lfptx::map_to_cta(lfptx::smem_u32(&sh->acc_empty[0]), 0);
        const unsigned lane_addr = tmem_base + ((unsigned)(quad * 32) << 16) + half * 128u;
        unsigned char* blk = epi + (warp - W::finish) * 4096;
        unsigned c = 0, st = 0, round = 0;
        bool ok = true;
        for (int t = pair; t < n_tiles && ok; t += n_pairs) {
            int tm, tn;
            lp_tile(t, P, tm, tn);
            const int row0 = (tm * 2 + (int)rank) * 128 + quad * 32, col0 = tn * 256 + half * 128;
            // one scale for the columns: scales of a block are sent for while the one before it is being added
            const float *sa = P.sa, *sb = P.sb;
            float sa_next = 0.f, sb_next = 0.f;
            if (!ROWS) {
                sa += min(row0 + lane, P.M - 1);
                sb += (size_t)min(col0 >> 7, (P.N - 1) >> 7) * n_k;
                sa_next = *sa;
                sb_next = *sb;
            }
            float acc[128];
#pragma unroll
            for (int i = 0; i < 128; ++i) acc[i] = 0.f;
#pragma unroll 1
            for (int ks = 0; ks < n_k; ++ks, ++c) {
                const unsigned ab = c & 1u, from = lane_addr + ab * 256u;
                float s = 0.f;
                if (!ROWS) {
                    s = sa_next * sb_next;
                    if (ks + 1 < n_k) {
                        sa += P.M;
                        ++sb;
                        sa_next = *sa;
                        sb_next = *sb;
                    }
                } else if (!lt_wait<false>(lfptx::smem_u32(&sh->scaled[c % LB_SLOTS]), (c / LB_SLOTS) & 1u, P, sh)) { ok = false; break; }
                if (!lt_wait<false>(lfptx::smem_u32(&sh->empty[st]), round & 1u, P, sh)) { ok = false; break; }
                if (++st == LB_STAGES) { st = 0; ++round; }
                lfptx::tc_fence_after();
                const float* slot = slots + (c % LB_SLOTS) * (LB_SLOT_BYTES / 4);
                float sr[4] = {0.f, 0.f, 0.f, 0.f};
                if (ROWS) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) sr[i] = slot[quad * 32 + 8 * i + (lane >> 2)];
                }
                const float2* sc = reinterpret_cast<const float2*>(slot + 128 + 128 * half) + (lane & 3);
                // 16 columns at a time, the next ones on their way
                float r[2][16];
                lb_ld<ROWS>(from, r[0]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    lfptx::tmem_wait_ld16(r[j & 1]);
                    if (j < 7) {
                        lb_ld<ROWS>(from + 16 * (j + 1), r[(j + 1) & 1]);
                    } else {
                        lfptx::tc_fence_before();
                        __syncwarp();
                        if (lane == 0) lt_arrive_cluster_relaxed(leader_acc_empty + ab * 8u);
                    }
                    if (ROWS) lb_scale_add(acc + 16 * j, r[j & 1], sr, sc + 8 * j);
                    else lb_scale_add<16>(acc + 16 * j, r[j & 1], s);
                }
                if (ROWS) {
                    __syncwarp();
                    if (lane == 0) lfptx::mbar_arrive(lfptx::smem_u32(&sh->scale_free[c % LB_SLOTS]));
                }
            }
            if (!ok) break;
            if constexpr (ROWS) {
                if (row0 + 32 <= P.M && col0 + 128 <= P.N) lb_finish_fragments<OUT, true>(acc, P, row0, col0);
                else lb_finish_fragments<OUT, false>(acc, P, row0, col0);
            } else {
                lb_finish<OUT>(acc, P, row0, col0, blk);
            }
        }
    }

    // Neither CTA may leave (or free tensor memory) while the other can still reach it.
    lfptx::tc_fence_before();
    __syncthreads();
    lfptx::cluster_sync_all();
    if (threadIdx.x == 0 && rank == 0) {
        // A launch that was given up: wait, with a limit, for the operand loads of both CTAs that are still on
        // their way.  All of them are credited to the leader's barriers; a phase that only one CTA
        // loaded for is first given what it would otherwise wait for.
        const bool gave_up = sh->abort_flag != 0u || lt_ld_cluster_u32(lfptx::map_to_cta(lfptx::smem_u32((const void*)&sh->abort_flag), 1)) != 0u;
        if (gave_up) {
            const unsigned it_l = sh->prog_it, it_p = lt_ld_cluster_u32(lfptx::map_to_cta(lfptx::smem_u32(&sh->prog_it), 1));
            const unsigned hi = max(it_l, it_p), lo = min(it_l, it_p);
            for (unsigned j = lo; j < hi; ++j) {
                const unsigned bar = lfptx::smem_u32(&sh->full[j % LB_STAGES]);
                if (j >= it_l) lfptx::mbar_arrive_expect_tx(bar, LT_STAGE_BYTES);                // only the peer loaded
                else lt_complete_tx(bar, LT_STAGE_BYTES);                                        // only the leader loaded
            }
            const unsigned long long t0 = lfptx::globaltimer_ns();
            for (unsigned j = hi > LB_STAGES ? hi - LB_STAGES : 0; j < hi; ++j) {
                const unsigned bar = lfptx::smem_u32(&sh->full[j % LB_STAGES]);
                while (!lfptx::mbar_try_wait(bar, (j / LB_STAGES) & 1u) && lfptx::globaltimer_ns() - t0 < 50000000ull) { }
            }
        }
    }
    lfptx::cluster_sync_all();
    if (warp == W::issue) {
        lfptx::tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

// ================================================================================================
// Split tiles
// ================================================================================================
// Every part leaves its fp32 tile in shared memory; after a cluster barrier each CTA adds its share of the rows that exist
// from all parts, in their order.  A row is a warp's: a lane has four columns.
template <typename OUT, bool ROWS, int SPLITS>
__global__ void __launch_bounds__(LBS_THREADS, 1)
k_blocks_split(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const LbParams P)
{
    typedef typename half_of<OUT>::type H;
    extern __shared__ unsigned char lb_smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(lb_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    float* tile = reinterpret_cast<float*>(ring + (size_t)LBS_STAGES * LT_STAGE_BYTES);     // [128][LBS_LD]
    unsigned char* scales = reinterpret_cast<unsigned char*>(tile) + LBS_TILE_BYTES;
    LtShared* sh = reinterpret_cast<LtShared*>(scales + LBS_SCALE_BYTES);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = (int)(blockIdx.x % (unsigned)SPLITS), t = (int)(blockIdx.x / (unsigned)SPLITS);
    const int tn = t / P.tiles_m, tm = t - tn * P.tiles_m;
    const int n_k_all = (P.K + LB_BK - 1) / LB_BK;
    const int ks0 = part * P.stages_per_split;
    const int n_k = max(0, min(P.stages_per_split, n_k_all - ks0));

    auto load_stage = [&](int ks) {                    // one thread; stage ks of this part into its slot
        const unsigned st = (unsigned)ks % LBS_STAGES, bar = lfptx::smem_u32(&sh->full[st]);
        lfptx::mbar_arrive_expect_tx(bar, LT_STAGE_BYTES);
        if (P.withhold && blockIdx.x == 0 && ks == 0) return;                       // test hook
        const unsigned dst = lfptx::smem_u32(ring + (size_t)st * LT_STAGE_BYTES);
        lt_load<false, false>(dst, &map_a, bar, tm * 128, (ks0 + ks) * LB_BK);
        lt_load<false, false>(dst + LT_BLOCK_BYTES, &map_b, bar, tn * 128, (ks0 + ks) * LB_BK);
    };
    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
        for (int i = 0; i < LBS_STAGES; ++i) {
            lfptx::mbar_init(lfptx::smem_u32(&sh->full[i]), 1);
            lfptx::mbar_init(lfptx::smem_u32(&sh->empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            lfptx::mbar_init(lfptx::smem_u32(&sh->acc_full[i]), 1);
            lfptx::mbar_init(lfptx::smem_u32(&sh->acc_empty[i]), 8);
        }
        sh->abort_flag = 0u;
        lfptx::mbar_fence_init();
        lf_grid_wait();
        for (int ks = 0; ks < min(n_k, LBS_STAGES); ++ks) load_stage(ks);            // under the rest of the set-up
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(lfptx::smem_u32(&sh->tmem_base)), "r"(256u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    lfptx::tc_fence_before();
    __syncthreads();
    lfptx::tc_fence_after();
    const unsigned tmem_base = sh->tmem_base;
    lf_grid_wait();
    lf_grid_release();

    if (warp == 0) {
        if (lane == 0) {
            int ks = LBS_STAGES;
            for (; ks < n_k; ++ks) {
                if (!lt_wait<false>(lfptx::smem_u32(&sh->empty[ks % LBS_STAGES]), (unsigned)(ks / LBS_STAGES - 1) & 1u, P, sh)) break;
                load_stage(ks);
            }
            // after giving up: do not let the CTA go on under loads that are still landing
            if (sh->abort_flag) {
                const unsigned long long t0 = lfptx::globaltimer_ns();
                const int n = min(ks, n_k);
                for (int j = max(0, n - LBS_STAGES); j < n; ++j)
                    while (!lfptx::mbar_try_wait(lfptx::smem_u32(&sh->full[j % LBS_STAGES]), (unsigned)(j / LBS_STAGES) & 1u) &&
                           lfptx::globaltimer_ns() - t0 < 50000000ull) { }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            for (int ks = 0; ks < n_k; ++ks) {
                const unsigned ab = (unsigned)ks & 1u, use = (unsigned)ks >> 1, st = (unsigned)ks % LBS_STAGES;
                if (use > 0 && !lt_wait<false>(lfptx::smem_u32(&sh->acc_empty[ab]), (use - 1) & 1u, P, sh)) break;
                if (!lt_wait<false>(lfptx::smem_u32(&sh->full[st]), (unsigned)(ks / LBS_STAGES) & 1u, P, sh)) break;
                lfptx::tc_fence_after();
                const unsigned a_addr = lfptx::smem_u32(ring + (size_t)st * LT_STAGE_BYTES);
                lb_products<false>(tmem_base + ab * 128u, lb_desc_low(a_addr), P.idesc);
                lt_commit<false>(lfptx::smem_u32(&sh->empty[st]));
                lt_commit<false>(lfptx::smem_u32(&sh->acc_full[ab]));
            }
        }
    } else if (warp < 10) {
        const int quad = warp & 3, half = (warp - 2) >> 2, row = tm * 128 + quad * 32 + lane, col0 = tn * 128 + half * 64;
        const float* sa = P.sa + (size_t)ks0 * P.M + min(row, P.M - 1);
        const float* sb = ROWS ? P.sb + (size_t)ks0 * P.N + min(col0 + 2 * lane, P.N - 2) : P.sb + (size_t)tn * n_k_all + ks0;
        const size_t sb_step = ROWS ? (size_t)P.N : 1;
        float acc[64];
#pragma unroll
        for (int i = 0; i < 64; ++i) acc[i] = 0.f;
        float sa_next = 0.f;
        float2 sb_next = f2(0.f);
        auto scales_of = [&]() {
            sa_next = *sa;
            if (ROWS) sb_next = *reinterpret_cast<const float2*>(sb);
            else sb_next.x = *sb;
        };
        if (n_k > 0) scales_of();
#pragma unroll 1
        for (int ks = 0; ks < n_k; ++ks) {
            const unsigned ab = (unsigned)ks & 1u;
            float* mine = reinterpret_cast<float*>(scales) + ((warp - 2) * 2 + (int)ab) * 96;
            const float both = sa_next * sb_next.x;
            if (ROWS) {
                mine[lane] = sa_next;
                reinterpret_cast<float2*>(mine + 32)[lane] = sb_next;
            }
            if (ks + 1 < n_k) {
                sa += P.M;
                sb += sb_step;
                scales_of();
            }
            if (ROWS) __syncwarp();
            if (!lt_wait<false>(lfptx::smem_u32(&sh->acc_full[ab]), ((unsigned)ks >> 1) & 1u, P, sh)) break;
            lfptx::tc_fence_after();
            float sr[4] = {0.f, 0.f, 0.f, 0.f};
            if (ROWS) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sr[i] = mine[8 * i + (lane >> 2)];
            }
            const float2* sc = reinterpret_cast<const float2*>(mine + 32) + (lane & 3);
            const unsigned from = tmem_base + ((unsigned)(quad * 32) << 16) + ab * 128u + half * 64u;
            // 32 columns at a time, or of fragments 16, the next ones on their way
            auto taken = [&]() {
                lfptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) lfptx::mbar_arrive(lfptx::smem_u32(&sh->acc_empty[ab]));
            };
            if constexpr (ROWS) {
                float r[2][16];
                lb_ld<true>(from, r[0]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    lfptx::tmem_wait_ld16(r[j & 1]);
                    if (j < 3) lb_ld<true>(from + 16 * (j + 1), r[(j + 1) & 1]);
                    else taken();
                    lb_scale_add(acc + 16 * j, r[j & 1], sr, sc + 8 * j);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float r[32];
                    lfptx::tmem_ld32_async(from + 32 * j, r);
                    lfptx::tmem_wait_ld32(r);
                    if (j == 1) taken();
                    lb_scale_add<32>(acc + 32 * j, r, both);
                }
            }
        }
        if (ROWS) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = 16 * (j >> 1) + 8 * (i >> 1) + 4 * (j & 1) + 2 * (i & 1);
                    *reinterpret_cast<float2*>(tile + (quad * 32 + 8 * i + (lane >> 2)) * LBS_LD + half * 64 + 8 * j + 2 * (lane & 3)) = make_float2(acc[at], acc[at + 1]);
                }
        } else {
            float* to = tile + (quad * 32 + lane) * LBS_LD + half * 64;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                *reinterpret_cast<float4*>(to + 4 * i) = make_float4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]);
        }
    }
    __syncwarp();
    lfptx::tc_fence_before();
    __syncthreads();
    if (SPLITS > 1) lfptx::cluster_sync_all();
    // this CTA's rows: its part of those that exist
    constexpr int R = 128 / SPLITS, SIDE = SPLITS == 8 ? 1 : 2;       // rows that a warp has in flight
    const int share = min(R, (P.M - tm * 128 + SPLITS - 1) / SPLITS);
    const int col = tn * 128 + 4 * lane;
    const bool live = sh->abort_flag == 0u && col < P.N;
    float4 bias = make_float4(0.f, 0.f, 0.f, 0.f);
    if (P.bias && live) bias = *reinterpret_cast<const float4*>(P.bias + col);
    for (int r0 = warp * SIDE; r0 < share; r0 += 16 * SIDE) {
        float4 x[SIDE][SPLITS];
        uint2 res[SIDE];
#pragma unroll
        for (int i = 0; i < SIDE; ++i) {
            const int r = part * share + r0 + i, row = tm * 128 + r;
            res[i] = make_uint2(0, 0);
            if (r0 + i >= share) continue;
#pragma unroll
            for (int p = 0; p < SPLITS; ++p) {
                const float* at = tile + r * LBS_LD + 4 * lane;
                if (SPLITS == 1) x[i][p] = *reinterpret_cast<const float4*>(at);
                else x[i][p] = lt_ld_cluster_f4(lfptx::map_to_cta(lfptx::smem_u32(at), (unsigned)p));
            }
            if (sizeof(OUT) == 2 && P.add && live && row < P.M) res[i] = *reinterpret_cast<const uint2*>(static_cast<const H*>(P.add) + (size_t)row * P.ld_add + col);
        }
#pragma unroll
        for (int i = 0; i < SIDE; ++i) {
            const int row = tm * 128 + part * share + r0 + i;
            if (r0 + i >= share || !live || row >= P.M) continue;
            float4 v = x[i][0];
#pragma unroll
            for (int p = 1; p < SPLITS; ++p) { v.x += x[i][p].x; v.y += x[i][p].y; v.z += x[i][p].z; v.w += x[i][p].w; }
            v.x += bias.x; v.y += bias.y; v.z += bias.z; v.w += bias.w;
            OUT* to = static_cast<OUT*>(P.d) + (size_t)row * P.ld_d + col;
            if (sizeof(OUT) == 2) {
                if (P.add) {
                    const float2 f0 = unpack2(res[i].x, H()), f1 = unpack2(res[i].y, H());
                    v.x += f0.x; v.y += f0.y; v.z += f1.x; v.w += f1.y;
                }
                *reinterpret_cast<uint2*>(to) = make_uint2(pack2(v.x, v.y, H()), pack2(v.z, v.w, H()));
            } else {
                *reinterpret_cast<float4*>(to) = v;
            }
        }
    }
    // no CTA may leave while another one reads its tile
    __syncwarp();
    if (SPLITS > 1) lfptx::cluster_sync_all();
    else __syncthreads();
    if (warp == 1) {
        lfptx::tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(256u) : "memory");
    }
}

int lb_threads(bool rows) { return rows ? lb_warps<true>::threads : lb_warps<false>::threads; }

typedef void (*lb_kernel)(const CUtensorMap, const CUtensorMap, const LbParams);

// kernel of a result type and kind of column scales; splits = 0: CTA pairs
template <typename OUT, bool ROWS>
lb_kernel lb_of(int splits)
{
    switch (splits) {
        case 0: return k_blocks_pair<OUT, ROWS>;
        case 1: return k_blocks_split<OUT, ROWS, 1>;
        case 2: return k_blocks_split<OUT, ROWS, 2>;
        case 4: return k_blocks_split<OUT, ROWS, 4>;
        default: return k_blocks_split<OUT, ROWS, 8>;
    }
}
lb_kernel lb_pick(int out_dtype, bool rows, int splits)
{
    if (out_dtype == LF_F32) return rows ? lb_of<float, true>(splits) : lb_of<float, false>(splits);
    if (out_dtype == LF_BF16) return rows ? lb_of<__nv_bfloat16, true>(splits) : lb_of<__nv_bfloat16, false>(splits);
    return rows ? lb_of<__half, true>(splits) : lb_of<__half, false>(splits);
}

// Parts of a split tile, or 0 for CTA pairs: the least estimated time in SM cycles.  A stage costs a 128 x 128 tile 600 (fetch), a pair
// 750; where the parts meet, 1500 and their bytes at 14 a cycle; the rest is launch, first loads and the end.  Measured, us,
// taken against the next best: 509 x 4096 -> 1024 4 parts 9.2, 2 parts 11.4; 512 x 4096 -> 4096 1 part 16.4, pairs 19.9; 1000 x 8192 -> 1000
// 2 parts 25.4, 4 parts 32.2; 2048 x 1024 -> 2304 pairs 15.6, 1 part 15.7; 2048 x 4096 -> 4096 pairs 37, 1 part 63.  Over 16 shapes it
// takes the best form or one within 4 %.
int lb_choose(const lf_ops* o, const lf_product_blocks_args& a, int n_k)
{
    auto waves = [](long long units, int at_once) { return (double)((units + at_once - 1) / at_once); };
    const long long m128 = (a.tokens + 127) / 128, n128 = (a.n_out + 127) / 128, tiles = ((a.tokens + 255) / 256) * (long long)((a.n_out + 255) / 256);
    const double rows = a.tokens < 128 ? a.tokens / 128.0 : 1.0;
    int best = 1;
    double least = 1e30;
    for (int i = 0, splits = 1; splits <= 8 && splits <= n_k; ++i, splits *= 2) {
        if (o->max_block_splits[i] == 0) continue;
        const double part = (double)((n_k + splits - 1) / splits);
        const double meet = splits > 1 ? 1500.0 + 65536.0 * rows * (splits - 1) / splits / 14.0 : 0.0;
        const double cycles = waves(m128 * n128 * splits, o->max_block_splits[i]) * (part * 600.0 + meet + 9000.0);
        if (cycles < least) { least = cycles; best = splits; }
    }
    if (o->max_block_pairs > 0 && waves(tiles, o->max_block_pairs) * (n_k * 750.0 + 4000.0) + 10000.0 < least) best = 0;
    return best;
}

}  // namespace

int lf_blocks_tc_init(lf_ops* o)
{
    o->max_block_pairs = -1;
    for (int& n : o->max_block_splits) n = -1;
    for (int type = 0; type < 3; ++type)
        for (int rows = 0; rows < 2; ++rows) {
            const int out = type == 0 ? LF_F32 : type == 1 ? LF_BF16 : LF_F16;
            // opts a kernel in; least: clusters of it that are resident at once, or fewer of another one
            auto resident = [&](lb_kernel f, int threads, int cluster, size_t smem, int* least) {
                cudaLaunchConfig_t cfg;
                cudaLaunchAttribute at[2];
                lt_cluster_config(&cfg, at, 32, threads, cluster, smem, nullptr);
                int n = 0;
                if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
                    cudaOccupancyMaxActiveClusters(&n, f, &cfg) != cudaSuccess) return false;
                if (*least < 0 || n < *least) *least = n;
                return true;
            };
            for (int i = 0; i < 4; ++i)
                if (!resident(lb_pick(out, rows, 1 << i), LBS_THREADS, 1 << i, LBS_SMEM, &o->max_block_splits[i])) return LF_ECUDA;
            if (!resident(lb_pick(out, rows, 0), lb_threads(rows != 0), 2, LB_SMEM, &o->max_block_pairs)) return LF_ECUDA;
        }
    for (int i = 0; i < 4; ++i) o->max_block_splits[i] <<= i;              // blocks
    return LF_OK;
}

int lf_blocks_tc(lf_ops* o, const lf_product_blocks_args& a)
{
    const int n_k = (a.n_in + LB_BK - 1) / LB_BK;
    LbParams P = {};
    P.M = a.tokens; P.N = a.n_out; P.K = a.n_in;
    P.sa = a.sa; P.sb = a.sb;
    P.bias = a.bias; P.add = a.add; P.ld_add = a.ld_add;
    P.d = a.d; P.ld_d = a.ld_d;
    P.wide_add = (a.ld_add & 15) == 0 && (reinterpret_cast<uintptr_t>(a.add) & 31) == 0;
    P.status = o->status_dev;
    P.budget_ns = (unsigned long long)o->wait_budget_us * 1000ull;
    P.withhold = o->withhold;
    const unsigned idesc = 1u << 4;                                 // fp32 accumulator; A and B: e4m3 (0), both K-major
    alignas(64) CUtensorMap map_a, map_b;
    if (!lt_map(&map_a, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.a, a.tokens, a.n_in, a.ld_a, LB_BK, 128) ||
        !lt_map(&map_b, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.b, a.n_out, a.n_in, a.ld_b, LB_BK, 128)) {
        o->last_cuda_error = (int)cudaErrorInvalidValue;
        return LF_ECUDA;
    }
    const int splits = lb_choose(o, a, n_k);
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute at[2];
    const lb_kernel f = lb_pick(a.out_dtype, a.b_tiles == 0, splits);
    if (splits == 0) {
        P.tiles_m = (P.M + 255) / 256; P.tiles_n = (P.N + 255) / 256;
        P.idesc = idesc | (256u >> 3) << 17 | (256u >> 4) << 24;
        P.band = 8;
        const long long tiles = (long long)P.tiles_m * P.tiles_n;
        const int pairs = tiles < o->max_block_pairs ? (int)tiles : o->max_block_pairs;
        lt_cluster_config(&cfg, at, 2 * pairs, lb_threads(a.b_tiles == 0), 2, LB_SMEM, o->stream);
        LF_OPS_TRY(o, cudaLaunchKernelEx(&cfg, f, map_a, map_b, P));
        o->stats.form = LF_FORM_PAIRS;
        o->stats.splits = 1;
    } else {
        P.tiles_m = (P.M + 127) / 128; P.tiles_n = (P.N + 127) / 128;
        P.idesc = idesc | (128u >> 3) << 17 | (128u >> 4) << 24;
        P.stages_per_split = (n_k + splits - 1) / splits;
        lt_cluster_config(&cfg, at, P.tiles_m * P.tiles_n * splits, LBS_THREADS, splits, LBS_SMEM, o->stream);
        LF_OPS_TRY(o, cudaLaunchKernelEx(&cfg, f, map_a, map_b, P));
        o->stats.form = LF_FORM_SPLIT;
        o->stats.splits = splits;
    }
    o->stats.launches += 1;
    return LF_OK;
}

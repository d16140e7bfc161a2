// The dense layer's three products in 16 bits on the 5th-generation tensor cores:
//     D[m][n] = sum_k A[m][k] B[n][k],   fp32 accumulators, epilogue on D
//   forward  A = x  [tokens][n_in],  B = w  [n_out][n_in]:  y = sigma(D + bias) + residual, z in 8 bits
//   grad_x   A = dz [tokens][n_out], B = w^T (w read MN-major): dx = D (.) sigma'(z from 8 bits) + add
//   grad_w   A = dz^T, B = x^T (both MN-major, the contraction runs over tokens):  gw = D
// Every operand is used where it lies; what differs is the box TMA fetches and the descriptor's
// majorness.  A K stage is 64 deep; a block of operand is 128 x 64 (16 KiB, 128-byte swizzle).
//
// Three kernels, chosen by an estimate of each one's time (lt_choose):
//   CTA pairs (k_product_pair): tcgen05.mma.cta_group::2, persistent.  256 x 256 tiles with two accumulators that take
//     turns, so that the epilogue of a tile runs under the next tile's products, or 512 x 256 tiles, an accumulator for
//     each 256 rows, which fetch 24 KiB for what 256 x 256 tiles fetch 32; the forward product's may be narrower.
//   Split tiles (k_product_split): one CTA per 128 x 128 tile and part of the contraction (1, 2, 4 or 8 parts); the
//     CTAs of a tile form a cluster, add their parts through distributed shared memory, and each finishes its
//     share of the rows.  Fills the device where there are few tiles.
//   Split pairs (k_product_pair_split): 256 x 256 tiles of CTA pairs, two pairs to a cluster and half of the
//     contraction each, for what lies between.
// What bounds them: large products the chip's power limit (8192 x 4096 -> 16384 in a loop: 1.35 PFLOP/s without an
// activation, 1.25 to 1.33 with GELU, by the card; the tensor cores are at work 85 % of the time in a single launch); middle ones the fetch
// of operands from L2; small ones launch, first loads and the meeting of the parts (5 to 6 us for a small layer, of
// which 2.3 is the launch).  Copies that reach several CTAs of a cluster at once would relieve the fetch; they are
// left out because operands may be any memory that the caller's device can address.
//
// The tensor core adds into its accumulator by truncation: over terms of one sign 1.0e-7 of the sum per instruction
// (16 terms), always towards zero.  An accumulator therefore takes a limited number of stages (lt_fill), and the fills are
// added in registers with round-to-nearest: 8 stages, 3e-6, for an fp32 result, which a weight gradient over thousands of
// tokens would show; 512 stages, 2.0e-4, for f16 and 1024, 4.1e-4, for bf16, below the smallest half unit of those
// types (2.4e-4, 2.0e-3).  Only contractions beyond 32768 and 65536 have more than one fill, in copies of
// the kernels made for them.  (Without a limit f16 results were 4.2e-4 short over 65536 terms, 8.4e-4 over 2^20 in eight parts.  With 256
// stages 2048 x 28672 -> 8192 took 890 us instead of 700, as only 256-row tiles have an accumulator to spare.)
// All waits are bounded; on expiry the status word is raised and the launch drains and ends.
#include "lf_ops_internal.h"
#include "lf_product_tc.cuh"
#include "lf_ptx.cuh"
#include "lf_rows.cuh"

namespace {

using namespace lfrow;

constexpr int LS_THREADS = 512;                          // split tiles: producer, issuer, eight warps that read the accumulator; all finish
constexpr int LP_RING_BYTES = LT_STAGES * LT_STAGE_BYTES;   // pairs: six stages of two blocks, or four of three
constexpr int LP_EPI_BYTES = 8 * 4096;                   // pairs: 32 rows x 128 bytes per epilogue warp
constexpr int LP_THREADS = 384;                          // pairs: a warpgroup with producer and issuer, two for the epilogue
constexpr int LP_REGS_LOW = 56, LP_REGS_HIGH = 224;      // 56 + 2 * 224 = 3 * 168: what the block was launched with
constexpr int LP_AHEAD = 4;                              // 512 x 256 tiles: stages by which block 0 runs ahead
constexpr int LS_LD = 132;                               // split tiles: padded row of the fp32 tile in shared memory
constexpr size_t LP_SMEM = (size_t)LP_RING_BYTES + LP_EPI_BYTES + 1024 + 512;
constexpr int LS_STAGES = 4;
constexpr int LS_TILE_BYTES = 128 * LS_LD * 4;
constexpr int LPS_SPLITS = 2;
constexpr int LD_PS = 260;                               // split pairs: padded row of a CTA's 128 x 256 fp32 tile
constexpr size_t LPS_SMEM = (size_t)LT_STAGES * LT_STAGE_BYTES + 1024 + 512;
static_assert(128 * LD_PS * 4 <= LT_STAGES * LT_STAGE_BYTES, "the fp32 tile overlays the operand ring");
constexpr size_t LS_SMEM = (size_t)LS_STAGES * LT_STAGE_BYTES + LS_TILE_BYTES + 1024 + 512;

// K stages that one accumulator takes of a result of type OUT
template <typename OUT> struct lt_fill { static constexpr int stages = 8; };
template <> struct lt_fill<__half> { static constexpr int stages = 512; };
template <> struct lt_fill<__nv_bfloat16> { static constexpr int stages = 1024; };

struct LtParams {
    int M, N, K;
    int tiles_m, tiles_n;
    int band;                          // pairs: tile rows of a band of the schedule
    int width;                         // pairs: columns of a tile, a multiple of 32 up to 256
    int stages_per_split;      // split tiles
    int act;
    unsigned idesc;
    const float* bias;
    const void* add; long long ld_add;
    void* d; long long ld_d;
    unsigned char *q, *s;
    int wide_q, wide_s, wide_add;      // 256-bit accesses to q and add, 32-bit ones to s, fit a lane's place
    unsigned* status;
    unsigned long long budget_ns;
    int withhold;
};

template <bool PAIR>
__device__ __forceinline__ void lt_mma(unsigned d_tmem, unsigned long long a, unsigned long long b, unsigned idesc, unsigned acc)
{
    if (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// ================================================================================================
// CTA pairs
// ================================================================================================
// What the epilogue reads for 32 columns of its row, fetched a step ahead of its use.
struct lp_operands {
    unsigned q[8];         // GRAD_X: 8-bit pre-activations ...
    unsigned s;            // ... and their scale
    unsigned add[16];      // residual, 16-bit
};
struct lp_place {
    int row0, col0, end, lane;     // (end: past the tile's last column)
    unsigned char* blk;    // this warp's 32 x 128 bytes of shared memory
    size_t groups;         // 8-bit scales per row
    bool full;             // every row and column of the block exists
    float4 bias;           // FORWARD: of columns col0 + 4 * lane ..
    lp_operands next;
};
// (256-bit accesses where a lane's 32 or 64 bytes allow them: its row is a line of its own, so every access less
// is 32 transactions less)
template <int PROD, typename T>
__device__ __forceinline__ void lp_fetch(lp_operands& o, const LtParams& P, const lp_place& e, int j)
{
    const int row = e.row0 + e.lane, col = e.col0 + j * 32;
    if (PROD == LF_PROD_GRAD_X && P.q && row < P.M && col < e.end) {
        const unsigned char* from = P.q + (size_t)row * P.N + col;
        if (e.full && P.wide_q) {
            ld256(from, o.q);
        } else {
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (col + 8 * g < e.end) {
                    const uint2 v = *reinterpret_cast<const uint2*>(from + 8 * g);
                    o.q[2 * g] = v.x; o.q[2 * g + 1] = v.y;
                }
        }
        o.s = P.s[(size_t)row * e.groups + (col >> 5)];
    }
    if (P.add && row < P.M && col < e.end) {
        const T* from = static_cast<const T*>(P.add) + (size_t)row * P.ld_add + col;
        if (e.full && P.wide_add) {
            ld256(from, *reinterpret_cast<unsigned(*)[8]>(o.add));
            ld256(from + 16, *reinterpret_cast<unsigned(*)[8]>(o.add + 8));
        } else {
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (col + 8 * g < e.end) {
                    const uint4 v = *reinterpret_cast<const uint4*>(from + 8 * g);
                    o.add[4 * g] = v.x; o.add[4 * g + 1] = v.y; o.add[4 * g + 2] = v.z; o.add[4 * g + 3] = v.w;
                }
        }
    }
}
// Epilogue of 32 rows x NC columns, a row per lane.  One copy per activation, straight-line: the accumulator's
// registers need constant indices, and choosing the activation per eight columns cost 1100 cycles for 32.  And one
// copy without 8-bit values and residual (OPERANDS = false), which then holds no registers for them.
template <int PROD, typename T, typename OUT, int KIND, int NC, bool OPERANDS>
__device__ __forceinline__ void lp_finish(float (&acc)[NC], const LtParams& P, lp_place& e)
{
    static_assert(NC == 128, "four scales of a row are one word");
    const int lane = e.lane, row = e.row0 + lane;
    unsigned scales = 0;
#pragma unroll
    for (int j = 0; j < NC / 32; ++j) {                         // 32 columns at a time
        const int col = e.col0 + j * 32;
        if (j % 2 == 0 && col >= e.end) break;                  // a narrower tile, or the last one
        const int valid = row < P.M ? min(32, e.end - col) : 0;   // a multiple of 8, or not positive
        float* v = acc + 32 * j;
        const lp_operands now = e.next;
        if (OPERANDS && j < NC / 32 - 1) lp_fetch<PROD, T>(e.next, P, e, j + 1);
        if (PROD == LF_PROD_FORWARD) {
            if (P.bias) {
#pragma unroll
                for (int g = 0; g < 8; ++g) {                   // lane 8 j + g holds the bias of these four columns
                    const int from = 8 * j + g;
                    const float2 lo = add2(make_float2(v[4 * g], v[4 * g + 1]), make_float2(__shfl_sync(0xFFFFFFFFu, e.bias.x, from), __shfl_sync(0xFFFFFFFFu, e.bias.y, from)));
                    const float2 hi = add2(make_float2(v[4 * g + 2], v[4 * g + 3]), make_float2(__shfl_sync(0xFFFFFFFFu, e.bias.z, from), __shfl_sync(0xFFFFFFFFu, e.bias.w, from)));
                    v[4 * g] = lo.x; v[4 * g + 1] = lo.y; v[4 * g + 2] = hi.x; v[4 * g + 3] = hi.y;
                }
            }
            if (OPERANDS && P.q && valid > 0) {
                unsigned m = 0;
                if (valid == 32) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) m = max(m, abs_bits(v[i]));
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) if (i < valid) m = max(m, abs_bits(v[i]));
                }
                const unsigned b = scale_byte(m);
                unsigned char* qp = P.q + (size_t)row * P.N + col;
                if (e.full && P.wide_q) {
                    unsigned w[8];
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const uint2 q8 = quantize8(*reinterpret_cast<float(*)[8]>(v + 8 * g), b);
                        w[2 * g] = q8.x; w[2 * g + 1] = q8.y;
                    }
                    st256(qp, w);
                } else {
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        if (8 * g < valid)
                            *reinterpret_cast<uint2*>(qp + 8 * g) = quantize8(*reinterpret_cast<float(*)[8]>(v + 8 * g), b);
                }
                if (e.full && P.wide_s && (e.col0 & 127) == 0) {                       // four scales at once
                    scales |= b << (8 * j);
                    if (j == NC / 32 - 1) *reinterpret_cast<unsigned*>(P.s + (size_t)row * e.groups + (e.col0 >> 5)) = scales;
                } else {
                    P.s[(size_t)row * e.groups + (col >> 5)] = (unsigned char)b;
                }
            }
            act_all<true, 32, KIND>(v);
        }
        if (OPERANDS && PROD == LF_PROD_GRAD_X && KIND != LF_ACT_NONE) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float z[8];
                dequantize8(make_uint2(now.q[2 * g], now.q[2 * g + 1]), prime_byte(now.s), z);
                prime_all<true, 8, KIND>(v + 8 * g, z, prime_nan(now.s));
            }
        }
        if (OPERANDS && P.add) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 r = add2(make_float2(v[8 * g + 2 * i], v[8 * g + 2 * i + 1]), unpack2(now.add[4 * g + i], T()));
                    v[8 * g + 2 * i] = r.x; v[8 * g + 2 * i + 1] = r.y;
                }
            }
        }
        constexpr int PER = sizeof(OUT) == 2 ? 2 : 1;            // blocks of 32 columns per stored line
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float(&w)[8] = *reinterpret_cast<const float(*)[8]>(v + 8 * g);
            // 16-byte units of a 128-byte line, turned by the row so that neither side meets a bank twice
            if (sizeof(OUT) == 2) {
                vec8<T> o;
                o.set(w);
                *reinterpret_cast<uint4*>(e.blk + lane * 128 + ((((j & 1) * 4 + g) ^ (lane & 7)) << 4)) = o.u;
            } else {
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    *reinterpret_cast<float4*>(e.blk + lane * 128 + (((g * 2 + u) ^ (lane & 7)) << 4)) =
                        make_float4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
            }
        }
        if (j % PER == PER - 1) {                               // a line of every row is complete: whole lines go out
            __syncwarp();
            constexpr int UC = 16 / (int)sizeof(OUT);           // columns of a 16-byte unit
            const int cu = col - (PER - 1) * 32 + (lane & 7) * UC, r0 = e.row0 + (lane >> 3);
            const unsigned char* from = e.blk + (lane >> 3) * 128;
            OUT* to = static_cast<OUT*>(P.d) + (size_t)r0 * P.ld_d + cu;
            const size_t step = (size_t)4 * P.ld_d;
            uint4 u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)                         // row (lane >> 3) + 4 i: its turn alternates
                u[i] = *reinterpret_cast<const uint4*>(from + i * 512 + (((lane & 7) ^ (((lane >> 3) + 4 * i) & 7)) << 4));
            if (cu < e.end) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (r0 + 4 * i < P.M) *reinterpret_cast<uint4*>(to + i * step) = u[i];
            }
            __syncwarp();
        }
    }
}

// MB: 128-row blocks per CTA.  MB = 1: 256 x 256 tiles, the two accumulators alternate between tiles (or
// fills).  MB = 2: 512 x 256 tiles, one accumulator per block: a 64-deep stage takes 1024 cycles for twice the
// products of MB = 1's 568 (8192 x 4096 -> 16384 without an activation: 813 us in a loop, 841 with MB = 1).
// Epilogue of 128 rows x 256 columns: 3700 cycles as it is, 7500 with GELU (half of it exponentials and
// reciprocals), 10000 with 8-bit values.  8192 x 1024 -> 4096: 53 us, with GELU 63, with GELU, checkpoint and residual 90.
// FILL: K stages per accumulator (MB = 1), or 0: one accumulator takes the whole contraction.
template <int PROD, typename T, typename OUT, int MB, int FILL>
__global__ void __launch_bounds__(LP_THREADS, 1)
k_product_pair(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const LtParams P)
{
    constexpr bool A_MN = PROD == LF_PROD_GRAD_W, B_MN = PROD != LF_PROD_FORWARD;
    static_assert(MB == 1 || FILL == 0, "with 512 rows both accumulators belong to one tile");
    constexpr int STAGES = MB == 2 ? 4 : 6;
    constexpr unsigned STAGE_BYTES = (unsigned)(MB + 1) * LT_BLOCK_BYTES;
    constexpr int NC = 128;                                  // columns of an epilogue warp
    static_assert(STAGES * STAGE_BYTES == LP_RING_BYTES, "both forms use the whole ring");
    extern __shared__ unsigned char lt_smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(lt_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    unsigned char* epi = ring + LP_RING_BYTES;
    LtShared* sh = reinterpret_cast<LtShared*>(epi + LP_EPI_BYTES);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned rank = lfptx::cluster_ctarank();
    const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const int n_tiles = P.tiles_m * P.tiles_n;
    const int n_k = (P.K + LT_BK - 1) / LT_BK;
    const int fill = FILL ? FILL : n_k;
    // bytes that this CTA's loads of a stage bring
    const unsigned stage_bytes = MB * LT_BLOCK_BYTES + (unsigned)(B_MN ? (P.width > 128 ? 128 : 64) : P.width / 2) * (LT_BK * 2);

    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
        for (int i = 0; i < STAGES; ++i) {
            lfptx::mbar_init(lfptx::smem_u32(&sh->full[i]), 1);
            lfptx::mbar_init(lfptx::smem_u32(&sh->empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            lfptx::mbar_init(lfptx::smem_u32(&sh->acc_full[i]), 1);
            lfptx::mbar_init(lfptx::smem_u32(&sh->acc_empty[i]), 16);   // eight epilogue warps of each CTA
        }
        sh->abort_flag = 0u;
        sh->prog_it = 0u;
        lfptx::mbar_fence_init();
    }
    if (warp == 1) {
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

    // registers move from the first warpgroup to the two that hold accumulators
    if (warp < 4) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LP_REGS_LOW));
      if (warp == 0) {
        // ------------------------------ TMA producer: this CTA's halves -------------------------
        if (lane == 0) {
            unsigned it = 0;
            bool ok = true;
            for (int t = pair; t < n_tiles && ok; t += n_pairs) {
                int tm, tn;
                lp_tile(t, P, tm, tn);
                const int m0 = (tm * 2 + (int)rank) * (MB * 128), n0 = tn * P.width + (int)rank * (P.width / 2);
                for (int ks = 0; ks < n_k; ++ks, ++it) {
                    const unsigned st = it % STAGES, use = it / STAGES;
                    if (use > 0 && !lt_wait(lfptx::smem_u32(&sh->empty[st]), (use - 1) & 1u, P, sh)) { ok = false; break; }
                    const unsigned lbar = lfptx::smem_u32(&sh->full[st]);
                    if (P.withhold && pair == 0 && rank == 1 && it == 0) continue;    // test hook
                    if (rank == 0) lfptx::mbar_arrive_expect_tx(lbar, 2u * stage_bytes);
                    const unsigned bar = lfptx::map_to_cta(lbar, 0);
                    const unsigned dst = lfptx::smem_u32(ring + (size_t)st * STAGE_BYTES);
#pragma unroll
                    for (int b = 0; b < MB; ++b) lt_load<A_MN, true>(dst + b * LT_BLOCK_BYTES, &map_a, bar, m0 + b * 128, ks * LT_BK);
                    lt_load<B_MN, true>(dst + MB * LT_BLOCK_BYTES, &map_b, bar, n0, ks * LT_BK, P.width / 2);
                }
            }
            sh->prog_it = it;
        }
      } else if (warp == 1) {
        // ------------------------------ MMA issuer (leader CTA) ---------------------------------
        if (lane == 0 && rank == 0) {
            auto full_wait = [&](unsigned it) {
                const bool ok = lt_wait(lfptx::smem_u32(&sh->full[it % STAGES]), (it / STAGES) & 1u, P, sh);
                lfptx::tc_fence_after();
                return ok;
            };
            auto acc_wait = [&](unsigned c) {           // fill c of the accumulators: buffer c & 1
                const bool ok = (c >> 1) == 0 || lt_wait(lfptx::smem_u32(&sh->acc_empty[c & 1u]), ((c >> 1) - 1) & 1u, P, sh);
                lfptx::tc_fence_after();
                return ok;
            };
            auto products = [&](unsigned it, int b, unsigned buffer, bool first) {      // block b of a stage
                const unsigned st_addr = lfptx::smem_u32(ring + (size_t)(it % STAGES) * STAGE_BYTES);
                const unsigned a_addr = st_addr + b * LT_BLOCK_BYTES, b_addr = st_addr + MB * LT_BLOCK_BYTES;
#pragma unroll
                for (int kk = 0; kk < LT_BK / 16; ++kk)
                    lt_mma<true>(tmem_base + buffer * 256u, lt_desc<A_MN>(a_addr + lt_step<A_MN>(kk)),
                                 lt_desc<B_MN>(b_addr + lt_step<B_MN>(kk)), P.idesc, (!first || kk > 0) ? 1u : 0u);
            };
            auto release = [&](unsigned it) { lt_commit<true>(lfptx::smem_u32(&sh->empty[it % STAGES])); };
            auto filled = [&](unsigned c) { lt_commit<true>(lfptx::smem_u32(&sh->acc_full[c & 1u])); };
            unsigned it = 0, c = 0;             // stages consumed, accumulators filled
            bool ok = true;
            for (int t = pair; t < n_tiles && ok; t += n_pairs) {
                if (MB == 1) {
                    for (int k0 = 0; k0 < n_k && ok; k0 += fill, ++c) {
                        if (!acc_wait(c)) { ok = false; break; }
                        const int k1 = min(k0 + fill, n_k);
                        for (int ks = k0; ks < k1; ++ks, ++it) {
                            if (!full_wait(it)) { ok = false; break; }
                            products(it, 0, c & 1u, ks == k0);
                            release(it);
                        }
                        if (ok) filled(c);
                    }
                } else {
                    // Both accumulators belong to this tile, so the epilogue can only run beside the products if one
                    // block is ahead of the other: the first stages are multiplied for block 0 before block
                    // 1's accumulator is asked for, the last ones for block 0 before block 1, whose
                    // products then cover block 0's epilogue.
                    const int head = min(LP_AHEAD, n_k), tail = min(LP_AHEAD, n_k - head), mid_end = n_k - tail;
                    if (!acc_wait(c)) break;
                    for (int ks = 0; ks < head && ok; ++ks) {
                        ok = full_wait(it + ks);
                        if (ok) products(it + ks, 0, 0u, ks == 0);
                    }
                    if (ok && n_k == head) filled(c);
                    if (!ok || !acc_wait(c + 1)) break;
                    for (int ks = 0; ks < head; ++ks) {
                        products(it + ks, 1, 1u, ks == 0);
                        release(it + ks);
                    }
                    for (int ks = head; ks < mid_end && ok; ++ks) {
                        ok = full_wait(it + ks);
                        if (!ok) break;
                        products(it + ks, 0, 0u, false);
                        products(it + ks, 1, 1u, false);
                        release(it + ks);
                    }
                    for (int ks = mid_end; ks < n_k && ok; ++ks) {
                        ok = full_wait(it + ks);
                        if (ok) products(it + ks, 0, 0u, false);
                    }
                    if (!ok) break;
                    if (tail > 0) filled(c);
                    for (int ks = mid_end; ks < n_k; ++ks) {
                        products(it + ks, 1, 1u, false);
                        release(it + ks);
                    }
                    filled(c + 1);
                    it += n_k;
                    c += 2;
                }
            }
        }
      }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(LP_REGS_HIGH));
        // ------------------------------ epilogue (warps 4..11 of both CTAs) ----------------------
        // A warp has one 32-lane quadrant (32 rows) and one half (NC columns) of an accumulator; a lane has a row.
        // It takes the columns into registers and hands the accumulator back before it works on
        // them.  Results are turned through a 32 x 128-byte block in shared memory, so that a warp
        // stores whole lines (a TMA store of the block instead made the next block wait for its read:
        // 6000 to 9000 cycles per accumulator against 2000).
        const int quad = warp & 3, half = (warp - 4) >> 2;
        const unsigned leader_acc_empty = lfptx::map_to_cta(lfptx::smem_u32(&sh->acc_empty[0]), 0);
        unsigned char* blk = epi + (warp - 4) * 4096;
        const size_t groups = (size_t)((P.N + 31) / 32);
        unsigned c = 0;
        bool ok = true;
        for (int tb = pair * MB; ok; tb += (tb % MB == MB - 1) ? n_pairs * MB - (MB - 1) : 1) {     // tile, block
            if (tb / MB >= n_tiles) break;
            int tm, tn;
            lp_tile(tb / MB, P, tm, tn);
            const int row0 = (tm * 2 + (int)rank) * (MB * 128) + (tb % MB) * 128 + quad * 32;
            const int col0 = tn * P.width + half * NC, end = min(P.N, (tn + 1) * P.width);
            const unsigned lane_addr = tmem_base + ((unsigned)(quad * 32) << 16) + half * (unsigned)NC;
            lp_place e = {row0, col0, end, lane, blk, groups, row0 + 32 <= P.M && col0 + NC <= end, make_float4(0.f, 0.f, 0.f, 0.f), {}};
            if (PROD == LF_PROD_FORWARD && P.bias && col0 + 4 * lane < P.N) e.bias = *reinterpret_cast<const float4*>(P.bias + col0 + 4 * lane);
            const bool operands = PROD != LF_PROD_GRAD_W && (P.q || P.add);
            if (operands) lp_fetch<PROD, T>(e.next, P, e, 0);   // on its way while the accumulator is waited for
            float acc[NC];
            if (FILL) {
#pragma unroll
                for (int i = 0; i < NC; ++i) acc[i] = 0.f;
                for (int k0 = 0; k0 < n_k; k0 += fill, ++c) {
                    const unsigned ab = c & 1u;
                    if (!lt_wait(lfptx::smem_u32(&sh->acc_full[ab]), (c >> 1) & 1u, P, sh)) { ok = false; break; }
                    lfptx::tc_fence_after();
#pragma unroll
                    for (int j = 0; j < NC / 16; ++j) {
                        unsigned r[16];
                        lfptx::tmem_ld16(lane_addr + ab * 256u + j * 16, r);
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[j * 16 + i] += __uint_as_float(r[i]);
                    }
                    lfptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) lt_arrive_cluster(leader_acc_empty + ab * 8u);
                }
                if (!ok) break;
            } else {
                const unsigned ab = c & 1u;
                if (!lt_wait(lfptx::smem_u32(&sh->acc_full[ab]), (c >> 1) & 1u, P, sh)) break;
                ++c;
                lfptx::tc_fence_after();
                lfptx::tmem_ld_row(lane_addr + ab * 256u, acc);
                lfptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) lt_arrive_cluster(leader_acc_empty + ab * 8u);
            }
            const int act = PROD == LF_PROD_GRAD_W || (PROD == LF_PROD_GRAD_X && !P.q) ? LF_ACT_NONE : P.act;
            if constexpr (PROD != LF_PROD_GRAD_W) {
                if (operands) {
                    switch (act) {
                        case LF_ACT_SIGMOID: lp_finish<PROD, T, OUT, LF_ACT_SIGMOID, NC, true>(acc, P, e); break;
                        case LF_ACT_TANH: lp_finish<PROD, T, OUT, LF_ACT_TANH, NC, true>(acc, P, e); break;
                        case LF_ACT_RELU: lp_finish<PROD, T, OUT, LF_ACT_RELU, NC, true>(acc, P, e); break;
                        case LF_ACT_SILU: lp_finish<PROD, T, OUT, LF_ACT_SILU, NC, true>(acc, P, e); break;
                        case LF_ACT_GELU: lp_finish<PROD, T, OUT, LF_ACT_GELU, NC, true>(acc, P, e); break;
                        default: lp_finish<PROD, T, OUT, LF_ACT_NONE, NC, true>(acc, P, e); break;
                    }
                    continue;
                }
            }
            if constexpr (PROD == LF_PROD_FORWARD) {
                switch (act) {
                    case LF_ACT_SIGMOID: lp_finish<PROD, T, OUT, LF_ACT_SIGMOID, NC, false>(acc, P, e); continue;
                    case LF_ACT_TANH: lp_finish<PROD, T, OUT, LF_ACT_TANH, NC, false>(acc, P, e); continue;
                    case LF_ACT_RELU: lp_finish<PROD, T, OUT, LF_ACT_RELU, NC, false>(acc, P, e); continue;
                    case LF_ACT_SILU: lp_finish<PROD, T, OUT, LF_ACT_SILU, NC, false>(acc, P, e); continue;
                    case LF_ACT_GELU: lp_finish<PROD, T, OUT, LF_ACT_GELU, NC, false>(acc, P, e); continue;
                    default: break;
                }
            }
            lp_finish<PROD, T, OUT, LF_ACT_NONE, NC, false>(acc, P, e);
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
                const unsigned bar = lfptx::smem_u32(&sh->full[j % STAGES]);
                if (j >= it_l) lfptx::mbar_arrive_expect_tx(bar, stage_bytes);                // only the peer loaded
                else lt_complete_tx(bar, stage_bytes);                                        // only the leader loaded
            }
            const unsigned long long t0 = lfptx::globaltimer_ns();
            for (unsigned j = hi > STAGES ? hi - STAGES : 0; j < hi; ++j) {
                const unsigned bar = lfptx::smem_u32(&sh->full[j % STAGES]);
                while (!lfptx::mbar_try_wait(bar, (j / STAGES) & 1u) && lfptx::globaltimer_ns() - t0 < 50000000ull) { }
            }
        }
    }
    lfptx::cluster_sync_all();
    if (warp == 1) {
        lfptx::tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

// ================================================================================================
// Split tiles: one CTA per 128 x 128 tile and part of the contraction, a cluster per tile
// ================================================================================================
// Bound by latency: of 5.4 us for 70 x 520 -> 1024 (8 parts; floor 0.2) the launch is 2.3, the rest set-up, first loads,
// meeting of the parts and store, one after another.  Distributed shared memory gives a multiprocessor 14 bytes a
// cycle, so 64 KB from the other parts are 4300 cycles: rows that do not exist are not exchanged (32 tokens, 4096 -> 4096:
// 10.8 us against 14.2).  509 x 4096 -> 1024 with 4 parts: 11.1 us, with 2: 14.9.
//
// What is left to do for a CTA's share of a tile's rows: add the parts, bias, 8 bits, activation, residual, store.  A
// piece is 128 columns of a row, half a warp's: a lane has columns 4 i .. and 64 + 4 i .., so that every
// access is a whole line, also to another CTA's tile, and eight neighbours hold an 8-bit scale group.  With eight
// parts a CTA has 16 rows, one for each warp: then a piece is a whole warp's (NK = 1: columns 4 i alone).
struct ls_share {
    const float* tile;         // [row][ld] fp32, the share's first row
    int ld;
    int row0, rows;            // first row of the share in the matrix, number of rows
    int col0;                  // first column of the tile
    int peer0, peer_step;      // CTA of the cluster that holds part p: peer0 + p * peer_step
    int live;                  // 0: a dry run, nothing is loaded or stored
    int leave;                 // arrive at the cluster's barrier as soon as the last part has been read
};
struct ls_operands {           // what a piece reads of the layer's matrices, fetched a piece ahead
    unsigned q[2], s[2];
    uint2 add[2];
};
template <int PROD, typename T, int NK>
__device__ __forceinline__ void ls_fetch(ls_operands& o, const LtParams& P, const ls_share& e, int row, int col)
{
#pragma unroll
    for (int k = 0; k < NK; ++k) {
        const int c = col + 64 * k;
        o.q[k] = o.s[k] = 0;
        o.add[k] = make_uint2(0, 0);
        if (PROD == LF_PROD_GRAD_W || !e.live || row >= e.row0 + e.rows || row >= P.M || c >= P.N) continue;
        if (PROD == LF_PROD_GRAD_X && P.q) {
            o.q[k] = *reinterpret_cast<const unsigned*>(P.q + (size_t)row * P.N + c);
            o.s[k] = P.s[(size_t)row * ((P.N + 31) / 32) + (c >> 5)];
        }
        if (P.add) o.add[k] = *reinterpret_cast<const uint2*>(static_cast<const T*>(P.add) + (size_t)row * P.ld_add + c);
    }
}
// HALVES: pieces per row.  One copy per activation: the choice stands outside of the loop.
template <int PROD, typename T, typename OUT, int SPLITS, int HALVES, int KIND>
__device__ __forceinline__ void ls_rows(const LtParams& P, const ls_share& e, ls_operands now)
{
    constexpr int NK = SPLITS == 8 ? 1 : 2, SIDE = NK;         // column groups of a lane, pieces a warp has side by side
    static_assert(HALVES == 1 || NK == 2, "two halves of a row are two pieces");
    const int lane = threadIdx.x & 31, i = NK == 1 ? lane : lane & 15;
    const int u0 = (threadIdx.x >> 5) * SIDE + (NK == 1 ? 0 : lane >> 4);
    const int half = HALVES == 2 ? (lane >> 4) : 0;
    const int col = e.col0 + half * 128 + 4 * i;
    const bool in0 = col < P.N, in1 = NK == 2 && col + 64 < P.N;
    float2 bias[4] = {f2(0.f), f2(0.f), f2(0.f), f2(0.f)};
    if (PROD == LF_PROD_FORWARD && P.bias) {
#pragma unroll
        for (int k = 0; k < NK; ++k)
            if (k ? in1 : in0) {
                const float4 b = *reinterpret_cast<const float4*>(P.bias + col + 64 * k);
                bias[2 * k] = make_float2(b.x, b.y);
                bias[2 * k + 1] = make_float2(b.z, b.w);
            }
    }
    const size_t groups = (size_t)((P.N + 31) / 32);
    const int pieces = e.rows * HALVES, steps = (pieces + 16 * SIDE - 1) / (16 * SIDE);      // 16 warps
    const bool reads = P.add != nullptr || (PROD == LF_PROD_GRAD_X && KIND != LF_ACT_NONE);
    if (SPLITS > 1 && e.leave && steps == 0) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
#pragma unroll 1
    for (int st = 0; st < steps; ++st) {
        const int u = u0 + st * 16 * SIDE, r = HALVES == 2 ? u >> 1 : u;
        const float* at = e.tile + r * e.ld + half * 128 + 4 * i;
        float4 x[SPLITS][2];
#pragma unroll
        for (int p = 0; p < SPLITS; ++p) {
            x[p][0] = x[p][1] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (u >= pieces) continue;                         // (reading along cost S = 8 twice the traffic between CTAs)
            if (SPLITS == 1) {
                x[p][0] = *reinterpret_cast<const float4*>(at);
                if (NK == 2) x[p][1] = *reinterpret_cast<const float4*>(at + 64);
            } else {
                const unsigned from = lfptx::map_to_cta(lfptx::smem_u32(at), (unsigned)(e.peer0 + p * e.peer_step));
                x[p][0] = lt_ld_cluster_f4(from);
                if (NK == 2) x[p][1] = lt_ld_cluster_f4(from + 256);
            }
        }
        if (SPLITS > 1 && e.leave && st + 1 == steps) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        const ls_operands mine = now;
        const int row = e.row0 + r, row_next = e.row0 + (HALVES == 2 ? (u + 32) >> 1 : u + 16 * SIDE);
        if (reads && st + 1 < steps) ls_fetch<PROD, T, NK>(now, P, e, row_next, col);
        float v[4 * NK];
#pragma unroll
        for (int k = 0; k < NK; ++k) {                         // parts in order: the sum does not depend on timing
            float2 lo = make_float2(x[0][k].x, x[0][k].y), hi = make_float2(x[0][k].z, x[0][k].w);
#pragma unroll
            for (int p = 1; p < SPLITS; ++p) {
                lo = add2(lo, make_float2(x[p][k].x, x[p][k].y));
                hi = add2(hi, make_float2(x[p][k].z, x[p][k].w));
            }
            if (PROD == LF_PROD_FORWARD) { lo = add2(lo, bias[2 * k]); hi = add2(hi, bias[2 * k + 1]); }
            v[4 * k] = lo.x; v[4 * k + 1] = lo.y; v[4 * k + 2] = hi.x; v[4 * k + 3] = hi.y;
        }
        const bool have = e.live && u < pieces && row < P.M;
        if (PROD == LF_PROD_FORWARD && P.q) {
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                const bool in = have && (k ? in1 : in0);
                const float* w = v + 4 * k;
                unsigned m = in ? max(max(abs_bits(w[0]), abs_bits(w[1])), max(abs_bits(w[2]), abs_bits(w[3]))) : 0u;
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
                const unsigned b = scale_byte(m);
                const float is = inv_scale(b);
                if (in) {
                    const int c = col + 64 * k;
                    *reinterpret_cast<unsigned*>(P.q + (size_t)row * P.N + c) = to_e4m3x4(w[0] * is, w[1] * is, w[2] * is, w[3] * is);
                    if ((c & 31) == 0) P.s[(size_t)row * groups + (c >> 5)] = (unsigned char)b;
                }
            }
        }
        if (PROD == LF_PROD_FORWARD) act_all<true, 4 * NK, KIND>(v);
        if (PROD == LF_PROD_GRAD_X && KIND != LF_ACT_NONE) {
            float z[4 * NK];
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                from_e4m3x4(mine.q[k], scale(prime_byte(mine.s[k])), z[4 * k], z[4 * k + 1], z[4 * k + 2], z[4 * k + 3]);
                prime_all<true, 4, KIND>(v + 4 * k, z + 4 * k, prime_nan(mine.s[k]));
            }
        }
        OUT* to = static_cast<OUT*>(P.d) + (size_t)row * P.ld_d + col;
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            float* w = v + 4 * k;
            if (PROD != LF_PROD_GRAD_W && P.add) {
                const float2 f0 = unpack2(mine.add[k].x, T()), f1 = unpack2(mine.add[k].y, T());
                w[0] += f0.x; w[1] += f0.y; w[2] += f1.x; w[3] += f1.y;
            }
            if (have && (k ? in1 : in0)) {
                if (sizeof(OUT) == 2) *reinterpret_cast<uint2*>(to + 64 * k) = make_uint2(pack2(w[0], w[1], T()), pack2(w[2], w[3], T()));
                else *reinterpret_cast<float4*>(to + 64 * k) = make_float4(w[0], w[1], w[2], w[3]);
            }
        }
    }
}
template <int PROD, typename T, typename OUT, int SPLITS, int HALVES>
__device__ __forceinline__ void ls_finish(const LtParams& P, const ls_share& e, const ls_operands& first)
{
    switch (PROD == LF_PROD_GRAD_W || (PROD == LF_PROD_GRAD_X && !P.q) ? LF_ACT_NONE : P.act) {
        case LF_ACT_SIGMOID: ls_rows<PROD, T, OUT, SPLITS, HALVES, LF_ACT_SIGMOID>(P, e, first); break;
        case LF_ACT_TANH: ls_rows<PROD, T, OUT, SPLITS, HALVES, LF_ACT_TANH>(P, e, first); break;
        case LF_ACT_RELU: ls_rows<PROD, T, OUT, SPLITS, HALVES, LF_ACT_RELU>(P, e, first); break;
        case LF_ACT_SILU: ls_rows<PROD, T, OUT, SPLITS, HALVES, LF_ACT_SILU>(P, e, first); break;
        case LF_ACT_GELU: ls_rows<PROD, T, OUT, SPLITS, HALVES, LF_ACT_GELU>(P, e, first); break;
        default: ls_rows<PROD, T, OUT, SPLITS, HALVES, LF_ACT_NONE>(P, e, first); break;
    }
}
// the first piece's operands, on their way while the accumulator is waited for
template <int PROD, typename T, int SPLITS, int HALVES>
__device__ __forceinline__ ls_operands ls_first(const LtParams& P, const ls_share& e)
{
    constexpr int NK = SPLITS == 8 ? 1 : 2;
    const int lane = threadIdx.x & 31, u = (threadIdx.x >> 5) * NK + (NK == 1 ? 0 : lane >> 4);
    ls_operands o;
    ls_fetch<PROD, T, NK>(o, P, e, e.row0 + (HALVES == 2 ? u >> 1 : u), e.col0 + (HALVES == 2 ? (lane >> 4) * 128 : 0) + 4 * (NK == 1 ? lane : lane & 15));
    return o;
}

// The parts of a tile meet in distributed shared memory: every part leaves its fp32 tile beside its operand ring,
// and after a cluster barrier each CTA adds its share of the rows, R = 128 / splits, from all parts,
// every load issued before the first addition.  (One part after the other cost 7000 to 11000 cycles,
// storing registers into the owners' shared memory, 16 bytes a row, 5000.)
// The epilogue warps go through their code once before the accumulator is complete, with nothing to load or store:
// a launch this short meets its instructions and parameters cold, 2400 cycles otherwise spent at its end.
template <int PROD, typename T, typename OUT, int SPLITS, int FILL>
__global__ void __launch_bounds__(LS_THREADS, 1)
k_product_split(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const LtParams P)
{
    constexpr bool A_MN = PROD == LF_PROD_GRAD_W, B_MN = PROD != LF_PROD_FORWARD;
    extern __shared__ unsigned char lt_smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(lt_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    float* tile = reinterpret_cast<float*>(ring + (size_t)LS_STAGES * LT_STAGE_BYTES);     // [128][LS_LD]
    LtShared* sh = reinterpret_cast<LtShared*>(ring + (size_t)LS_STAGES * LT_STAGE_BYTES + LS_TILE_BYTES);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = (int)(blockIdx.x % (unsigned)SPLITS), t = (int)(blockIdx.x / (unsigned)SPLITS);
    const int tn = t / P.tiles_m, tm = t - tn * P.tiles_m;
    const int n_k_all = (P.K + LT_BK - 1) / LT_BK;
    const int ks0 = part * P.stages_per_split;
    const int n_k = max(0, min(P.stages_per_split, n_k_all - ks0));
    const int fill = FILL ? FILL : (n_k > 0 ? n_k : 1);

    auto load_stage = [&](int ks) {                    // one thread; stage ks of this part into its slot
        const unsigned st = (unsigned)ks % LS_STAGES, bar = lfptx::smem_u32(&sh->full[st]);
        lfptx::mbar_arrive_expect_tx(bar, LT_STAGE_BYTES);
        if (P.withhold && blockIdx.x == 0 && ks == 0) return;                       // test hook
        const unsigned dst = lfptx::smem_u32(ring + (size_t)st * LT_STAGE_BYTES);
        lt_load<A_MN, false>(dst, &map_a, bar, tm * 128, (ks0 + ks) * LT_BK);
        lt_load<B_MN, false>(dst + LT_BLOCK_BYTES, &map_b, bar, tn * 128, (ks0 + ks) * LT_BK);
    };
    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
        for (int i = 0; i < LS_STAGES; ++i) {
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
        for (int ks = 0; ks < min(n_k, LS_STAGES); ++ks) load_stage(ks);            // under the rest of the set-up
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
            int ks = LS_STAGES;
            for (; ks < n_k; ++ks) {
                if (!lt_wait(lfptx::smem_u32(&sh->empty[ks % LS_STAGES]), (unsigned)(ks / LS_STAGES - 1) & 1u, P, sh)) break;
                load_stage(ks);
            }
            // after giving up: do not let the CTA go on under loads that are still landing
            if (sh->abort_flag) {
                const unsigned long long t0 = lfptx::globaltimer_ns();
                const int n = min(ks, n_k);
                for (int j = max(0, n - LS_STAGES); j < n; ++j)
                    while (!lfptx::mbar_try_wait(lfptx::smem_u32(&sh->full[j % LS_STAGES]), (unsigned)(j / LS_STAGES) & 1u) &&
                           lfptx::globaltimer_ns() - t0 < 50000000ull) { }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            unsigned it = 0, c = 0;
            bool ok = true;
            for (int k0 = 0; k0 < n_k && ok; k0 += fill, ++c) {
                const unsigned ab = c & 1u, ab_use = c >> 1;
                if (ab_use > 0 && !lt_wait(lfptx::smem_u32(&sh->acc_empty[ab]), (ab_use - 1) & 1u, P, sh)) break;
                lfptx::tc_fence_after();
                const int k1 = min(k0 + fill, n_k);
                for (int ks = k0; ks < k1; ++ks, ++it) {
                    const unsigned st = it % LS_STAGES, use = it / LS_STAGES;
                    if (!lt_wait(lfptx::smem_u32(&sh->full[st]), use & 1u, P, sh)) { ok = false; break; }
                    lfptx::tc_fence_after();
                    const unsigned a_addr = lfptx::smem_u32(ring + (size_t)st * LT_STAGE_BYTES);
                    const unsigned b_addr = a_addr + LT_BLOCK_BYTES;
#pragma unroll
                    for (int kk = 0; kk < LT_BK / 16; ++kk)
                        lt_mma<false>(tmem_base + ab * 128u, lt_desc<A_MN>(a_addr + lt_step<A_MN>(kk)),
                                      lt_desc<B_MN>(b_addr + lt_step<B_MN>(kk)), P.idesc, (ks > k0 || kk > 0) ? 1u : 0u);
                    lt_commit<false>(lfptx::smem_u32(&sh->empty[st]));
                }
                if (ok) lt_commit<false>(lfptx::smem_u32(&sh->acc_full[ab]));
            }
        }
    }
    __syncwarp();
    // this CTA's rows: its part of those that exist
    constexpr int R = 128 / SPLITS;
    const int share = min(R, (P.M - tm * 128 + SPLITS - 1) / SPLITS);
    ls_share e = {tile + part * share * LS_LD, LS_LD, tm * 128 + part * share, share, tn * 128, 0, 1, 1, 0};
    const ls_operands first = ls_first<PROD, T, SPLITS, 1>(P, e);
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        if (pass == 1) {
            if (warp >= 2 && warp < 10) {
                const int quad = warp & 3, half = (warp - 2) >> 2;
                float acc[64];
#pragma unroll
                for (int i = 0; i < 64; ++i) acc[i] = 0.f;
                unsigned c = 0;
                for (int k0 = 0; k0 < n_k; k0 += fill, ++c) {
                    const unsigned ab = c & 1u;
                    if (!lt_wait(lfptx::smem_u32(&sh->acc_full[ab]), (c >> 1) & 1u, P, sh)) break;
                    lfptx::tc_fence_after();
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        unsigned r[32];
                        lfptx::tmem_ld32(tmem_base + ((unsigned)(quad * 32) << 16) + ab * 128u + half * 64u + j * 32, r);
#pragma unroll
                        for (int i = 0; i < 32; ++i) acc[j * 32 + i] += __uint_as_float(r[i]);
                    }
                    lfptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) lfptx::mbar_arrive(lfptx::smem_u32(&sh->acc_empty[ab]));
                }
                float* to = tile + (quad * 32 + lane) * LS_LD + half * 64;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    *reinterpret_cast<float4*>(to + 4 * i) = make_float4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]);
            }
            lfptx::tc_fence_before();
            if (SPLITS > 1) lfptx::cluster_sync_all();
            else __syncthreads();
        }
        e.live = pass == 1 && !sh->abort_flag;
        e.rows = pass == 1 ? share : min(share, 1);
        e.peer0 = pass == 1 ? 0 : part;                          // (a dry run reads its own CTA's memory only)
        e.peer_step = pass == 1 ? 1 : 0;
        e.leave = pass;
        ls_finish<PROD, T, OUT, SPLITS, 1>(P, e, first);
    }
    // no CTA may leave while another one reads its tile
    if (SPLITS > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (warp == 1) {
        __syncwarp();
        lfptx::tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(256u) : "memory");
    }
}

// ================================================================================================
// Split pairs: 256 x 256 tiles of CTA pairs, the contraction split over the two pairs of a cluster
// ================================================================================================
// For outputs with too few 256 x 256 tiles to fill the device and too many bytes of operands for 128 x 128 ones: a
// stage costs a pair 568 cycles for four times the products of a 128 x 128 tile's 560.  The parts meet as
// above (the fp32 tile of a CTA, 128 x 256, overlays its operand ring here: every product that reads
// the ring is done when the accumulator is).  16-bit results only, and no more stages a part than one accumulator takes.  512 x 4096 x 4096: 19 us, against 27 with either
// of the other forms.  (Four pairs to a cluster leave 60 multiprocessors idle -- 15 such clusters are resident -- and were
// never ahead.)
template <int PROD, typename T>
__global__ void __launch_bounds__(LS_THREADS, 1)
k_product_pair_split(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const LtParams P)
{
    constexpr bool A_MN = PROD == LF_PROD_GRAD_W, B_MN = PROD != LF_PROD_FORWARD;
    constexpr int SPLITS = LPS_SPLITS, CTAS = 2 * SPLITS;
    extern __shared__ unsigned char lt_smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(lt_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    float* tile = reinterpret_cast<float*>(ring);            // [128][LD_PS], once every product is done
    LtShared* sh = reinterpret_cast<LtShared*>(ring + (size_t)LT_STAGES * LT_STAGE_BYTES);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int member = (int)lfptx::cluster_ctarank(), part = member >> 1, rank = member & 1;
    const unsigned leader = (unsigned)(member & ~1);
    const int t = (int)(blockIdx.x / (unsigned)CTAS);
    const int tn = t / P.tiles_m, tm = t - tn * P.tiles_m;
    const int n_k_all = (P.K + LT_BK - 1) / LT_BK;
    const int ks0 = part * P.stages_per_split;
    const int n_k = max(0, min(P.stages_per_split, n_k_all - ks0));
    const int row_base = tm * 256 + rank * 128;

    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
        for (int i = 0; i < LT_STAGES; ++i) {
            lfptx::mbar_init(lfptx::smem_u32(&sh->full[i]), 1);
            lfptx::mbar_init(lfptx::smem_u32(&sh->empty[i]), 1);
        }
        lfptx::mbar_init(lfptx::smem_u32(&sh->acc_full[0]), 1);
        sh->abort_flag = 0u;
        sh->prog_it = 0u;
        lfptx::mbar_fence_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(lfptx::smem_u32(&sh->tmem_base)), "r"(256u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    lfptx::tc_fence_before();
    __syncthreads();
    lfptx::cluster_sync_all();       // the pair's barriers exist before anything can arrive on them
    lfptx::tc_fence_after();
    const unsigned tmem_base = sh->tmem_base;
    lf_grid_wait();
    lf_grid_release();

    const unsigned short both = (unsigned short)(3u << leader);
    auto commit = [&](unsigned bar) {
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"(both) : "memory");
    };
    if (warp == 0) {
        if (lane == 0) {
            int ks = 0;
            for (; ks < n_k; ++ks) {
                const unsigned st = (unsigned)ks % LT_STAGES, use = (unsigned)ks / LT_STAGES;
                if (use > 0 && !lt_wait(lfptx::smem_u32(&sh->empty[st]), (use - 1) & 1u, P, sh)) break;
                const unsigned lbar = lfptx::smem_u32(&sh->full[st]);
                if (P.withhold && blockIdx.x == 1 && ks == 0) continue;                   // test hook
                if (rank == 0) lfptx::mbar_arrive_expect_tx(lbar, 2u * LT_STAGE_BYTES);
                const unsigned bar = lfptx::map_to_cta(lbar, leader);
                const unsigned dst = lfptx::smem_u32(ring + (size_t)st * LT_STAGE_BYTES);
                lt_load<A_MN, true>(dst, &map_a, bar, row_base, (ks0 + ks) * LT_BK);
                lt_load<B_MN, true>(dst + LT_BLOCK_BYTES, &map_b, bar, tn * 256 + rank * 128, (ks0 + ks) * LT_BK);
            }
            sh->prog_it = (unsigned)ks;
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            bool ok = true;
            for (int ks = 0; ks < n_k; ++ks) {
                const unsigned st = (unsigned)ks % LT_STAGES, use = (unsigned)ks / LT_STAGES;
                if (!lt_wait(lfptx::smem_u32(&sh->full[st]), use & 1u, P, sh)) { ok = false; break; }
                lfptx::tc_fence_after();
                const unsigned a_addr = lfptx::smem_u32(ring + (size_t)st * LT_STAGE_BYTES);
                const unsigned b_addr = a_addr + LT_BLOCK_BYTES;
#pragma unroll
                for (int kk = 0; kk < LT_BK / 16; ++kk)
                    lt_mma<true>(tmem_base, lt_desc<A_MN>(a_addr + lt_step<A_MN>(kk)), lt_desc<B_MN>(b_addr + lt_step<B_MN>(kk)), P.idesc,
                                 (ks > 0 || kk > 0) ? 1u : 0u);
                commit(lfptx::smem_u32(&sh->empty[st]));
            }
            if (ok && n_k > 0) commit(lfptx::smem_u32(&sh->acc_full[0]));
        }
    }
    __syncwarp();
    // this CTA's rows: its part of those that exist
    constexpr int R = 128 / SPLITS;
    const int share = min(R, max(0, (P.M - row_base + SPLITS - 1) / SPLITS));
    ls_share e = {tile + part * share * LD_PS, LD_PS, row_base + part * share, share, tn * 256, rank, 2, 1, 0};
    const ls_operands first = ls_first<PROD, T, SPLITS, 2>(P, e);
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        if (pass == 1) {
            if (warp >= 2 && warp < 10) {
                const int quad = warp & 3, half = (warp - 2) >> 2;
                const bool ok = n_k > 0 && lt_wait(lfptx::smem_u32(&sh->acc_full[0]), 0u, P, sh);
                lfptx::tc_fence_after();
                float* to = tile + (quad * 32 + lane) * LD_PS + half * 128;
#pragma unroll 1
                for (int j = 0; j < 4 && (ok || n_k == 0); ++j) {
                    unsigned r[32];
                    if (ok) lfptx::tmem_ld32(tmem_base + ((unsigned)(quad * 32) << 16) + half * 128u + j * 32, r);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<float4*>(to + j * 32 + 4 * i) =
                            ok ? make_float4(__uint_as_float(r[4 * i]), __uint_as_float(r[4 * i + 1]), __uint_as_float(r[4 * i + 2]), __uint_as_float(r[4 * i + 3]))
                               : make_float4(0.f, 0.f, 0.f, 0.f);
                }
            }
            lfptx::tc_fence_before();
            lfptx::cluster_sync_all();
        }
        // (a dry run reads its own CTA's memory only, which holds operands still: nothing is kept of it)
        e.live = pass == 1 && sh->abort_flag == 0u;
        e.rows = pass == 1 ? share : min(share, 1);
        e.peer0 = pass == 1 ? rank : member;
        e.peer_step = pass == 1 ? 2 : 0;
        e.leave = pass;
        ls_finish<PROD, T, T, SPLITS, 2>(P, e, first);
    }
    // No CTA may leave (or free tensor memory) while another one reads its tile or the pair's products can reach it.
    lfptx::tc_fence_before();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (threadIdx.x == 0 && rank == 0) {
        // given up: as in the persistent form, the loads of both CTAs that are on their way are waited for, with a limit
        const bool any = sh->abort_flag != 0u || lt_ld_cluster_u32(lfptx::map_to_cta(lfptx::smem_u32((const void*)&sh->abort_flag), leader + 1)) != 0u;
        if (any) {
            const unsigned it_l = sh->prog_it, it_p = lt_ld_cluster_u32(lfptx::map_to_cta(lfptx::smem_u32(&sh->prog_it), leader + 1));
            const unsigned hi = max(it_l, it_p), lo = min(it_l, it_p);
            for (unsigned j = lo; j < hi; ++j) {
                const unsigned bar = lfptx::smem_u32(&sh->full[j % LT_STAGES]);
                if (j >= it_l) lfptx::mbar_arrive_expect_tx(bar, LT_STAGE_BYTES);
                else lt_complete_tx(bar, LT_STAGE_BYTES);
            }
            const unsigned long long t0 = lfptx::globaltimer_ns();
            for (unsigned j = hi > LT_STAGES ? hi - LT_STAGES : 0; j < hi; ++j) {
                const unsigned bar = lfptx::smem_u32(&sh->full[j % LT_STAGES]);
                while (!lfptx::mbar_try_wait(bar, (j / LT_STAGES) & 1u) && lfptx::globaltimer_ns() - t0 < 50000000ull) { }
            }
        }
    }
    lfptx::cluster_sync_all();
    if (warp == 1) {
        lfptx::tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(256u) : "memory");
    }
}

typedef void (*lt_kernel)(const CUtensorMap, const CUtensorMap, const LtParams);

// Kernel of a product: index = prod * 2 + (f16); 6 and 7: grad_w with an fp32 result.  Pairs: tile 0 256 x 256,
// 1 512 x 256 (16-bit results), 2 256 x 256 with more than one fill of the accumulator.  Split tiles: splits = 1, 2, 4, 8, and
// LT_LONG_SPLITS for eight parts of more than one fill.
constexpr int LT_KERNELS = 8, LT_LONG_SPLITS = 16;
enum lt_tile { LT_256x256 = 0, LT_512x256 = 1, LT_256x256_LONG = 2, LT_TILES = 3 };
template <int PROD, typename T, typename OUT>
lt_kernel lt_pair_of(int tile)
{
    constexpr int FILL = lt_fill<OUT>::stages;
    if constexpr (sizeof(OUT) == 2) {
        if (tile == LT_512x256) return k_product_pair<PROD, T, OUT, 2, 0>;
        if (tile == LT_256x256_LONG) return k_product_pair<PROD, T, OUT, 1, FILL>;
        return k_product_pair<PROD, T, OUT, 1, 0>;
    }
    return tile == LT_256x256 ? k_product_pair<PROD, T, OUT, 1, FILL> : nullptr;
}
template <int PROD, typename T, typename OUT>
lt_kernel lt_split_of(int splits)
{
    constexpr int FILL = lt_fill<OUT>::stages, SHORT = sizeof(OUT) == 2 ? 0 : FILL;
    switch (splits) {
        case 1: return k_product_split<PROD, T, OUT, 1, SHORT>;
        case 2: return k_product_split<PROD, T, OUT, 2, SHORT>;
        case 4: return k_product_split<PROD, T, OUT, 4, SHORT>;
        case 8: return k_product_split<PROD, T, OUT, 8, SHORT>;
        default: return k_product_split<PROD, T, OUT, 8, FILL>;
    }
}
// stages that one accumulator takes without being added up
int lt_one_fill(const lf_product& p)
{
    return p.out_dtype == LF_F32 ? 1 << 30 : p.out_dtype == LF_F16 ? lt_fill<__half>::stages : lt_fill<__nv_bfloat16>::stages;
}
lt_kernel lt_pick_pair(int i, int tile)
{
    switch (i) {
        case 0: return lt_pair_of<LF_PROD_FORWARD, __nv_bfloat16, __nv_bfloat16>(tile);
        case 1: return lt_pair_of<LF_PROD_FORWARD, __half, __half>(tile);
        case 2: return lt_pair_of<LF_PROD_GRAD_X, __nv_bfloat16, __nv_bfloat16>(tile);
        case 3: return lt_pair_of<LF_PROD_GRAD_X, __half, __half>(tile);
        case 4: return lt_pair_of<LF_PROD_GRAD_W, __nv_bfloat16, __nv_bfloat16>(tile);
        case 5: return lt_pair_of<LF_PROD_GRAD_W, __half, __half>(tile);
        case 6: return lt_pair_of<LF_PROD_GRAD_W, __nv_bfloat16, float>(tile);
        default: return lt_pair_of<LF_PROD_GRAD_W, __half, float>(tile);
    }
}
lt_kernel lt_pick_pair_split(int i)
{
    switch (i) {
        case 0: return k_product_pair_split<LF_PROD_FORWARD, __nv_bfloat16>;
        case 1: return k_product_pair_split<LF_PROD_FORWARD, __half>;
        case 2: return k_product_pair_split<LF_PROD_GRAD_X, __nv_bfloat16>;
        case 3: return k_product_pair_split<LF_PROD_GRAD_X, __half>;
        case 4: return k_product_pair_split<LF_PROD_GRAD_W, __nv_bfloat16>;
        case 5: return k_product_pair_split<LF_PROD_GRAD_W, __half>;
        default: return nullptr;
    }
}
lt_kernel lt_pick_split(int i, int splits)
{
    switch (i) {
        case 0: return lt_split_of<LF_PROD_FORWARD, __nv_bfloat16, __nv_bfloat16>(splits);
        case 1: return lt_split_of<LF_PROD_FORWARD, __half, __half>(splits);
        case 2: return lt_split_of<LF_PROD_GRAD_X, __nv_bfloat16, __nv_bfloat16>(splits);
        case 3: return lt_split_of<LF_PROD_GRAD_X, __half, __half>(splits);
        case 4: return lt_split_of<LF_PROD_GRAD_W, __nv_bfloat16, __nv_bfloat16>(splits);
        case 5: return lt_split_of<LF_PROD_GRAD_W, __half, __half>(splits);
        case 6: return lt_split_of<LF_PROD_GRAD_W, __nv_bfloat16, float>(splits);
        default: return lt_split_of<LF_PROD_GRAD_W, __half, float>(splits);
    }
}

}  // namespace

int lf_product_tc_init(lf_ops* o)
{
    if (!lt_encode()) return LF_ECUDA;
    o->max_pairs = o->max_pair_splits = -1;
    for (int i = 0; i < LT_KERNELS; ++i) {
        for (int splits = 1; splits <= LT_LONG_SPLITS; splits *= 2)
            if (cudaFuncSetAttribute(lt_pick_split(i, splits), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)LS_SMEM) != cudaSuccess) return LF_ECUDA;
        auto resident = [&](lt_kernel f, int threads, int cluster, size_t smem, int* least) {
            if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return false;
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute at[2];
            lt_cluster_config(&cfg, at, 32, threads, cluster, smem, nullptr);
            int n = 0;
            if (cudaOccupancyMaxActiveClusters(&n, f, &cfg) != cudaSuccess) return false;
            if (*least < 0 || n < *least) *least = n;
            return true;
        };
        if (const lt_kernel f = lt_pick_pair_split(i))
            if (!resident(f, LS_THREADS, 2 * LPS_SPLITS, LPS_SMEM, &o->max_pair_splits)) return LF_ECUDA;
        for (int tile = 0; tile < LT_TILES; ++tile) {
            const lt_kernel f = lt_pick_pair(i, tile);
            if (f && !resident(f, LP_THREADS, 2, LP_SMEM, &o->max_pairs)) return LF_ECUDA;
        }
    }
    return LF_OK;
}

namespace {

struct lt_choice { int splits, tile, width; };      // splits = 0: CTA pairs on `tile`, `width` columns wide; < 0: split pairs; else split tiles

// The form with the least estimated time, in SM cycles; constants measured on B200 (widths 72 .. 16384, 17 .. 8192
// tokens).  A 64-deep stage costs what is most of: its products (a pair: 2 cycles per column and 128-row block of a
// CTA), a multiprocessor's own fetch at 57 bytes a cycle, and all multiprocessors' fetch at 7600 bytes a cycle from
// L2, which is what limits 256 x 256 tiles when all are busy.  Rows that do not begin on a 32-byte sector cost a fetch
// five sectors for four (6998 x 1976 -> 6744: 293,000 cycles, 6998 x 1984 -> 6744: 220,000).  Narrower tiles only pay where
// they fill the last wave better (408 x 4576 -> 12728: 49 us with 512 x 192 tiles, 55 with 256 x 256); their MN-major operand
// comes in boxes of 64 columns per CTA, so they are taken for the forward product.  Switching tiles
// costs 600, but no tile takes less than the epilogue before it, or with 512 rows 4300 and the epilogue, of which little
// runs beside the products there; where the parts of a split tile meet, 1500 and the bytes from the other parts at 14 a
// cycle; the rest is the launch, the first loads and the last epilogue (a split tile's: 128 columns, more warps).
lt_choice lt_choose(const lf_ops* o, const lf_product& p, int n_k)
{
    auto waves = [](long long units, int at_once) { return (double)((units + at_once - 1) / at_once); };
    lt_choice best = {1, 0, 0};
    double least = 1e30;
    auto offer = [&](lt_choice c, double cycles) { if (cycles < least) { least = cycles; best = c; } };
    const long long m128 = (p.M + 127) / 128, m256 = (p.M + 255) / 256, m512 = (p.M + 511) / 512;
    const long long n128 = (p.N + 127) / 128, n256 = (p.N + 255) / 256;
    const double rows = p.M < 128 ? p.M / 128.0 : 1.0;
    auto sectors = [](const void* base, long long ld) { return ((reinterpret_cast<uintptr_t>(base) | (uintptr_t)(2 * ld)) & 31) ? 1.25 : 1.0; };
    const double row_a = 128.0 * sectors(p.a, p.ld_a), row_b = 128.0 * sectors(p.b, p.ld_b);      // a row of a stage, as fetched
    // a stage of `a` rows of A and `b` of B per CTA, `ctas` of them at work
    auto stage = [&](double products, int a, int b, double ctas) {
        const double bytes = a * row_a + b * row_b, own = bytes / 57.0, all = bytes * ctas / 7600.0;
        return products > own ? (products > all ? products : all) : (own > all ? own : all);
    };
    auto busy = [](long long units, int at_once) { return (double)(units < at_once ? units : at_once); };
    // epilogue of 128 rows x 256 columns: as it is, an activation, 8-bit values one way or the other
    const double epilogue = p.q ? 10000.0 : p.prod == LF_PROD_FORWARD && p.act != LF_ACT_NONE ? 7500.0 : 3700.0;
    const int one_fill = lt_one_fill(p);
    for (int splits = 1; splits <= 8 && splits <= n_k; splits *= 2) {
        const double part = (double)((n_k + splits - 1) / splits);
        if (part > one_fill && splits < 8) continue;               // (of more than one fill there are copies of eight parts)
        const double meet = splits > 1 ? 1500.0 + 65536.0 * rows * (splits - 1) / splits / 14.0 : 0.0;
        const int at_once = splits == 8 ? 120 : splits == 4 ? 132 : o->sm_count;      // resident clusters
        const long long ctas = m128 * n128 * splits;
        offer({splits, 0, 0}, waves(ctas, at_once) * (part * stage(256.0, 128, 128, busy(ctas, at_once)) + meet + 6300.0 + 0.86 * epilogue / splits));
    }
    if (o->max_pair_splits > 0 && n_k >= LPS_SPLITS && n_k <= LPS_SPLITS * one_fill && p.out_dtype != LF_F32) {
        const double part = (double)((n_k + LPS_SPLITS - 1) / LPS_SPLITS), meet = 2000.0 + 65536.0 * rows / 14.0;
        const long long tiles = m256 * n256;
        offer({-LPS_SPLITS, 0, 0}, waves(tiles, o->max_pair_splits) *
              (part * stage(512.0, 128, 128, 2.0 * LPS_SPLITS * busy(tiles, o->max_pair_splits)) + meet + 9600.0 + 0.5 * epilogue));
    }
    if (o->max_pairs > 0) {
        for (int width = 256; width >= (p.prod == LF_PROD_FORWARD ? 160 : 256); width -= 32) {
            const long long n = (p.N + width - 1) / width, t256 = m256 * n, t512 = m512 * n;
            const double products = n_k * stage(2.0 * width, 128, width / 2, 2.0 * busy(t256, o->max_pairs));
            offer({0, LT_256x256, width}, products + 600.0 + (waves(t256, o->max_pairs) - 1.0) * ((products > epilogue ? products : epilogue) + 600.0) + 10300.0 + epilogue);
            if (p.out_dtype != LF_F32 && n_k <= one_fill)
                offer({0, LT_512x256, width}, waves(t512, o->max_pairs) *
                      (n_k * stage(4.0 * width, 256, width / 2, 2.0 * busy(t512, o->max_pairs)) + 4300.0 + epilogue) + 14000.0);
        }
    }
    return best;
}

}  // namespace

int lf_product_tc(lf_ops* o, const lf_product& p)
{
    const bool a_mn = p.prod == LF_PROD_GRAD_W, b_mn = p.prod != LF_PROD_FORWARD;
    const CUtensorMapDataType in_type = p.dtype == LF_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const bool out32 = p.out_dtype == LF_F32;
    const int kernel = (out32 ? 6 : p.prod * 2) + (p.dtype == LF_F16 ? 1 : 0);

    LtParams P = {};
    P.M = p.M; P.N = p.N; P.K = p.K;
    P.act = p.act;
    P.bias = p.bias; P.add = p.add; P.ld_add = p.ld_add;
    P.d = p.d; P.ld_d = p.ld_d;
    P.q = p.q; P.s = p.s;
    P.wide_q = (p.N & 31) == 0 && (reinterpret_cast<uintptr_t>(p.q) & 31) == 0;
    P.wide_s = (p.N & 127) == 0 && (reinterpret_cast<uintptr_t>(p.s) & 3) == 0;
    P.wide_add = (p.ld_add & 15) == 0 && (reinterpret_cast<uintptr_t>(p.add) & 31) == 0;
    P.status = o->status_dev;
    P.budget_ns = (unsigned long long)o->wait_budget_us * 1000ull;
    P.withhold = o->withhold;
    unsigned idesc = 1u << 4;                                       // fp32 accumulator
    if (p.dtype == LF_BF16) idesc |= (1u << 7) | (1u << 10);        // A and B: bf16 (f16: 0)
    if (a_mn) idesc |= 1u << 15;
    if (b_mn) idesc |= 1u << 16;

    const int n_k = (p.K + LT_BK - 1) / LT_BK;
    const lt_choice c = lt_choose(o, p, n_k);
    const int one_fill = lt_one_fill(p);
    alignas(64) CUtensorMap map_a, map_b;
    const bool ok = (a_mn ? lt_map(&map_a, in_type, p.a, p.K, p.M, p.ld_a, 64, 64) : lt_map(&map_a, in_type, p.a, p.M, p.K, p.ld_a, 64, 128)) &&
                    (b_mn ? lt_map(&map_b, in_type, p.b, p.K, p.N, p.ld_b, 64, 64) : lt_map(&map_b, in_type, p.b, p.N, p.K, p.ld_b, 64, c.splits == 0 ? c.width / 2 : 128));
    if (!ok) { o->last_cuda_error = (int)cudaErrorInvalidValue; return LF_ECUDA; }

    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute at[2];
    if (c.splits < 0) {
        P.tiles_m = (p.M + 255) / 256; P.tiles_n = (p.N + 255) / 256;
        P.idesc = idesc | (256u >> 3) << 17 | (256u >> 4) << 24;
        P.stages_per_split = (n_k + LPS_SPLITS - 1) / LPS_SPLITS;
        lt_cluster_config(&cfg, at, P.tiles_m * P.tiles_n * 2 * LPS_SPLITS, LS_THREADS, 2 * LPS_SPLITS, LPS_SMEM, o->stream);
        LF_OPS_TRY(o, cudaLaunchKernelEx(&cfg, lt_pick_pair_split(kernel), map_a, map_b, P));
        o->stats.form = LF_FORM_SPLIT_PAIRS;
        o->stats.splits = LPS_SPLITS;
    } else if (c.splits == 0) {
        const int bm = c.tile == LT_512x256 ? 512 : 256;
        P.width = c.width;
        P.tiles_m = (p.M + bm - 1) / bm; P.tiles_n = (p.N + c.width - 1) / c.width;
        P.idesc = idesc | ((unsigned)c.width >> 3) << 17 | (256u >> 4) << 24;
        P.band = 2048 / bm;
        const int tiles = P.tiles_m * P.tiles_n, pairs = tiles < o->max_pairs ? tiles : o->max_pairs;
        lt_cluster_config(&cfg, at, 2 * pairs, LP_THREADS, 2, LP_SMEM, o->stream);
        LF_OPS_TRY(o, cudaLaunchKernelEx(&cfg, lt_pick_pair(kernel, c.tile == LT_256x256 && n_k > one_fill ? LT_256x256_LONG : c.tile), map_a, map_b, P));
        o->stats.form = LF_FORM_PAIRS;
        o->stats.splits = 1;
    } else {
        P.tiles_m = (p.M + 127) / 128; P.tiles_n = (p.N + 127) / 128;
        P.idesc = idesc | (128u >> 3) << 17 | (128u >> 4) << 24;
        P.stages_per_split = (n_k + c.splits - 1) / c.splits;
        lt_cluster_config(&cfg, at, P.tiles_m * P.tiles_n * c.splits, LS_THREADS, c.splits, LS_SMEM, o->stream);
        LF_OPS_TRY(o, cudaLaunchKernelEx(&cfg, lt_pick_split(kernel, P.stages_per_split > one_fill ? LT_LONG_SPLITS : c.splits), map_a, map_b, P));
        o->stats.form = LF_FORM_SPLIT;
        o->stats.splits = c.splits;
    }
    o->stats.launches += 1;
    return LF_OK;
}

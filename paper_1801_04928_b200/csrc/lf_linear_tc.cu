// The dense layer's three products in 16 bits on the 5th-generation tensor cores:
//     D[m][n] = sum_k A[m][k] B[n][k],   fp32 accumulators, epilogue on D
//   forward  A = x  [tokens][n_in],  B = w  [n_out][n_in]:  y = sigma(D + bias) + residual, z in 8 bits
//   grad_x   A = dz [tokens][n_out], B = w^T (w read MN-major): dx = D (.) sigma'(z from 8 bits) + add
//   grad_w   A = dz^T, B = x^T (both MN-major, the contraction runs over tokens):  gw = D
// Every operand is used where it lies; what differs is the box TMA fetches and the descriptor's
// majorness.  A K stage is 64 deep; a CTA fetches a 128 x 64 block of A and one of B (16 KiB each, 128-byte
// swizzle) per stage, six stages in flight.
//
// Two forms.  CTA pairs (k_product_pair): tcgen05.mma.cta_group::2 on 256 x 256 tiles, each CTA fetching half
// of both operands, so a stage of 512 tensor-core cycles needs 32 KiB per CTA; persistent, two
// accumulators in tensor memory, so the epilogue of a tile runs under the next tile's products.  Split tiles
// (k_product_split): one CTA per 128 x 128 tile and part of the contraction; the CTAs of a tile form
// a cluster and add their parts through distributed shared memory, each finishing its share of the rows.
// The first form needs the fewest operand bytes per product, the second fills the device when
// there are few tiles.
//
// The tensor core adds into its accumulator by truncation.  Results that are rounded to 16 bits do not see
// it; an fp32 weight gradient over thousands of tokens would (about 1e-5 relative after 512
// instructions), so there an accumulator only takes CHUNK stages (32 instructions) and the chunks are added in
// registers with round-to-nearest.
// All waits are bounded; on expiry the status word is raised and the launch drains and ends.
#include "lf_ops_internal.h"
#include "lf_ptx.cuh"
#include "lf_rows.cuh"

namespace {

using namespace lfrow;

constexpr int LT_BK = 64;
constexpr int LT_BLOCK_BYTES = 128 * LT_BK * 2;          // 16 KiB: 128 rows (or columns) x 64 contraction steps
constexpr int LT_STAGE_BYTES = 2 * LT_BLOCK_BYTES;
constexpr int LT_STAGES = 6;
constexpr int LT_THREADS = 320;                          // producer, issuer, eight epilogue warps
constexpr int LT_CHUNK = 8;                              // K stages per accumulator of an fp32 result
constexpr int LP_EPI_BYTES = 8 * 4096;                   // pairs: 32 rows x 128 bytes per epilogue warp
constexpr int LS_LD = 132;                               // split tiles: padded row of the fp32 tile in shared memory
constexpr size_t LP_SMEM = (size_t)LT_STAGES * LT_STAGE_BYTES + LP_EPI_BYTES + 1024 + 512;
constexpr size_t LS_SMEM = (size_t)LT_STAGES * LT_STAGE_BYTES + 1024 + 512;
static_assert(128 * LS_LD * 4 <= LT_STAGES * LT_STAGE_BYTES, "the fp32 tile overlays the operand ring");

struct LtParams {
    int M, N, K;
    int tiles_m, tiles_n;
    int splits, stages_per_split;      // split tiles
    int act;
    unsigned idesc;
    const float* bias;
    const void* add; long long ld_add;
    void* d; long long ld_d;
    unsigned char *q, *s;
    unsigned* status;
    unsigned long long budget_ns;
    int withhold;
};

struct LtShared {
    unsigned long long full[LT_STAGES];
    unsigned long long empty[LT_STAGES];
    unsigned long long acc_full[2];
    unsigned long long acc_empty[2];
    unsigned tmem_base;
    volatile unsigned abort_flag;
    unsigned prog_it;                  // stage loads this CTA's producer has issued
};
static_assert(sizeof(LtShared) <= 512, "the barrier block must fit into the space reserved for it");

// Bounded wait (acquire at cluster scope: the peer's arrivals count too); false once this CTA has given up.
__device__ __forceinline__ bool lt_wait(unsigned bar, unsigned parity, const LtParams& P, LtShared* sh)
{
    if (lfptx::mbar_try_wait_cluster(bar, parity)) return true;
    if (sh->abort_flag) return false;
    const unsigned long long t0 = lfptx::globaltimer_ns();
    unsigned spins = 0;
    while (!lfptx::mbar_try_wait_cluster(bar, parity)) {
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

// One operand block of a stage: `mn` the first row/column, `k` the first contraction step.
template <bool MN, bool PAIR>
__device__ __forceinline__ void lt_load(unsigned dst, const CUtensorMap* map, unsigned bar, int mn, int k)
{
    if (MN) {
        if (PAIR) {
            lfptx::tma_load_2d_pair(dst, map, bar, mn, k);
            lfptx::tma_load_2d_pair(dst + 8192, map, bar, mn + 64, k);
        } else {
            lfptx::tma_load_2d(dst, map, bar, mn, k);
            lfptx::tma_load_2d(dst + 8192, map, bar, mn + 64, k);
        }
    } else {
        if (PAIR) lfptx::tma_load_2d_pair(dst, map, bar, k, mn);
        else lfptx::tma_load_2d(dst, map, bar, k, mn);
    }
}

// ---- epilogue on eight columns of one row -----------------------------------------------------------
// FORWARD, first half: z = D + bias (in place)
__device__ __forceinline__ void epi_bias8(float (&v)[8], const LtParams& P, int col)
{
    if (!P.bias) return;
    float b[8];
    vec8<float> bv;
    bv.load(P.bias + col);
    bv.get(b);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += b[k];
}
template <typename T>
__device__ __forceinline__ void epi_add8(float (&v)[8], const LtParams& P, int row, int col)
{
    if (!P.add) return;
    float r[8];
    vec8<T> rv;
    rv.load(static_cast<const T*>(P.add) + (size_t)row * P.ld_add + col);
    rv.get(r);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += r[k];
}
__device__ __forceinline__ void epi_act8(float (&v)[8], int kind)
{
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = act<true>(v[k], kind);
}
__device__ __forceinline__ void epi_prime8(float (&v)[8], uint2 q, unsigned byte, int kind)
{
    float z[8];
    dequantize8(q, byte, z);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= act_prime<true>(z[k], kind);
}

// ================================================================================================
// CTA pairs, 256 x 256 tiles
// ================================================================================================
// tile of a persistent schedule: bands of eight row blocks, column by column inside a band, so that the
// tiles worked on at one time share both operands in L2
__device__ __forceinline__ void lp_tile(int t, const LtParams& P, int& tm, int& tn)
{
    const int per_band = 8 * P.tiles_n, band = t / per_band, in = t - band * per_band;
    const int rows = min(8, P.tiles_m - band * 8);
    tn = in / rows;
    tm = band * 8 + (in - tn * rows);
}

template <int PROD, typename T, typename OUT>
__global__ void __launch_bounds__(LT_THREADS, 1)
k_product_pair(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ CUtensorMap map_d, const LtParams P)
{
    constexpr bool A_MN = PROD == LF_PROD_GRAD_W, B_MN = PROD != LF_PROD_FORWARD;
    constexpr bool PROMOTE = sizeof(OUT) == 4;
    extern __shared__ unsigned char lt_smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(lt_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    unsigned char* epi = ring + (size_t)LT_STAGES * LT_STAGE_BYTES;
    LtShared* sh = reinterpret_cast<LtShared*>(epi + LP_EPI_BYTES);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned rank = lfptx::cluster_ctarank();
    const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const int n_tiles = P.tiles_m * P.tiles_n;
    const int n_k = (P.K + LT_BK - 1) / LT_BK;
    const int chunk = PROMOTE ? LT_CHUNK : n_k;

    if (threadIdx.x == 0) {
        for (int i = 0; i < LT_STAGES; ++i) {
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

    if (warp == 0) {
        // ------------------------------ TMA producer: this CTA's halves -------------------------
        if (lane == 0) {
            unsigned it = 0;
            bool ok = true;
            for (int t = pair; t < n_tiles && ok; t += n_pairs) {
                int tm, tn;
                lp_tile(t, P, tm, tn);
                const int m0 = tm * 256 + (int)rank * 128, n0 = tn * 256 + (int)rank * 128;
                for (int ks = 0; ks < n_k; ++ks, ++it) {
                    const unsigned st = it % LT_STAGES, use = it / LT_STAGES;
                    if (use > 0 && !lt_wait(lfptx::smem_u32(&sh->empty[st]), (use - 1) & 1u, P, sh)) { ok = false; break; }
                    const unsigned lbar = lfptx::smem_u32(&sh->full[st]);
                    if (P.withhold && pair == 0 && rank == 1 && it == 0) continue;    // test hook
                    if (rank == 0) lfptx::mbar_arrive_expect_tx(lbar, 2u * LT_STAGE_BYTES);
                    const unsigned bar = lfptx::map_to_cta(lbar, 0);
                    const unsigned dst = lfptx::smem_u32(ring + (size_t)st * LT_STAGE_BYTES);
                    lt_load<A_MN, true>(dst, &map_a, bar, m0, ks * LT_BK);
                    lt_load<B_MN, true>(dst + LT_BLOCK_BYTES, &map_b, bar, n0, ks * LT_BK);
                }
            }
            sh->prog_it = it;
        }
    } else if (warp == 1) {
        // ------------------------------ MMA issuer (leader CTA) ---------------------------------
        if (lane == 0 && rank == 0) {
            unsigned it = 0, c = 0;             // c counts accumulator fills
            bool ok = true;
            for (int t = pair; t < n_tiles && ok; t += n_pairs) {
                for (int k0 = 0; k0 < n_k && ok; k0 += chunk, ++c) {
                    const unsigned ab = c & 1u, ab_use = c >> 1;
                    if (ab_use > 0 && !lt_wait(lfptx::smem_u32(&sh->acc_empty[ab]), (ab_use - 1) & 1u, P, sh)) { ok = false; break; }
                    lfptx::tc_fence_after();
                    const unsigned d_tmem = tmem_base + ab * 256u;
                    const int k1 = min(k0 + chunk, n_k);
                    for (int ks = k0; ks < k1; ++ks, ++it) {
                        const unsigned st = it % LT_STAGES, use = it / LT_STAGES;
                        if (!lt_wait(lfptx::smem_u32(&sh->full[st]), use & 1u, P, sh)) { ok = false; break; }
                        lfptx::tc_fence_after();
                        const unsigned a_addr = lfptx::smem_u32(ring + (size_t)st * LT_STAGE_BYTES);
                        const unsigned b_addr = a_addr + LT_BLOCK_BYTES;
#pragma unroll
                        for (int kk = 0; kk < LT_BK / 16; ++kk)
                            lt_mma<true>(d_tmem, lt_desc<A_MN>(a_addr + lt_step<A_MN>(kk)), lt_desc<B_MN>(b_addr + lt_step<B_MN>(kk)),
                                         P.idesc, (ks > k0 || kk > 0) ? 1u : 0u);
                        lt_commit<true>(lfptx::smem_u32(&sh->empty[st]));
                    }
                    if (ok) lt_commit<true>(lfptx::smem_u32(&sh->acc_full[ab]));
                }
            }
        }
    } else {
        // ------------------------------ epilogue (warps 2..9 of both CTAs) ----------------------
        // A warp has one 32-lane quadrant (32 rows) and one half (128 columns) of the tile; a lane has a
        // row.  Results leave through a 32 x 128-byte block in shared memory and a TMA store, which
        // clips ragged edges.
        const int quad = warp & 3, half = (warp - 2) >> 2;
        const unsigned leader_acc_empty = lfptx::map_to_cta(lfptx::smem_u32(&sh->acc_empty[0]), 0);
        unsigned char* blk = epi + (warp - 2) * 4096;
        const unsigned blk_addr = lfptx::smem_u32(blk);
        constexpr int OC = 128 / (int)sizeof(OUT);             // columns of a stored block: 64 or 32
        unsigned c = 0;
        bool ok = true;
        for (int t = pair; t < n_tiles && ok; t += n_pairs) {
            int tm, tn;
            lp_tile(t, P, tm, tn);
            const int row0 = tm * 256 + (int)rank * 128 + quad * 32, row = row0 + lane;
            const int col0 = tn * 256 + half * 128;
            const unsigned lane_addr = tmem_base + ((unsigned)(quad * 32) << 16) + half * 128u;
            float acc[PROMOTE ? 128 : 1];
            if (PROMOTE) {
#pragma unroll
                for (int i = 0; i < 128; ++i) acc[(PROMOTE ? i : 0)] = 0.f;
                for (int k0 = 0; k0 < n_k; k0 += chunk, ++c) {
                    const unsigned ab = c & 1u;
                    if (!lt_wait(lfptx::smem_u32(&sh->acc_full[ab]), (c >> 1) & 1u, P, sh)) { ok = false; break; }
                    lfptx::tc_fence_after();
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        unsigned r[16];
                        lfptx::tmem_ld16(lane_addr + ab * 256u + j * 16, r);
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[(PROMOTE ? j * 16 + i : 0)] += __uint_as_float(r[i]);
                    }
                    lfptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) lt_arrive_cluster(leader_acc_empty + ab * 8u);
                }
                if (!ok) break;
            } else {
                if (!lt_wait(lfptx::smem_u32(&sh->acc_full[c & 1u]), (c >> 1) & 1u, P, sh)) break;
                lfptx::tc_fence_after();
            }
#pragma unroll (PROMOTE ? 4 : 1)
            for (int j = 0; j < 128 / OC; ++j) {
                const int colj = col0 + j * OC;
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");   // blk is free again
                __syncwarp();
#pragma unroll
                for (int h = 0; h < OC / 32; ++h) {            // 32 columns at a time
                    const int col = colj + h * 32;
                    float v[32];
                    if (PROMOTE) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = acc[(PROMOTE ? j * 32 + i : 0)];
                    } else {
                        unsigned r[32];
                        lfptx::tmem_ld32(lane_addr + (c & 1u) * 256u + j * OC + h * 32, r);
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
                    }
                    const int valid = row < P.M ? min(32, P.N - col) : 0;    // a multiple of 8
                    if (PROD == LF_PROD_FORWARD) {
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            if (col + 8 * g < P.N) epi_bias8(*reinterpret_cast<float(*)[8]>(v + 8 * g), P, col + 8 * g);
                        if (P.q && valid > 0) {
                            unsigned m = 0;
#pragma unroll
                            for (int i = 0; i < 32; ++i) if (i < valid) m = max(m, abs_bits(v[i]));
                            const unsigned b = scale_byte(m);
                            unsigned char* qp = P.q + (size_t)row * P.N + col;
#pragma unroll
                            for (int g = 0; g < 4; ++g)
                                if (8 * g < valid)
                                    *reinterpret_cast<uint2*>(qp + 8 * g) = quantize8(*reinterpret_cast<float(*)[8]>(v + 8 * g), b);
                            P.s[(size_t)row * ((P.N + 31) / 32) + (col >> 5)] = (unsigned char)b;
                        }
                    }
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        float(&w)[8] = *reinterpret_cast<float(*)[8]>(v + 8 * g);
                        if (PROD == LF_PROD_FORWARD) epi_act8(w, P.act);
                        if (PROD == LF_PROD_GRAD_X && P.q && 8 * g < valid)
                            epi_prime8(w, *reinterpret_cast<const uint2*>(P.q + (size_t)row * P.N + col + 8 * g),
                                       P.s[(size_t)row * ((P.N + 31) / 32) + (col >> 5)], P.act);
                        if (PROD != LF_PROD_GRAD_W && 8 * g < valid) epi_add8<T>(w, P, row, col + 8 * g);
                        // 16-byte units of a 128-byte line, turned as the 128-byte swizzle has them
                        if (sizeof(OUT) == 2) {
                            vec8<T> o;
                            o.set(w);
                            const int unit = h * 4 + g;
                            *reinterpret_cast<uint4*>(blk + lane * 128 + ((unit ^ (lane & 7)) << 4)) = o.u;
                        } else {
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                const int unit = g * 2 + u;
                                *reinterpret_cast<float4*>(blk + lane * 128 + ((unit ^ (lane & 7)) << 4)) =
                                    make_float4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
                            }
                        }
                    }
                }
                if (!PROMOTE && j == 128 / OC - 1) {           // the accumulator has been read
                    lfptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) lt_arrive_cluster(leader_acc_empty + (c & 1u) * 8u);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    if (row0 < P.M && colj < P.N)
                        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                                     ::"l"(&map_d), "r"(blk_addr), "r"(colj), "r"(row0) : "memory");
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
            }
            if (!PROMOTE) ++c;
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
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
                const unsigned bar = lfptx::smem_u32(&sh->full[j % LT_STAGES]);
                if (j >= it_l) lfptx::mbar_arrive_expect_tx(bar, (unsigned)LT_STAGE_BYTES);   // only the peer loaded
                else lt_complete_tx(bar, (unsigned)LT_STAGE_BYTES);                           // only the leader loaded
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
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

// ================================================================================================
// Split tiles: one CTA per 128 x 128 tile and part of the contraction, a cluster per tile
// ================================================================================================
template <int PROD, typename T, typename OUT>
__global__ void __launch_bounds__(LT_THREADS, 1)
k_product_split(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const LtParams P)
{
    constexpr bool A_MN = PROD == LF_PROD_GRAD_W, B_MN = PROD != LF_PROD_FORWARD;
    constexpr bool PROMOTE = sizeof(OUT) == 4;
    extern __shared__ unsigned char lt_smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(lt_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    LtShared* sh = reinterpret_cast<LtShared*>(ring + (size_t)LT_STAGES * LT_STAGE_BYTES);
    float* tile = reinterpret_cast<float*>(ring);            // [128][LS_LD], once every product is done

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = (int)(blockIdx.x % (unsigned)P.splits), t = (int)(blockIdx.x / (unsigned)P.splits);
    const int tn = t / P.tiles_m, tm = t - tn * P.tiles_m;
    const int n_k_all = (P.K + LT_BK - 1) / LT_BK;
    const int ks0 = part * P.stages_per_split;
    const int n_k = max(0, min(P.stages_per_split, n_k_all - ks0));
    const int chunk = PROMOTE ? LT_CHUNK : (n_k > 0 ? n_k : 1);

    if (threadIdx.x == 0) {
        for (int i = 0; i < LT_STAGES; ++i) {
            lfptx::mbar_init(lfptx::smem_u32(&sh->full[i]), 1);
            lfptx::mbar_init(lfptx::smem_u32(&sh->empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            lfptx::mbar_init(lfptx::smem_u32(&sh->acc_full[i]), 1);
            lfptx::mbar_init(lfptx::smem_u32(&sh->acc_empty[i]), 8);
        }
        sh->abort_flag = 0u;
        lfptx::mbar_fence_init();
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

    float acc[64];
    if (warp == 0) {
        if (lane == 0) {
            unsigned it = 0;
            for (int ks = 0; ks < n_k; ++ks, ++it) {
                const unsigned st = it % LT_STAGES, use = it / LT_STAGES;
                if (use > 0 && !lt_wait(lfptx::smem_u32(&sh->empty[st]), (use - 1) & 1u, P, sh)) break;
                const unsigned bar = lfptx::smem_u32(&sh->full[st]);
                lfptx::mbar_arrive_expect_tx(bar, LT_STAGE_BYTES);
                if (P.withhold && blockIdx.x == 0 && it == 0) continue;              // test hook
                const unsigned dst = lfptx::smem_u32(ring + (size_t)st * LT_STAGE_BYTES);
                lt_load<A_MN, false>(dst, &map_a, bar, tm * 128, (ks0 + ks) * LT_BK);
                lt_load<B_MN, false>(dst + LT_BLOCK_BYTES, &map_b, bar, tn * 128, (ks0 + ks) * LT_BK);
            }
            // after giving up: do not let the CTA go on under loads that are still landing
            if (sh->abort_flag) {
                const unsigned long long t0 = lfptx::globaltimer_ns();
                for (unsigned j = it > LT_STAGES ? it - LT_STAGES : 0; j < it; ++j)
                    while (!lfptx::mbar_try_wait(lfptx::smem_u32(&sh->full[j % LT_STAGES]), (j / LT_STAGES) & 1u) &&
                           lfptx::globaltimer_ns() - t0 < 50000000ull) { }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            unsigned it = 0, c = 0;
            bool ok = true;
            for (int k0 = 0; k0 < n_k && ok; k0 += chunk, ++c) {
                const unsigned ab = c & 1u, ab_use = c >> 1;
                if (ab_use > 0 && !lt_wait(lfptx::smem_u32(&sh->acc_empty[ab]), (ab_use - 1) & 1u, P, sh)) break;
                lfptx::tc_fence_after();
                const int k1 = min(k0 + chunk, n_k);
                for (int ks = k0; ks < k1; ++ks, ++it) {
                    const unsigned st = it % LT_STAGES, use = it / LT_STAGES;
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
    } else {
        const int quad = warp & 3, half = (warp - 2) >> 2;
#pragma unroll
        for (int i = 0; i < 64; ++i) acc[i] = 0.f;
        unsigned c = 0;
        for (int k0 = 0; k0 < n_k; k0 += chunk, ++c) {
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
        // every product of this CTA is done (the last accumulator was complete), so the ring is free
        if (!sh->abort_flag) {
            float* to = tile + (quad * 32 + lane) * LS_LD + half * 64;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                *reinterpret_cast<float4*>(to + 4 * i) = make_float4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]);
        }
    }
    lfptx::tc_fence_before();
    __syncthreads();
    if (P.splits > 1) lfptx::cluster_sync_all();
    if (warp >= 2 && !sh->abort_flag) {
        // this CTA finishes 128 / splits rows; a lane takes eight columns, half a warp a row
        const int tid = threadIdx.x - 64;
        const int rows = 128 / P.splits;
        const unsigned tile_addr = lfptx::smem_u32(tile);
        for (int u = tid; u < rows * 16; u += 256) {           // (a multiple of 256: whole warps)
            const int r = part * rows + (u >> 4), cv = (u & 15) * 8;
            const int row = tm * 128 + r, col = tn * 128 + cv;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.f;
            const unsigned at = tile_addr + (unsigned)(r * LS_LD + cv) * 4u;
            for (int p = 0; p < P.splits; ++p) {               // parts in order: the sum does not depend on timing
                const unsigned from = P.splits > 1 ? lfptx::map_to_cta(at, (unsigned)p) : at;
                const float4 x = lt_ld_cluster_f4(from), y = lt_ld_cluster_f4(from + 16);
                v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
                v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
            }
            const bool in = row < P.M && col < P.N;
            if (PROD == LF_PROD_FORWARD) {
                if (in) epi_bias8(v, P, col);
                if (P.q) {
                    float z[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) z[k] = in ? v[k] : 0.f;
                    const unsigned b = group_byte(z);
                    if (in) {
                        *reinterpret_cast<uint2*>(P.q + (size_t)row * P.N + col) = quantize8(z, b);
                        if ((col & 31) == 0) P.s[(size_t)row * ((P.N + 31) / 32) + (col >> 5)] = (unsigned char)b;
                    }
                }
                epi_act8(v, P.act);
            }
            if (!in) continue;
            if (PROD == LF_PROD_GRAD_X && P.q)
                epi_prime8(v, *reinterpret_cast<const uint2*>(P.q + (size_t)row * P.N + col),
                           P.s[(size_t)row * ((P.N + 31) / 32) + (col >> 5)], P.act);
            if (PROD != LF_PROD_GRAD_W) epi_add8<T>(v, P, row, col);
            vec8<OUT> o;
            o.set(v);
            o.store(static_cast<OUT*>(P.d) + (size_t)row * P.ld_d + col);
        }
    }
    if (P.splits > 1) lfptx::cluster_sync_all();               // the other parts have read this CTA's tile
    else __syncthreads();
    if (warp == 1) {
        lfptx::tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(256u) : "memory");
    }
}

lf_encode_fn lt_encode()
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
bool lt_map(CUtensorMap* m, CUtensorMapDataType type, int esize, const void* base, int rows, int cols, long long ld, int bc, int br)
{
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * (cuuint64_t)esize};
    cuuint32_t box[2] = {(cuuint32_t)bc, (cuuint32_t)br};
    cuuint32_t estr[2] = {1, 1};
    return lt_encode()(m, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

typedef void (*lt_pair_kernel)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const LtParams);
typedef void (*lt_split_kernel)(const CUtensorMap, const CUtensorMap, const LtParams);

template <int PROD, typename T, typename OUT>
struct lt_kernels {
    static lt_pair_kernel pair() { return k_product_pair<PROD, T, OUT>; }
    static lt_split_kernel split() { return k_product_split<PROD, T, OUT>; }
};

// kernel of a product; index = prod * 2 + (f16), 6 and 7: grad_w with an fp32 result
lt_pair_kernel lt_pick_pair(int i)
{
    switch (i) {
        case 0: return lt_kernels<LF_PROD_FORWARD, __nv_bfloat16, __nv_bfloat16>::pair();
        case 1: return lt_kernels<LF_PROD_FORWARD, __half, __half>::pair();
        case 2: return lt_kernels<LF_PROD_GRAD_X, __nv_bfloat16, __nv_bfloat16>::pair();
        case 3: return lt_kernels<LF_PROD_GRAD_X, __half, __half>::pair();
        case 4: return lt_kernels<LF_PROD_GRAD_W, __nv_bfloat16, __nv_bfloat16>::pair();
        case 5: return lt_kernels<LF_PROD_GRAD_W, __half, __half>::pair();
        case 6: return lt_kernels<LF_PROD_GRAD_W, __nv_bfloat16, float>::pair();
        default: return lt_kernels<LF_PROD_GRAD_W, __half, float>::pair();
    }
}
lt_split_kernel lt_pick_split(int i)
{
    switch (i) {
        case 0: return lt_kernels<LF_PROD_FORWARD, __nv_bfloat16, __nv_bfloat16>::split();
        case 1: return lt_kernels<LF_PROD_FORWARD, __half, __half>::split();
        case 2: return lt_kernels<LF_PROD_GRAD_X, __nv_bfloat16, __nv_bfloat16>::split();
        case 3: return lt_kernels<LF_PROD_GRAD_X, __half, __half>::split();
        case 4: return lt_kernels<LF_PROD_GRAD_W, __nv_bfloat16, __nv_bfloat16>::split();
        case 5: return lt_kernels<LF_PROD_GRAD_W, __half, __half>::split();
        case 6: return lt_kernels<LF_PROD_GRAD_W, __nv_bfloat16, float>::split();
        default: return lt_kernels<LF_PROD_GRAD_W, __half, float>::split();
    }
}

void lt_cluster_config(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* at, int grid, int cluster, size_t smem, cudaStream_t s)
{
    *cfg = cudaLaunchConfig_t{};
    cfg->gridDim = dim3((unsigned)grid);
    cfg->blockDim = dim3(LT_THREADS);
    cfg->dynamicSmemBytes = smem;
    cfg->stream = s;
    at->id = cudaLaunchAttributeClusterDimension;
    at->val.clusterDim.x = (unsigned)cluster;
    at->val.clusterDim.y = 1;
    at->val.clusterDim.z = 1;
    cfg->attrs = at;
    cfg->numAttrs = 1;
}

}  // namespace

int lf_product_tc_init(lf_ops* o)
{
    if (!lt_encode()) return LF_ECUDA;
    o->max_pairs = 0;
    for (int i = 0; i < 8; ++i) {
        if (cudaFuncSetAttribute(lt_pick_pair(i), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)LP_SMEM) != cudaSuccess ||
            cudaFuncSetAttribute(lt_pick_split(i), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)LS_SMEM) != cudaSuccess)
            return LF_ECUDA;
        cudaLaunchConfig_t cfg;
        cudaLaunchAttribute at[1];
        lt_cluster_config(&cfg, at, 32, 2, LP_SMEM, nullptr);
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, lt_pick_pair(i), &cfg) != cudaSuccess) return LF_ECUDA;
        if (i == 0 || n < o->max_pairs) o->max_pairs = n;
    }
    return LF_OK;
}

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
    P.status = o->status_dev;
    P.budget_ns = (unsigned long long)o->wait_budget_us * 1000ull;
    P.withhold = o->withhold;
    unsigned idesc = 1u << 4;                                       // fp32 accumulator
    if (p.dtype == LF_BF16) idesc |= (1u << 7) | (1u << 10);        // A and B: bf16 (f16: 0)
    if (a_mn) idesc |= 1u << 15;
    if (b_mn) idesc |= 1u << 16;

    alignas(64) CUtensorMap map_a, map_b, map_d;
    bool ok = a_mn ? lt_map(&map_a, in_type, 2, p.a, p.K, p.M, p.ld_a, 64, 64) : lt_map(&map_a, in_type, 2, p.a, p.M, p.K, p.ld_a, 64, 128);
    ok = ok && (b_mn ? lt_map(&map_b, in_type, 2, p.b, p.K, p.N, p.ld_b, 64, 64) : lt_map(&map_b, in_type, 2, p.b, p.N, p.K, p.ld_b, 64, 128));

    const int n_k = (p.K + LT_BK - 1) / LT_BK;
    const long long pair_tiles = (long long)((p.M + 255) / 256) * ((p.N + 255) / 256);
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute at[1];
    if (o->max_pairs > 0 && pair_tiles * 2 >= o->max_pairs) {
        P.tiles_m = (p.M + 255) / 256; P.tiles_n = (p.N + 255) / 256;
        P.idesc = idesc | (256u >> 3) << 17 | (256u >> 4) << 24;
        ok = ok && (out32 ? lt_map(&map_d, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, p.d, p.M, p.N, p.ld_d, 32, 32)
                          : lt_map(&map_d, in_type, 2, p.d, p.M, p.N, p.ld_d, 64, 32));
        if (!ok) { o->last_cuda_error = (int)cudaErrorInvalidValue; return LF_ECUDA; }
        const int pairs = pair_tiles < o->max_pairs ? (int)pair_tiles : o->max_pairs;
        lt_cluster_config(&cfg, at, 2 * pairs, 2, LP_SMEM, o->stream);
        LF_OPS_TRY(o, cudaLaunchKernelEx(&cfg, lt_pick_pair(kernel), map_a, map_b, map_d, P));
        o->stats.form = LF_FORM_PAIRS;
        o->stats.splits = 1;
    } else {
        if (!ok) { o->last_cuda_error = (int)cudaErrorInvalidValue; return LF_ECUDA; }
        P.tiles_m = (p.M + 127) / 128; P.tiles_n = (p.N + 127) / 128;
        P.idesc = idesc | (128u >> 3) << 17 | (128u >> 4) << 24;
        const long long tiles = (long long)P.tiles_m * P.tiles_n;
        int splits = 1;
        while (splits < 8 && tiles * splits * 2 <= o->sm_count && n_k >= splits * 4) splits *= 2;
        P.splits = splits;
        P.stages_per_split = (n_k + splits - 1) / splits;
        lt_cluster_config(&cfg, at, (int)(tiles * splits), splits, LS_SMEM, o->stream);
        LF_OPS_TRY(o, cudaLaunchKernelEx(&cfg, lt_pick_split(kernel), map_a, map_b, P));
        o->stats.form = LF_FORM_SPLIT;
        o->stats.splits = splits;
    }
    o->stats.launches += 1;
    return LF_OK;
}

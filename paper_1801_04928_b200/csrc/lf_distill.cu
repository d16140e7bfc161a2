// The loss of a network against a teacher's top logits, and its gradient:
//     loss = w T^2 sum_k p_k (ln p_k - ln q_{i_k}),   dz_v = w T (q_v - sum of p_k with i_k = v)
// with p the softmax of the teacher's entries and q the softmax of the whole row of logits, both at temperature T.
//
// Mathematics: with m and t_m the largest logit and entry, S and P the sums of e^((z - m) / T) and e^((t - t_m) / T),
//     sum_k p_k (ln p_k - ln q_{i_k}) = sum_k p_k ((t_k - t_m) - (z_{i_k} - m)) / T + ln S - ln P,
// so the loss needs of a row only m and S, taken together in one pass with S rescaled where m grows, and the picked
// logits.  Differences come first throughout, so a row of nothing but a type's lowest number is a uniform softmax.  What there is
// one of per row is in 64 bits.
//
// Bound by memory: the loss reads a row once, the gradient reads it and writes one.  A row is cut into parts, a block
// each, which are a cluster and meet once, over distributed shared memory, with their m and s.  Where the gradient is
// written too, a part keeps what it has read in shared memory, so that the row is read from memory once.
// The teacher's entries and the loss are one warp's work, beside the others' passes over the row; the dense part of the gradient is
// written first, then the entries that fall into the part are put right.  Measured, bf16: loss alone 8192 x 131072 331 us, 6.49 TB/s; gradient
// alone 8192 x 32768 170 us, 6.3; both at once 8192 x 131072 with 64 entries a token 815 to 857 us in a row by the card, 5.0 to 5.27 TB/s, up to 885 among other work.
#include <algorithm>

#include <math_constants.h>

#include "lf_ops_internal.h"
#include "lf_ptx.cuh"
#include "lf_rows.cuh"

namespace {

using namespace lfrow;

// Threads for a row (RT in what follows): 256, or 64 where rows are short; beside them a warp for the teacher's entries and the loss.
constexpr int DT_LONG = 256, DT_SHORT = 64;
constexpr int DT_TABLE_LOG2 = 10, DT_TABLE_ROUNDS = 12;
constexpr int DT_UNROLL = 4;                    // pieces of 16 bytes that a thread has in flight
constexpr int DT_MAX_PARTS = 8;                 // blocks of a cluster
constexpr float DT_LARGE_LSE = 1024.f;          // from here on lse in fp32 is off by 3e-5, so much of the gradient
// Rows up to here are short, where there are so many tokens that a row need not be cut; up to twice as much (the joint kernel: half as much again)
// where there are eight for a multiprocessor.  Measured, us, short against long: both at once 5554 x 5249 f16 42 and 71, 8192 x 12000 bf16 94
// and 101, 8192 x 16384 131 and 114; loss 8192 x 16384 50 and 70, 400 x 30000 11.8 and 10.0; gradient 8192 x 16384 95 and 113, 8192 x 30000 190 and 167.
constexpr int DT_SHORT_BYTES = 16 * 1024;
constexpr int DT_PART_BYTES = 32 * 1024;        // of a row that a block of the joint kernel has, where eight parts are enough
// The same of the gradient alone (fp32 logits), which needs no more blocks than there are multiprocessors: through shared memory 64 x 50001 in four parts 7.5 us, in
// eight of 32 KB 10.9; 1000 x 30000 43.8 and 49.5, 400 x 131072 78 and 94.
constexpr int DT_ALONE_BYTES = 64 * 1024;
constexpr int DT_HELD = DT_ALONE_BYTES / (16 * DT_UNROLL * DT_LONG);         // so much in a thread's registers
// of shared memory for one of so many blocks, beside its variables and what every block takes
constexpr int dt_room(int blocks) { return 227 * 1024 / blocks - 1024 - 2304; }

// ---- 16 bytes of a row -------------------------------------------------------------------------------
template <typename T>
struct piece16 {
    static constexpr int N = 16 / (int)sizeof(T);
    uint4 u;
    __device__ __forceinline__ void get(float (&v)[N]) const
    {
        if constexpr (sizeof(T) == 2) {
            vec8<T> w;
            w.u = u;
            w.get(v);
        } else {
            v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[N])
    {
        if constexpr (sizeof(T) == 2) {
            vec8<T> w;
            w.set(v);
            u = w.u;
        } else {
            u = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        }
    }
};
__device__ __forceinline__ unsigned minus_infinity(float) { return 0xFF800000u; }
__device__ __forceinline__ unsigned minus_infinity(__nv_bfloat16) { return 0xFF80FF80u; }
__device__ __forceinline__ unsigned minus_infinity(__half) { return 0xFC00FC00u; }
__device__ __forceinline__ uint4 ld16(const void* p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// The part of a row that a block has: elements [e0, e1), of which pieces [0, pieces) of 16 aligned bytes begin at `body`; fewer than a
// piece's elements lie before and behind them.
template <typename T>
struct part_of {
    long long e0, e1, body;
    int pieces, edge;           // edge: elements before and behind
    // per: elements of a part, a multiple of a piece's
    __device__ __forceinline__ part_of(const T* row, int vocab, int part, long long per)
    {
        constexpr int N = 16 / (int)sizeof(T);
        e0 = min((long long)vocab, per * part);
        e1 = min((long long)vocab, e0 + per);
        const int off = (int)((reinterpret_cast<uintptr_t>(row + e0) & 15u) / sizeof(T));
        body = min(e1, e0 + (off ? N - off : 0));
        pieces = (int)((e1 - body) / N);
        edge = (int)(e1 - e0) - pieces * N;
    }
    // element of the i-th one that is in no piece
    __device__ __forceinline__ long long at_edge(int i) const
    {
        const int before = (int)(body - e0);
        return i < before ? e0 + i : body + (long long)pieces * (16 / (int)sizeof(T)) + (i - before);
    }
};

// ---- running maximum and sum of e^((z - m) / T); c = log2(e) / T --------------------------------------
// e^t comes from the special-function unit, for fp32 logits too: its argument is rounded twice, and over 64 x 50001 q is off by 2.5e-7 in the mean square, that of
// elementary fp32 operations by 1.6e-7; losses over two dozen random shapes by 1.0 to 1.3 times theirs, dz as a whole the same; a single row whose sum hangs on a few terms by up to
// 2.6 times (1 x 30056: dz 1.7e-7 and 6.5e-8).  The library's function of an argument rounded once has the errors of those operations, and takes a loss of 8192 x 32768
// 182 us instead of 160, of 4096 x 5249 20.6 instead of 14.4, and both calls of 64 x 50001 17.4 instead of 15.0; giving back to 2^t what its argument's rounding
// takes, 16.5, helps q alone.
__device__ __forceinline__ unsigned max2(unsigned a, unsigned b, __nv_bfloat16)
{
    const __nv_bfloat162 r = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const unsigned*>(&r);
}
__device__ __forceinline__ unsigned max2(unsigned a, unsigned b, __half)
{
    const __half2 r = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const unsigned*>(&r);
}
struct online {
    float m, s;
    __device__ __forceinline__ void clear() { m = -CUDART_INF_F; s = 0.f; }
    // DT_UNROLL pieces; 16-bit maxima two at a time, the rest in packed fp32
    template <typename T>
    __device__ __forceinline__ void add(const uint4 (&r)[DT_UNROLL], float c)
    {
        constexpr int W = 4 * DT_UNROLL;
        const unsigned(&w)[W] = reinterpret_cast<const unsigned(&)[W]>(r);
        float top;
        if constexpr (sizeof(T) == 2) {
            unsigned t[4] = {w[0], w[1], w[2], w[3]};
#pragma unroll
            for (int i = 4; i < W; ++i) t[i & 3] = max2(t[i & 3], w[i], T());
            const float2 f = unpack2(max2(max2(t[0], t[1], T()), max2(t[2], t[3], T()), T()), T());
            top = fmaxf(f.x, f.y);
        } else {
            float t[4] = {__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3])};
#pragma unroll
            for (int i = 4; i < W; ++i) t[i & 3] = fmaxf(t[i & 3], __uint_as_float(w[i]));
            top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
        }
        const float now = fmaxf(m, top), about = now == -CUDART_INF_F ? 0.f : now;
        float2 sum[2] = {make_float2(s * ex2((m - about) * c), 0.f), f2(0.f)};
        auto pair = [&](int k, float2 v) {
            const float2 t = mul2(add2(v, f2(-about)), f2(c));
            sum[k & 1] = add2(sum[k & 1], make_float2(ex2(t.x), ex2(t.y)));
        };
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < W; ++i) pair(i, unpack2(w[i], T()));
        } else {
#pragma unroll
            for (int i = 0; i < W; i += 2) pair(i >> 1, make_float2(__uint_as_float(w[i]), __uint_as_float(w[i + 1])));
        }
        sum[0] = add2(sum[0], sum[1]);
        s = sum[0].x + sum[0].y;
        m = now;
    }
    __device__ __forceinline__ void add(float v, float c)
    {
        const float now = fmaxf(m, v), about = now == -CUDART_INF_F ? 0.f : now;
        s = s * ex2((m - about) * c) + ex2((v - about) * c);
        m = now;
    }
    // over the lanes of a warp: the maximum first, then the sums of what is left, in a fixed order
    __device__ __forceinline__ void join_lanes(float c)
    {
        // (floats in the order of signed integers)
        const int b = __float_as_int(m), k = __reduce_max_sync(0xFFFFFFFFu, b ^ ((b >> 31) & 0x7FFFFFFF));
        const float now = __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF)), about = now == -CUDART_INF_F ? 0.f : now;
        s *= ex2((m - about) * c);
#pragma unroll
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
        m = now;
    }
    // Over the row's warps of all blocks of a cluster: every warp leaves its own, and after one barrier takes all of them, the same ones on a lane.
    // `mine`: this warp has a share of the row.
    template <int RT>
    __device__ __forceinline__ void join_row(float2* warp_ms, bool mine, int parts, float c)
    {
        constexpr int WARPS = RT / 32, EACH = (WARPS * DT_MAX_PARTS + 31) / 32;
        const int lane = threadIdx.x & 31;
        if (mine) {
            join_lanes(c);
            if (lane == 0) warp_ms[threadIdx.x >> 5] = make_float2(m, s);
        }
        __syncwarp();
        if (parts > 1) lfptx::cluster_sync_all();
        else __syncthreads();
        const unsigned at = lfptx::smem_u32(warp_ms + (lane & (WARPS - 1)));
        float2 v[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int part = lane / WARPS + 32 / WARPS * i;
            v[i] = make_float2(-CUDART_INF_F, 0.f);
            if (parts == 1) {
                if (part == 0) v[i] = warp_ms[lane & (WARPS - 1)];
            } else if (part < parts) {
                asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v[i].x), "=f"(v[i].y) : "r"(lfptx::map_to_cta(at, (unsigned)part)) : "memory");
            }
        }
        __syncwarp();
        m = v[0].x;
#pragma unroll
        for (int i = 1; i < EACH; ++i) m = fmaxf(m, v[i].x);
        const float about = m == -CUDART_INF_F ? 0.f : m;
        s = 0.f;
#pragma unroll
        for (int i = 0; i < EACH; ++i) s += v[i].y * ex2((v[i].x - about) * c);
        join_lanes(c);
    }
};

struct entry_facts {                   // of a token's entries
    double sum;                        // P
    float top;                         // t_m
    int any, bad;                      // entries at all; an index beyond the vocabulary
    int mine;                          // entries in this part of the row
};
struct entries {                       // the teacher's, of one token
    int* at;                           // -1: not there
    float* p;                          // 0: not there
    float* t;                          // the teacher's logit
    float* z;                          // the student's
    float* total;                      // of the first of this part's entries on an element: what all of them have; of others < 0
    short* mine;                       // this part's entries, in their order
    entry_facts* facts;
    __host__ __device__ static constexpr size_t bytes(int top) { return (size_t)top * 22; }
    __device__ __forceinline__ entries(void* space, int top, entry_facts* f) : facts(f)
    {
        at = static_cast<int*>(space);
        p = reinterpret_cast<float*>(at + top);
        t = p + top;
        z = t + top;
        total = z + top;
        mine = reinterpret_cast<short*>(total + top);
    }
};
__device__ __forceinline__ void copy4(void* to, const void* from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(lfptx::smem_u32(to)), "l"(from) : "memory");
}
// whether the four bytes that an element lies in are the row's
template <typename T>
__device__ __forceinline__ bool in_word(const T* z, int at, int vocab)
{
    if (sizeof(T) == 4) return true;
    return (reinterpret_cast<uintptr_t>(z + at) & 2) ? at > 0 : at + 1 < vocab;
}
// By one warp, in steps: what is read of the row (the logits of elements [e0, e1); of 16-bit ones the four bytes that they lie in, where the row has both
// halves) and which entries are of the part [p0, p1), ...
template <typename T>
__device__ __forceinline__ void gather(const entries& e, const lf_distill_args& a, int token, const T* z, long long e0, long long e1, long long p0, long long p1)
{
    const int lane = threadIdx.x & 31;
    const int* index = a.index + (size_t)token * a.top;
    const float* value = a.value + (size_t)token * a.top;
    float top = -CUDART_INF_F;
    int bad = 0, any = 0, mine = 0;
    // (copies without registers: the whole list is under way at once, then all the logits, so that its length costs no further trip to memory)
    for (int k = lane; k < a.top; k += 32) {
        copy4(e.at + k, index + k);
        copy4(e.t + k, value + k);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    for (int first = 0; first < a.top; first += 32) {
        const int k = first + lane, at = k < a.top ? e.at[k] : -1;
        const float t = k < a.top ? e.t[k] : -CUDART_INF_F;
        const bool there = at >= 0 && t != -CUDART_INF_F, here = there && at >= p0 && at < p1;
        const unsigned all_here = __ballot_sync(0xFFFFFFFFu, here);
        if (here) e.mine[mine + __popc(all_here & ((1u << lane) - 1u))] = (short)k;
        mine += __popc(all_here);
        bad |= there && at >= a.vocab;
        any |= there;
        if (there) top = fmaxf(top, t);
        if (k < a.top) {
            if (!there) e.t[k] = -CUDART_INF_F;
            if (there && at >= e0 && at < e1) {
                if (in_word(z, at, a.vocab)) copy4(e.z + k, reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(z + at) & ~(uintptr_t)3));
                else e.z[k] = (float)z[at];
            } else {
                e.z[k] = 0.f;
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    bad = __any_sync(0xFFFFFFFFu, bad);
    any = __any_sync(0xFFFFFFFFu, any);
    if (lane == 0) {
        e.facts->any = any;
        e.facts->bad = bad;
        e.facts->top = top;
        e.facts->mine = mine;
    }
    __syncwarp();
}
// ... the weights (a sum over lanes adds in a fixed order) and, where four bytes hold two logits, the one that is meant, ...
// Weights of fp32 logits are in 64 bits until they are rounded once: dz is little else than they are, and with the roundings of an fp32 argument,
// exponential and quotient it was off by 5.2e-8 (64 x 50001, relative norm), now 3.8e-8.  What is rounded to 16 bits gains nothing by that (8192 x 32768 bf16
// with 64 entries 212 us, with 64-bit weights 224).
template <typename T>
__device__ __forceinline__ void weigh(const entries& e, const lf_distill_args& a, const T* z, long long e0, long long e1)
{
    const int lane = threadIdx.x & 31;
    double sum = 0.0;
    if constexpr (sizeof(T) == 4) {
        const double inv_t = 1.0 / (double)a.temperature, top = (double)e.facts->top;
        for (int k = lane; k < a.top; k += 32) {
            const double p = e.t[k] != -CUDART_INF_F ? exp(((double)e.t[k] - top) * inv_t) : 0.0;
            sum += p;
            e.p[k] = (float)p;                            // (two numbers hold it until the sum is known)
            e.total[k] = (float)(p - (double)(float)p);
        }
    } else {
        const float inv_t = 1.0f / a.temperature, top = e.facts->top;
#pragma unroll 4
        for (int k = lane; k < a.top; k += 32) {
            const float p = e.t[k] != -CUDART_INF_F ? expf((e.t[k] - top) * inv_t) : 0.f;
            sum += (double)p;
            e.p[k] = p;
            const int at = e.at[k];
            if (at >= e0 && at < e1 && e.t[k] != -CUDART_INF_F && in_word(z, at, a.vocab)) {
                const float2 f = unpack2(__float_as_uint(e.z[k]), T());
                e.z[k] = (reinterpret_cast<uintptr_t>(z + at) & 2) ? f.y : f.x;
            }
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if constexpr (sizeof(T) == 4) {
        const double inv = 1.0 / sum;
        for (int k = lane; k < a.top; k += 32) e.p[k] = (float)(((double)e.p[k] + (double)e.total[k]) * inv);
    } else {
        const float inv = 1.0f / (float)sum;
#pragma unroll 4
        for (int k = lane; k < a.top; k += 32) e.p[k] *= inv;
    }
    if (lane == 0) e.facts->sum = sum;
    __syncwarp();
}
// ... and what each element of the part has of them, for the gradient.
__device__ __forceinline__ void gather_totals(const entries& e, short* table)
{
    const int lane = threadIdx.x & 31, mine = e.facts->mine;
    // Several entries on one element: the first adds them up, in their order.  Whether there are any is found with a table: an entry
    // leaves its number at its element's place there and looks who is there then: itself, or an entry on the same element, or on another
    // one, and then it tries again with the others that did, by another multiplier.  (Every entry against every other: 102 of them took longer than a row of 5249.)
    bool several = false;
    unsigned mult = 2654435769u;
    for (int i = lane; i < mine; i += 32) e.total[e.mine[i]] = e.p[e.mine[i]];
    if (mine <= 32) {                      // a lane each, compared at once
        const int at = lane < mine ? e.at[e.mine[lane]] : -1;
        const unsigned same = __match_any_sync(0xFFFFFFFFu, at);
        several = __any_sync(0xFFFFFFFFu, at >= 0 && (same & (same - 1)) != 0);
    }
    for (int round = 0, left = mine > 32; left && !several; ++round, mult = mult * 5u + 0x9E3779B8u) {
        left = 0;
#pragma unroll 2
        for (int i = lane; i < mine; i += 32) {
            const int k = e.mine[i];
            if (round == 0 || e.total[k] < 0.f) table[(mult * (unsigned)e.at[k]) >> (32 - DT_TABLE_LOG2)] = (short)k;
        }
        __syncwarp();
#pragma unroll 2
        for (int i = lane; i < mine; i += 32) {
            const int k = e.mine[i], at = e.at[k];
            if (round > 0 && !(e.total[k] < 0.f)) continue;
            const int there = table[(mult * (unsigned)at) >> (32 - DT_TABLE_LOG2)];
            const bool again = there != k && e.at[there] != at;
            several |= there != k && !again;
            left |= again;
            e.total[k] = again ? -1.f : e.p[k];             // (a mark: weights are not below zero)
        }
        left = __any_sync(0xFFFFFFFFu, left);
        several = __any_sync(0xFFFFFFFFu, several) || round == DT_TABLE_ROUNDS;
        __syncwarp();
    }
    if (!several) return;
    for (int i = lane; i < mine; i += 32) {
        const int k = e.mine[i], at = e.at[k];
        bool first = true;
        float total = 0.f;
        for (int o = 0; o < mine; ++o) {
            const int j = e.mine[o];
            if (e.at[j] == at) {
                total += e.p[j];
                first &= j >= k;
            }
        }
        e.total[k] = first ? total : -1.f;
    }
}
// The loss, by one warp.  A weight p that fp32 does not tell from zero has no part in it, whatever logit it falls on.
__device__ __forceinline__ void loss_of(const entries& e, const lf_distill_args& a, int token, float m, float s)
{
    const double tau = (double)a.temperature, log_s = log((double)s);
    const entry_facts facts = *e.facts;
    double dot = 0.0;
    for (int k = threadIdx.x & 31; k < a.top; k += 32)
        if (e.p[k] != 0.f) dot += (double)e.p[k] * (((double)e.t[k] - (double)facts.top) - ((double)e.z[k] - (double)m));
#pragma unroll
    for (int o = 16; o; o >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, o);
    if ((threadIdx.x & 31) == 0) {
        const float w = a.weight ? a.weight[token] : 1.f;
        const double kl = facts.bad ? CUDART_NAN : dot / tau + log_s - log(facts.sum);
        if (a.lse) a.lse[token] = (float)((double)m / tau + log_s);
        a.loss[token] = w == 0.f || !facts.any ? 0.f : (float)(kl * tau * tau * (double)w);
    }
}
// By the row's threads: dz of the entries that fall on elements [e0, e1)
template <typename T, int RT, typename F>
__device__ __forceinline__ void put_right(const entries& e, T* dz, float wt, F q_of)
{
    const int mine = e.facts->mine;
    for (int i = threadIdx.x; i < mine; i += RT) {
        const int k = e.mine[i];
        // (NaN, the weight of a list that holds one, is no number below zero)
        if (!(e.total[k] < 0.f)) dz[e.at[k]] = (T)(wt * (q_of(e.z[k]) - e.total[k]));
    }
}
template <typename T>
__device__ __forceinline__ void store_piece(T* to, const float (&v)[16 / sizeof(T)], bool aligned)
{
    if (aligned) {
        piece16<T> o;
        o.set(v);
        *reinterpret_cast<uint4*>(to) = o.u;
    } else {
#pragma unroll
        for (int i = 0; i < 16 / (int)sizeof(T); ++i) to[i] = (T)v[i];
    }
}

// a piece of dz: f e^((z - m) / T)
template <typename T>
__device__ __forceinline__ void gradient_piece(float (&v)[16 / sizeof(T)], uint4 u, float m, float c, float f)
{
    piece16<T> p;
    p.u = u;
    p.get(v);
#pragma unroll
    for (int k = 0; k < 16 / (int)sizeof(T); k += 2) {
        const float2 t = mul2(add2(make_float2(v[k], v[k + 1]), f2(-m)), f2(c));
        const float2 g = mul2(make_float2(ex2(t.x), ex2(t.y)), f2(f));
        v[k] = g.x; v[k + 1] = g.y;
    }
}
// pieces [first, last) of a part's dz, a thread's of them, from pieces that `at` gives, BATCH of them before the first is used
template <typename T, int RT, int BATCH, typename F>
__device__ __forceinline__ void gradient_pieces(T* to, int first, int last, float m, float c, float f, bool aligned, F at)
{
    constexpr int N = 16 / (int)sizeof(T), STEP = RT * BATCH;
    float v[N];
    int i = first + (int)threadIdx.x;
    if (aligned) {
        for (; i + STEP - RT < last; i += STEP) {
            uint4 r[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) r[u] = at(i + u * RT);
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                gradient_piece<T>(v, r[u], m, c, f);
                piece16<T> o;
                o.set(v);
                reinterpret_cast<uint4*>(to)[i + u * RT] = o.u;
            }
        }
    }
    for (; i < last; i += RT) {
        gradient_piece<T>(v, at(i), m, c, f);
        store_piece<T>(to + (long long)i * N, v, aligned);
    }
}
template <typename T>
__device__ __forceinline__ void gradient_edge(T* dz, const T* z, const part_of<T>& mine, float m, float c, float f)
{
    if ((int)threadIdx.x < mine.edge) {
        const long long at = mine.at_edge(threadIdx.x);
        dz[at] = (T)(f * ex2(((float)z[at] - m) * c));
    }
}
template <typename T, int RT>
__device__ __forceinline__ void fill_part(T* dz, const part_of<T>& mine, float with, bool aligned)
{
    float v[16 / sizeof(T)];
#pragma unroll
    for (int k = 0; k < 16 / (int)sizeof(T); ++k) v[k] = with;
    for (int i = threadIdx.x; i < mine.pieces; i += RT) store_piece<T>(dz + mine.body + (long long)i * (16 / (int)sizeof(T)), v, aligned);
    if ((int)threadIdx.x < mine.edge) dz[mine.at_edge(threadIdx.x)] = (T)with;
}
template <typename T, int RT>
__device__ __forceinline__ void zero_part(T* dz, const part_of<T>& mine, bool aligned) { fill_part<T, RT>(dz, mine, 0.f, aligned); }

// pieces [first, last) of a part, a thread's of them, from pieces that `at` gives, DT_UNROLL at a time
template <typename T, int RT, typename F>
__device__ __forceinline__ void online_pieces(online& o, int first, int last, float c, F at)
{
    constexpr int STEP = RT * DT_UNROLL;
    uint4 r[DT_UNROLL];
    int i = first + (int)threadIdx.x;
    for (; i + STEP - RT < last; i += STEP) {
#pragma unroll
        for (int u = 0; u < DT_UNROLL; ++u) r[u] = at(i + u * RT);
        o.add<T>(r, c);
    }
    if (i < last) {
        const unsigned none = minus_infinity(T());
#pragma unroll
        for (int u = 0; u < DT_UNROLL; ++u) r[u] = i + u * RT < last ? at(i + u * RT) : make_uint4(none, none, none, none);
        o.add<T>(r, c);
    }
}
template <typename T>
__device__ __forceinline__ void online_edge(online& o, const T* z, const part_of<T>& mine, float c)
{
    if ((int)threadIdx.x < mine.edge) o.add((float)z[mine.at_edge(threadIdx.x)], c);
}

// Loss and lse of a token's row; a cluster of 2^log2 blocks has a token, each of them `per` elements.
// (Registers: left to itself the compiler takes 32 of them for long rows and has fewer loads under way: 64 x 50001 f32 7.4 us, with room for 56 6.1;
// the short rows' blocks want to be many: 8192 x 8000 bf16 33.6 us with 56, 32.5 with 40.)
template <typename T, int RT>
__global__ void __launch_bounds__(RT + 32, RT == DT_LONG ? 4 : 16) k_distill(const lf_distill_args a, int log2, long long per)
{
    extern __shared__ __align__(16) unsigned char space[];
    __shared__ entry_facts facts;
    __shared__ float2 warp_ms[RT / 32];
    const int parts = 1 << log2, token = blockIdx.x >> log2, part = blockIdx.x & (parts - 1), tid = threadIdx.x;
    const T* z = static_cast<const T*>(a.z) + (size_t)token * a.ld_z;
    const part_of<T> mine(z, a.vocab, part, per);
    const uint4* from = reinterpret_cast<const uint4*>(z + mine.body);
    const float c = LOG2E / a.temperature;
    const bool row_warp = tid < RT;
    const entries ent(space, a.top, &facts);
    lf_grid_wait();
    lf_grid_release();
    online o;
    o.clear();
    if (row_warp) {
        online_pieces<T, RT>(o, 0, mine.pieces, c, [&](int i) { return ld16(from + i); });
        online_edge<T>(o, z, mine, c);
    } else if (part == 0) {
        gather<T>(ent, a, token, z, 0, a.vocab, 0, 0);
        weigh<T>(ent, a, z, 0, a.vocab);
    }
    __syncwarp();
    o.join_row<RT>(warp_ms, row_warp, parts, c);
    if (parts > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    if (part == 0 && !row_warp) loss_of(ent, a, token, o.m, o.s);
    __syncwarp();
    if (parts > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");       // nobody leaves while its sums are being read
}

// The same and the gradient, or (loss NULL) the gradient alone, with z read once from memory: a part of a row stays in shared memory between the sums and the
// gradient (`staged` pieces of it; what is more, of rows beyond eight parts, is read again).  Blocks are small and many, so that
// some load while others add or store: 8192 x 131072 bf16 849 us with six blocks to a multiprocessor (five: 938, four: 1072), 815 since a part looks after its own entries only; persistent
// ones with the next part on its way 1345, a row to a block that reads it again from L2 1154.  The warp with the teacher's entries is waited for where it has read the row, which dz may be, and at
// the end: a list of nothing, or an index beyond the vocabulary, is rare enough for the part to be written again.
// HELD: a thread holds so many times DT_UNROLL pieces in registers instead, of fp32 rows whose gradient alone is wanted and that are all at work at once: their
// blocks need not be small, and no multiprocessor has to divide its memory differently for them than for the loss before them (both calls on other rows each time:
// 64 x 50001 15.2 us, through shared memory 19.3; 148 x 16000 11.3 and 14.2; not all at once, 2048 x 131072, 611 and 583).
template <typename T, int RT, int HELD>
__global__ void __launch_bounds__(RT + 32, HELD ? 2 : RT == DT_LONG ? 6 : 16) k_distill_both(const lf_distill_args a, int log2, long long per, int staged)
{
    extern __shared__ __align__(16) unsigned char space[];     // staged pieces, entries
    __shared__ entry_facts facts;
    __shared__ short table[1 << DT_TABLE_LOG2];
    __shared__ float2 warp_ms[RT / 32];
    const int parts = 1 << log2, token = blockIdx.x >> log2, part = blockIdx.x & (parts - 1), tid = threadIdx.x;
    const bool row_warp = tid < RT, whole = part == 0 && a.loss;      // the first part has the loss
    const T* z = static_cast<const T*>(a.z) + (size_t)token * a.ld_z;
    const part_of<T> mine(z, a.vocab, part, per);
    const uint4* from = reinterpret_cast<const uint4*>(z + mine.body);
    const int kept = min(HELD ? HELD * DT_UNROLL * RT : staged, mine.pieces);
    uint4 held[HELD ? HELD : 1][DT_UNROLL];
    const float c = LOG2E / a.temperature;
    uint4* own = reinterpret_cast<uint4*>(space);
    const entries ent(space + (size_t)staged * 16, a.top, &facts);
    lf_grid_wait();
    lf_grid_release();
    online o;
    o.clear();
    if (row_warp) {
        if constexpr (HELD > 0) {
            const unsigned none = minus_infinity(T());
#pragma unroll
            for (int k = 0; k < HELD; ++k)
#pragma unroll
                for (int u = 0; u < DT_UNROLL; ++u) {
                    const int i = tid + (k * DT_UNROLL + u) * RT;
                    held[k][u] = i < kept ? ld16(from + i) : make_uint4(none, none, none, none);
                }
        } else {
            // (a thread reads what it copied itself)
            for (int i = tid; i < kept; i += RT) cp_async16(lfptx::smem_u32(own + i), from + i);
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        online_pieces<T, RT>(o, kept, mine.pieces, c, [&](int i) { return ld16(from + i); });
        online_edge<T>(o, z, mine, c);
        if constexpr (HELD > 0) {
#pragma unroll
            for (int k = 0; k < HELD; ++k)
                if (tid + k * DT_UNROLL * RT < kept) o.add<T>(held[k], c);
        } else {
            asm volatile("cp.async.wait_all;" ::: "memory");
            online_pieces<T, RT>(o, 0, kept, c, [&](int i) { return own[i]; });
        }
    } else {
        gather<T>(ent, a, token, z, whole ? 0 : mine.e0, whole ? a.vocab : mine.e1, mine.e0, mine.e1);
    }
    __syncwarp();
    o.join_row<RT>(warp_ms, row_warp, parts, c);                     // (every part has read the logits that its entries need)
    if (parts > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    T* dz = static_cast<T*>(a.dz) + (size_t)token * a.ld_dz;
    const float w = a.weight ? a.weight[token] : 1.f, wt = w * a.temperature, m = o.m;
    const bool aligned = (reinterpret_cast<uintptr_t>(dz + mine.body) & 15u) == 0, none = w == 0.f || !facts.any;
    if (!row_warp) {
        weigh<T>(ent, a, z, whole ? 0 : mine.e0, whole ? a.vocab : mine.e1);
        gather_totals(ent, table);
    } else if (!none) {
        const float f = facts.bad ? CUDART_NAN_F : wt / o.s;
        if constexpr (HELD > 0) {
#pragma unroll
            for (int k = 0; k < HELD; ++k)
#pragma unroll
                for (int u = 0; u < DT_UNROLL; ++u) {
                    const int i = tid + (k * DT_UNROLL + u) * RT;
                    float v[16 / sizeof(T)];
                    gradient_piece<T>(v, held[k][u], m, c, f);
                    if (i < kept) store_piece<T>(dz + mine.body + (long long)i * (16 / (int)sizeof(T)), v, aligned);
                }
        } else {
            gradient_pieces<T, RT, 1>(dz + mine.body, 0, kept, m, c, f, aligned, [&](int i) { return own[i]; });
        }
        gradient_pieces<T, RT, 1>(dz + mine.body, kept, mine.pieces, m, c, f, aligned, [&](int i) { return ld16(from + i); });
        gradient_edge<T>(dz, z, mine, m, c, f);
    } else {
        zero_part<T, RT>(dz, mine, aligned);
    }
    __syncthreads();
    if (row_warp) {
        if (!none) {
            const float inv_s = 1.0f / o.s;
            put_right<T, RT>(ent, dz, facts.bad ? CUDART_NAN_F : wt, [&](float zk) { return inv_s * ex2((zk - m) * c); });
        }
    } else if (whole) {
        loss_of(ent, a, token, o.m, o.s);
    }
    __syncwarp();
    if (parts > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");       // nobody leaves while its sums are being read
}

// dz from z and lse, 16-bit logits: no part of a row needs to know another.  Where lse is so large that fp32 does not hold enough of
// its fraction (a row of nothing but a type's lowest number), the first part takes the whole row, with its own maximum and sum.
// (Of fp32 logits, lse as an fp32 number is never good enough: its rounding, 2^-24 of itself, is in every q of the row, 5e-7 for an lse of 11 and 1.5e-5 for one of
// 260, where q is good for 1e-7.  Their maximum and sum are taken again, by k_distill_both without a loss.  Both calls on other rows each time: 64 x 50001 15.2 us,
// from lse 14.5; 1 x 50001 7.4 and 6.4; 8192 x 32768 565 and 501; 2048 x 131072 583 and 495.  A row that eight parts do not hold is read twice: 64 x 600001 139 for 55.)
template <typename T, int RT>
__global__ void __launch_bounds__(RT + 32, RT == DT_LONG ? 4 : 16) k_distill_backward(const lf_distill_args a, int parts, long long per)
{
    static_assert(sizeof(T) == 2, "fp32 logits: k_distill_both");
    extern __shared__ __align__(16) unsigned char space[];
    __shared__ entry_facts facts;
    __shared__ short table[1 << DT_TABLE_LOG2];
    __shared__ float2 warp_ms[RT / 32];
    const int token = blockIdx.x / parts, part = blockIdx.x - token * parts, tid = threadIdx.x;
    const T* z = static_cast<const T*>(a.z) + (size_t)token * a.ld_z;
    T* dz = static_cast<T*>(a.dz) + (size_t)token * a.ld_dz;
    const bool row_warp = tid < RT;
    const entries ent(space, a.top, &facts);
    lf_grid_wait();
    lf_grid_release();
    const float w = a.weight ? a.weight[token] : 1.f, lse = a.lse[token], c = LOG2E / a.temperature;
    const bool large = fabsf(lse) >= DT_LARGE_LSE;
    if (large && part > 0) return;
    const part_of<T> mine(z, a.vocab, part, large ? (1ll << 40) : per);
    const uint4* from = reinterpret_cast<const uint4*>(z + mine.body);
    if (!row_warp) gather<T>(ent, a, token, z, mine.e0, mine.e1, mine.e0, mine.e1);
    if (a.dz == a.z) __syncthreads();      // the entries' logits have been read
    if (!row_warp) {
        weigh<T>(ent, a, z, mine.e0, mine.e1);
        gather_totals(ent, table);
    }
    const bool aligned = (reinterpret_cast<uintptr_t>(dz + mine.body) & 15u) == 0;
    if (w == 0.f) {
        if (row_warp) zero_part<T, RT>(dz, mine, aligned);
        return;
    }
    const float wt = w * a.temperature;
    float m = lse * a.temperature, scale = 1.f;        // q = scale e^((z - m) / T)
    if (large) {
        online o;
        o.clear();
        if (row_warp) {
            online_pieces<T, RT>(o, 0, mine.pieces, c, [&](int i) { return ld16(from + i); });
            online_edge<T>(o, z, mine, c);
        }
        __syncwarp();
        o.join_row<RT>(warp_ms, row_warp, 1, c);
        m = o.m;
        scale = 1.0f / o.s;
    }
    const float f = wt * scale;
    if (row_warp) {
        gradient_pieces<T, RT, DT_UNROLL>(dz + mine.body, 0, mine.pieces, m, c, f, aligned, [&](int i) { return ld16(from + i); });
        gradient_edge<T>(dz, z, mine, m, c, f);
    }
    __syncthreads();
    if (!row_warp) return;
    if (!facts.any) zero_part<T, RT>(dz, mine, aligned);               // (rare: what was written is written again)
    else if (facts.bad) fill_part<T, RT>(dz, mine, CUDART_NAN_F, aligned);
    else put_right<T, RT>(ent, dz, wt, [&](float zk) { return scale * ex2((zk - m) * c); });
}

// elements of a part, whole pieces
template <typename T>
long long per_part(const lf_distill_args& a, long long parts)
{
    constexpr long long N = 16 / (long long)sizeof(T);
    return ((a.vocab + parts - 1) / parts + N - 1) / N * N;
}
// Blocks of a cluster, as a power of two: enough for `blocks` of them and to have `most` bytes at most, up to eight; parts of fewer than 4 KB
// are not worth a meeting.
int parts_log2(const lf_distill_args& a, long long blocks, long long most)
{
    const long long bytes = (long long)a.vocab * (a.dtype == LF_F32 ? 4 : 2);
    int n = 0;
    while ((1 << n) < DT_MAX_PARTS && (bytes >> n) > 4096 && ((bytes >> n) > most || ((long long)a.tokens << n) < blocks)) ++n;
    return n;
}

template <typename T>
cudaError_t distill_of(const lf_ops* o, const lf_distill_args& a)
{
    const int sm_count = o->sm_count;
    const cudaStream_t s = o->stream;
    const int part_bytes = a.loss ? DT_PART_BYTES : DT_ALONE_BYTES;
    const int log2 = parts_log2(a, a.loss ? 2 * sm_count : sm_count, a.dz ? part_bytes : 1ll << 40), parts = 1 << log2;
    const long long row = (long long)a.vocab * (long long)sizeof(T);
    const bool brief = log2 == 0 && (row <= DT_SHORT_BYTES || (a.tokens >= 8 * sm_count && row <= DT_SHORT_BYTES / 2 * (a.dz ? 3 : 4)));
    const dim3 grid((unsigned)((long long)a.tokens << log2));
    const long long per = per_part<T>(a, parts);
    if (!a.dz)
        return brief ? lf_launch(k_distill<T, DT_SHORT>, grid, DT_SHORT + 32, entries::bytes(a.top), s, a, log2, per)
                     : lf_launch_clusters(k_distill<T, DT_LONG>, grid, DT_LONG + 32, entries::bytes(a.top), parts, s, a, log2, per);
    const long long bytes = per * (long long)sizeof(T);
    if constexpr (sizeof(T) == 4)
        if (!a.loss && !brief && bytes <= DT_ALONE_BYTES && a.tokens <= o->max_held_rows[log2])
            return lf_launch_clusters(k_distill_both<T, DT_LONG, DT_HELD>, grid, DT_LONG + 32, entries::bytes(a.top), parts, s, a, log2, per, 0);
    // (long lists take room from the row, not from the six, or alone three, blocks: 8192 x 131072 with 300 entries 1257 us when they did)
    const long long most = brief ? part_bytes : std::min((long long)part_bytes, (dt_room(a.loss ? 6 : 3) - (long long)entries::bytes(a.top)) / 16 * 16);
    const int staged = (int)((bytes < most ? bytes : most) / 16);
    const size_t smem = (size_t)staged * 16 + entries::bytes(a.top);
    return brief ? lf_launch(k_distill_both<T, DT_SHORT, 0>, grid, DT_SHORT + 32, smem, s, a, log2, per, staged)
                 : lf_launch_clusters(k_distill_both<T, DT_LONG, 0>, grid, DT_LONG + 32, smem, parts, s, a, log2, per, staged);
}
template <typename T>
cudaError_t distill_backward_of(const lf_ops* o, const lf_distill_args& a)
{
    const int sm_count = o->sm_count;
    const cudaStream_t s = o->stream;
    const long long bytes = (long long)a.vocab * sizeof(T);
    long long parts = (bytes + 65535) / 65536;                    // (16 pieces a thread)
    while ((long long)a.tokens * parts < 2 * sm_count && bytes / parts > 4096) parts *= 2;
    const dim3 grid((unsigned)((long long)a.tokens * parts));
    return parts == 1 && (bytes <= DT_SHORT_BYTES || (a.tokens >= 8 * sm_count && bytes <= 2 * DT_SHORT_BYTES))
               ? lf_launch(k_distill_backward<T, DT_SHORT>, grid, DT_SHORT + 32, entries::bytes(a.top), s, a, 1, per_part<T>(a, 1))
               : lf_launch(k_distill_backward<T, DT_LONG>, grid, DT_LONG + 32, entries::bytes(a.top), s, a, (int)parts, per_part<T>(a, parts));
}
template <typename T>
bool distill_ready()
{
    return cudaFuncSetAttribute(k_distill_both<T, DT_LONG, 0>, cudaFuncAttributeMaxDynamicSharedMemorySize, dt_room(sizeof(T) == 4 ? 3 : 6)) == cudaSuccess;
}

}  // namespace

int lf_distill_init(lf_ops* o)
{
    for (int i = 0; i < 4; ++i) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute at[1];
        cfg.gridDim = dim3(8);
        cfg.blockDim = dim3(DT_LONG + 32);
        cfg.dynamicSmemBytes = entries::bytes(LF_DISTILL_MAX_TOP);
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = 1u << i;
        at[0].val.clusterDim.y = 1;
        at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&o->max_held_rows[i], k_distill_both<float, DT_LONG, DT_HELD>, &cfg) != cudaSuccess) return LF_ECUDA;
    }
    return distill_ready<float>() && distill_ready<__nv_bfloat16>() && distill_ready<__half>() ? LF_OK : LF_ECUDA;
}

cudaError_t lfk_distill(const lf_ops* o, const lf_distill_args& a)
{
    if (a.dtype == LF_F32) return distill_of<float>(o, a);
    if (a.dtype == LF_BF16) return distill_of<__nv_bfloat16>(o, a);
    return distill_of<__half>(o, a);
}
cudaError_t lfk_distill_backward(const lf_ops* o, const lf_distill_args& a)
{
    if (a.dtype == LF_F32) {
        lf_distill_args alone = a;
        alone.loss = alone.lse = nullptr;
        return distill_of<float>(o, alone);
    }
    if (a.dtype == LF_BF16) return distill_backward_of<__nv_bfloat16>(o, a);
    return distill_backward_of<__half>(o, a);
}

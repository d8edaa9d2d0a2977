// Beam search's selection: the best (score, beam, token) of each sequence over the logits of its beams, total = score + (logit - log sum exp logits).
//
// Two launches.  The first reads every logit once: a block takes a piece of a row into registers, finds the sums of exponentials of its granules and its `keep` best
// logits: totals of a row are in the order of its logits.  The second joins a sequence's rows in binary64 and picks among them.
//
// How a row is cut depends on the batch, its totals do not, nor on where the row begins: they are compared with other rows', where an equal total has to be equal in every bit.  Sums are formed over
// granules of 64 vectors of 16 bytes from the row's first value on, each under its own largest value, and over blocks of eight granules, in the same order in every cut; a piece is one block or eight of them.
//
// The best of a piece: the `keep`-th largest of the maxima of its groups of threads is no more than the `keep`-th largest value of all.  What reaches it (18 values for keep = 16 and
// logits in no order) goes to a list in LDS, which is ranked by counting.
#include "../../include/samp.h"
#include "decoder.h"
#include "decoder_rules.h"

#include <type_traits>

namespace samp {
namespace {

constexpr int SLOTS = 128, ROOM = 512;                                // threads of a piece whose values are looked through, and values that are ranked (1000 take longer than the way round: 4096 rows of 1000 equal
                                                                      // logits 413 us, 39)
constexpr float LOG2E = 1.44269504088896340736f;                      // (1.3e-8 of it off: as much of the mean distance from the largest logit, 2e-7 at most)

enum { F16 = 0, BF16 = 1, F32 = 2 };
typedef int v4i_at_2 __attribute__((ext_vector_type(4), aligned(2)));              // 16 bytes at any value's address: one load, wherever they lie
typedef int v4i_at_4 __attribute__((ext_vector_type(4), aligned(4)));
template <int T> struct Logit {
    static constexpr int SIZE = T == F32 ? 4 : 2, VEC = 16 / SIZE;
    typedef typename std::conditional<T == F32, v4i_at_4, v4i_at_2>::type Raw;
    static constexpr unsigned MINUS_INF_BITS = T == F16 ? 0xfc00u : T == BF16 ? 0xff80u : 0xff800000u;
    static __device__ __forceinline__ float value(const v4i &raw, int e)
    {
        if constexpr (T == F32) return __int_as_float(raw[e]);
        else if constexpr (T == BF16) return __int_as_float(e & 1 ? raw[e >> 1] & (int)0xffff0000u : raw[e >> 1] << 16);
        else return (float)__builtin_bit_cast(_Float16, (unsigned short)((unsigned)raw[e >> 1] >> 16 * (e & 1)));
    }
    static __device__ __forceinline__ float value(const void *at, int i)
    {
        if constexpr (T == F32) return static_cast<const float *>(at)[i];
        else if constexpr (T == BF16) return __uint_as_float((unsigned)static_cast<const unsigned short *>(at)[i] << 16);
        else return (float)static_cast<const _Float16 *>(at)[i];
    }
};
__device__ __forceinline__ float max_of_wave(float x)
{
    x = max3(x, x, other_lane<0xb1>(x));                              // lanes 1 0 3 2, then 2 3 0 1 of four, eight mirrored, sixteen mirrored
    x = max3(x, x, other_lane<0x4e>(x));
    x = max3(x, x, other_lane<0x141>(x));
    x = max3(x, x, other_lane<0x140>(x));
    const float a = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 0)), b = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 16));
    const float c = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 32)), d = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 48));
    return max3(max3(a, b, c), d, d);
}
// Of each of N values the largest (the sum) over the wave, in the lanes GRAIN n .. GRAIN n + GRAIN - 1 that of value n.  Lanes meet in the same order for every N
template <bool MAX> __device__ __forceinline__ float met(const Met &m) { return MAX ? max3(m.x, m.x, m.y) : m.x + m.y; }
template <bool MAX, int N> __device__ __forceinline__ float of_each(float (&x)[N], int lane)
{
    static_assert(N == 2 || N == 8, "pieces have two vectors a thread or eight");
    constexpr int A = N / 2, B = N == 8 ? 2 : 1;
    float a[A], b[B], c;
    if constexpr (MAX) settle<N>(x);
#pragma unroll
    for (int i = 0; i < A; i++) a[i] = met<MAX>(meet<32>(x[i], x[i + A], lane));
    if constexpr (MAX) settle<A>(a);
#pragma unroll
    for (int i = 0; i < B; i++) b[i] = met<MAX>(meet<16>(a[i], a[i + (N == 8 ? B : 0)], lane));
    c = met<MAX>(meet<8>(b[0], b[B - 1], lane));
    c = met<MAX>(Met{c, other_lane<0x141>(c)});                       // eight mirrored, then lanes 2 3 0 1 of four, 1 0 3 2
    c = met<MAX>(Met{c, other_lane<0x4e>(c)});
    return met<MAX>(Met{c, other_lane<0xb1>(c)});
}

struct Candidate { float logit; int token; };                         // token -1: none
constexpr int BLOCK_OF = 8;                                           // granules of a block
struct BlockSum { float top, sum; };                                  // sum of exp(x - top)
// The order of a value with the place behind it, the lower one first
__device__ __forceinline__ unsigned long long listed_of(float x, int place) { return (unsigned long long)order_of(x) << 32 | (unsigned)~place; }
__device__ __forceinline__ bool before(unsigned long long a, unsigned long long b) { return a > b; }

// How many of `all` come before `mine`, counted by 2^n lanes `step` that have each every step-th; and f(entry, how many come before it) for each of n entries, by THREADS threads.
// Eight (numbers of 16 bytes: four) are read together; one at a time took 110 clocks each.
template <class T> __device__ __forceinline__ int count_before(const T *all, int n, int first, int step, const T &mine)
{
    constexpr int BATCH = 64 / sizeof(T);
    int better = 0, j = first;
    for (; j + (BATCH - 1) * step < n; j += BATCH * step) {
        T x[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; u++) x[u] = all[j + u * step];
#pragma unroll
        for (int u = 0; u < BATCH; u++) better += before(x[u], mine);
    }
    for (; j < n; j += step) better += before(all[j], mine);
    return better;
}
template <int THREADS, class T, class F> __device__ __forceinline__ void rank_entries(const T *all, int n, F &&f)
{
    int share = 1;
    while (share < 64 && n * share * 2 <= THREADS) share *= 2;
    const int mine = threadIdx.x & (share - 1);
    for (int i = (int)threadIdx.x / share; i < n; i += THREADS / share) {
        const T e = all[i];
        int better = count_before(all, n, mine, share, e);
        for (int o = 1; o < share; o <<= 1) better += __shfl_xor(better, o, 64);
        if (mine == 0) f(i, e, better);
    }
}

__device__ __forceinline__ bool row_counts(const float *scores, const uint8_t *finished, int row)
{
    return __builtin_isfinite(scores[row]) && !(finished && finished[row]);
}

// One piece of one row: what bounds it is HBM where there are rows enough (512 rows of 128256, of which a quarter are finished or have no score and are not read: 97 MB, 25.7 us, 3.8 TB/s;
// the vector ALUs issue six tenths of that time, eleven instructions a logit), else its chain of one trip to memory, two reductions and the list: 35 rows of 50265
// binary32 6.6 us, 4 rows of 21128 4.8.  Vectors of 16 bytes are counted from the row's first value, wherever that lies; what of the last one lies behind the row counts as minus infinity.
template <int T, int THREADS, int VECTORS, int GROUPS>
__global__ __launch_bounds__(THREADS, 8) void beam_pieces_kernel(const char *__restrict__ logits, long ld, const float *__restrict__ scores,
                                                              const uint8_t *__restrict__ finished, int vocab, int keep, int chunks,
                                                              BlockSum *__restrict__ sums, Candidate *__restrict__ best)
{
    typedef Logit<T> L;
    constexpr int VEC = L::VEC, PER = VECTORS * VEC, TEAM = THREADS / GROUPS, WAVES = THREADS / 64, GRANULES = WAVES * VECTORS, GRAIN = 64 / VECTORS;
    static_assert(GRANULES % BLOCK_OF == 0 && GRANULES <= 64, "whole blocks, a granule a lane");
    static_assert(GROUPS == 64 || (GROUPS % 64 == 0 && TEAM <= 2), "the same lane of every wave, or one or two neighbours");
    __shared__ __attribute__((aligned(16))) unsigned long long list[ROOM];
    __shared__ __attribute__((aligned(16))) v4i held[SLOTS][VECTORS];
    __shared__ int owner[SLOTS];
    __shared__ __attribute__((aligned(16))) float tops[GROUPS == 64 ? THREADS : GROUPS];
    __shared__ float granule_top[GRANULES], granule_sum[GRANULES], least[GROUPS / 64];
    __shared__ int slots, listed, wave_count[WAVES];

    const int row = blockIdx.x / chunks, piece = blockIdx.x - row * chunks;
    if (VECTORS > 2 && !row_counts(scores, finished, row)) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const char *from = logits + (size_t)row * ld * L::SIZE;
    const int first = piece * THREADS * PER;                          // the piece's first token

    v4i raw[VECTORS];
    typedef typename L::Raw Raw;
    if (first + THREADS * PER <= vocab) {
        const Raw *const all = reinterpret_cast<const Raw *>(from + (long)first * L::SIZE) + tid;
#pragma unroll
        for (int i = 0; i < VECTORS; i++) raw[i] = all[i * THREADS];
    } else {
#pragma unroll
        for (int i = 0; i < VECTORS; i++) {
            const int at = first + (i * THREADS + tid) * VEC;
            if (at + VEC <= vocab) raw[i] = *reinterpret_cast<const Raw *>(from + (long)at * L::SIZE);
            else {
                unsigned x[VEC];
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    x[e] = L::MINUS_INF_BITS;
                    if (at + e < vocab) {
                        if constexpr (T == F32) x[e] = *reinterpret_cast<const unsigned *>(from + (long)(at + e) * 4);
                        else x[e] = *reinterpret_cast<const unsigned short *>(from + (long)(at + e) * 2);
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; e++) raw[i][e] = T == F32 ? (int)x[e] : (int)(x[(2 * e) % VEC] | x[(2 * e + 1) % VEC] << 16);
            }
        }
    }
    // (a short piece waits for its logits and for the row's flags at the same time)
    if (VECTORS <= 2 && !row_counts(scores, finished, row)) return;
    if (tid == 0) slots = listed = 0;
    float each[VECTORS];
#pragma unroll
    for (int i = 0; i < VECTORS; i++) {
        each[i] = max3(L::value(raw[i], 0), L::value(raw[i], 1), L::value(raw[i], 2));
#pragma unroll
        for (int e = 3; e < VEC; e += 2) each[i] = max3(each[i], L::value(raw[i], e), L::value(raw[i], min(e + 1, VEC - 1)));
    }
    float top = max3(each[0], each[0], each[1]);
#pragma unroll
    for (int i = 2; i < VECTORS; i += 2) top = max3(top, each[i], each[i + 1]);
    if constexpr (GROUPS == 64) tops[tid] = top;
    else {
        const float pair = TEAM == 2 ? max3(top, top, other_lane<0xb1>(top)) : top;
        if (tid % TEAM == 0) tops[tid / TEAM] = pair;
    }
    // the largest of the granule of vector lane / GRAIN of the wave's threads
    float m = of_each<true>(each, lane);
    if (m == -INFINITY) m = 0.0f;
    // (converted again for each use: 32 registers, and waves enough to wait for memory.  With the values kept, 178 registers, 64 x 8 x 128256 took 84 us)
    auto again = [&]() {
#pragma unroll
        for (int i = 0; i < VECTORS; i++) asm("" : "+v"(raw[i]));
    };
    again();
    // exp(x - m) as 2^(x log2(e) - reference), one multiply-add in front of each; the reference is m log2(e) but for its rounding, at most 1, which the sum makes
    // up for.  Of larger logits (a row of the type's lowest value) the difference comes first.
    constexpr float PLAIN = 0x1p24f;
    float sums_of[VECTORS];
#pragma unroll
    for (int i = 0; i < VECTORS; i++) {
        const float reference = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(m), GRAIN * i)) * LOG2E;
        float part[4] = {};
#pragma unroll
        for (int e = 0; e < VEC; e++) part[e & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(L::value(raw[i], e), LOG2E, -reference));
        sums_of[i] = (part[0] + part[1]) + (part[2] + part[3]);
    }
    if (__any(!(__builtin_fabsf(m) < PLAIN))) {
        again();
#pragma unroll
        for (int i = 0; i < VECTORS; i++) {
            const float of = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(m), GRAIN * i));
            if (__builtin_fabsf(of) < PLAIN) continue;
            float part[4] = {};
#pragma unroll
            for (int e = 0; e < VEC; e++) part[e & 3] += __builtin_amdgcn_exp2f((L::value(raw[i], e) - of) * LOG2E);
            sums_of[i] = (part[0] + part[1]) + (part[2] + part[3]);
        }
    }
    again();
    float sum = of_each<false>(sums_of, lane);
    if (__builtin_fabsf(m) < PLAIN) sum *= __builtin_amdgcn_exp2f(-__builtin_fmaf(m, LOG2E, -(m * LOG2E)));
    if (lane % GRAIN == 0) {
        granule_top[lane / GRAIN * WAVES + w] = m;
        granule_sum[lane / GRAIN * WAVES + w] = sum;
    }
    __syncthreads();
    if (tid < GROUPS) {
        // the `keep`-th largest of the groups' maxima: the smallest of those that fewer than `keep` are above
        float mine = tops[tid];
        int above = 0;
        if constexpr (GROUPS == 64) {
#pragma unroll
            for (int i = 1; i < WAVES; i++) mine = max3(mine, mine, tops[64 * i + tid]);
#pragma unroll
            for (int i = 0; i < 64; i++) above += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), i)) > mine;
        } else {
            const v4f *const all = reinterpret_cast<const v4f *>(tops);
#pragma unroll 16
            for (int i = 0; i < GROUPS / 4; i++)
#pragma unroll
                for (int e = 0; e < 4; e++) above += all[i][e] > mine;
        }
        const float t = -max_of_wave(above < keep ? -mine : -INFINITY);
        if (lane == 0) least[w] = t;
    }
    if (w == WAVES - 1) {
        // eight neighbouring lanes have a block's granules
        const bool some = lane < GRANULES && granule_sum[lane % GRANULES] != 0.0f;
        const float u = some ? granule_top[lane % GRANULES] : -INFINITY;
        float all = max3(u, u, other_lane<0xb1>(u));
        all = max3(all, all, other_lane<0x4e>(all));
        all = max3(all, all, other_lane<0x141>(all));
        float s = some ? granule_sum[lane % GRANULES] * __builtin_amdgcn_exp2f((u - all) * LOG2E) : 0.0f;
        s += other_lane<0xb1>(s);
        s += other_lane<0x4e>(s);
        s += other_lane<0x141>(s);
        if (lane < GRANULES && lane % BLOCK_OF == 0) sums[(size_t)blockIdx.x * (GRANULES / BLOCK_OF) + lane / BLOCK_OF] = BlockSum{all, s};
    }
    __syncthreads();
    float limit = least[0];
#pragma unroll
    for (int i = 1; i < GROUPS / 64; i++) limit = __builtin_fminf(limit, least[i]);
    limit = __builtin_fmaxf(limit, -3.40282347e38f);                  // (minus infinity is no candidate)

    // threads that have a value that reaches `limit` leave all of theirs in LDS, where the block looks through them
    if (top >= limit) {
        int *count = &slots;
        asm("" : "+v"(count));                                        // (few lanes: an addition of theirs each, not one of the wave's)
        const int slot = atomicAdd(count, 1);
        if (slot < SLOTS) {
            owner[slot] = tid;
#pragma unroll
            for (int i = 0; i < VECTORS; i++) held[slot][i] = raw[i];
        }
    }
    __syncthreads();
    int n = slots;                                                    // (this and what follows from it: the same for the whole block)
    if (n <= SLOTS) {
        for (int at = tid; at < n * PER; at += THREADS) {
            const int slot = at / PER, e = at % PER;
            const float x = L::value(&held[slot][0], e);
            if (x >= limit) {
                int *count = &listed;
                asm("" : "+v"(count));
                const int to = atomicAdd(count, 1);                   // (in any order: they are ranked)
                if (to < ROOM) list[to] = listed_of(x, (e / VEC * THREADS + owner[slot]) * VEC + e % VEC);
            }
        }
        __syncthreads();
        n = listed;
    } else n = ROOM + 1;
    if (n > ROOM) {
        // Many reach the limit, as in rows whose tokens have one value but for a few.  The `keep`-th largest value itself: the limit, which `keep` values reach, if fewer are above it, and
        // else bit by bit from the top; what is above it, less than `keep` values; and those that equal it, in the order of their places, as far as they are wanted.
        unsigned t = 0;
        bool is_limit = false;
#pragma unroll 1
        for (int bit = 32; bit >= 0 && !is_limit; bit--) {
            again();
            const float v = value_of_order(bit < 32 ? t | 1u << bit : order_of(limit) + 1);
            int reach = 0;
#pragma unroll
            for (int i = 0; i < VECTORS; i++)
#pragma unroll
                for (int e = 0; e < VEC; e++) reach += L::value(raw[i], e) >= v;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) reach += __shfl_xor(reach, o, 64);
            __syncthreads();
            if (lane == 0) wave_count[w] = reach;
            __syncthreads();
            reach = 0;
#pragma unroll
            for (int i = 0; i < WAVES; i++) reach += wave_count[i];
            if (bit == 32) is_limit = reach < keep;
            else if (reach >= keep) t |= 1u << bit;
        }
        if (!is_limit) limit = __builtin_fmaxf(value_of_order(t), -3.40282347e38f);
        again();
        __syncthreads();
        if (tid == 0) listed = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VECTORS; i++)
#pragma unroll
            for (int e = 0; e < VEC; e++)
                if (L::value(raw[i], e) > limit) {
                    const int to = atomicAdd(&listed, 1);
                    if (to < ROOM) list[to] = listed_of(L::value(raw[i], e), (i * THREADS + tid) * VEC + e);
                }
        __syncthreads();
        n = listed;
        again();
#pragma unroll
        for (int i = 0; i < VECTORS; i++) {
            if (n < keep) {                                           // (the same for the whole block)
                int at = tid;
                asm("" : "+v"(at));
                unsigned equal = 0;
#pragma unroll
                for (int e = 0; e < VEC; e++) equal |= (unsigned)(L::value(raw[i], e) == limit) << e;
                int before = __popc(equal);
                const int mine = before;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const int other = __shfl_up(before, o, 64);
                    if (lane >= o) before += other;
                }
                __syncthreads();
                if (lane == 63) wave_count[w] = before;
                __syncthreads();
                int to = n + before - mine;
#pragma unroll
                for (int u = 0; u < WAVES; u++) {
                    to += u < w ? wave_count[u] : 0;
                    n += wave_count[u];
                }
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    if ((equal >> e & 1) && to < ROOM) list[to] = listed_of(limit, (i * THREADS + at) * VEC + e);
                    to += equal >> e & 1;
                }
            }
        }
        __syncthreads();
        n = min(n, keep);                                             // (those above come first in the list)
    }
    Candidate *const to = best + (size_t)blockIdx.x * keep;
    rank_entries<THREADS>(list, n, [&](int, unsigned long long e, int better) {
        if (better < keep) to[better] = Candidate{value_of_order((unsigned)(e >> 32)), first + (int)~(unsigned)e};
    });
    if (tid < keep && tid >= n) to[tid] = Candidate{-INFINITY, -1};
}

// One sequence.  The pieces' lists are sorted: entry p of the list whose first entry is the r-th best of all first entries can be among the `keep` best only where r + p < keep; of those
// keep (keep + 1) / 2 the ones that reach a total that `keep` entries reach are ranked by counting, several lanes to an entry.  Entries are a total as a whole number of the same order, then row, logit and token.
constexpr int JOIN = 1024;
struct __attribute__((aligned(16))) Entry { unsigned long long total, then; };
constexpr Entry NO_ENTRY{0, ~0ull};
__device__ __forceinline__ bool before(const Entry &a, const Entry &b) { return (a.total > b.total) | ((a.total == b.total) & (a.then < b.then)); }
__device__ __forceinline__ Entry entry_of(double total, int r, float logit, int token)
{
    if (!(total > -INFINITY)) return NO_ENTRY;
    const unsigned long long t = (unsigned long long)__double_as_longlong(total + 0.0);
    const unsigned l = __float_as_uint(logit + 0.0f), high_first = l >> 31 ? l : ~(l | 0x80000000u);
    return Entry{t >> 63 ? ~t : t | 1ull << 63, (unsigned long long)r << 52 | (unsigned long long)high_first << 20 | (unsigned)token};
}
__device__ __forceinline__ double total_of(const Entry &e)
{
    return __longlong_as_double((long long)(e.total >> 63 ? e.total & ~(1ull << 63) : ~e.total));
}
// f(entry's place, entry, how many of the n come before it) for the `keep` best that are there, and perhaps for more.  Of many, only those are ranked that reach the `keep`-th largest of the
// maxima of TOPS groups, by the upper half of their totals: `keep` entries do.  1088 lists, keep = 64, 18 us, all ranked against all 85; 512, keep = 32, 9.0
// and 19.8; up to FEW entries that is as fast (136 of 64 sequences 6.9, this way 8.5).
constexpr int FEW = 192, TOPS = 128, RANKED = 512;
struct Best { __attribute__((aligned(16))) unsigned top[TOPS]; unsigned bound; int n, at[RANKED]; };
template <class F> __device__ __forceinline__ void rank_best(const Entry *all, int n, int keep, Best &best, F &&f)
{
    const int tid = threadIdx.x;
    int some = n;
    if (n > FEW) {
        if (tid < TOPS) best.top[tid] = 0;
        if (tid == 0) best.bound = ~0u, best.n = 0;
        __syncthreads();
        for (int i = tid; i < n; i += JOIN) atomicMax(&best.top[i % TOPS], (unsigned)(all[i].total >> 32));
        __syncthreads();
        if (tid < TOPS) {
            const unsigned mine = best.top[tid];
            const v4i *const tops = reinterpret_cast<const v4i *>(best.top);
            int above = 0;
#pragma unroll 8
            for (int j = 0; j < TOPS / 4; j++) {
                const v4i t = tops[j];
#pragma unroll
                for (int e = 0; e < 4; e++) above += (unsigned)t[e] > mine;
            }
            if (above < keep) atomicMin(&best.bound, mine);
        }
        __syncthreads();
        const unsigned bound = best.bound;
        for (int i = tid; i < n; i += JOIN) {
            const unsigned long long total = all[i].total;
            if (!total || (unsigned)(total >> 32) < bound) continue;
            const int to = atomicAdd(&best.n, 1);                     // (in any order: they are ranked)
            if (to < RANKED) best.at[to] = i;
        }
        __syncthreads();
        some = best.n;
    }
    if (n <= FEW || some > RANKED) {
        rank_entries<JOIN>(all, n, [&](int i, const Entry &e, int better) {
            if (e.total) f(i, e, better);
        });
        return;
    }
    int share = 1;
    while (share < 64 && some * share * 2 <= JOIN) share *= 2;
    const int mine = tid & (share - 1), i = tid / share;
    if (i >= some) return;                                            // (all lanes of an entry: no more than RANKED of them, JOIN threads)
    const Entry e = all[best.at[i]];
    int better = 0;
#pragma unroll 4
    for (int j = mine; j < some; j += share) better += before(all[best.at[j]], e);
    for (int o = 1; o < share; o <<= 1) better += __shfl_xor(better, o, 64);
    if (mine == 0) f(best.at[i], e, better);
}

// A block a sequence.  A few dependent steps over some thousand numbers: 7.4 us for 64 sequences of 8 rows in 4 pieces each, keep = 16; 5.2 for one of 4 rows in 6.
__global__ __launch_bounds__(JOIN) void beam_join_kernel(const BlockSum *__restrict__ sums, const Candidate *__restrict__ best, const float *__restrict__ scores,
                                                         const uint8_t *__restrict__ finished, int end, int beams, int keep, int chunks, int blocks, float *__restrict__ out,
                                                         int *__restrict__ parents, int *__restrict__ tokens)
{
    extern __shared__ __attribute__((aligned(16))) Entry first[];
    const int lists = beams * chunks;
    Entry *const pair = first + lists;
    __shared__ double lse[SAMP_MAX_BEAMS];                            // log sum exp; NaN where a row's logits have no candidates
    __shared__ float score[SAMP_MAX_BEAMS];                           // NaN where a row has none
    __shared__ bool done[SAMP_MAX_BEAMS];
    __shared__ int list_of[SAMP_MAX_KEEP], there;
    __shared__ Best ranked;
    __shared__ unsigned long long enough;                             // a total that at least `keep` entries reach, or 0
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const size_t row0 = (size_t)b * beams;
    // (of rows that do not count nothing was written: what is read of them is not used)
    const Candidate head = tid < lists ? best[(row0 * chunks + tid) * keep] : Candidate{0.0f, -1};
    if (tid < beams) {
        const float s = scores[row0 + tid];
        score[tid] = __builtin_isfinite(s) ? s : __builtin_nanf("");
        done[tid] = finished && finished[row0 + tid];
    }
    if (tid < keep) list_of[tid] = -1;
    if (tid == 0) there = 0, enough = 0;
    for (int r = w; r < beams; r += JOIN / 64) {
        const BlockSum *const of = sums + (row0 + r) * blocks;
        const BlockSum mine = lane < blocks ? of[lane] : BlockSum{0.0f, 0.0f};
        float top = mine.sum == 0.0f ? -INFINITY : mine.top;          // (a sum of 0: nothing finite there)
        for (int c = lane + 64; c < blocks; c += 64)
            if (!(of[c].sum == 0.0f)) top = __builtin_fmaxf(top, of[c].top);
        top = wave_max(top);
        double sum = mine.sum == 0.0f ? 0.0 : (double)mine.sum * exp((double)mine.top - (double)top);
        for (int c = lane + 64; c < blocks; c += 64)
            if (!(of[c].sum == 0.0f)) sum += (double)of[c].sum * exp((double)of[c].top - (double)top);
        sum = wave_sum(sum);
        // (no finite logit: a sum of 0; NaN or plus infinity: a sum of NaN)
        if (lane == 0) lse[r] = sum > 0.0 ? (double)top + log(sum) : __builtin_nan("");
    }
    __syncthreads();
    auto entry = [&](int list, int p, const Candidate &x) {
        const int r = list / chunks;
        if (done[r]) return list == r * chunks && p == 0 ? entry_of((double)score[r], r, 0.0f, 0) : NO_ENTRY;
        return x.token >= 0 ? entry_of((double)score[r] + ((double)x.logit - lse[r]), r, x.logit, x.token) : NO_ENTRY;
    };
    if (tid < lists) first[tid] = entry(tid, 0, head);
    for (int i = tid + JOIN; i < lists; i += JOIN) first[i] = entry(i, 0, best[(row0 * chunks + i) * keep]);
    __syncthreads();
    rank_best(first, lists, keep, ranked, [&](int i, const Entry &e, int better) {
        if (better < keep) list_of[better] = i;
        if (better == keep - 1) enough = e.total;
    });
    __syncthreads();
    if (lists < keep) {
        // of few lists entry `deep` - 1 of the `deep`-th part of `keep` lists
        const int deep = (keep + lists - 1) / lists, part = (keep + deep - 1) / deep;
        if (tid < lists) pair[tid] = entry(tid, deep - 1, best[(row0 * chunks + tid) * keep + deep - 1]);
        __syncthreads();
        rank_entries<JOIN>(pair, lists, [&](int, const Entry &e, int better) {
            if (e.total && better == part - 1) enough = e.total;
        });
        __syncthreads();
    }
    for (int at = tid; at < keep * keep; at += JOIN) {
        const int r = at / keep, p = at - r * keep, list = list_of[r];
        if (r + p >= keep) continue;
        const Entry e = list >= 0 ? entry(list, p, best[(row0 * chunks + list) * keep + p]) : NO_ENTRY;
        if (e.total && e.total >= enough) pair[atomicAdd(&there, 1)] = e;              // (in any order: they are ranked)
    }
    __syncthreads();
    const size_t to = (size_t)b * keep;
    rank_best(pair, there, keep, ranked, [&](int, const Entry &e, int better) {
        if (better >= keep) return;
        const int r = (int)(e.then >> 52);
        out[to + better] = (float)total_of(e);
        parents[to + better] = (int)row0 + r;
        tokens[to + better] = done[r] ? end : (int)(e.then & 0xfffff);
    });
    if (tid < keep && tid >= there) {
        out[to + tid] = -INFINITY;
        parents[to + tid] = tokens[to + tid] = -1;
    }
}

template <int T, int THREADS, int VECTORS>
void pieces(const void *logits, long ld, const float *scores, const uint8_t *finished, int rows, int vocab, int keep, int chunks, BlockSum *sums, Candidate *best,
            hipStream_t st)
{
    auto kern = keep <= 16 ? beam_pieces_kernel<T, THREADS, VECTORS, 64> : beam_pieces_kernel<T, THREADS, VECTORS, 256>;
    hipLaunchKernelGGL(kern, dim3((unsigned)(rows * chunks)), dim3(THREADS), 0, st, (const char *)logits, ld, scores, finished,
                       vocab, keep, chunks, sums, best);
}
template <int T>
void pieces(const void *logits, long ld, const float *scores, const uint8_t *finished, int rows, int vocab, int keep, BeamCut cut, BlockSum *sums, Candidate *best,
            hipStream_t st)
{
    if (cut.large) pieces<T, LONG_PIECE.threads, LONG_PIECE.vectors>(logits, ld, scores, finished, rows, vocab, keep, cut.chunks, sums, best, st);
    else pieces<T, SHORT_PIECE.threads, SHORT_PIECE.vectors>(logits, ld, scores, finished, rows, vocab, keep, cut.chunks, sums, best, st);
}

}  // namespace

BeamCut beam_cut(int type, int rows, int vocab)
{
    const bool wide = type == F32, large = long_pieces(wide, rows, vocab);
    const BeamPiece piece = large ? LONG_PIECE : SHORT_PIECE;
    const int chunks = piece_chunks(piece, wide, vocab);
    return BeamCut{large, chunks, chunks * (piece.threads * piece.vectors / 64 / BLOCK_OF)};
}

size_t beam_workspace(int type, int batch, int beams, int vocab, int keep)
{
    const BeamCut cut = beam_cut(type, batch * beams, vocab);
    return (size_t)batch * beams * (cut.blocks * sizeof(BlockSum) + (size_t)cut.chunks * keep * sizeof(Candidate));
}

hipError_t launch_beam_select(const void *logits, long ld, int type, const float *scores, const uint8_t *finished, int end, int batch, int beams, int vocab, int keep,
                              float *best, int *parents, int *tokens, void *ws, hipStream_t st)
{
    const BeamCut cut = beam_cut(type, batch * beams, vocab);
    const int rows = batch * beams;
    Candidate *const candidates = static_cast<Candidate *>(ws);
    BlockSum *const sums = reinterpret_cast<BlockSum *>(candidates + (size_t)rows * cut.chunks * keep);
    if (type == F16) pieces<F16>(logits, ld, scores, finished, rows, vocab, keep, cut, sums, candidates, st);
    else if (type == BF16) pieces<BF16>(logits, ld, scores, finished, rows, vocab, keep, cut, sums, candidates, st);
    else pieces<F32>(logits, ld, scores, finished, rows, vocab, keep, cut, sums, candidates, st);
    if (hipError_t err = hipGetLastError()) return err;               // (the join reads what they wrote)
    const size_t lds = sizeof(Entry) * ((size_t)beams * cut.chunks + (size_t)keep * (keep + 1) / 2);
    if (lds > 56 << 10)
        if (hipError_t err = hipFuncSetAttribute((const void *)beam_join_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) return err;
    hipLaunchKernelGGL(beam_join_kernel, dim3((unsigned)batch), dim3(JOIN), lds, st, sums, candidates, scores, finished, end, beams, keep, cut.chunks, cut.blocks, best, parents,
                       tokens);
    return hipGetLastError();
}

}  // namespace samp

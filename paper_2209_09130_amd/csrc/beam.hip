// Beam search's selection: the best (score, beam, token) of each sequence over the logits of its beams, total = score + logit - log sum exp logits.
//
// Two launches.  The first reads every logit once: a block takes a piece of a row into registers, finds its largest value, the sum of exponentials under it and its `keep` best
// logits: totals of a row are in the order of its logits.  The second joins the pieces of a sequence's rows in binary64 and picks among them.
//
// The best of a piece are found by their order as integers: a key holds a logit (as a whole number of the same order) above its index, so keys differ, and the lower
// index wins among equal logits.  The `keep`-th largest of the threads' own best keys is no more than the `keep`-th largest of all, and no more than `keep` threads have a key that reaches
// it: only their registers are looked through again.
#include "../../include/samp.h"
#include "decoder.h"

#include <type_traits>

namespace samp {
namespace {

constexpr int THREADS = 256;
// log2(e) in two parts
constexpr double LOG2E = 1.44269504088896340736;
constexpr float LOG2E_HI = (float)LOG2E, LOG2E_LO = (float)(LOG2E - (double)LOG2E_HI);

enum { F16 = 0, BF16 = 1, F32 = 2 };
template <int T> struct Logit {
    static constexpr int SIZE = T == F32 ? 4 : 2, VEC = 16 / SIZE;
    typedef typename std::conditional<T == F32, int64_t, int32_t>::type Key;
    static constexpr Key NONE = T == F32 ? (Key)INT64_MIN : (Key)INT32_MIN;
    static constexpr int SHIFT = T == F32 ? 32 : 16;
    static constexpr int MINUS_INF = T == F16 ? -0x7c00 : T == BF16 ? -0x7f80 : -0x7f800000;
    static constexpr unsigned MINUS_INF_BITS = T == F16 ? 0xfc00u : T == BF16 ? 0xff80u : 0xff800000u;
    // a value's bits as a whole number of the same order (both zeros are 0), and back
    static __device__ __forceinline__ int order(unsigned bits)
    {
        if constexpr (T == F32) {
            const int s = (int)bits >> 31;
            return ((int)bits ^ (s & 0x7fffffff)) - s;
        } else {
            const int v = (int16_t)bits, s = v >> 15;
            return (v ^ (s & 0x7fff)) - s;
        }
    }
    static __device__ __forceinline__ float value_of_order(int t)
    {
        const unsigned m = (unsigned)(t < 0 ? -t : t);
        if constexpr (T == F32) return __uint_as_float(t < 0 ? m | 0x80000000u : m);
        else return value(t < 0 ? m | 0x8000u : m);
    }
    static __device__ __forceinline__ float value(unsigned bits)
    {
        if constexpr (T == F32) return __uint_as_float(bits);
        else if constexpr (T == BF16) return __uint_as_float(bits << 16);
        else return (float)__builtin_bit_cast(_Float16, (unsigned short)bits);
    }
    static __device__ __forceinline__ unsigned bits(const v4i &raw, int e)
    {
        if constexpr (T == F32) return (unsigned)raw[e];
        else return (unsigned)raw[e >> 1] >> 16 * (e & 1) & 0xffffu;
    }
    static __device__ __forceinline__ Key key(unsigned bits, int index)
    {
        if constexpr (T == F32) return (Key)order(bits) * ((Key)1 << 32) + (Key)(uint32_t)~index;
        else return (Key)((unsigned)order(bits) << 16 | (0xffffu - (unsigned)index));
    }
    static __device__ __forceinline__ int order_of(Key k) { return (int)(k >> SHIFT); }
    static __device__ __forceinline__ int index_of(Key k)
    {
        if constexpr (T == F32) return (int)~(uint32_t)k;
        else return (int)(0xffffu - ((unsigned)k & 0xffffu));
    }
};

struct Candidate { float logit; int token; };                         // token -1: none
struct PieceSum { float top, sum; };                                  // sum of exp(x - top)

__device__ __forceinline__ bool row_counts(const float *scores, const uint8_t *finished, int row)
{
    return __builtin_isfinite(scores[row]) && !(finished && finished[row]);
}

// One piece of one row.  Vectors of 16 bytes are numbered from the aligned address at or before the row's first value; what of them lies outside the row counts as minus infinity.
template <int T, int VECTORS>
__global__ __launch_bounds__(THREADS) void beam_pieces_kernel(const char *__restrict__ logits, long ld, const float *__restrict__ scores,
                                                              const uint8_t *__restrict__ finished, int vocab, int keep, int chunks,
                                                              PieceSum *__restrict__ sums, Candidate *__restrict__ best)
{
    typedef Logit<T> L;
    typedef typename L::Key Key;
    constexpr int PER = VECTORS * L::VEC;                             // values of a thread
    extern __shared__ __attribute__((aligned(16))) char shared[];
    v4i *const held = reinterpret_cast<v4i *>(shared);                // [keep][VECTORS]: registers of the threads that are looked through
    Key *const list = reinterpret_cast<Key *>(shared + (size_t)keep * VECTORS * 16);         // [keep * PER]
    __shared__ Key tops[THREADS];
    __shared__ int owner[SAMP_MAX_KEEP];
    __shared__ Key wave_top[4];
    __shared__ float wave_part[4];
    __shared__ Key least;
    __shared__ int listed;

    const int row = blockIdx.x / chunks, piece = blockIdx.x - row * chunks;
    if (!row_counts(scores, finished, row)) return;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const char *from = logits + (size_t)row * ld * L::SIZE;
    const int phase = (int)(reinterpret_cast<uintptr_t>(from) & 15) / L::SIZE;
    const int first = piece * THREADS * PER - phase;                  // token of the piece's first place

    v4i raw[VECTORS];
#pragma unroll
    for (int i = 0; i < VECTORS; i++) {
        const int at = first + (i * THREADS + tid) * L::VEC;
        if (at >= 0 && at + L::VEC <= vocab) raw[i] = *reinterpret_cast<const v4i *>(from + (long)at * L::SIZE);
        else {
            unsigned x[L::VEC];
#pragma unroll
            for (int e = 0; e < L::VEC; e++) {
                x[e] = L::MINUS_INF_BITS;
                if (at + e >= 0 && at + e < vocab) {
                    if constexpr (T == F32) x[e] = *reinterpret_cast<const unsigned *>(from + (long)(at + e) * 4);
                    else x[e] = *reinterpret_cast<const unsigned short *>(from + (long)(at + e) * 2);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; e++) raw[i][e] = T == F32 ? (int)x[e] : (int)(x[(2 * e) % L::VEC] | x[(2 * e + 1) % L::VEC] << 16);
        }
    }
    Key top = L::NONE;
#pragma unroll
    for (int i = 0; i < VECTORS; i++)
#pragma unroll
        for (int e = 0; e < L::VEC; e++) top = max(top, L::key(L::bits(raw[i], e), (i * THREADS + tid) * L::VEC + e));
    tops[tid] = top;
    Key most = top;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) most = max(most, (Key)__shfl_xor(most, o, 64));
    if (lane == 0) wave_top[w] = most;
    if (tid == 0) {
        least = L::NONE;
        listed = 0;
    }
    if (tid < keep) owner[tid] = -1;
    __syncthreads();
    most = max(max(wave_top[0], wave_top[1]), max(wave_top[2], wave_top[3]));
    // (NaN of negative sign lie below, of positive sign above all numbers)
    const float m = L::order_of(most) > L::MINUS_INF ? L::value_of_order(L::order_of(most)) : 0.0f;

    // how many threads have a better key: the first `keep` of them are looked through
    if (L::order_of(top) > L::MINUS_INF) {
        int better = 0;
        for (int i = 0; i < THREADS; i++) better += tops[i] > top;
        if (better < keep) {
            owner[better] = tid;
#pragma unroll
            for (int i = 0; i < VECTORS; i++) held[better * VECTORS + i] = raw[i];
            if (better == keep - 1) least = top;
        }
    }
    float part[4] = {};
#pragma unroll
    for (int i = 0; i < VECTORS; i++)
#pragma unroll
        for (int e = 0; e < L::VEC; e++) {
            const float d = L::value(L::bits(raw[i], e)) - m;          // (logits of the type's lowest value alone: zeros)
            part[e & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(d, LOG2E_HI, d * LOG2E_LO));
        }
    float sum = (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) wave_part[w] = sum;
    __syncthreads();
    if (tid == 0) sums[blockIdx.x] = PieceSum{m, (wave_part[0] + wave_part[1]) + (wave_part[2] + wave_part[3])};

    for (int at = tid; at < keep * PER; at += THREADS) {
        const int slot = at / PER, who = owner[slot];
        if (who < 0) continue;
        const int i = at % PER / L::VEC, e = at % L::VEC;
        unsigned b;
        if constexpr (T == F32) b = (unsigned)reinterpret_cast<const int *>(held)[(slot * VECTORS + i) * 4 + e];
        else b = reinterpret_cast<const unsigned short *>(held)[(slot * VECTORS + i) * 8 + e];
        const Key k = L::key(b, (i * THREADS + who) * L::VEC + e);
        if (k >= least && L::order_of(k) > L::MINUS_INF) list[atomicAdd(&listed, 1)] = k;     // (in any order: they are ranked)
    }
    __syncthreads();
    const int n = listed;
    Candidate *const to = best + (size_t)blockIdx.x * keep;
    for (int at = tid; at < n; at += THREADS) {
        const Key k = list[at];
        int better = 0;
        for (int i = 0; i < n; i++) better += list[i] > k;
        if (better < keep) to[better] = Candidate{L::value_of_order(L::order_of(k)), first + L::index_of(k)};
    }
    if (tid < keep && tid >= n) to[tid] = Candidate{-INFINITY, -1};
}

// One sequence.  The pieces' lists are sorted: entry p of the list whose first entry is the r-th best of all first entries can be among the `keep` best only where r + p < keep, and those
// keep (keep + 1) / 2 are ranked by counting.  place = beam << 20 | token.
struct __attribute__((aligned(16))) Entry { double total; float logit; int place; };
constexpr Entry NONE{-INFINITY, 0.0f, INT32_MAX};
__device__ __forceinline__ bool before(const Entry &a, const Entry &b)
{
    if (a.total != b.total) return a.total > b.total;
    const bool one_row = (a.place ^ b.place) >> 20 == 0;
    return one_row && a.logit != b.logit ? a.logit > b.logit : a.place < b.place;
}

__global__ __launch_bounds__(THREADS) void beam_join_kernel(const PieceSum *__restrict__ sums, const Candidate *__restrict__ best, const float *__restrict__ scores,
                                                            const uint8_t *__restrict__ finished, int end, int beams, int keep, int chunks,
                                                            float *__restrict__ out, int *__restrict__ parents, int *__restrict__ tokens)
{
    extern __shared__ __attribute__((aligned(16))) char shared[];
    const int lists = beams * chunks, pairs = keep * (keep + 1) / 2;
    Entry *const first = reinterpret_cast<Entry *>(shared), *const pair = first + lists;
    __shared__ double lse[SAMP_MAX_BEAMS];                            // log sum exp; NaN where a row's logits have no candidates
    __shared__ int list_of[SAMP_MAX_KEEP];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    for (int r = w; r < beams; r += THREADS / 64) {
        const int row = b * beams + r;
        double o = __builtin_nan("");
        if (row_counts(scores, finished, row)) {
            float top = -INFINITY;
            for (int c = lane; c < chunks; c += 64) {
                const PieceSum p = sums[(size_t)row * chunks + c];
                if (!(p.sum == 0.0f)) top = __builtin_fmaxf(top, p.top);
            }
            top = wave_max(top);
            double sum = 0.0;
            for (int c = lane; c < chunks; c += 64) {
                const PieceSum p = sums[(size_t)row * chunks + c];
                if (!(p.sum == 0.0f)) sum += (double)p.sum * exp((double)p.top - (double)top);
            }
            sum = wave_sum(sum);
            // (no finite logit: a sum of 0; NaN or plus infinity: a sum of NaN)
            if (sum > 0.0) o = (double)top + log(sum);
        }
        if (lane == 0) lse[r] = o;
    }
    if (tid < keep) list_of[tid] = -1;
    __syncthreads();
    auto entry = [&](int list, int p) {
        const int r = list / chunks, c = list - r * chunks, row = b * beams + r;
        Entry e = NONE;
        if (finished && finished[row]) {
            const float s = scores[row];
            if (c == 0 && p == 0 && __builtin_isfinite(s)) e = Entry{(double)s, 0.0f, r << 20};
        } else if (__builtin_isfinite(lse[r])) {
            const Candidate x = best[((size_t)row * chunks + c) * keep + p];
            if (x.token >= 0) e = Entry{(double)scores[row] + ((double)x.logit - lse[r]), x.logit, r << 20 | x.token};
        }
        return e;
    };
    for (int i = tid; i < lists; i += THREADS) first[i] = entry(i, 0);
    __syncthreads();
    for (int i = tid; i < lists; i += THREADS) {
        const Entry e = first[i];
        if (e.place == INT32_MAX) continue;
        int better = 0;
        for (int j = 0; j < lists; j++) better += before(first[j], e);
        if (better < keep) list_of[better] = i;
    }
    __syncthreads();
    for (int at = tid; at < keep * keep; at += THREADS) {
        const int r = at / keep, p = at - r * keep;
        if (r + p >= keep) continue;
        pair[r * keep - r * (r - 1) / 2 + p] = list_of[r] >= 0 ? entry(list_of[r], p) : NONE;
    }
    __syncthreads();
    int there = 0;
    for (int i = 0; i < pairs; i++) there += pair[i].place != INT32_MAX;
    for (int i = tid; i < pairs; i += THREADS) {
        const Entry e = pair[i];
        if (e.place == INT32_MAX) continue;
        int better = 0;
        for (int j = 0; j < pairs; j++) better += before(pair[j], e);
        if (better < keep) {
            const int r = e.place >> 20, row = b * beams + r;
            out[(size_t)b * keep + better] = (float)e.total;
            parents[(size_t)b * keep + better] = row;
            tokens[(size_t)b * keep + better] = finished && finished[row] ? end : e.place & 0xfffff;
        }
    }
    for (int i = tid; i < keep; i += THREADS)
        if (i >= there) {
            out[(size_t)b * keep + i] = -INFINITY;
            parents[(size_t)b * keep + i] = tokens[(size_t)b * keep + i] = -1;
        }
}

int values_of(int type, int vectors) { return THREADS * vectors * (type == F32 ? 4 : 8); }

template <int T>
void pieces(const void *logits, long ld, const float *scores, const uint8_t *finished, int rows, int vocab, int keep, BeamCut cut, PieceSum *sums, Candidate *best,
            hipStream_t st)
{
    auto kern = cut.vectors == 8 ? beam_pieces_kernel<T, 8> : beam_pieces_kernel<T, 2>;
    const size_t lds = (size_t)keep * cut.vectors * (16 + Logit<T>::VEC * sizeof(typename Logit<T>::Key));
    hipLaunchKernelGGL(kern, dim3((unsigned)(rows * cut.chunks)), dim3(THREADS), lds, st, (const char *)logits, ld, scores, finished, vocab, keep, cut.chunks, sums, best);
}

}  // namespace

BeamCut beam_cut(int type, int rows, int vocab)
{
    const int phase = (type == F32 ? 4 : 8) - 1;                      // places that a row may begin behind an aligned address
    auto chunks = [&](int vectors) { return (vocab + phase + values_of(type, vectors) - 1) / values_of(type, vectors); };
    const int vectors = (long)rows * chunks(8) >= 512 ? 8 : 2;
    return BeamCut{vectors, chunks(vectors)};
}

size_t beam_workspace(int type, int batch, int beams, int vocab, int keep)
{
    const BeamCut cut = beam_cut(type, batch * beams, vocab);
    return (size_t)batch * beams * cut.chunks * (sizeof(PieceSum) + (size_t)keep * sizeof(Candidate));
}

hipError_t launch_beam_select(const void *logits, long ld, int type, const float *scores, const uint8_t *finished, int end, int batch, int beams, int vocab, int keep,
                              float *best, int *parents, int *tokens, void *ws, hipStream_t st)
{
    const BeamCut cut = beam_cut(type, batch * beams, vocab);
    Candidate *const candidates = static_cast<Candidate *>(ws);
    PieceSum *const sums = reinterpret_cast<PieceSum *>(candidates + (size_t)batch * beams * cut.chunks * keep);
    if (type == F16) pieces<F16>(logits, ld, scores, finished, batch * beams, vocab, keep, cut, sums, candidates, st);
    else if (type == BF16) pieces<BF16>(logits, ld, scores, finished, batch * beams, vocab, keep, cut, sums, candidates, st);
    else pieces<F32>(logits, ld, scores, finished, batch * beams, vocab, keep, cut, sums, candidates, st);
    const size_t lds = sizeof(Entry) * ((size_t)beams * cut.chunks + (size_t)keep * (keep + 1) / 2);
    if (lds > 64 << 10)
        if (hipError_t e = hipFuncSetAttribute((const void *)beam_join_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) return e;
    hipLaunchKernelGGL(beam_join_kernel, dim3((unsigned)batch), dim3(THREADS), lds, st, sums, candidates, scores, finished, end, beams, keep, cut.chunks, best, parents,
                       tokens);
    return hipGetLastError();
}

}  // namespace samp

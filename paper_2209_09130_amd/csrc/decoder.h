// What the kernels of the 8-bit decoder's operators share: their 16-bit types, the quantiser of a row, the cache's geometry, and the launchers
// behind the C ABI's decoder entry points (api_decoder.hip).
#pragma once
#include "samp_common.h"

#include <type_traits>

namespace samp {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// Eight 16-bit values of a 16-byte load as binary32, and back (one rounding, to nearest even)
template <bool BF> __device__ __forceinline__ void widen8(const v4i &raw, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const unsigned u = (unsigned)raw[i];
        if constexpr (BF) {
            x[2 * i] = __uint_as_float(u << 16);
            x[2 * i + 1] = __uint_as_float(u & 0xffff0000u);
        } else {
            x[2 * i] = (float)__builtin_bit_cast(_Float16, (unsigned short)u);
            x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (unsigned short)(u >> 16));
        }
    }
}
template <bool BF> __device__ __forceinline__ int narrow2(float lo, float hi)
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef typename std::conditional<BF, __bf16, _Float16>::type half2 __attribute__((ext_vector_type(2)));
    asm("" : "+v"(lo), "+v"(hi));
    return __builtin_bit_cast(int, __builtin_convertvector((v2f{lo, hi}), half2));          // one instruction
}

// A barrier for what the threads of a block hand each other in LDS: loads from memory and stores to it stay on their way
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// the sum of the lanes up to this one (row shifts, then the last lanes of rows 0 and 2, then of row 1)
__device__ __forceinline__ int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// The largest, the smallest of three.  (The compiler's own quiet signalling NaN in front: another instruction each.)  A lane exchange that reads a result has to wait two states, for which the compiler
// does not look into asm where the exchange is a swap of halves: settle() in front of those.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float min3(float a, float b, float c)
{
    float r;
    asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ void settle(float &a, float &b) { asm("s_nop 1" : "+v"(a), "+v"(b)); }
__device__ __forceinline__ void settle(float &a, float &b, float &c, float &d) { asm("s_nop 1" : "+v"(a), "+v"(b), "+v"(c), "+v"(d)); }
// of the first M
template <int M, int N> __device__ __forceinline__ void settle(float (&x)[N])
{
    static_assert(M <= N && (M == 1 || M == 2 || M % 4 == 0), "one, two or fours");
    if constexpr (M <= 2) settle(x[0], x[M - 1]);
    else
#pragma unroll
        for (int i = 0; i < M; i += 4) settle(x[i], x[i + 1], x[i + 2], x[i + 3]);
}
template <int CTRL> __device__ __forceinline__ float other_lane(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true)); }
// Lanes l and l ^ HALF of two values: the lower of the two lanes gets the first value of both, the upper the second
struct Met { float x, y; };
template <int HALF> __device__ __forceinline__ Met meet(float a, float b, int lane)
{
    if constexpr (HALF == 32) {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return Met{__uint_as_float(both[0]), __uint_as_float(both[1])};
    } else if constexpr (HALF == 16) {
        const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return Met{__uint_as_float(both[0]), __uint_as_float(both[1])};
    } else {
        const bool upper = lane & HALF;
        const int give = __float_as_int(upper ? a : b);
        return Met{upper ? b : a, __int_as_float(HALF == 8 ? __builtin_amdgcn_update_dpp(0, give, 0x128, 0xf, 0xf, true) : __builtin_amdgcn_ds_swizzle(give, HALF << 10 | 0x1f))};
    }
}

// A whole number of the order of the values, the two zeros the same (not for NaN), and back: numbers outside the infinities' are NaN, which nothing reaches
__device__ __forceinline__ unsigned order_of(float x)
{
    const unsigned u = __float_as_uint(x + 0.0f);
    return u >> 31 ? ~u : u | 1u << 31;
}
__device__ __forceinline__ float value_of_order(unsigned t) { return __uint_as_float(t >> 31 ? t & 0x7fffffffu : ~t); }

// The largest magnitude of 16-bit values, by their bits (two running maxima, in the halves of a dword): infinities come above every number and NaN above them
typedef unsigned short v2u16 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned max_halves(unsigned a, unsigned b)
{ return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(v2u16, a), __builtin_bit_cast(v2u16, b))); }
__device__ __forceinline__ unsigned bits_max16(const v4i &raw)
{
    const unsigned M = 0x7fff7fffu;
    return max_halves(max_halves((unsigned)raw[0] & M, (unsigned)raw[1] & M), max_halves((unsigned)raw[2] & M, (unsigned)raw[3] & M));
}
// over sixteen lanes (row rotations) or all 64 of the wave; then of the two halves
__device__ __forceinline__ unsigned max_of_16_lanes(unsigned top)
{
    top = max_halves(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0x128, 0xf, 0xf, true));
    top = max_halves(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0x124, 0xf, 0xf, true));
    top = max_halves(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0x122, 0xf, 0xf, true));
    top = max_halves(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0x121, 0xf, 0xf, true));
    return max(top & 0xffffu, top >> 16);
}
__device__ __forceinline__ unsigned max_of_wave(unsigned top)
{
    top = max_of_16_lanes(top);
    top = max(top, (unsigned)__shfl_xor((int)top, 16, 64));
    return max(top, (unsigned)__shfl_xor((int)top, 32, 64));
}

// The quantiser of a row that brings its own step: step = absmax / 127 and code = 127 x / absmax rounded half to even, decided exactly.  127 x / absmax is
// a quotient of short integers: where it is no tie it is further than 2^-19 of itself from one (254 x is at least one unit from an odd multiple of absmax, x has 11 bits), so
// a product with a relative error of 2^-28 that is rounded to binary32 lies on the right side, and a tie is a binary32 number, to which it rounds.  The reciprocal therefore comes in two parts, an approximate one and what it
// leaves; so does 1 / 127 (quotients by 127 have bits of period seven: none is near a rounding boundary).  True divisions in their place made the cache's
// writing 30 % longer: every lane of a row forms them.
// A row without a number of at least 2^-60 is a row of zeros (step 1, as for a weight row of zeros); a row with an infinity or NaN has codes 0 and a step of
// NaN, so that what is computed from it is NaN as well.
struct RowQuant { float step, hi, lo; bool finite; };
template <bool BF> __device__ __forceinline__ RowQuant row_quant(unsigned absmax_bits)
{
    const float top = BF ? __uint_as_float(absmax_bits << 16) : (float)__builtin_bit_cast(_Float16, (unsigned short)absmax_bits);
    RowQuant q;
    q.finite = absmax_bits < (BF ? 0x7f80u : 0x7c00u);
    const bool some = q.finite && top >= 0x1p-60f;
    const float t = some ? top : 1.0f, m = __builtin_amdgcn_frexp_mantf(t), inverse = __builtin_amdgcn_rcpf(m), hi = 127.0f * inverse;
    const int down = -__builtin_amdgcn_frexp_expf(t);
    q.hi = some ? __builtin_amdgcn_ldexpf(hi, down) : 0.0f;
    q.lo = some ? __builtin_amdgcn_ldexpf(__builtin_fmaf(-hi, m, 127.0f) * inverse, down) : 0.0f;
    constexpr double C = 1.0 / 127.0;
    constexpr float CH = (float)C, CL = (float)(C - (double)CH);
    q.step = !q.finite ? __builtin_nanf("") : some ? __builtin_fmaf(top, CH, top * CL) : 1.0f;
    return q;
}
// eight codes; |127 x / absmax| <= 127, so adding 1.5 * 2^23 leaves the code in the low byte without a clamp
__device__ __forceinline__ v2i quant8(const float (&x)[8], const RowQuant &q)
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = __builtin_fmaf(x[i], q.hi, x[i] * q.lo) + SAMP_RNE_MAGIC;
    v2i c = {pack_codes(f[0], f[1], f[2], f[3]), pack_codes(f[4], f[5], f[6], f[7])};
    if (!q.finite) c = v2i{0, 0};
    return c;
}

// The cache: codes [pages, kv_heads, page_len, head_dim], steps [pages, kv_heads, page_len]; page_len a power of two, 16 or more
struct KvCache { int8_t *k, *v; float *k_step, *v_step; int pages, kv_heads, page_shift; };
// Which positions of which sequences the packed rows of a call are: rows cu[b] .. cu[b + 1] - 1 (cu null: max_rows each) are the last of the lens[b]
// positions of sequence b, whose pages are row b of the table
// (tables: 1, or kv_heads where each key head has a table of its own, behind each other for a sequence; only the attention reads such)
struct KvRows { const int *table; int width; const int *cu, *lens; int batch, max_rows, rows, tables = 1; };
// Bounds of the keys of a page: codes [pages, kv_heads, 2, head_dim] (largest, smallest), steps [pages, kv_heads]
struct KeyBounds { int8_t *codes; float *steps; };

// n = 0 where cu names rows that the tensors do not have; todo: those of the n that the caller counted with; len: at most what the table has room for
struct SeqRows { int first_row, n, todo, len; };
__device__ __forceinline__ SeqRows seq_rows(const KvRows &r, int b, int page_shift)
{
    SeqRows s;
    s.first_row = r.cu ? r.cu[b] : b * r.max_rows;
    s.n = (r.cu ? r.cu[b + 1] : s.first_row + r.max_rows) - s.first_row;
    if (s.first_row < 0 || s.n < 0 || s.first_row > r.rows - s.n) s.n = 0;
    s.todo = min(s.n, r.max_rows);
    const long room = (long)r.width << page_shift;
    s.len = r.lens[b];
    if (s.len > room) s.len = (int)room;
    return s;
}

hipError_t launch_quantize_tokens(const void *x, long ldx, bool bf16, int M, int K, int8_t *codes, float *steps, hipStream_t st);
hipError_t launch_gemm_i8_tokens(const int8_t *codes, const float *steps, const int8_t *Wp, const float *s_w, const float *bias, bool gelu, void *out,
                                 bool bf16, int M, int N, int K, hipStream_t st);
// both in one launch (tokens_fused())
hipError_t launch_linear_few(const void *x, long ldx, bool bf16, const int8_t *Wp, const float *s_w, const float *bias, bool gelu, void *out, int M, int N, int K,
                             hipStream_t st);
hipError_t launch_cache_write(const KvCache &cache, const void *k, long ldk, const void *v, long ldv, bool bf16, int head_dim, const KvRows &rows,
                              hipStream_t st);
hipError_t launch_cache_read(const KvCache &cache, void *k, void *v, bool bf16, int head_dim, const KvRows &rows, hipStream_t st);
// how a call cuts contexts: pieces of so many tiles of 32 keys, at most `splits` of them, each with a partial result in the workspace if there are several
struct Cut { int splits, piece; };
Cut cached_attention_cut(int batch, int heads, int kv_heads, int max_new, int max_len);
hipError_t launch_cached_attention(const void *q, long ldq, bool bf16, int heads, int head_dim, const KvCache &cache, const KvRows &rows, float scale,
                                   const uint64_t *tree, Cut cut, float *partials, void *out, hipStream_t st);
hipError_t launch_causal_attention(const void *q, long ldq, const void *k, long ldk, const void *v, long ldv, bool bf16, int heads, int kv_heads,
                                   int head_dim, const int *cu, int batch, int max_len, int rows, float scale, void *out, hipStream_t st);

// Beam search: type as in samp.h; the bytes of the workspace follow from how a row is cut
struct BeamCut { bool large; int chunks, blocks; };                   // kind and number of a row's pieces; blocks whose exponentials are summed
BeamCut beam_cut(int type, int rows, int vocab);
size_t beam_workspace(int type, int batch, int beams, int vocab, int keep);
hipError_t launch_beam_select(const void *logits, long ld, int type, const float *scores, const uint8_t *finished, int end, int batch, int beams, int vocab, int keep,
                              float *best, int *parents, int *tokens, void *ws, hipStream_t st);

// Pages: row i of `to` continues row parents[i] of `from`
struct PageFork {
    const int *refs, *table, *lens, *parents, *cu;
    int pages, rows_from, width, page_shift, max_new, rows;
    int *refs_out, *table_out, *lens_out, *copies, *lacking;
};
size_t pages_fork_workspace(int pages, int rows_from, int width, int rows);
hipError_t launch_pages_fork(const PageFork &f, void *ws, hipStream_t st);
size_t pages_compact_workspace(int pages, int entries);
hipError_t launch_pages_compact(const int *refs, int pages, const int *table, int entries, int page_len, int *refs_out, int *table_out, int *copies, int *used, void *ws,
                                hipStream_t st);
hipError_t launch_cache_copy(const KvCache &cache, int head_dim, const KeyBounds &bounds, const int *copies, int n, hipStream_t st);

hipError_t launch_cache_bounds(const KvCache &cache, int head_dim, const KeyBounds &bounds, const KvRows &rows, hipStream_t st);
size_t cache_select_workspace(int batch, int kv_heads, int width);
hipError_t launch_cache_select(const void *q, long ldq, bool bf16, int heads, int head_dim, const KvCache &cache, const KeyBounds &bounds, const KvRows &rows, int keep,
                               int sinks, int recent, int *tables, int *lens_out, void *ws, hipStream_t st);

}  // namespace samp

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

// The larger of two magnitudes of 16-bit values, by their bits: infinities come above every number and NaN above them
__device__ __forceinline__ unsigned bits_max16(const v4i &raw)
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) m = max(m, max((unsigned)raw[i] & 0x7fffu, ((unsigned)raw[i] >> 16) & 0x7fffu));
    return m;
}

// The quantiser of a row that brings its own step: step = absmax / 127 and code = 127 x / absmax rounded half to even, decided exactly.  127 x / absmax is
// a quotient of short integers: where it is no tie it is further than 2^-12 from one, so a product with error 2^-40 that is rounded to binary32
// lies on the right side, and a tie is a binary32 number, to which it rounds.  The reciprocal therefore comes in two parts.
// A row without a number of at least 2^-60 is a row of zeros (step 1, as for a weight row of zeros); a row with an infinity or NaN has codes 0 and a step of
// NaN, so that what is computed from it is NaN as well.
struct RowQuant { float step, hi, lo; bool finite; };
template <bool BF> __device__ __forceinline__ RowQuant row_quant(unsigned absmax_bits)
{
    const float top = BF ? __uint_as_float(absmax_bits << 16) : (float)__builtin_bit_cast(_Float16, (unsigned short)absmax_bits);
    RowQuant q;
    q.finite = absmax_bits < (BF ? 0x7f80u : 0x7c00u);
    const bool some = q.finite && top >= 0x1p-60f;
    const float t = some ? top : 1.0f;
    q.hi = __fdiv_rn(127.0f, t);
    q.lo = __fdiv_rn(__builtin_fmaf(-q.hi, t, 127.0f), t);
    q.hi = some ? q.hi : 0.0f;
    q.lo = some ? q.lo : 0.0f;
    q.step = !q.finite ? __builtin_nanf("") : some ? __fdiv_rn(top, 127.0f) : 1.0f;
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
struct KvRows { const int *table; int width; const int *cu, *lens; int batch, max_rows, rows; };

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
// few rows: both in one launch
bool linear_tokens_is_fused(int M, int K);
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

}  // namespace samp

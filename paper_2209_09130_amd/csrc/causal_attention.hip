// Causal attention over packed prompts with grouped heads: O = softmax(scale q K^T) V, a query sees the keys of its sequence up to itself.
//
// What bounds it is the matrix cores, with the softmax's vector work close behind: 4 head_dim operations per (query, key) pair on the one side, some ten
// vector operations and an exponential on the other.  A wave owns 32 queries for the whole loop and keeps them, their output (as O^T) and the softmax in
// registers: S^T = K Q^T leaves a lane one query and 32 of a tile's 64 keys, and what it makes of them is, as it stands, the operand of
// O^T += V^T P^T.  The key tiles (64 keys, K and V) are shared by the block's waves: direct loads into one half of LDS while the other is worked on, V
// transposed by the reads.  One pass, with a reference per query that moves (and rescales) only when a score exceeds it by 2^8.
// Two documents of 8192 tokens, 32 query heads on 8 key heads of 128: fp16 1.03 to 1.08 ms between cards (1.01 to 1.06 PFLOP/s), bfloat16 0.99 ms; torch's products of
// 8192 x 8192 x 8192 reach 1.23 to 1.26 and 1.47.  Eight of 300 to 2048, bfloat16: 142 us, 0.79 PFLOP/s: 6 % more products than needed, and a block holds 21 % more tiles than
// that for all its waves (long documents 1 % and 3 %): waves wait at the barrier where the diagonal or the sequence's end lies before the block's last.  The matrix cores are busy 58 % of the clocks (at 1.67 GHz: the chip is at its power limit), the vector ALUs nearly as long.  Tried and dropped: blocks
// of eight waves (long documents -1 to -3 %, eight of 300 to 2048 tokens +12 %), two groups of waves that alternate between products and softmax behind barriers (+12 %
// at head size 64, spills at 128), half tiles with the next scores' products dealt out between the exponentials (+11 % at 64, spills at 128), wave priorities
// (+-0), the sum of probabilities by dot products (+2 %).
// Rounding a probability to 16 bits is off by half a step of each, as the result's own rounding is.  The reference lies where the type's range is best used: in binary16
// 2^7 below the scores, so that probabilities run up to 2^15 and have all their bits down to 2^-21 of the largest (half a step is 2^-32 of it below), for
// the sake of rows whose largest probability falls on a key with little or no value; in bfloat16, whose range is binary32's, 2^24 above them, so that the sums of the largest
// values stay inside binary32.
//
// A key that a query does not see has no part in its result, whatever it holds.  On the diagonal the product multiplies such keys' V by a probability of 0,
// which an infinity or NaN survives; so a block with a result that is not finite goes over its tiles again, with V's infinities and NaN left out of the
// product on the diagonal and added to the queries that see them.
#include "decoder.h"
#include "mfma_tile.h"

namespace samp {
namespace {

constexpr float LOWEST = -3.0e38f, SLACK = 8.0f;
template <bool BF> constexpr float ABOVE = BF ? 24.0f : -7.0f;
constexpr int KEYS = 64;

template <bool BF> __device__ __forceinline__ v16f mma32(const v4i &a, const v4i &b, const v16f &c)
{
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// Positions of 16-byte chunks inside a row of a tile in LDS (D * 2 bytes a row).  K is read 16 bytes a lane, eight rows at a time over all banks; V by
// transposing reads, four rows of 64 bytes at a time.
template <int D> __device__ __forceinline__ int swz_k(int row) { return D == 128 ? row & 15 : swz<128>(row); }
template <int D> __device__ __forceinline__ int swz_v(int row) { return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; }

template <int OFFSET> __device__ __forceinline__ v2i lds_read_tr64(unsigned addr)
{
    v2i v;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFFSET));
    return v;
}

// Of two halves: bits 15 and 31 where one is an infinity or NaN (the exponent's carry); the pair with zeros in their place
template <bool BF> __device__ __forceinline__ unsigned odd_halves(int two)
{ return (((unsigned)two & 0x7fff7fffu) + (BF ? 0x00800080u : 0x04000400u)) & 0x80008000u; }
template <bool BF> __device__ __forceinline__ v4i without_odd(v4i v)
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const unsigned odd = odd_halves<BF>(v[i]);
        if (odd & 0x8000u) v[i] &= (int)0xffff0000u;
        if (odd >> 16) v[i] &= 0xffff;
    }
    return v;
}

template <int D, int NW> struct CausalTile {
    static constexpr int ROW = 2 * D, TILE = KEYS * ROW, STAGE = 2 * TILE;            // bytes; K then V
    static constexpr int LOADS = TILE / 1024 / NW;                                  // direct loads of a wave per tile and matrix
    static constexpr int OUT = 32 * (ROW + 16) * NW;                              // the output tile takes the ring's place
    static constexpr int LDS = 2 * STAGE > OUT ? 2 * STAGE : OUT;
};

template <bool BF, int D, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2)))
void causal_attention_kernel(const char *__restrict__ Q, const char *__restrict__ K, const char *__restrict__ V, long ldq, long ldk, long ldv,
                             const int *__restrict__ cu, int rows, int max_len, int heads, int group, int batch, int strips, float scale, char *__restrict__ out)
{
    typedef CausalTile<D, NW> T;
    constexpr int QB = 32 * NW, KS = D / 16, DB = D / 32;
    __shared__ __attribute__((aligned(1024))) char lds[T::LDS];

    // Strips of queries from the last (longest) to the first; a strip's heads, which have the same work, follow each other, so that the XCDs and their shader engines, to
    // which blocks go in turn, have the same share (sequences following each other, eight of 300 to 2048 tokens: 230 us, the engine that gets the long one's
    // blocks holds the others up).  Key heads run fastest: where they are a multiple of eight an XCD's L2 holds the keys of its own.
    const int kv_heads = heads / group, kvh = blockIdx.x % kv_heads;
    int rest = blockIdx.x / kv_heads;
    const int head = kvh * group + rest % group;
    rest /= group;
    const int b = rest % batch, strip = strips - 1 - rest / batch;
    const int t0 = cu ? cu[b] : b * max_len;
    int n = (cu ? cu[b + 1] : t0 + max_len) - t0;
    if (t0 < 0 || n < 0 || t0 > rows - n) return;                          // rows that the tensors do not have
    n = min(n, max_len);
    const int q0 = strip * QB;
    if (q0 >= n) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, g = lane >> 5;
    const int qw = q0 + 32 * w, wave_end = qw < n ? qw + 31 : -1;          // the wave's first query; its last, -1 if the sequence ends before it
    const unsigned ldkb = 2 * (unsigned)ldk, ldvb = 2 * (unsigned)ldv;
    const char *kbase = K + (size_t)t0 * ldkb + kvh * T::ROW, *vbase = V + (size_t)t0 * ldvb + kvh * T::ROW;

    v4i qf[KS];
    {
        const char *from = Q + 2 * ((size_t)(t0 + min(qw + r, n - 1)) * ldq + (size_t)head * D + 8 * g);
#pragma unroll
        for (int i = 0; i < KS; i++) qf[i] = *reinterpret_cast<const v4i *>(from + 32 * i);
    }
    // direct loads: a wave's j-th fills 1 KB, 1024 / ROW rows; past the sequence the descriptor makes them zeros
    constexpr int CH = T::ROW / 16, RPL = 64 / CH;                        // chunks of a row; rows of a load
    unsigned offk[T::LOADS], offv[T::LOADS];
#pragma unroll
    for (int j = 0; j < T::LOADS; j++) {
        const int row = (w * T::LOADS + j) * RPL + lane / CH, chunk = lane % CH;
        offk[j] = row * ldkb + ((chunk ^ swz_k<D>(row)) << 4);
        offv[j] = row * ldvb + ((chunk ^ swz_v<D>(row)) << 4);
    }
    auto request = [&](int tile, int buffer) {
        const int j0 = tile * KEYS, left = min(n - j0, KEYS);              // rows of the tile that are there
        const auto kr = buffer_of(kbase + (size_t)j0 * ldkb, (int)((left - 1) * ldkb + T::ROW));
        const auto vr = buffer_of(vbase + (size_t)j0 * ldvb, (int)((left - 1) * ldvb + T::ROW));
        char *to = lds + buffer * T::STAGE + w * T::LOADS * 1024;
#pragma unroll
        for (int j = 0; j < T::LOADS; j++) buffer_to_lds128(kr, offk[j], 0, to + j * 1024);
#pragma unroll
        for (int j = 0; j < T::LOADS; j++) buffer_to_lds128(vr, offv[j], 0, to + T::TILE + j * 1024);
    };
    // A lane's operand reads, as LDS addresses in a stage: K row r (+ 32), chunk 2 i + g at address ^ (i << 5); V key vkey of a group of eight, channels 16 (lane >> 4 & 1)
    // + 4 (lane & 3) of 32 at address ^ (i << 6) for the i-th 32.  (The reads are asm with waits of their own, as in the GEMMs: the compiler would wait for the direct
    // loads of the next tile in front of every read of this one, which costs a memory latency per tile: two documents of 8192 tokens 1150 us.)
    const int vkey = 4 * g + ((lane >> 2) & 3), vchunk = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
    const unsigned lds_base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const unsigned kat = lds_base + r * T::ROW + ((g ^ swz_k<D>(r)) << 4);
    const unsigned vat = lds_base + T::TILE + vkey * T::ROW + ((vchunk ^ swz_v<D>(vkey)) << 4) + 8 * (lane & 1);

    const float factor = scale * 1.44269504088896341f;
    const int tiles = (min(n, q0 + QB) + KEYS - 1) / KEYS;
    v16f o[DB];
    float m, l;
    auto sweep = [&](auto careful_tag) {
        constexpr bool CAREFUL = decltype(careful_tag)::value;
#pragma unroll
        for (int i = 0; i < DB; i++)
#pragma unroll
            for (int e = 0; e < 16; e++) o[i][e] = 0.0f;
        m = LOWEST;
        l = 0.0f;
        request(0, 0);
        for (int t = 0; t < tiles; t++) {
            wait_vm_and_barrier<0>();                                     // tile t is there, and tile t - 1 has been read by all
            if (t + 1 < tiles) request(t + 1, (t + 1) & 1);
            const int j0 = t * KEYS;
            if (j0 > wave_end) continue;                                  // (wave-uniform) keys behind all of the wave's queries
            const unsigned stage = (t & 1) * T::STAGE, ka = kat + stage, va = vat + stage;
            // scores: four fragments of K on their way while four are multiplied
            constexpr int HALF = KS / 2;                                  // fragments of a step; steps (h, first or second half of the channels)
            v16f sc[2];
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int e = 0; e < 16; e++) sc[h][e] = 0.0f;
            v4i kf[2][HALF];
            auto fetch_k = [&](auto step_tag) {
                constexpr int S = decltype(step_tag)::value;
#pragma unroll
                for (int i = 0; i < HALF; i++) kf[S & 1][i] = lds_read128<(S >> 1) * 32 * T::ROW>(ka ^ (((S & 1) * HALF + i) << 5));
            };
            v2i vf[2][DB][2];
            auto fetch_v = [&](auto u_tag) {                              // keys 16 u + 4 g + (0..3, 8..11)
                constexpr int U = decltype(u_tag)::value;
#pragma unroll
                for (int i = 0; i < DB; i++) {
                    vf[U & 1][i][0] = lds_read_tr64<U * 16 * T::ROW>(va ^ (i << 6));
                    vf[U & 1][i][1] = lds_read_tr64<U * 16 * T::ROW + 8 * T::ROW>(va ^ (i << 6));
                }
            };
            constexpr std::integral_constant<int, 0> c0;
            fetch_k(c0);
            each_index([&](auto step_tag) {
                constexpr int S = decltype(step_tag)::value, HB = S >> 1;
                if constexpr (S < 3) fetch_k(std::integral_constant<int, S + 1>());
                else fetch_v(c0);
                wait_lds_reads<S < 3 ? HALF : 2 * DB>();
                tie(kf[S & 1], std::make_integer_sequence<int, HALF>());
#pragma unroll
                for (int i = 0; i < HALF; i++) sc[HB] = mma32<BF>(kf[S & 1][i], qf[(S & 1) * HALF + i], sc[HB]);
            }, std::make_integer_sequence<int, 4>());
            const bool edge = j0 + KEYS - 1 > qw;                         // the diagonal crosses the tile (the sequence's end lies behind it)
            if (edge) {
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int e = 0; e < 16; e++)
                        if (j0 + 32 * h + 8 * (e >> 2) + 4 * g + (e & 3) > qw + r) sc[h][e] = -INFINITY;
            }
            float top = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int e = 0; e < 16; e++) top = __builtin_fmaxf(top, sc[h][e]);
            top *= factor;
            constexpr float MOVES = SLACK - ABOVE<BF>;
            if (__any(top > m + MOVES)) {
                top = __builtin_fmaxf(top, __shfl_xor(top, 32, 64));
                const float to = top > m + MOVES ? top + ABOVE<BF> : m, down = __builtin_amdgcn_exp2f(m - to);   // (a query's result does not depend on the wave's others)
                m = to;
                l *= down;
#pragma unroll
                for (int i = 0; i < DB; i++)
#pragma unroll
                    for (int e = 0; e < 16; e++) o[i][e] *= down;
            }
            v4i pf[4];
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[h][e], factor, -m)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[h][e + 1], factor, -m));
                    l += p0 + p1;
                    pf[2 * h + (e >> 3)][(e & 7) >> 1] = narrow2<BF>(p0, p1);
                }
            each_index([&](auto u_tag) {
                constexpr int U = decltype(u_tag)::value;
                if constexpr (U < 3) fetch_v(std::integral_constant<int, U + 1>());
                wait_lds_reads<U < 3 ? 2 * DB : 0>();
#pragma unroll
                for (int i = 0; i < DB; i++) {
                    asm volatile("" : "+v"(vf[U & 1][i][0]), "+v"(vf[U & 1][i][1]));          // (read from here on)
                    v4i v = {vf[U & 1][i][0][0], vf[U & 1][i][0][1], vf[U & 1][i][1][0], vf[U & 1][i][1][1]};
                    if (CAREFUL && edge) v = without_odd<BF>(v);
                    o[i] = mma32<BF>(v, pf[U], o[i]);
                }
            }, std::make_integer_sequence<int, 4>());
            if (CAREFUL && edge) {
                const char *vt = lds + stage + T::TILE;
                for (int key = 0; key < KEYS && j0 + key < n; key++) {
                    const char *row = vt + key * T::ROW;
                    if (!__any(odd_halves<BF>(*reinterpret_cast<const int *>(row + 4 * (lane % (D / 2)))))) continue;
                    const bool sees = j0 + key <= qw + r;
#pragma unroll
                    for (int i = 0; i < DB; i++)
#pragma unroll
                        for (int e = 0; e < 16; e += 4) {                 // channels 32 i + 2 e + 4 g + (0..3)
                            const v2i four = *reinterpret_cast<const v2i *>(row + (((4 * i + (e >> 2)) ^ swz_v<D>(key)) << 4) + 8 * g);
#pragma unroll
                            for (int c = 0; c < 4; c++) {
                                const unsigned half = (unsigned)four[c >> 1] >> (16 * (c & 1)) & 0xffffu;
                                if (sees && odd_halves<BF>((int)half))
                                    o[i][e + c] += BF ? __uint_as_float(half << 16) : (float)__builtin_bit_cast(_Float16, (unsigned short)half);
                            }
                        }
                }
            }
        }
    };
    sweep(std::false_type());
    {
        float all = 0.0f;
#pragma unroll
        for (int i = 0; i < DB; i++)
#pragma unroll
            for (int e = 0; e < 16; e++) all = __builtin_fmaf(o[i][e], 0.0f, all);
        if (__syncthreads_or(!(all == 0.0f))) {                           // (the same for all waves; behind it the tiles have been read)
            sweep(std::true_type());
            __syncthreads();
        }
    }
    l += __shfl_xor(l, 32, 64);
    const float by = l != 0.0f ? __fdiv_rn(1.0f, l) : 0.0f;
    char *mine = lds + w * 32 * (T::ROW + 16);
#pragma unroll
    for (int i = 0; i < DB; i++)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<v2i *>(mine + r * (T::ROW + 16) + 2 * (32 * i + 2 * e + 4 * g)) =
                v2i{narrow2<BF>(o[i][e] * by, o[i][e + 1] * by), narrow2<BF>(o[i][e + 2] * by, o[i][e + 3] * by)};
    wait_lds();
#pragma unroll
    for (int p = 0; p < 32 / RPL; p++) {
        const int row = p * RPL + lane / CH;
        if (qw + row < n)
            *reinterpret_cast<v4i *>(out + 2 * ((size_t)(t0 + qw + row) * heads + head) * D + lane % CH * 16) =
                *reinterpret_cast<const v4i *>(mine + row * (T::ROW + 16) + lane % CH * 16);
    }
}

template <bool BF, int D>
hipError_t causal_attention(const void *q, long ldq, const void *k, long ldk, const void *v, long ldv, int heads, int kv_heads, const int *cu, int batch,
                            int max_len, int rows, float scale, void *out, hipStream_t st)
{
    constexpr int NW = 4;
    const int strips = (max_len + 32 * NW - 1) / (32 * NW);
    hipLaunchKernelGGL((causal_attention_kernel<BF, D, NW>), dim3((unsigned)strips * heads * batch), dim3(64 * NW), 0, st, (const char *)q, (const char *)k,
                       (const char *)v, ldq, ldk, ldv, cu, rows, max_len, heads, heads / kv_heads, batch, strips, scale, (char *)out);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_causal_attention(const void *q, long ldq, const void *k, long ldk, const void *v, long ldv, bool bf16, int heads, int kv_heads, int D,
                                   const int *cu, int batch, int max_len, int rows, float scale, void *out, hipStream_t st)
{
    if (D == 128) return bf16 ? causal_attention<true, 128>(q, ldq, k, ldk, v, ldv, heads, kv_heads, cu, batch, max_len, rows, scale, out, st)
                              : causal_attention<false, 128>(q, ldq, k, ldk, v, ldv, heads, kv_heads, cu, batch, max_len, rows, scale, out, st);
    return bf16 ? causal_attention<true, 64>(q, ldq, k, ldk, v, ldv, heads, kv_heads, cu, batch, max_len, rows, scale, out, st)
                : causal_attention<false, 64>(q, ldq, k, ldk, v, ldv, heads, kv_heads, cu, batch, max_len, rows, scale, out, st);
}

}  // namespace samp

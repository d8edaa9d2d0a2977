// y[m, n] = act(steps[m] * s_w[n] * sum_k codes[m, k] W[n, k] + bias[n]): the int8 product whose activation rows bring their own steps, on weights in the
// order of pack_weight_kernel, with a 16-bit result.  The sum is exact in int32; it becomes binary32 (2^-24), is multiplied by the row's step (2^-24) and, in one
// fused operation with the bias, by the channel's (2^-24), and is rounded once to 16 bits.  In between the row's step is 2^-24 of itself and the channel's
// 2^24, so that a sum of 2^31 steps of 2^121 (rows of the largest bfloat16) does not overflow where the channel's step brings it back; no other bit
// changes (the quantiser's steps are 2^-67 or more).
#include "decoder.h"
#include "decoder_rules.h"
#include "mfma_tile.h"

namespace samp {
namespace {

struct TokensEpi { const float *steps, *s_w, *bias; int gelu; };

constexpr float ROW_SHIFT = 0x1p-24f, CHANNEL_SHIFT = 0x1p24f;
template <bool BF> __device__ __forceinline__ v2i finish4(const v4i &acc, float step, const v4f &sw, const v4f &b, int gelu)
{
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
        y[e] = __builtin_fmaf((float)acc[e] * step, sw[e], b[e]);
        if (gelu) y[e] = gelu_fast(y[e]);
    }
    return v2i{narrow2<BF>(y[0], y[1]), narrow2<BF>(y[2], y[3])};
}

// ---- many rows -------------------------------------------------------------------------------------
// The tile loop on packed weights (mfma_tile.h): 16 MT tokens x 64 NTW channels per block, weights straight into registers, token rows through LDS.
// 8192 x 4096 x 4096: 133 us in the median, 2.06 POP/s, at least 125 (torch's int8 product, 8192 x 8192 x 4096, on that card: 2.08).
// K need only be a multiple of 64: what is left after whole rounds of the ring (D stages of 128 bytes) is multiplied from memory, without a pipeline.
// N need only be a multiple of 16: a wave's blocks past the last one repeat it and are not stored.
template <bool BF, int MT, int NTW, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void gemm_tokens_kernel(const char *__restrict__ A, const char *__restrict__ Wp, int M, int N, int K, int tiles_m, int tiles_n, int band, TokensEpi epi, char *__restrict__ out)
{
    constexpr int BM = 16 * MT, BN = 64 * NTW, NLDA = stream_loads<false, MT>(), STRIDE = BN * 2 + 16;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    // tiles in bands of `band` row tiles, in a band column by column
    const int tile = xcd_contiguous(blockIdx.x, tiles_m * tiles_n), first = tile / (band * tiles_n) * band, high = min(band, tiles_m - first);
    const int in_band = tile - first * tiles_n, m0 = (first + in_band % high) * BM, n0 = in_band / high * BN;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, q = lane >> 4;

    unsigned offa[NLDA];
#pragma unroll
    for (int j = 0; j < NLDA; j++) {
        const int srow = 8 * (wave + 4 * j) + (lane >> 3);
        offa[j] = (unsigned)min(srow, M - 1 - m0) * (unsigned)K + (((lane & 7) ^ swz<128>(srow)) << 4);
    }
    const int nb = N / 16, block0 = min(n0 / 16 + NTW * wave, nb - 1);
    const char *wbase = Wp + (size_t)block0 * 16 * K, *abase = A + (size_t)m0 * K;
    unsigned woff[NTW];
    int chan[NTW];                                                // the first of a lane's four channels of block t
#pragma unroll
    for (int t = 0; t < NTW; t++) {
        const int block = min(n0 / 16 + NTW * wave + t, nb - 1);
        woff[t] = (unsigned)(block - block0) * 16 * K;
        chan[t] = block * 16 + 4 * q;
    }
    v4i acc[NTW][MT];
#pragma unroll
    for (int t = 0; t < NTW; t++)
#pragma unroll
        for (int i = 0; i < MT; i++) acc[t][i] = v4i{0, 0, 0, 0};
    v4f sw[NTW], bb[NTW];
    float step[MT];
    auto tables = [&]() {
#pragma unroll
        for (int t = 0; t < NTW; t++) {
            sw[t] = *reinterpret_cast<const v4f *>(epi.s_w + chan[t]);
            bb[t] = *reinterpret_cast<const v4f *>((epi.bias ? epi.bias : epi.s_w) + chan[t]);
        }
#pragma unroll
        for (int i = 0; i < MT; i++) step[i] = epi.steps[min(m0 + 16 * i + r, M - 1)];
    };
    const int rounds = K / (128 * D);
    if (rounds)
        stream_tile_loop<false, MT, NTW, D>(abase, offa, wbase, woff, rounds * D, lds, wave, lane, tables,
            [&](int t, int i, const v4i &w, const v4i &f) { acc[t][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, f, acc[t][i], 0, 0, 0); });
    else tables();
    for (int k = rounds * 128 * D; k < K; k += 64) {
        v4i w[NTW], f[MT];
#pragma unroll
        for (int t = 0; t < NTW; t++) w[t] = *reinterpret_cast<const v4i *>(wbase + woff[t] + (size_t)k * 16 + 16 * lane);
#pragma unroll
        for (int i = 0; i < MT; i++) f[i] = *reinterpret_cast<const v4i *>(abase + (size_t)min(16 * i + r, M - 1 - m0) * K + k + 16 * q);
#pragma unroll
        for (int t = 0; t < NTW; t++)
#pragma unroll
            for (int i = 0; i < MT; i++) acc[t][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[t], f[i], acc[t][i], 0, 0, 0);
    }
#pragma unroll
    for (int t = 0; t < NTW; t++) {
        if (!epi.bias) bb[t] = v4f{0.f, 0.f, 0.f, 0.f};
        sw[t] *= CHANNEL_SHIFT;
#pragma unroll
        for (int i = 0; i < MT; i++)
            *reinterpret_cast<v2i *>(lds + (16 * i + r) * STRIDE + (16 * (NTW * wave + t) + 4 * q) * 2) = finish4<BF>(acc[t][i], step[i] * ROW_SHIFT, sw[t], bb[t], epi.gelu);
    }
    __syncthreads();
    constexpr int CHUNKS = BN / 8;
#pragma unroll 4
    for (int idx = tid; idx < BM * CHUNKS; idx += 256) {
        const int row = m0 + idx / CHUNKS, n = n0 + idx % CHUNKS * 8;
        if (row < M && n < N)
            *reinterpret_cast<v4i *>(out + ((size_t)row * N + n) * 2) = *reinterpret_cast<const v4i *>(lds + (idx / CHUNKS) * STRIDE + idx % CHUNKS * 16);
    }
}

template <bool BF, int MT, int NTW, int D>
hipError_t launch_tile(const int8_t *A, const int8_t *Wp, const TokensEpi &epi, void *out, int M, int N, int K, int band, hipStream_t st)
{
    constexpr int RING = stream_ring_bytes<false, MT, D>(), OUT = 16 * MT * (64 * NTW * 2 + 16), LDS = RING > OUT ? RING : OUT;
    auto kern = gemm_tokens_kernel<BF, MT, NTW, D>;
    static_assert(LDS <= 65536, "more needs an attribute of the kernel");
    const int tm = (M + 16 * MT - 1) / (16 * MT), tn = (N + 64 * NTW - 1) / (64 * NTW);
    hipLaunchKernelGGL(kern, dim3((unsigned)tm * tn), dim3(256), LDS, st, (const char *)A, (const char *)Wp, M, N, K, tm, tn, band, epi, (char *)out);
    return hipGetLastError();
}

// ---- up to sixteen rows ------------------------------------------------------------------------------
// One token tile; what it costs is the weights' way from HBM and the latencies around it.  A block owns 16 channels and splits K over its eight waves, so that
// all of its weights (KB blocks of 1 KB a wave) are requested before anything else happens; the int32 partial tiles meet in LDS.  FUSED: the rows come in 16
// bits and every block quantises them for itself while its weights are on the way, into LDS (rows 16 bytes more than K apart, so that the sixteen rows of an
// operand read lie in different banks), which saves a launch.  Eight, four, two or one waves share a row, the fewer the more rows there are.  One row, 4096 -> 6144,
// 25 MB of weights: 8.1 us in a chain of launches with weights from memory (the quantiser in front 8.6), 7.3 with weights in the memory-side cache; with every lane quantising
// what it multiplies, sixteen times over, some 2 us more.  When it is used: decoder_rules.h.
struct FewRows { const void *x; long ld; const float *steps; };        // FUSED: 16-bit rows, ld values apart; else codes, K apart, and their steps
template <bool BF, bool FUSED, int KB>
__global__ __launch_bounds__(64 * FEW_WAVES) void gemm_tokens_few_kernel(const char *__restrict__ Wp, int K, int N, int M, int sharers, FewRows in, TokensEpi epi,
                                                                           char *__restrict__ out)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];             // FUSED: codes
    __shared__ unsigned tops[FEW_WAVES];
    __shared__ float row_steps[16];
    __shared__ __attribute__((aligned(16))) v4i part[FEW_WAVES][64];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, q = lane >> 4, kblocks = K >> 6;
    const auto weights = buffer_of(Wp + (size_t)blockIdx.x * 16 * K, 16 * K);
    const int row = min(r, M - 1);
    v4i wf[KB], f[KB];
    auto request_weights = [&]() {                                          // past the end: zeros
#pragma unroll
        for (int i = 0; i < KB; i++) wf[i] = __builtin_amdgcn_raw_buffer_load_b128(weights, (w + FEW_WAVES * i) * 1024 + 16 * lane, 0, 0);
    };
    // the lane of the result: token r, channels 4 q .. 4 q + 3
    const int chan = blockIdx.x * 16 + 4 * q;
    v4f sw = {0.f, 0.f, 0.f, 0.f}, bb = sw;
    auto request_tables = [&]() {
        if (w) return;
        sw = *reinterpret_cast<const v4f *>(epi.s_w + chan);
        if (epi.bias) bb = *reinterpret_cast<const v4f *>(epi.bias + chan);
    };
    float step = 1.0f;
    if constexpr (FUSED) {
        const int pitch = K + 16, rows_at_once = FEW_WAVES / sharers, first = (w & (sharers - 1)) * 64 + lane, stride = 64 * sharers;
        for (int m0 = 0; m0 < M; m0 += rows_at_once) {                      // (one round where waves share a row)
            const int m = m0 + w / sharers;
            const auto from = buffer_of((const char *)in.x + 2 * (size_t)min(m, M - 1) * in.ld, m < M ? 2 * K : 0);
            v4i x[KB];
#pragma unroll
            for (int i = 0; i < KB; i++) x[i] = __builtin_amdgcn_raw_buffer_load_b128(from, 16 * (first + i * stride), 0, 0);
            if (m0 == 0) {
                request_weights();
                request_tables();
            }
            unsigned top = 0;
#pragma unroll
            for (int i = 0; i < KB; i++) top = max_halves(top, bits_max16(x[i]));
            top = max_of_wave(top);
            if (sharers > 1) {
                if (lane == 0) tops[w] = top;
                __syncthreads();
                for (int u = 0; u < sharers; u++) top = max(top, tops[(w & ~(sharers - 1)) + u]);
            }
            const RowQuant rq = row_quant<BF>(top);
            if (m < M) {
#pragma unroll
                for (int i = 0; i < KB; i++) {
                    float v[8];
                    widen8<BF>(x[i], v);
                    if (8 * (first + i * stride) < K) *reinterpret_cast<v2i *>(lds + m * pitch + 8 * (first + i * stride)) = quant8(v, rq);
                }
                if (first == 0) row_steps[m] = rq.step;
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < KB; i++) f[i] = *reinterpret_cast<const v4i *>(lds + row * pitch + min(w + FEW_WAVES * i, kblocks - 1) * 64 + 16 * q);
        step = row_steps[row];
    } else {
        const auto codes = buffer_of(in.x, M * K);
#pragma unroll
        for (int i = 0; i < KB; i++)
            f[i] = __builtin_amdgcn_raw_buffer_load_b128(codes, row * K + min(w + FEW_WAVES * i, kblocks - 1) * 64 + 16 * q, 0, 0);
        request_weights();
        request_tables();
        if (w == 0) step = in.steps[row];
    }
    v4i acc = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < KB; i++) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[i], f[i], acc, 0, 0, 0);
    part[w][lane] = acc;
    __syncthreads();
    if (w || r >= M) return;
#pragma unroll
    for (int u = 1; u < FEW_WAVES; u++) acc += part[u][lane];
    *reinterpret_cast<v2i *>(out + 2 * ((size_t)r * N + chan)) = finish4<BF>(acc, step * ROW_SHIFT, sw * CHANNEL_SHIFT, bb, epi.gelu);
}

template <bool BF, bool FUSED>
hipError_t launch_few(const FewRows &in, const int8_t *Wp, const TokensEpi &epi, void *out, int M, int N, int K, hipStream_t st)
{
    const int kb = tokens_few_blocks(K), sharers = M == 1 ? 8 : M == 2 ? 4 : M <= 4 ? 2 : 1;
    auto kern = kb == 2 ? gemm_tokens_few_kernel<BF, FUSED, 2> : kb == 4 ? gemm_tokens_few_kernel<BF, FUSED, 4> : kb == 8 ? gemm_tokens_few_kernel<BF, FUSED, 8>
                        : gemm_tokens_few_kernel<BF, FUSED, 16>;
    hipLaunchKernelGGL(kern, dim3(N / 16), dim3(64 * FEW_WAVES), FUSED ? M * (K + 16) : 0, st, (const char *)Wp, K, N, M, sharers, in, epi, (char *)out);
    return hipGetLastError();
}

// ---- which kernel: decoder_rules.h ---------------------------------------------------------------------
template <bool BF>
hipError_t gemm_tokens(const int8_t *A, const int8_t *Wp, const TokensEpi &epi, void *out, int M, int N, int K, hipStream_t st)
{
    if (tokens_few(M, K)) return launch_few<BF, false>(FewRows{A, K, epi.steps}, Wp, epi, out, M, N, K, st);
    const int tile = tokens_tile(M, N), band = tokens_band(tile);
    const bool deep = tokens_depth(tile, K) == 4;
    switch (tile) {
    case 0: return deep ? launch_tile<BF, 2, 1, 4>(A, Wp, epi, out, M, N, K, band, st) : launch_tile<BF, 2, 1, 2>(A, Wp, epi, out, M, N, K, band, st);
    case 1: return deep ? launch_tile<BF, 4, 1, 4>(A, Wp, epi, out, M, N, K, band, st) : launch_tile<BF, 4, 1, 2>(A, Wp, epi, out, M, N, K, band, st);
    case 2: return deep ? launch_tile<BF, 4, 2, 4>(A, Wp, epi, out, M, N, K, band, st) : launch_tile<BF, 4, 2, 2>(A, Wp, epi, out, M, N, K, band, st);
    case 3: return launch_tile<BF, 8, 2, 2>(A, Wp, epi, out, M, N, K, band, st);
    }
    return launch_tile<BF, 8, 3, 2>(A, Wp, epi, out, M, N, K, band, st);
}

}  // namespace

hipError_t launch_gemm_i8_tokens(const int8_t *codes, const float *steps, const int8_t *Wp, const float *s_w, const float *bias, bool gelu, void *out,
                                 bool bf16, int M, int N, int K, hipStream_t st)
{
    const TokensEpi epi{steps, s_w, bias, gelu};
    return bf16 ? gemm_tokens<true>(codes, Wp, epi, out, M, N, K, st) : gemm_tokens<false>(codes, Wp, epi, out, M, N, K, st);
}

hipError_t launch_linear_few(const void *x, long ldx, bool bf16, const int8_t *Wp, const float *s_w, const float *bias, bool gelu, void *out, int M, int N, int K,
                             hipStream_t st)
{
    const TokensEpi epi{nullptr, s_w, bias, gelu};
    const FewRows in{x, ldx, nullptr};
    return bf16 ? launch_few<true, true>(in, Wp, epi, out, M, N, K, st) : launch_few<false, true>(in, Wp, epi, out, M, N, K, st);
}

}  // namespace samp

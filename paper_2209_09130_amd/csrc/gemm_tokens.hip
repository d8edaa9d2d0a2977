// y[m, n] = act(steps[m] * s_w[n] * sum_k codes[m, k] W[n, k] + bias[n]): the int8 product whose activation rows bring their own steps, on weights in the
// order of pack_weight_kernel, with a 16-bit result.
#include "decoder.h"
#include "divisor.h"
#include "mfma_tile.h"

namespace samp {
namespace {

struct TokensEpi { const float *steps, *s_w, *bias; int gelu; };

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
// K need only be a multiple of 64: what is left after whole rounds of the ring (D stages of 128 bytes) is multiplied from memory, without a pipeline.
// N need only be a multiple of 16: a wave's blocks past the last one repeat it and are not stored.
template <bool BF, int MT, int NTW, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void gemm_tokens_kernel(const char *__restrict__ A, const char *__restrict__ Wp, int M, int N, int K, int tiles_m, int tiles_n, TokensEpi epi, char *__restrict__ out)
{
    constexpr int BM = 16 * MT, BN = 64 * NTW, NLDA = stream_loads<false, MT>(), STRIDE = BN * 2 + 16;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int tile = xcd_contiguous(blockIdx.x, tiles_m * tiles_n);
    const int m0 = tile / tiles_n * BM, n0 = tile % tiles_n * BN;
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
#pragma unroll
        for (int i = 0; i < MT; i++)
            *reinterpret_cast<v2i *>(lds + (16 * i + r) * STRIDE + (16 * (NTW * wave + t) + 4 * q) * 2) = finish4<BF>(acc[t][i], step[i], sw[t], bb[t], epi.gelu);
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
hipError_t launch_tile(const int8_t *A, const int8_t *Wp, const TokensEpi &epi, void *out, int M, int N, int K, hipStream_t st)
{
    constexpr int RING = stream_ring_bytes<false, MT, D>(), OUT = 16 * MT * (64 * NTW * 2 + 16), LDS = RING > OUT ? RING : OUT;
    auto kern = gemm_tokens_kernel<BF, MT, NTW, D>;
    if constexpr (LDS > 65536) {
        static std::atomic<bool> set{false};
        if (!set.load(std::memory_order_acquire)) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
            if (e != hipSuccess) return e;
            set.store(true, std::memory_order_release);
        }
    }
    const int tm = (M + 16 * MT - 1) / (16 * MT), tn = (N + 64 * NTW - 1) / (64 * NTW);
    hipLaunchKernelGGL(kern, dim3((unsigned)tm * tn), dim3(256), LDS, st, (const char *)A, (const char *)Wp, M, N, K, tm, tn, epi, (char *)out);
    return hipGetLastError();
}

template <bool BF>
hipError_t gemm_tokens(const int8_t *A, const int8_t *Wp, const TokensEpi &epi, void *out, int M, int N, int K, hipStream_t st)
{
    return launch_tile<BF, 2, 1, 2>(A, Wp, epi, out, M, N, K, st);
}

}  // namespace

hipError_t launch_gemm_i8_tokens(const int8_t *codes, const float *steps, const int8_t *Wp, const float *s_w, const float *bias, bool gelu, void *out,
                                 bool bf16, int M, int N, int K, hipStream_t st)
{
    const TokensEpi epi{steps, s_w, bias, gelu};
    return bf16 ? gemm_tokens<true>(codes, Wp, epi, out, M, N, K, st) : gemm_tokens<false>(codes, Wp, epi, out, M, N, K, st);
}

}  // namespace samp

// Rows that bring their own steps: activation rows quantised as they come, keys and values quantised as they are written to the cache, and the cache
// read back.  All of them move each byte once; what bounds them is HBM, and for a few rows the launch.
#include "decoder.h"
#include "decoder_rules.h"

namespace samp {
namespace {

// ---- activation rows -----------------------------------------------------------------------------
// WPR waves share a row, each lane holds C chunks of 8 values of it, so that the row is read once: its largest magnitude, then its codes.
template <bool BF, int WPR, int C>
__global__ __launch_bounds__(256) void quantize_tokens_kernel(const char *__restrict__ x, long ldx, int M, int K, int8_t *__restrict__ codes,
                                                              float *__restrict__ steps)
{
    constexpr int ROWS = 4 / WPR;
    __shared__ unsigned tops[4];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = blockIdx.x * ROWS + w / WPR, first = (w % WPR) * 64 + lane, chunks = K >> 3;
    if (WPR == 1 && row >= M) return;
    const char *from = x + 2 * (size_t)row * ldx;
    v4i raw[C];
    unsigned top = 0;
#pragma unroll
    for (int c = 0; c < C; c++) {
        const int at = first + c * 64 * WPR;
        raw[c] = at < chunks ? *reinterpret_cast<const v4i *>(from + 16 * (size_t)at) : v4i{0, 0, 0, 0};
    }
#pragma unroll
    for (int c = 0; c < C; c++) top = max_halves(top, bits_max16(raw[c]));
    top = max_of_wave(top);
    if constexpr (WPR > 1) {
        if (lane == 0) tops[w] = top;
        __syncthreads();
        top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    }
    const RowQuant q = row_quant<BF>(top);
    int8_t *to = codes + (size_t)row * K;
#pragma unroll
    for (int c = 0; c < C; c++) {
        const int at = first + c * 64 * WPR;
        float v[8];
        widen8<BF>(raw[c], v);
        const v2i code = quant8(v, q);
        if (at < chunks) *reinterpret_cast<v2i *>(to + 8 * (size_t)at) = code;
    }
    if (first == 0) steps[row] = q.step;
}

// rows longer than the registers of a block hold are read twice, the second time from the caches
template <bool BF>
__global__ __launch_bounds__(256) void quantize_tokens_long_kernel(const char *__restrict__ x, long ldx, int K, int8_t *__restrict__ codes,
                                                                   float *__restrict__ steps)
{
    __shared__ unsigned tops[4];
    const int tid = threadIdx.x, row = blockIdx.x, chunks = K >> 3;
    const char *from = x + 2 * (size_t)row * ldx;
    unsigned top = 0;
    for (int at = tid; at < chunks; at += 256) top = max_halves(top, bits_max16(*reinterpret_cast<const v4i *>(from + 16 * (size_t)at)));
    top = max_of_wave(top);
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
    const RowQuant q = row_quant<BF>(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
    for (int at = tid; at < chunks; at += 256) {
        float v[8];
        widen8<BF>(*reinterpret_cast<const v4i *>(from + 16 * (size_t)at), v);
        *reinterpret_cast<v2i *>(codes + (size_t)row * K + 8 * (size_t)at) = quant8(v, q);
    }
    if (tid == 0) steps[row] = q.step;
}

template <bool BF>
hipError_t quantize_tokens(const void *x, long ldx, int M, int K, int8_t *codes, float *steps, hipStream_t st)
{
    const char *from = (const char *)x;
    if (K <= 512) hipLaunchKernelGGL((quantize_tokens_kernel<BF, 1, 1>), dim3((M + 3) / 4), dim3(256), 0, st, from, ldx, M, K, codes, steps);
    else if (K <= 1024) hipLaunchKernelGGL((quantize_tokens_kernel<BF, 1, 2>), dim3((M + 3) / 4), dim3(256), 0, st, from, ldx, M, K, codes, steps);
    else if (K <= 2048) hipLaunchKernelGGL((quantize_tokens_kernel<BF, 4, 1>), dim3(M), dim3(256), 0, st, from, ldx, M, K, codes, steps);
    else if (K <= 4096) hipLaunchKernelGGL((quantize_tokens_kernel<BF, 4, 2>), dim3(M), dim3(256), 0, st, from, ldx, M, K, codes, steps);
    else if (K <= 8192) hipLaunchKernelGGL((quantize_tokens_kernel<BF, 4, 4>), dim3(M), dim3(256), 0, st, from, ldx, M, K, codes, steps);
    else if (K <= 16384) hipLaunchKernelGGL((quantize_tokens_kernel<BF, 4, 8>), dim3(M), dim3(256), 0, st, from, ldx, M, K, codes, steps);
    else hipLaunchKernelGGL(quantize_tokens_long_kernel<BF>, dim3(M), dim3(256), 0, st, from, ldx, K, codes, steps);
    return hipGetLastError();
}

// ---- cache -----------------------------------------------------------------------------------------
// Sixteen lanes a row of head_dim values; a block's sixteen rows are 2^TOKENS_LOG2 tokens of 16 >> TOKENS_LOG2 of the 2 kv_heads keys and values, so
// that a page's neighbouring rows and steps are written together and a block of a decode step (one token) is not left idle.  PASSES: so many times that many
// tokens, all requested before the first is worked on.  Heads run fastest over the blocks, so that those at work at a time read whole rows of the tensors.
struct RowAt { int token, head; bool is_v; };
template <int PASSES> __device__ __forceinline__ RowAt row_at(int tokens_log2, int kv_heads)
{
    const int group = threadIdx.x >> 4;
    RowAt a;
    a.token = ((int)blockIdx.y * PASSES << tokens_log2) + (group & ((1 << tokens_log2) - 1));
    const int part = blockIdx.x * (16 >> tokens_log2) + (group >> tokens_log2);
    a.is_v = part >= kv_heads;
    a.head = a.is_v ? part - kv_heads : part;
    return a;
}
// the page of a position, and -1 where the table has none of the cache's pages
__device__ __forceinline__ int page_of(const KvRows &r, const KvCache &c, int b, int pos)
{
    if (pos < 0 || (pos >> c.page_shift) >= r.width) return -1;
    const int p = r.table[(size_t)b * r.width + (pos >> c.page_shift)];
    return (unsigned)p < (unsigned)c.pages ? p : -1;
}

template <bool BF, int D, int PASSES>
__global__ __launch_bounds__(256) void cache_write_kernel(KvCache c, const char *__restrict__ k, long ldk, const char *__restrict__ v, long ldv, KvRows r,
                                                          int tokens_log2)
{
    constexpr int PER = D / 16;                                       // values of a lane
    const SeqRows s = seq_rows(r, blockIdx.z, c.page_shift);
    const RowAt a = row_at<PASSES>(tokens_log2, c.kv_heads);
    if (a.token >= s.todo || a.head >= c.kv_heads) return;
    const int lane = threadIdx.x & 15;
    const char *from = (a.is_v ? v : k) + 2 * ((size_t)s.first_row * (a.is_v ? ldv : ldk) + a.head * D + lane * PER);
    const size_t ld = 2 * (size_t)(a.is_v ? ldv : ldk);
    v4i raw[PASSES];
    int pos[PASSES], page[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; i++) {
        const int token = a.token + (i << tokens_log2);
        raw[i] = v4i{0, 0, 0, 0};
        page[i] = -1;
        if (token >= s.todo) continue;
        pos[i] = r.lens[blockIdx.z] - s.n + token;
        page[i] = page_of(r, c, blockIdx.z, pos[i]);
        if constexpr (PER == 8) raw[i] = *reinterpret_cast<const v4i *>(from + token * ld);
        else {
            const v2i half = *reinterpret_cast<const v2i *>(from + token * ld);
            raw[i][0] = half[0];
            raw[i][1] = half[1];
        }
    }
#pragma unroll
    for (int i = 0; i < PASSES; i++) {
        const unsigned top = max_of_16_lanes(bits_max16(raw[i]));
        if (page[i] < 0) continue;
        const RowQuant q = row_quant<BF>(top);
        float x[8];
        widen8<BF>(raw[i], x);
        const v2i code = quant8(x, q);
        const size_t row = (((size_t)page[i] * c.kv_heads + a.head) << c.page_shift) + (pos[i] & ((1 << c.page_shift) - 1));
        int8_t *to = (a.is_v ? c.v : c.k) + row * D + lane * PER;
        if constexpr (PER == 8) *reinterpret_cast<v2i *>(to) = code;
        else *reinterpret_cast<int *>(to) = code[0];
        if (lane == 0) (a.is_v ? c.v_step : c.k_step)[row] = q.step;
    }
}

template <bool BF, int D, int PASSES>
__global__ __launch_bounds__(256) void cache_read_kernel(KvCache c, char *__restrict__ k, char *__restrict__ v, KvRows r, int tokens_log2)
{
    constexpr int PER = D / 16;
    const SeqRows s = seq_rows(r, blockIdx.z, c.page_shift);
    const RowAt a = row_at<PASSES>(tokens_log2, c.kv_heads);
    if (a.token >= s.todo || a.head >= c.kv_heads) return;
    const int lane = threadIdx.x & 15;
    v2i code[PASSES];
    float step[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; i++) {
        const int token = a.token + (i << tokens_log2), pos = r.lens[blockIdx.z] - s.n + token, page = token < s.todo ? page_of(r, c, blockIdx.z, pos) : -1;
        code[i] = v2i{0, 0};
        step[i] = 0.0f;
        if (page < 0) continue;
        const size_t row = (((size_t)page * c.kv_heads + a.head) << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
        const int8_t *from = (a.is_v ? c.v : c.k) + row * D + lane * PER;
        if constexpr (PER == 8) code[i] = *reinterpret_cast<const v2i *>(from);
        else code[i][0] = *reinterpret_cast<const int *>(from);
        step[i] = (a.is_v ? c.v_step : c.k_step)[row];
    }
#pragma unroll
    for (int i = 0; i < PASSES; i++) {
        const int token = a.token + (i << tokens_log2);
        if (token >= s.todo) continue;
        v4i out;
#pragma unroll
        for (int e = 0; e < PER / 2; e++) {
            const int two = code[i][e >> 1] >> (16 * (e & 1));
            out[e] = narrow2<BF>((float)(int8_t)two * step[i], (float)(int8_t)(two >> 8) * step[i]);
        }
        char *to = (a.is_v ? v : k) + 2 * (((size_t)(s.first_row + token) * c.kv_heads + a.head) * D + lane * PER);
        if constexpr (PER == 8) *reinterpret_cast<v4i *>(to) = out;
        else *reinterpret_cast<v2i *>(to) = v2i{out[0], out[1]};
    }
}

int tokens_log2_for(int max_rows)
{
    int n = 0;
    while (n < 4 && (1 << n) < max_rows) n++;
    return n;
}
dim3 cache_grid(const KvCache &c, const KvRows &r, int log2, int passes)
{
    const int tokens = passes << log2;
    return dim3((unsigned)((2 * c.kv_heads + (16 >> log2) - 1) / (16 >> log2)), (unsigned)((r.max_rows + tokens - 1) / tokens), (unsigned)r.batch);
}

template <bool BF, int D>
hipError_t cache_write(const KvCache &c, const void *k, long ldk, const void *v, long ldv, const KvRows &r, hipStream_t st)
{
    const int n = tokens_log2_for(r.max_rows), passes = cache_passes(r.rows, c.kv_heads);
    auto kern = passes == 4 ? cache_write_kernel<BF, D, 4> : cache_write_kernel<BF, D, 1>;
    hipLaunchKernelGGL(kern, cache_grid(c, r, n, passes), dim3(256), 0, st, c, (const char *)k, ldk, (const char *)v, ldv, r, n);
    return hipGetLastError();
}

template <bool BF, int D>
hipError_t cache_read(const KvCache &c, void *k, void *v, const KvRows &r, hipStream_t st)
{
    const int n = tokens_log2_for(r.max_rows), passes = cache_passes(r.rows, c.kv_heads);
    auto kern = passes == 4 ? cache_read_kernel<BF, D, 4> : cache_read_kernel<BF, D, 1>;
    hipLaunchKernelGGL(kern, cache_grid(c, r, n, passes), dim3(256), 0, st, c, (char *)k, (char *)v, r, n);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_tokens(const void *x, long ldx, bool bf16, int M, int K, int8_t *codes, float *steps, hipStream_t st)
{
    return bf16 ? quantize_tokens<true>(x, ldx, M, K, codes, steps, st) : quantize_tokens<false>(x, ldx, M, K, codes, steps, st);
}

hipError_t launch_cache_write(const KvCache &c, const void *k, long ldk, const void *v, long ldv, bool bf16, int D, const KvRows &r, hipStream_t st)
{
    if (D == 128) return bf16 ? cache_write<true, 128>(c, k, ldk, v, ldv, r, st) : cache_write<false, 128>(c, k, ldk, v, ldv, r, st);
    return bf16 ? cache_write<true, 64>(c, k, ldk, v, ldv, r, st) : cache_write<false, 64>(c, k, ldk, v, ldv, r, st);
}

hipError_t launch_cache_read(const KvCache &c, void *k, void *v, bool bf16, int D, const KvRows &r, hipStream_t st)
{
    if (D == 128) return bf16 ? cache_read<true, 128>(c, k, v, r, st) : cache_read<false, 128>(c, k, v, r, st);
    return bf16 ? cache_read<true, 64>(c, k, v, r, st) : cache_read<false, 64>(c, k, v, r, st);
}

}  // namespace samp

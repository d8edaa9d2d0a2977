// Which pages of a long context a query reads: bounds of the keys of each page, kept beside the cache, and the choice of the pages whose bounds promise most.
//
// A page's bounds are the largest and the smallest key in each channel, in 8 bits like the cache (2 head_dim + 4 bytes for page_len (head_dim + 4)).  No key of the page has a product with a
// query above sum_d max(q_d high_d, q_d low_d), which is the product of (positive part of q, negative part) and (high, low): one int8 matrix product of twice the length, exact,
// so that the choice is the same however it is computed.
#include "../../include/samp.h"
#include "decoder.h"

namespace samp {
namespace {

constexpr float INV_127 = 1.0f / 127.0f;

// ---- bounds ------------------------------------------------------------------------------------------
// A wave takes a page of a key head: D / 16 lanes hold 16 channels each of 1024 / D keys at a time; then the lanes of the same channels meet.  What bounds it is HBM for whole prompts, and
// the launch for a decode step, in which few pages become full and the other waves end at once.
template <int D>
__global__ __launch_bounds__(256) void cache_bounds_kernel(KvCache c, KeyBounds bounds, KvRows rows)
{
    constexpr int LANES = D / 16, KEYS = 64 / LANES;
    const SeqRows s = seq_rows(rows, blockIdx.z, c.page_shift);
    const int lane = threadIdx.x & 63, from = max(rows.lens[blockIdx.z] - s.n, 0), to = min(rows.lens[blockIdx.z] - s.n + s.todo, s.len);
    const int index = (from >> c.page_shift) + blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), head = blockIdx.x;
    if (s.todo <= 0 || to <= 0 || index >= to >> c.page_shift) return;
    const int page = rows.table[(size_t)blockIdx.z * rows.width + index];
    if ((unsigned)page >= (unsigned)c.pages) return;
    const size_t row = ((size_t)page * c.kv_heads + head) << c.page_shift;
    const int8_t *const k = c.k + row * D + 16 * lane;
    const float *const steps = c.k_step + row + lane / LANES;
    float high[16], low[16];
#pragma unroll
    for (int e = 0; e < 16; e++) {
        high[e] = -INFINITY;
        low[e] = INFINITY;
    }
    bool odd = false;                                                 // a step that is not finite: that of a key that is not
    for (int i0 = 0; i0 < 1 << c.page_shift; i0 += 16) {              // sixteen keys a turn: page_len is a multiple
        v4i raw[16 / KEYS];
        float step[16 / KEYS];
#pragma unroll
        for (int i = 0; i < 16 / KEYS; i++) {
            raw[i] = *reinterpret_cast<const v4i *>(k + (size_t)(i0 + i * KEYS) * D);
            step[i] = steps[i0 + i * KEYS];
        }
#pragma unroll
        for (int i = 0; i < 16 / KEYS; i++) {
            odd |= !__builtin_isfinite(step[i]);
#pragma unroll
            for (int e = 0; e < 16; e++) {
                const float x = (float)(int8_t)(raw[i][e >> 2] >> 8 * (e & 3)) * step[i];
                high[e] = __builtin_fmaxf(high[e], x);
                low[e] = __builtin_fminf(low[e], x);
            }
        }
    }
#pragma unroll
    for (int o = LANES; o < 64; o <<= 1)
#pragma unroll
        for (int e = 0; e < 16; e++) {
            high[e] = __builtin_fmaxf(high[e], __shfl_xor(high[e], o, 64));
            low[e] = __builtin_fminf(low[e], __shfl_xor(low[e], o, 64));
        }
    odd = __any(odd);
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; e++) top = __builtin_fmaxf(top, __builtin_fmaxf(__builtin_fabsf(high[e]), __builtin_fabsf(low[e])));
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, o, 64));
    const bool some = top > 0.0f && !odd;
    const float step = odd ? __builtin_nanf("") : some ? top * INV_127 : 1.0f;
    const size_t at = (size_t)page * c.kv_heads + head;
    if (lane < 2 * LANES) {                                           // the first lanes write the high codes, the next ones the low codes
        const bool is_low = lane >= LANES;
        int code[16];
#pragma unroll
        for (int e = 0; e < 16; e++) {
            const float q = __fdiv_rn(is_low ? low[e] : high[e], step), r = is_low ? __builtin_fmaxf(__builtin_floorf(q), -127.0f) : __builtin_fminf(__builtin_ceilf(q), 127.0f);
            code[e] = some ? (int)r : 0;
        }
        v4i packed;
#pragma unroll
        for (int i = 0; i < 4; i++) packed[i] = pack4(code[4 * i], code[4 * i + 1], code[4 * i + 2], code[4 * i + 3]);
        *reinterpret_cast<v4i *>(bounds.codes + at * 2 * D + 16 * lane) = packed;
    }
    if (lane == 0) bounds.steps[at] = step;
}

// ---- choice ------------------------------------------------------------------------------------------
// A binary32 number as a whole number of the same order; NaN counts as plus infinity
__device__ __forceinline__ unsigned order_of(float x)
{
    const unsigned u = __float_as_uint(x);
    if (x != x) return 0xff800000u;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
template <bool BF> __device__ __forceinline__ float largest(unsigned bits)
{
    return BF ? __uint_as_float(bits << 16) : (float)__builtin_bit_cast(_Float16, (unsigned short)bits);
}
constexpr unsigned ALWAYS = 0xffffffffu;                              // above the order of every number

// One block: a sequence and a key head.  The pages' scores go to LDS as whole numbers, then the `keep`-th largest of them is found eight bits at a time, and the pages that
// are chosen are written in order.
template <bool BF, int D>
__global__ __launch_bounds__(1024) void select_pages_kernel(const char *__restrict__ Q, long ldq, KvCache c, KeyBounds bounds, KvRows rows, int group, int keep, int sinks, int recent,
                                    int *__restrict__ tables, int *__restrict__ lens_out)
{
    extern __shared__ __attribute__((aligned(16))) unsigned score[];  // [width]
    __shared__ __attribute__((aligned(16))) int8_t codes[16][2 * D];  // positive parts, negative parts of sixteen rows of queries
    __shared__ float steps[16];
    __shared__ int count[256], parts[16];
    __shared__ int found[2];                                          // a digit, and how many are above it
    const int b = blockIdx.x / c.kv_heads, head = blockIdx.x - b * c.kv_heads, tid = threadIdx.x, lane = tid & 63, waves = blockDim.x >> 6;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    const SeqRows s = seq_rows(rows, b, c.page_shift);
    const int pages = (max(s.len, 0) + (1 << c.page_shift) - 1) >> c.page_shift, chosen = min(pages, keep);
    const int *const table = rows.table + (size_t)b * rows.width;
    int *const to = tables + (size_t)blockIdx.x * keep;
    if (head == 0 && tid == 0) lens_out[b] = rows.lens[b] - ((pages - chosen) << c.page_shift);
    if (pages <= keep) {
        for (int i = tid; i < keep; i += blockDim.x) to[i] = i < pages ? table[i] : -1;
        return;
    }

    const int all = s.todo * group;
    for (int r0 = 0; r0 < all || r0 == 0; r0 += 16) {
        // sixteen lanes a row of queries
        for (int row = tid >> 4; row < 16; row += blockDim.x >> 4) {
            constexpr int PER = D / 16;
            const int token = (r0 + row) / group, h = head * group + (r0 + row) - token * group;
            v4i raw = {0, 0, 0, 0};
            if (r0 + row < all) {
                const char *from = Q + 2 * ((size_t)(s.first_row + token) * ldq + h * D + r * PER);
                if constexpr (PER == 8) raw = *reinterpret_cast<const v4i *>(from);
                else {
                    const v2i half = *reinterpret_cast<const v2i *>(from);
                    raw[0] = half[0];
                    raw[1] = half[1];
                }
            }
            const unsigned top = max_of_16_lanes(bits_max16(raw));
            const RowQuant q = row_quant<BF>(top);
            float x[8];
            widen8<BF>(raw, x);
            const v2i code = quant8(x, q);
#pragma unroll
            for (int i = 0; i < PER / 4; i++) {
                int pos = 0, neg = 0;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int v = (int8_t)(code[i] >> 8 * e);
                    pos |= (max(v, 0) & 0xff) << 8 * e;
                    neg |= (min(v, 0) & 0xff) << 8 * e;
                }
                *reinterpret_cast<int *>(&codes[row][r * PER + 4 * i]) = pos;
                *reinterpret_cast<int *>(&codes[row][D + r * PER + 4 * i]) = neg;
            }
            // (the product is the definition's step; the quantiser's own is the quotient)
            if (r == 0) steps[row] = !q.finite || q.hi == 0.0f ? q.step : largest<BF>(top) * INV_127;
        }
        __syncthreads();
        v4i qf[2 * D / 64];
#pragma unroll
        for (int i = 0; i < 2 * D / 64; i++) qf[i] = *reinterpret_cast<const v4i *>(&codes[r][64 * i + 16 * g]);
        const v4f qs = *reinterpret_cast<const v4f *>(&steps[4 * g]);
        for (int p0 = 16 * w; p0 < pages; p0 += 16 * waves) {
            const int p = p0 + r, entry = p < pages ? table[p] : -1;
            const bool ok = (unsigned)entry < (unsigned)c.pages;
            const size_t at = (size_t)(ok ? entry : 0) * c.kv_heads + head;
            const int8_t *from = bounds.codes + at * 2 * D + 16 * g;
            v4i sum = {0, 0, 0, 0}, bf[2 * D / 64];
#pragma unroll
            for (int i = 0; i < 2 * D / 64; i++) bf[i] = *reinterpret_cast<const v4i *>(from + 64 * i);
            const float step = bounds.steps[at];
#pragma unroll
            for (int i = 0; i < 2 * D / 64; i++) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(qf[i], bf[i], sum, 0, 0, 0);
            unsigned best = 0;
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (r0 + 4 * g + e < all) best = max(best, order_of((float)sum[e] * (qs[e] * step)));
            best = max(best, (unsigned)__shfl_xor((int)best, 16, 64));
            best = max(best, (unsigned)__shfl_xor((int)best, 32, 64));
            if (!ok) best = order_of(-INFINITY);
            if (p < sinks || p >= pages - recent) best = ALWAYS;
            if (g == 0 && p < pages) score[p] = r0 ? max(score[p], best) : best;
        }
        __syncthreads();
    }

    // the `keep`-th largest, and how many pages of just that score are kept
    unsigned known = 0;
    int left = keep;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += blockDim.x) count[i] = 0;
        __syncthreads();
        for (int p = tid; p < pages; p += blockDim.x) {
            const unsigned x = score[p];
            if (shift == 24 || (x ^ known) >> (shift + 8) == 0) atomicAdd(&count[x >> shift & 255], 1);
        }
        __syncthreads();
        if (tid < 64) {                                               // digits 4 lane .. 4 lane + 3, from above
            int n[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) sum += n[i] = count[255 - 4 * tid - i];
            int before = sum;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int other = __shfl_up(before, o, 64);
                if (tid >= o) before += other;
            }
            before -= sum;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (before < left && before + n[i] >= left) {
                    found[0] = 255 - 4 * tid - i;
                    found[1] = before;
                }
                before += n[i];
            }
        }
        __syncthreads();
        known |= (unsigned)found[0] << shift;
        left -= found[1];
    }

    int written = 0, equal = 0;
    for (int p0 = 0; p0 < pages; p0 += blockDim.x) {
        const int p = p0 + tid;
        const unsigned x = p < pages ? score[p] : 0;
        const bool above = p < pages && x > known, same = p < pages && x == known;
        const unsigned long long below = (1ull << lane) - 1, m_above = __ballot(above), m_same = __ballot(same);
        __syncthreads();
        if (lane == 0) parts[w] = __popcll(m_above) | __popcll(m_same) << 16;
        __syncthreads();
        int n_above = 0, n_same = 0, all_above = 0, all_same = 0;
        for (int i = 0; i < waves; i++) {
            const int v = parts[i];
            n_above += i < w ? v & 0xffff : 0;
            n_same += i < w ? v >> 16 : 0;
            all_above += v & 0xffff;
            all_same += v >> 16;
        }
        n_above += __popcll(m_above & below);
        n_same += equal + __popcll(m_same & below);
        if (above || (same && n_same < left)) to[written + n_above + min(n_same, left) - min(equal, left)] = table[p];
        written += all_above + min(equal + all_same, left) - min(equal, left);
        equal += all_same;
    }
}

template <bool BF, int D>
hipError_t select_pages(const void *q, long ldq, int heads, const KvCache &c, const KeyBounds &bounds, const KvRows &rows, int keep, int sinks, int recent, int *tables,
                        int *lens_out, hipStream_t st)
{
    auto kern = select_pages_kernel<BF, D>;
    const size_t lds = 4 * (size_t)rows.width;
    if (lds > 48 << 10)
        if (hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) return e;
    const int threads = rows.width <= 64 ? 256 : rows.width <= 512 ? 512 : 1024;
    hipLaunchKernelGGL(kern, dim3((unsigned)(rows.batch * c.kv_heads)), dim3(threads), lds, st, (const char *)q, ldq, c, bounds, rows, heads / c.kv_heads, keep, sinks,
                       recent, tables, lens_out);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_bounds(const KvCache &c, int D, const KeyBounds &bounds, const KvRows &r, hipStream_t st)
{
    const int most = min(r.width, ((r.max_rows - 1) >> c.page_shift) + 1);             // pages that max_rows positions in a row can fill
    const dim3 grid((unsigned)c.kv_heads, (unsigned)((most + 3) / 4), (unsigned)r.batch);
    auto kern = D == 128 ? cache_bounds_kernel<128> : cache_bounds_kernel<64>;
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, c, bounds, r);
    return hipGetLastError();
}

hipError_t launch_cache_select(const void *q, long ldq, bool bf16, int heads, int D, const KvCache &c, const KeyBounds &bounds, const KvRows &rows, int keep, int sinks,
                               int recent, int *tables, int *lens_out, hipStream_t st)
{
    if (D == 128) return bf16 ? select_pages<true, 128>(q, ldq, heads, c, bounds, rows, keep, sinks, recent, tables, lens_out, st)
                              : select_pages<false, 128>(q, ldq, heads, c, bounds, rows, keep, sinks, recent, tables, lens_out, st);
    return bf16 ? select_pages<true, 64>(q, ldq, heads, c, bounds, rows, keep, sinks, recent, tables, lens_out, st)
                : select_pages<false, 64>(q, ldq, heads, c, bounds, rows, keep, sinks, recent, tables, lens_out, st);
}

}  // namespace samp

// Which pages of a long context a query reads: bounds of the keys of each page, kept beside the cache, and the choice of the pages whose bounds promise most.
//
// A page's bounds are the largest and the smallest key in each channel, in 8 bits like the cache (2 head_dim + 4 bytes for page_len (head_dim + 4)).  No key of the page has a product with a
// query above sum_d max(q_d high_d, q_d low_d), which is the product of (positive part of q, negative part) and (high, low): one int8 matrix product of twice the length, exact,
// so that the choice is the same however it is computed.
#include "../../include/samp.h"
#include "decoder.h"
#include "decoder_rules.h"

namespace samp {
namespace {

constexpr float INV_127 = 1.0f / 127.0f;

// ---- bounds ------------------------------------------------------------------------------------------
// A wave takes a page of a key head: D / 16 lanes hold 16 channels each of 1024 / D keys at a time; then the lanes of the same channels meet and share them out, D / 64 of them a lane.
// What bounds it is HBM for whole prompts (16 of 2000 to 8192 positions, 8 key heads of 128: 88 MB, 18.5 us, 4.8 TB/s), and the launch for a decode step (3.4 us), in which few pages become
// full and the other waves end at once.
// Of two channels the lower half of the lanes (or of each 32, 16, 8) gets the first, the upper the second, each from both halves
template <int HALF, bool MAX> __device__ __forceinline__ float share(float a, float b, int lane)
{
    const Met m = meet<HALF>(a, b, lane);
    return MAX ? max3(m.x, m.x, m.y) : min3(m.x, m.x, m.y);
}

// AT: keys at a time, 32, or 16 for pages of no more (138 MB, inputs that change from call to call: in pages of 64 32.9 us, of 16 42.6, bound by the vector ALUs; the kernel of 32, each key twice,
// takes a quarter longer for those)
template <int D, int AT>
__global__ __launch_bounds__(256) void cache_bounds_kernel(KvCache c, KeyBounds bounds, KvRows rows)
{
    constexpr int LANES = D / 16, KEYS = 64 / LANES, TURN = AT / KEYS;
    const SeqRows s = seq_rows(rows, blockIdx.z, c.page_shift);
    const int lane = threadIdx.x & 63, from = max(rows.lens[blockIdx.z] - s.n, 0), to = min(rows.lens[blockIdx.z] - s.n + s.todo, s.len);
    const int index = (from >> c.page_shift) + blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), head = blockIdx.x;
    if (s.todo <= 0 || to <= 0 || index >= to >> c.page_shift) return;
    const int page = rows.table[(size_t)blockIdx.z * rows.width + index];
    if ((unsigned)page >= (unsigned)c.pages) return;
    const size_t at = (size_t)page * c.kv_heads + head, row = at << c.page_shift;
    const int8_t *const k = c.k + row * D + 16 * (lane % LANES);
    const float *const steps = c.k_step + row;
    const int len = 1 << c.page_shift;
    float high[16], low[16];
#pragma unroll
    for (int e = 0; e < 16; e++) {
        high[e] = -INFINITY;
        low[e] = INFINITY;
    }
    float odd = 0.0f;                                                 // NaN with a step that is not finite, that of a key that is not
    for (int i0 = 0; i0 < len; i0 += AT) {
        v4i raw[TURN];
        float step[TURN];
#pragma unroll
        for (int i = 0; i < TURN; i++) {
            const int key = i0 + i * KEYS + lane / LANES;
            raw[i] = *reinterpret_cast<const v4i *>(k + key * D);
            step[i] = steps[key];
        }
#pragma unroll
        for (int i = 0; i < TURN; i += 2) {
            constexpr int NEXT = TURN > 1;
            odd += step[i] * 0.0f + step[i + NEXT] * 0.0f;
#pragma unroll
            for (int e = 0; e < 16; e++) {
                const float x = (float)(int8_t)(raw[i][e >> 2] >> 8 * (e & 3)) * step[i], y = (float)(int8_t)(raw[i + NEXT][e >> 2] >> 8 * (e & 3)) * step[i + NEXT];
                high[e] = max3(high[e], x, y);
                low[e] = min3(low[e], x, y);
            }
        }
    }
    const bool bad = __any(!(odd == 0.0f));
    settle<16>(high);
    settle<16>(low);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        high[e] = share<32, true>(high[e], high[e + 8], lane);
        low[e] = share<32, false>(low[e], low[e + 8], lane);
    }
    settle<8>(high);
    settle<8>(low);
#pragma unroll
    for (int e = 0; e < 4; e++) {
        high[e] = share<16, true>(high[e], high[e + 4], lane);
        low[e] = share<16, false>(low[e], low[e + 4], lane);
    }
#pragma unroll
    for (int e = 0; e < 2; e++) {
        high[e] = share<8, true>(high[e], high[e + 2], lane);
        low[e] = share<8, false>(low[e], low[e + 2], lane);
    }
    constexpr int MINE = D / 64;                                      // channels of a lane
    int channel = 16 * (lane % LANES) + (lane >> 5 & 1) * 8 + (lane >> 4 & 1) * 4 + (lane >> 3 & 1) * 2;
    if constexpr (MINE == 1) {
        high[0] = share<4, true>(high[0], high[1], lane);
        low[0] = share<4, false>(low[0], low[1], lane);
        channel += lane >> 2 & 1;
    }
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < MINE; e++) top = max3(top, __builtin_fabsf(high[e]), __builtin_fabsf(low[e]));
    top = wave_max(top);
    const bool some = top > 0.0f && !bad;
    const float step = bad ? __builtin_nanf("") : some ? top * INV_127 : 1.0f;
    int codes[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < MINE; e++) {
        const float up = __builtin_fminf(__builtin_ceilf(__fdiv_rn(high[e], step)), 127.0f), down = __builtin_fmaxf(__builtin_floorf(__fdiv_rn(low[e], step)), -127.0f);
        codes[0] |= (some ? (int)up & 0xff : 0) << 8 * e;
        codes[1] |= (some ? (int)down & 0xff : 0) << 8 * e;
    }
#pragma unroll
    for (int i = 0; i < 2; i++) {
        int8_t *const to_codes = bounds.codes + (2 * at + i) * D + channel;
        if constexpr (MINE == 2) *reinterpret_cast<short *>(to_codes) = (short)codes[i];
        else *to_codes = (int8_t)codes[i];
    }
    if (lane == 0) bounds.steps[at] = step;
}

// ---- choice ------------------------------------------------------------------------------------------
// NaN counts as plus infinity
__device__ __forceinline__ unsigned order_of_score(float x) { return x != x ? order_of(INFINITY) : order_of(x); }
template <bool BF> __device__ __forceinline__ float largest(unsigned bits)
{
    return BF ? __uint_as_float(bits << 16) : (float)__builtin_bit_cast(_Float16, (unsigned short)bits);
}
constexpr unsigned ALWAYS = 0xfffffffeu;                              // above the order of every number, and a number above it

constexpr int BINS = 1024, LIST = 512, WORDS = SAMP_MAX_TABLE / 64;
struct Scored { unsigned score; int page; };

// What scores are made with: a sequence, a key head, its table and the queries that see it
struct Seen { SeqRows s; int b, head, group, pages, sinks, recent; const int *table; };

// The scores of the pages first .. first + 16 TILES - 1 of a sequence, a page a lane of the wave: f(page of the lane, score).  All waves of the block, four, call it together.  entry: the
// table's of the lane's page.  A wave requests the bounds of its pages together and keeps them for all rows of queries: 16 of them are the columns of a product, 16 rows of queries, which the
// block quantises while the bounds or the last product's operands are on their way, its rows.
template <bool BF, int D, int TILES, class F>
__device__ __forceinline__ void score_pages(const char *__restrict__ Q, long ldq, const KvCache &c, const KeyBounds &bounds, const Seen &seen, int first, int entry, F &&f)
{
    constexpr int STEPS = 2 * D / 64, PER = D / 16;                   // products of 64 codes; values of a lane, sixteen lanes a row of queries
    __shared__ __attribute__((aligned(16))) int8_t codes[16][2 * D];  // positive parts, negative parts of sixteen rows of queries
    __shared__ float steps[16];
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4, all = seen.s.todo * seen.group, pages = seen.pages, row = tid >> 4;
    auto request = [&](int r0) __attribute__((always_inline)) {
        v4i raw = {0, 0, 0, 0};
        if (r0 + row < all) {
            const int token = (r0 + row) / seen.group, h = seen.head * seen.group + (r0 + row) - token * seen.group;
            const char *from = Q + 2 * ((size_t)(seen.s.first_row + token) * ldq + h * D + r * PER);
            if constexpr (PER == 8) raw = *reinterpret_cast<const v4i *>(from);
            else {
                const v2i half = *reinterpret_cast<const v2i *>(from);
                raw[0] = half[0];
                raw[1] = half[1];
            }
        }
        return raw;
    };
    v4i raw = request(0);                                             // in front of the bounds: loads arrive in their order
    const bool ok = (unsigned)entry < (unsigned)c.pages;
    const float page_step = bounds.steps[(size_t)(ok ? entry : 0) * c.kv_heads + seen.head];
    v4i bf[TILES][STEPS];
#pragma unroll
    for (int t = 0; t < TILES; t++) {
        const int e = __shfl(ok ? entry : 0, 16 * t + r, 64);
        const int8_t *from = bounds.codes + ((size_t)e * c.kv_heads + seen.head) * (2 * D) + 16 * g;
#pragma unroll
        for (int i = 0; i < STEPS; i++) bf[t][i] = *reinterpret_cast<const v4i *>(from + 64 * i);
    }
    unsigned best[TILES];                                             // of the lane's rows of queries: minus infinity without any, as for a page that is none of the cache's
#pragma unroll
    for (int t = 0; t < TILES; t++) best[t] = order_of(-INFINITY);
    for (int r0 = 0; r0 < all; r0 += 16) {
        const unsigned top = max_of_16_lanes(bits_max16(raw));
        const RowQuant q = row_quant<BF>(top);
        float x[8];
        widen8<BF>(raw, x);
        const v2i code = quant8(x, q);
        if (r0) lds_barrier();
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
        raw = request(r0 + 16);
        lds_barrier();
        v4i qf[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; i++) qf[i] = *reinterpret_cast<const v4i *>(&codes[r][64 * i + 16 * g]);
        const v4f qs = *reinterpret_cast<const v4f *>(&steps[4 * g]);
#pragma unroll
        for (int t = 0; t < TILES; t++) {
            v4i sum = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < STEPS; i++) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(qf[i], bf[t][i], sum, 0, 0, 0);
            const float s = __shfl(page_step, 16 * t + r, 64);
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (r0 + 4 * g + e < all) best[t] = max(best[t], order_of_score((float)sum[e] * (qs[e] * s)));
        }
    }
    unsigned mine = 0;
#pragma unroll
    for (int t = 0; t < TILES; t++) {
        best[t] = max(best[t], (unsigned)__shfl_xor((int)best[t], 16, 64));
        best[t] = max(best[t], (unsigned)__shfl_xor((int)best[t], 32, 64));
        if (g == t) mine = best[t];
    }
    const int p = first + lane;
    if (!ok) mine = order_of(-INFINITY);
    if (p < seen.sinks || p >= pages - seen.recent) mine = ALWAYS;
    if (lane < 16 * TILES && p < pages) f(p, mine);
}

// Of a sequence that keeps only some of its pages and has more new tokens than max_rows, those behind the last row that is computed are none: what follows that row it does not see
__device__ __forceinline__ Seen what_is_seen(const KvCache &c, const KvRows &rows, int b, int head, int group, int keep, int sinks, int recent)
{
    Seen seen{seq_rows(rows, b, c.page_shift), b, head, group, 0, sinks, recent, rows.table + (size_t)b * rows.width};
    const int last = (1 << c.page_shift) - 1;
    seen.pages = (max(seen.s.len, 0) + last) >> c.page_shift;
    if (seen.pages > keep && seen.s.n > seen.s.todo) {
        const long upto = (long)rows.lens[b] - (seen.s.n - seen.s.todo);
        if (upto < seen.s.len) seen.pages = (int)(max(upto, 0l) + last) >> c.page_shift;
    }
    return seen;
}

// scores [batch, kv_heads, width]; a wave has 32 pages of a sequence and a key head.  What bounds it is a chain of dependent loads (lengths and page numbers, bounds) and then HBM: 64 contexts of 900 to 32768 tokens in
// pages of 64, 8 key heads of 128 (35 MB) 13.0 us, one of 100000 4.3; 25 of 85000 in pages of 32, 4 key heads, 35 rows of queries each (69 MB) 21 us, 37 where the bounds were read
// again for every sixteen rows.  (64 pages a wave: 13.5 and 5.4; blocks of the key heads of a page on one XCD, which shares their steps: no difference.)
constexpr int OF_WAVE = SCORES_BLOCK / 4;
template <bool BF, int D>
__global__ __launch_bounds__(256, 4) void page_scores_kernel(const char *__restrict__ Q, long ldq, KvCache c, KeyBounds bounds, KvRows rows, int group, int keep, int sinks,
                                                          int recent, unsigned *__restrict__ scores)
{
    const int head = blockIdx.x % c.kv_heads, item = blockIdx.x / c.kv_heads, chunk = item / rows.batch, b = item - chunk * rows.batch;
    const int first = chunk * SCORES_BLOCK + __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) * OF_WAVE), page = first + (threadIdx.x & 63);
    const int entry = rows.table[(size_t)b * rows.width + min(page, rows.width - 1)];              // (on its way with the lengths)
    const Seen seen = what_is_seen(c, rows, b, head, group, keep, sinks, recent);
    if (seen.pages <= keep || chunk * SCORES_BLOCK >= seen.pages) return;
    unsigned *const to = scores + ((size_t)b * c.kv_heads + head) * rows.width;
    score_pages<BF, D, OF_WAVE / 16>(Q, ldq, c, bounds, seen, first, page < seen.pages ? entry : -1,
                       [&](int p, unsigned x) { to[p] = x; });
}

// Whether a sequence keeps all its pages, which are its table then; and its length without those that it does not keep
__device__ __forceinline__ bool keeps_all(const KvCache &c, const KvRows &rows, const Seen &seen, int keep, int *__restrict__ to, int *__restrict__ lens_out)
{
    if (seen.head == 0 && threadIdx.x == 0) lens_out[seen.b] = rows.lens[seen.b] - ((seen.pages - min(seen.pages, keep)) << c.page_shift);
    if (seen.pages > keep) return false;
    for (int i = threadIdx.x; i < keep; i += blockDim.x) to[i] = i < seen.pages ? seen.table[i] : -1;
    return true;
}

// Scores formed by the block that chooses, a page a thread: a page is kept if fewer than `keep` come before it.  72 blocks of up to 157 pages 6.5 us; counting steps instead, as below, 7.0.
template <bool BF, int D>
__global__ __launch_bounds__(SCORED_TOGETHER, 4) void select_pages_kernel(const char *__restrict__ Q, long ldq, KvCache c, KeyBounds bounds, KvRows rows, int group, int keep,
                                                                          int sinks, int recent, int *__restrict__ tables, int *__restrict__ lens_out)
{
    constexpr int WAVES = SCORED_TOGETHER / 64;
    __shared__ __attribute__((aligned(16))) unsigned score[SCORED_TOGETHER];
    __shared__ unsigned long long bits[WAVES];
    const int b = blockIdx.x / c.kv_heads, page = threadIdx.x, lane = page & 63, w = __builtin_amdgcn_readfirstlane(page >> 6);
    const int entry = rows.table[(size_t)b * rows.width + min(page, rows.width - 1)];
    const Seen seen = what_is_seen(c, rows, b, blockIdx.x - b * c.kv_heads, group, keep, sinks, recent);
    int *const to = tables + (size_t)blockIdx.x * keep;
    if (keeps_all(c, rows, seen, keep, to, lens_out)) return;
    if (page >= seen.pages) score[page] = 0;
    score_pages<BF, D, 4>(Q, ldq, c, bounds, seen, __builtin_amdgcn_readfirstlane(page & ~63), page < seen.pages ? entry : -1,
                          [&](int p, unsigned x) { score[p] = x; });
    lds_barrier();
    const unsigned mine = score[page];
    int better = 0;
    for (int v = 0; v < WAVES && 64 * v < seen.pages; v++) {
        const int others = (int)score[64 * v + lane];                 // of 64 pages, each to all lanes in turn
        // an equal score counts where its page is an earlier one
        if (v == w) {
#pragma unroll
            for (int i = 0; i < 64; i++) better += (unsigned)__builtin_amdgcn_readlane(others, i) >= mine + (i >= lane);
        } else {
            const unsigned least = mine + (v > w);
#pragma unroll
            for (int i = 0; i < 64; i++) better += (unsigned)__builtin_amdgcn_readlane(others, i) >= least;
        }
    }
    const bool kept = page < seen.pages && better < keep;
    const unsigned long long word = __ballot(kept);
    if (lane == 0) bits[w] = word;
    lds_barrier();
    int at = __popcll(word & ((1ull << lane) - 1));
    for (int v = 0; v < w; v++) at += __popcll(bits[v]);
    if (kept) to[at] = entry;
}

// Scores that are there already.  They are counted in BINS steps between the smallest and the largest; the pages of the step in which the `keep`-th largest lies are ranked by counting, and
// where they are too many (equal scores), that score is found eight bits at a time.  A chain of steps on one CU a key head: 8 blocks of 1563 pages 5.5 us, 512 of up to 512 5.1, 8 of
// 32768 28.
__global__ __launch_bounds__(1024) void select_scored_kernel(KvCache c, KvRows rows, int keep, int sinks, int recent, const unsigned *__restrict__ scores,
                                                             int *__restrict__ tables, int *__restrict__ lens_out)
{
    extern __shared__ __attribute__((aligned(16))) unsigned score[];  // [width]
    __shared__ __attribute__((aligned(16))) int count[BINS];
    __shared__ Scored list[LIST];
    __shared__ unsigned long long bits[WORDS];
    __shared__ float lows[16], highs[16];
    __shared__ int found[2], listed;                                  // a digit, and how many are above it
    const int b = blockIdx.x / c.kv_heads, step = blockDim.x, tid = threadIdx.x, lane = tid & 63, waves = step >> 6, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned *const from = scores + (size_t)blockIdx.x * rows.width;
    unsigned x[4];
#pragma unroll
    for (int u = 0; u < 4; u++) x[u] = from[min(tid + u * step, rows.width - 1)];              // (on their way with the lengths; what nobody wrote is not used)
    const Seen seen = what_is_seen(c, rows, b, blockIdx.x - b * c.kv_heads, 1, keep, sinks, recent);
    const int pages = seen.pages, groups = (pages + 63) >> 6;
    const int *const table = seen.table;
    int *const to = tables + (size_t)blockIdx.x * keep;
    if (keeps_all(c, rows, seen, keep, to, lens_out)) return;
    for (int i = tid; i < BINS; i += step) count[i] = 0;
    if (tid == 0) listed = 0;
    // steps of the scores that are finite
    float low = INFINITY, high = -INFINITY;
    auto have = [&](int p, unsigned x) __attribute__((always_inline)) {
        if (p >= pages) return;
        score[p] = x;
        const float value = value_of_order(x);
        if (x != ALWAYS && __builtin_isfinite(value)) {
            low = __builtin_fminf(low, value);
            high = __builtin_fmaxf(high, value);
        }
    };
#pragma unroll
    for (int u = 0; u < 4; u++) have(tid + u * step, x[u]);
    for (int p0 = tid + 4 * step; p0 < pages; p0 += 8 * step) {
        unsigned more[8];
#pragma unroll
        for (int u = 0; u < 8; u++) more[u] = from[min(p0 + u * step, pages - 1)];
#pragma unroll
        for (int u = 0; u < 8; u++) have(p0 + u * step, more[u]);
    }
    low = -wave_max(-low);
    high = wave_max(high);
    if (lane == 0) {
        lows[w] = low;
        highs[w] = high;
    }
    lds_barrier();
    for (int i = 0; i < waves; i++) {
        low = __builtin_fminf(low, lows[i]);
        high = __builtin_fmaxf(high, highs[i]);
    }
    const float rate = high > low ? (float)(BINS - 1) / (high - low) : 0.0f;
    // (rising with the score whatever the roundings: differences, products and whole parts do)
    auto bin_of = [&](unsigned x) {
        const float v = value_of_order(x), f = (v - low) * rate;
        return v <= low ? 0 : v >= high ? BINS - 1 : f < (float)(BINS - 1) ? (int)f : BINS - 1;
    };
    for (int p = 64 * w + lane; p < pages; p += 64 * waves)
        if (score[p] != ALWAYS) atomicAdd(&count[bin_of(score[p])], 1);
    lds_barrier();
    const int want = keep - min(sinks, pages) - min(recent, pages);   // of the pages that are not kept anyway
    if (w == 0) {
        // lane l has the steps 16 l .. 16 l + 15 from above; then sixteen lanes have one each of those of the lane in which the `want`-th lies
        int sum = 0;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const v4i four = *reinterpret_cast<const v4i *>(&count[BINS - 16 * lane - 4 * i - 4]);
            sum += (four[0] + four[1]) + (four[2] + four[3]);
        }
        const int upto = wave_scan(sum), owner = min((int)__popcll(__ballot(upto < want)), 63);
        const int in_front = owner ? __builtin_amdgcn_readlane(upto, owner - 1) : 0;
        const int one = lane < 16 ? count[BINS - 1 - 16 * owner - lane] : 0, then = in_front + wave_scan(one);
        if (lane < 16 && then >= want && then - one < want) {
            found[0] = BINS - 1 - 16 * owner - lane;
            found[1] = then - one;
        }
        if (want <= 0 && lane == 0) {
            found[0] = BINS;
            found[1] = 0;
        }
    }
    lds_barrier();
    const int step_of_last = found[0], left = want - found[1];
    for (int p0 = 64 * w; p0 < pages; p0 += 64 * waves) {
        const int p = p0 + lane;
        const unsigned x = score[min(p, pages - 1)];
        const int bin = p >= pages ? -1 : x == ALWAYS ? BINS + 1 : bin_of(x);      // (found[0] is BINS where only those that are always kept are)
        const unsigned long long word = __ballot(bin > step_of_last);
        if (lane == 0) bits[p0 >> 6] = word;
        if (bin == step_of_last && x != ALWAYS) {
            const int at = atomicAdd(&listed, 1);                     // (in any order: they are ranked)
            if (at < LIST) list[at] = Scored{x, p};
        }
    }
    lds_barrier();
    const int n = listed;
    if (n <= LIST) {
        for (int i = tid; i < n; i += blockDim.x) {
            const Scored mine = list[i];
            int better = 0;
#pragma unroll 4
            for (int j = 0; j < n; j++) better += (list[j].score > mine.score) | ((list[j].score == mine.score) & (list[j].page < mine.page));
            if (better < left) atomicOr(&bits[mine.page >> 6], 1ull << (mine.page & 63));
        }
    } else {
        unsigned least = 0;                                           // scores above it are kept too, of pages of that step
        int rest = left;
        for (int shift = 24; shift >= 0; shift -= 8) {
            lds_barrier();
            for (int i = tid; i < 256; i += blockDim.x) count[i] = 0;
            lds_barrier();
            for (int p = 64 * w + lane; p < pages; p += 64 * waves) {
                const unsigned x = score[p];
                if (x != ALWAYS && bin_of(x) == step_of_last && (shift == 24 || (x ^ least) >> (shift + 8) == 0)) atomicAdd(&count[x >> shift & 255], 1);
            }
            lds_barrier();
            if (w == 0) {
                int m[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; i++) sum += m[i] = count[255 - 4 * lane - i];
                int before = wave_scan(sum) - sum;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    if (before < rest && before + m[i] >= rest) {
                        found[0] = 255 - 4 * lane - i;
                        found[1] = before;
                    }
                    before += m[i];
                }
            }
            lds_barrier();
            least |= (unsigned)found[0] << shift;
            rest -= found[1];
        }
        // of the pages of just that score the first `rest`
        for (int p0 = 64 * w; p0 < pages; p0 += 64 * waves) {
            const unsigned long long word = __ballot(p0 + lane < pages && score[p0 + lane] == least);
            if (lane == 0) bits[p0 >> 6] = word;
        }
        lds_barrier();
        if (w == 0) {
            int before = 0;
            for (int i0 = 0; i0 < groups; i0 += 64) {
                unsigned long long word = i0 + lane < groups ? bits[i0 + lane] : 0;
                const int m = __popcll(word), upto = wave_scan(m);
                int drop = before + upto - rest;                      // of this word the last `drop` go
                for (; drop > 0 && word; drop--) word &= ~(1ull << (63 - __builtin_clzll(word)));
                if (i0 + lane < groups) bits[i0 + lane] = word;
                before += __shfl(upto, 63, 64);
            }
        }
        lds_barrier();
        for (int p0 = 64 * w; p0 < pages; p0 += 64 * waves) {
            const unsigned x = p0 + lane < pages ? score[p0 + lane] : 0;
            const int bin = x == ALWAYS ? BINS : bin_of(x);
            const unsigned long long word = __ballot(p0 + lane < pages && (x == ALWAYS || bin > step_of_last || (bin == step_of_last && x > least)));
            if (lane == 0) bits[p0 >> 6] |= word;
        }
    }
    lds_barrier();
    // the pages that are kept, in order, where the scores were; then their numbers
    int before = 0;
    for (int i0 = 0; i0 < groups; i0 += 64) {
        const int upto = wave_scan(i0 + lane < groups ? __popcll(bits[i0 + lane]) : 0);
        for (int i = (i0 + waves - 1 - w) / waves * waves + w; i < min(i0 + 64, groups); i += waves) {
            const unsigned long long word = bits[i];
            const int at = before + (i > i0 ? __builtin_amdgcn_readlane(upto, max(i - i0 - 1, 0)) : 0);
            if (word >> lane & 1) score[at + __popcll(word & ((1ull << lane) - 1))] = 64 * i + lane;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    lds_barrier();
    for (int i = tid; i < keep; i += step) to[i] = table[score[i]];
}

template <bool BF, int D>
hipError_t select_pages(const void *q, long ldq, int heads, const KvCache &c, const KeyBounds &bounds, const KvRows &rows, int keep, int sinks, int recent, int *tables,
                        int *lens_out, unsigned *scores, hipStream_t st)
{
    const size_t lds = 4 * (size_t)rows.width;
    const int group = heads / c.kv_heads;
    const dim3 grid((unsigned)(rows.batch * c.kv_heads));
    if (!scores_apart(rows.width)) {
        hipLaunchKernelGGL((select_pages_kernel<BF, D>), grid, dim3(SCORED_TOGETHER), 0, st, (const char *)q, ldq, c, bounds, rows, group, keep, sinks, recent, tables, lens_out);
        return hipGetLastError();
    }
    if (lds > 40 << 10)
        if (hipError_t e = hipFuncSetAttribute((const void *)select_scored_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) return e;
    const unsigned items = (unsigned)((rows.width + SCORES_BLOCK - 1) / SCORES_BLOCK) * rows.batch;
    hipLaunchKernelGGL((page_scores_kernel<BF, D>), dim3(items * c.kv_heads), dim3(256), 0, st, (const char *)q, ldq, c, bounds, rows, group, keep, sinks, recent,
                       scores);
    if (hipError_t e = hipGetLastError()) return e;                   // (the choice reads what they wrote)
    hipLaunchKernelGGL(select_scored_kernel, grid, dim3(choice_threads(rows.width)), lds, st, c, rows, keep, sinks, recent, scores, tables, lens_out);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_bounds(const KvCache &c, int D, const KeyBounds &bounds, const KvRows &r, hipStream_t st)
{
    const int most = min(r.width, ((r.max_rows - 1) >> c.page_shift) + 1);             // pages that max_rows positions in a row can fill
    const dim3 grid((unsigned)c.kv_heads, (unsigned)((most + 3) / 4), (unsigned)r.batch);
    auto kern = c.page_shift == 4 ? (D == 128 ? cache_bounds_kernel<128, 16> : cache_bounds_kernel<64, 16>) : D == 128 ? cache_bounds_kernel<128, 32> : cache_bounds_kernel<64, 32>;
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, c, bounds, r);
    return hipGetLastError();
}

size_t cache_select_workspace(int batch, int kv_heads, int width) { return scores_apart(width) ? 4 * (size_t)batch * kv_heads * width : 0; }

hipError_t launch_cache_select(const void *q, long ldq, bool bf16, int heads, int D, const KvCache &c, const KeyBounds &bounds, const KvRows &rows, int keep, int sinks,
                               int recent, int *tables, int *lens_out, void *ws, hipStream_t st)
{
    unsigned *const scores = static_cast<unsigned *>(ws);
    if (D == 128) return bf16 ? select_pages<true, 128>(q, ldq, heads, c, bounds, rows, keep, sinks, recent, tables, lens_out, scores, st)
                              : select_pages<false, 128>(q, ldq, heads, c, bounds, rows, keep, sinks, recent, tables, lens_out, scores, st);
    return bf16 ? select_pages<true, 64>(q, ldq, heads, c, bounds, rows, keep, sinks, recent, tables, lens_out, scores, st)
                : select_pages<false, 64>(q, ldq, heads, c, bounds, rows, keep, sinks, recent, tables, lens_out, scores, st);
}

}  // namespace samp

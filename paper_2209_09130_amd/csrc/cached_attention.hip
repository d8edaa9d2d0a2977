// Attention of a few new tokens per sequence over the int8 cache: O = softmax(scale q K^T) V with K = step_k[key] codes, V = step_v[key] codes.
//
// What bounds it is HBM: 2 (head_dim + 4) bytes per token and key head, against which the products are small.  So the loop is a stream: every wave
// takes key tiles of its own (32 keys) straight from the pages into registers, there is no LDS and no barrier before its end, and the
// query heads of a group (and the new tokens of a sequence) share what was read as the columns of the matrix products.  Long contexts are cut into
// pieces (splits), each with a partial result, which a second kernel joins.  Medians, both kernels: 64 contexts of 17 to 8192 tokens, 32 query heads on 8 key heads of 128
// (556 MB), 112.5 + 5.0 us, 4.7 TB/s; one context of 4000 5.9 + 4.0 us, a chain of dependent loads (offsets, page numbers, keys) and a launch.  Tried and dropped: the
// next tile's loads ahead of this one's work (64 contexts +-0, 16 drafts +3 %: other waves hide it, and it costs one of three per SIMD).  The last block of a row could join its
// pieces, stored and read at device scope, if a counter of theirs started at zero: the workspace is the caller's and holds anything.
//
// Products are 16 x 16 x 32.  S^T = K Q^T is in the queries' type, in which int8 codes are exact.  In binary16 1024 + (code + 128) is a code's byte under the
// exponent byte 0x64, and one packed addition takes 1152 off again; in bfloat16 a code is the upper half of its binary32.  A lane gets four keys of one
// query, two such tiles are the eight keys that it needs as the operand of O^T += V^T P^T.  V^T is formed on the way: a lane holds head_dim / 16 neighbouring channels
// of eight keys, and the byte permute that packs widened codes takes the two halves of a dword from two keys.  The steps of the keys multiply products (K)
// and probabilities (V) in binary32.
//
// O^T += V^T P^T is in bfloat16, in which codes are exact too and whose range is binary32's: p step_v of a key may be any size next to that of another (rows of zeros
// have step 1, and one large channel makes the step of a row in all of them), so no power of two for all of them would keep binary16 from losing the small
// ones.  Its 8 bits are made 16 by a second product with what was rounded off, 2^-16 of each p step_v and below (the matrix cores are idle most of the time).
//
// Softmax in one pass with a running reference m per query, which is ABOVE the scores (in powers of two), so that p times the largest step (2^121) and the sums stay
// inside binary32.  m moves (and the sums are scaled) only when a score exceeds what it was set for by 2^8, not for every new maximum.
#include "decoder.h"
#include "mfma_tile.h"

namespace samp {
namespace {

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
constexpr float LOWEST = -3.0e38f, SLACK = 8.0f, ABOVE = 24.0f;
constexpr int TILE = 32;                                              // keys of a wave's step

// halves 1024 + 128 + code from the dword whose bytes 0 and 2 are codes and 1 and 3 are zero; codes as binary16
__device__ __forceinline__ int to_halves(unsigned bytes)
{
    const v2h biased = __builtin_bit_cast(v2h, bytes ^ 0x64806480u);
    return __builtin_bit_cast(int, biased - v2h{(_Float16)1152.0f, (_Float16)1152.0f});
}

// bytes LO and HI of two dwords as two bfloat16 (a code's binary32 has no more than the upper half)
template <int LO, int HI> __device__ __forceinline__ int to_bfloats(int lo, int hi)
{
    const float a = (float)(int8_t)(lo >> 8 * LO), b = (float)(int8_t)(hi >> 8 * HI);
    return (int)__builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
template <bool BF> __device__ __forceinline__ v4f mma(const v4i &a, const v4i &b, const v4f &c)
{
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

template <int D> struct KeyTile {
    v4i k[2][D / 64];                                                 // two rows (keys r, 16 + r), 16 codes of each 64
    int v[8][D / 64];                                                 // eight keys, D / 16 codes
    v4f ks[2], vs[2];                                                 // steps of keys 4 g .. 4 g + 3 and 16 + 4 g ..
    unsigned known;                                                   // bit h: the page of keys 16 h .. 16 h + 15 is one of the cache's
};

// entries: the table's, of the tile's two groups of 16 keys (which lie in one page each)
template <int D>
__device__ __forceinline__ KeyTile<D> load_tile(const KvCache &c, const int (&entries)[2], int head, int j0, int last, int r, int g)
{
    KeyTile<D> t;
    t.known = 0;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int pos = min(j0 + 16 * h, last);                       // past the end the last keys are read again, and masked
        const bool ok = (unsigned)entries[h] < (unsigned)c.pages;
        t.known |= (unsigned)ok << h;
        const int page = ok ? entries[h] : 0;
        const size_t row = (((size_t)page * c.kv_heads + head) << c.page_shift) + (pos & ((1 << c.page_shift) - 1) & ~15);
        const int8_t *k = c.k + row * D, *v = c.v + row * D;
#pragma unroll
        for (int i = 0; i < D / 64; i++) t.k[h][i] = *reinterpret_cast<const v4i *>(k + r * D + 64 * i + 16 * g);
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int8_t *at = v + (4 * g + u) * D + r * (D / 16);
            if constexpr (D == 128) {
                const v2i two = *reinterpret_cast<const v2i *>(at);
                t.v[4 * h + u][0] = two[0];
                t.v[4 * h + u][1] = two[1];
            } else t.v[4 * h + u][0] = *reinterpret_cast<const int *>(at);
        }
        t.ks[h] = *reinterpret_cast<const v4f *>(c.k_step + row + 4 * g);
        t.vs[h] = *reinterpret_cast<const v4f *>(c.v_step + row + 4 * g);
    }
    return t;
}

// A context of more than `piece` tiles is cut into pieces of so many, at most `splits` of them (the last takes what is left); the parts of one that is not are the result
__device__ __forceinline__ int pieces_of(int tiles, int piece, int splits) { return min(max((tiles + piece - 1) / piece, 1), splits); }

// One block: sequence, key head, 16 QT rows (row = new token x query heads of the group + head in the group) and one split's key tiles, which its
// four waves take in turn.  partials: per row of the call and split head_dim sums, then the rows' (reference, sum of exponentials).
template <bool BF, int D, int QT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void cached_attention_kernel(const char *__restrict__ Q, long ldq, KvCache c, KvRows rows, int group, int chunks, int splits, int piece, float scale,
                             const uint64_t *__restrict__ tree, float *__restrict__ partials, char *__restrict__ out)
{
    constexpr int QR = 16 * QT, DV = D / 16;
    __shared__ __attribute__((aligned(16))) float so[4][QR][D + 4];
    __shared__ float sm[4][QR], sl[4][QR];
    // key heads run fastest: their work is alike, so the XCDs, to which blocks go in turn, have the same share whatever the lengths are (pieces running
    // fastest, 64 contexts of 17 to 8192 tokens in pieces of 1024: 149 us, of 768 119.5)
    int item = blockIdx.x;
    const int head = item % c.kv_heads;
    item /= c.kv_heads;
    const int b = item % rows.batch;
    item /= rows.batch;
    const int chunk = item % chunks, split = item / chunks;
    const SeqRows s = seq_rows(rows, b, c.page_shift);
    const int r0 = chunk * QR, all = s.todo * group, tiles = (max(s.len, 0) + TILE - 1) / TILE, pieces = pieces_of(tiles, piece, splits);
    if (r0 >= all || split >= pieces) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    const int heads = c.kv_heads * group, len = max(s.len, 0);
    const int first = rows.lens[b] - s.n;                             // position of the first new token (negative: more new tokens than positions)
    const int *table = rows.table + (size_t)b * rows.width;

    // Table entries of the wave's tiles, 32 at a time (lane 2 i + h: group h of its i-th tile): looked up one by one, each would stand in front of its tile's loads
    const int end = split == pieces - 1 ? tiles : (split + 1) * piece, last = (len - 1) & ~15;
    int t = split * piece + w, entries = -1;
    auto look_up = [&]() {
        const int pos = min((t + 4 * (lane >> 1)) * TILE + 16 * (lane & 1), last);
        entries = table[max(pos, 0) >> c.page_shift];
    };
    look_up();

    // queries: operand step (i, half) holds channels 64 i + 16 g + 8 half .. + 7
    v4i qf[QT][D / 32];
    int limit[QT];                                                    // positions below it are seen; from `first` on the word's bits decide if there are drafts
    uint64_t word[QT];
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        const int row = min(r0 + 16 * qt + r, all - 1), token = row / group, h = head * group + row - token * group;
        const char *from = Q + 2 * ((size_t)(s.first_row + token) * ldq + h * D + 16 * g);
        limit[qt] = min(tree ? len : first + token + 1, len);
        word[qt] = tree ? tree[s.first_row + token] : ~0ull;
#pragma unroll
        for (int i = 0; i < D / 32; i++) qf[qt][i] = *reinterpret_cast<const v4i *>(from + 128 * (i >> 1) + 16 * (i & 1));
    }
    const float factor = scale * 1.44269504088896341f;
    v4f o[QT][DV];
    float m[QT], l[QT];
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        m[qt] = LOWEST;
        l[qt] = 0.0f;
#pragma unroll
        for (int j = 0; j < DV; j++) o[qt][j] = v4f{0.f, 0.f, 0.f, 0.f};
    }

    const int whole = min(first, len) / TILE;                         // tiles below it are seen by every row
    for (int i = 0; t < end; t += 4, i++) {
        if (i == 32) {
            look_up();
            i = 0;
        }
        const int mine[2] = {__builtin_amdgcn_readlane(entries, 2 * i), __builtin_amdgcn_readlane(entries, 2 * i + 1)};
        const KeyTile<D> kt = load_tile<D>(c, mine, head, t * TILE, last, r, g);
        v4i kf[2][D / 32];
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
            for (int i = 0; i < D / 64; i++)
#pragma unroll
                for (int half = 0; half < 2; half++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const int four = kt.k[h][i][2 * half + e];
                        v4i &to = kf[h][2 * i + half];
                        if constexpr (BF) {
                            to[2 * e] = to_bfloats<0, 1>(four, four);
                            to[2 * e + 1] = to_bfloats<2, 3>(four, four);
                        } else {
                            to[2 * e] = to_halves(__builtin_amdgcn_perm(0u, (unsigned)four, 0x0c010c00u));
                            to[2 * e + 1] = to_halves(__builtin_amdgcn_perm(0u, (unsigned)four, 0x0c030c02u));
                        }
                    }
        v4i pf[QT], pl[QT];
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            float sc[2][4], top = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                v4f acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < D / 32; i++) acc = mma<BF>(kf[h][i], qf[qt][i], acc);
#pragma unroll
                for (int e = 0; e < 4; e++) sc[h][e] = acc[e] * kt.ks[h][e];
            }
            unsigned masked = 0;                                      // bit 4 h + e
            if (t >= whole || kt.known != 3u) {
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const int pos = t * TILE + 16 * h + 4 * g + e, draft = pos - first;
                        const bool seen = pos < limit[qt] && (kt.known >> h & 1u) && (draft < 0 || (draft < 64 ? (word[qt] >> draft) & 1 : tree == nullptr));
                        if (!seen) sc[h][e] = -INFINITY;
                        masked |= (unsigned)!seen << (4 * h + e);
                    }
            }
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int e = 0; e < 4; e++) top = __builtin_fmaxf(top, sc[h][e]);
            top *= factor;
            if (__any(top > m[qt] - (ABOVE - SLACK))) {
                top = __builtin_fmaxf(top, __shfl_xor(top, 16, 64));
                top = __builtin_fmaxf(top, __shfl_xor(top, 32, 64));
                const float to = top > m[qt] - (ABOVE - SLACK) ? top + ABOVE : m[qt], down = __builtin_amdgcn_exp2f(m[qt] - to);
                m[qt] = to;
                l[qt] *= down;
#pragma unroll
                for (int j = 0; j < DV; j++) o[qt][j] *= down;
            }
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    float pv[2];
#pragma unroll
                    for (int u = 0; u < 2; u++) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[h][e + u], factor, -m[qt]));
                        l[qt] += p;
                        pv[u] = masked >> (4 * h + e + u) & 1u ? 0.0f : p * kt.vs[h][e + u];
                    }
                    const int first_part = narrow2<true>(pv[0], pv[1]);
                    pf[qt][2 * h + (e >> 1)] = first_part;
                    pl[qt][2 * h + (e >> 1)] = narrow2<true>(pv[0] - __uint_as_float((unsigned)first_part << 16), pv[1] - __uint_as_float((unsigned)first_part & 0xffff0000u));
                }
        }
        each_index([&](auto j_tag) {
            constexpr int J = decltype(j_tag)::value;
            v4i x;
#pragma unroll
            for (int u = 0; u < 4; u++) x[u] = to_bfloats<J & 3, J & 3>(kt.v[2 * u][J >> 2], kt.v[2 * u + 1][J >> 2]);
#pragma unroll
            for (int qt = 0; qt < QT; qt++) {
                o[qt][J] = mma<true>(x, pf[qt], o[qt][J]);
                o[qt][J] = mma<true>(x, pl[qt], o[qt][J]);
            }
        }, std::make_integer_sequence<int, DV>());
    }

    // the waves' parts meet: the lane's channels are DV (4 g + e) + j of query r
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        l[qt] += __shfl_xor(l[qt], 16, 64);
        l[qt] += __shfl_xor(l[qt], 32, 64);
        if (g == 0) {
            sm[w][16 * qt + r] = m[qt];
            sl[w][16 * qt + r] = l[qt];
        }
#pragma unroll
        for (int e = 0; e < 4; e++)
#pragma unroll
            for (int j = 0; j < DV; j += 4)
                *reinterpret_cast<v4f *>(&so[w][16 * qt + r][DV * (4 * g + e) + j]) = v4f{o[qt][j][e], o[qt][j + 1][e], o[qt][j + 2][e], o[qt][j + 3][e]};
    }
    __syncthreads();
    constexpr int LANES = D / 8;                                      // lanes of a row, eight channels each
    for (int at = tid / LANES; at < QR && r0 + at < all; at += 256 / LANES) {
        const int row = r0 + at, token = row / group, h = head * group + row - token * group, d = tid % LANES * 8;
        float top = sm[0][at], sum = 0.0f, f[4], y[8];
#pragma unroll
        for (int u = 1; u < 4; u++) top = __builtin_fmaxf(top, sm[u][at]);
#pragma unroll
        for (int u = 0; u < 4; u++) {
            f[u] = __builtin_amdgcn_exp2f(sm[u][at] - top);
            sum += sl[u][at] * f[u];
        }
#pragma unroll
        for (int e = 0; e < 8; e++) {
            y[e] = 0.0f;
#pragma unroll
            for (int u = 0; u < 4; u++) y[e] += so[u][at][d + e] * f[u];
        }
        const size_t to = (size_t)(s.first_row + token) * heads + h;
        if (pieces == 1) {
            const float by = sum != 0.0f ? __fdiv_rn(1.0f, sum) : 0.0f;        // a row that sees nothing is zeros
            const v4i packed = {narrow2<BF>(y[0] * by, y[1] * by), narrow2<BF>(y[2] * by, y[3] * by), narrow2<BF>(y[4] * by, y[5] * by),
                                narrow2<BF>(y[6] * by, y[7] * by)};
            *reinterpret_cast<v4i *>(out + 2 * (to * D + d)) = packed;
        } else {
            float *p = partials + (to * splits + split) * D + d;
            *reinterpret_cast<v4f *>(p) = v4f{y[0], y[1], y[2], y[3]};
            *reinterpret_cast<v4f *>(p + 4) = v4f{y[4], y[5], y[6], y[7]};
            if (d == 0) {
                float *ml = partials + (size_t)rows.rows * heads * splits * D + 2 * (to * splits + split);
                ml[0] = top;
                ml[1] = sum;
            }
        }
    }
}

// Joins the pieces of the sequences that have several: a wave per row, D / 8 lanes of eight channels, the others of the wave taking pieces of their own.
constexpr int MAX_SPLITS = 64;
template <bool BF, int D>
__global__ __launch_bounds__(256) void join_pieces_kernel(KvRows rows, int heads, int splits, int piece, int page_shift, const float *__restrict__ partials,
                                                          char *__restrict__ out)
{
    constexpr int LANES = D / 8, AT_ONCE = 64 / LANES;
    const SeqRows s = seq_rows(rows, blockIdx.y, page_shift);
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), d = lane % LANES * 8;
    const int pieces = pieces_of((max(s.len, 0) + TILE - 1) / TILE, piece, splits);
    if (row >= s.todo * heads || pieces == 1) return;
    const size_t at = (size_t)s.first_row * heads + row;
    const float *ml = partials + (size_t)rows.rows * heads * splits * D + 2 * at * splits, *p = partials + at * splits * D + d;
    const float m = lane < pieces ? ml[2 * lane] : LOWEST, l = lane < pieces ? ml[2 * lane + 1] : 0.0f;
    constexpr int BATCH = 4;
    float y[8] = {}, factor = 0.0f, sum = 0.0f;
    for (int i0 = 0; i0 < pieces; i0 += BATCH * AT_ONCE) {
        v4f a[BATCH][2];
#pragma unroll
        for (int u = 0; u < BATCH; u++) {
            const float *from = p + (size_t)min(i0 + u * AT_ONCE + lane / LANES, pieces - 1) * D;
            a[u][0] = *reinterpret_cast<const v4f *>(from);
            a[u][1] = *reinterpret_cast<const v4f *>(from + 4);
        }
        if (i0 == 0) {
            factor = __builtin_amdgcn_exp2f(m - wave_max(m));
            sum = l * factor;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        }
#pragma unroll
        for (int u = 0; u < BATCH; u++) {
            const int i = i0 + u * AT_ONCE + lane / LANES;
            const float f = __shfl(factor, min(i, pieces - 1), 64);
            if (i < pieces) {
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    y[e] += a[u][0][e] * f;
                    y[4 + e] += a[u][1][e] * f;
                }
            }
        }
    }
#pragma unroll
    for (int o = LANES; o < 64; o <<= 1)
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] += __shfl_xor(y[e], o, 64);
    const float by = sum != 0.0f ? __fdiv_rn(1.0f, sum) : 0.0f;
    if (lane < LANES)
        *reinterpret_cast<v4i *>(out + 2 * (at * D + d)) = v4i{narrow2<BF>(y[0] * by, y[1] * by), narrow2<BF>(y[2] * by, y[3] * by),
                                                               narrow2<BF>(y[4] * by, y[5] * by), narrow2<BF>(y[6] * by, y[7] * by)};
}

int row_tiles(long rows) { return rows > 16 ? 2 : 1; }

template <bool BF, int D>
hipError_t cached_attention(const void *q, long ldq, int heads, const KvCache &c, const KvRows &rows, float scale, const uint64_t *tree, Cut cut,
                            float *partials, void *out, hipStream_t st)
{
    const int group = heads / c.kv_heads, most = rows.max_rows * group, qt = row_tiles(most), chunks = (most + 16 * qt - 1) / (16 * qt);
    auto kern = qt == 1 ? cached_attention_kernel<BF, D, 1> : cached_attention_kernel<BF, D, 2>;
    hipLaunchKernelGGL(kern, dim3((unsigned)rows.batch * c.kv_heads * cut.splits * chunks), dim3(256), 0, st, (const char *)q, ldq, c, rows, group, chunks, cut.splits,
                       cut.piece, scale, tree, partials, (char *)out);
    if (cut.splits > 1)
        hipLaunchKernelGGL((join_pieces_kernel<BF, D>), dim3((unsigned)((most * c.kv_heads + 3) / 4), (unsigned)rows.batch), dim3(256), 0, st,
                           rows, heads, cut.splits, cut.piece, c.page_shift, partials, (char *)out);
    return hipGetLastError();
}

}  // namespace

// Pieces of so many tiles that 512 blocks have them all, but no less than four tiles (a tile for each wave; eight where a block has two row tiles), below which
// the blocks' own latencies count for more than their number, and no more than 48, so that blocks of contexts of different lengths end together: 48 for 512 blocks
// without a cut, more in proportion where there are more.  None at all where a context has at most sixteen tiles more than a piece, or where blocks of two row
// tiles (many new tokens) are 512 without and no context has more than a million positions (some 20 ms of one block): their partial results are what costs
// then.  us and MB of those, in pieces of 48 / uncut, 32 query heads on 8 of 128: 512 tokens of a context of 4500 114 and 24 / 93, of 64 contexts up to 4500 4580 and
// 1560 / 4440, 128 tokens of 16 contexts up to 8192 504 and 195 / 433; one token of 128 contexts up to 8192 223 in pieces of 48 or 96, 231 to 235 uncut.  Joining
// costs a launch.  Both kernels, us, by tiles of a piece (4 / 8 / 16 / 32 / 64 / uncut): 32 query heads on 8
// key heads of 128, one context of 4000 8.5 / 9.2 / 11.7 / 16.0 / 23.9 / 36; 64 of 17 to 8192 176 / 139 / 124 / 120 / 121 / 131; 32 of 500 to 1000 21.7 / 19.4 /
// 18.0 / 15.3 (uncut); 16 drafts on 8 contexts of 300 to 2100, 16 heads of 64, 17.3 / 14.4 / 14.0 / 15.6 / 21.7; one context of 8192, five tokens of 28 heads on 4,
// 18.1 / 15.3 / 16.6 / 21.6 / 32.0 / 91; 64 contexts of 100 to 300, 12 heads of 64, 15.8 / 13.8 / 10.0 (uncut)
Cut cached_attention_cut(int batch, int heads, int kv_heads, int max_new, int max_len)
{
    const long most = (long)max_new * (heads / kv_heads), qt = row_tiles(most);
    const long items = (long)batch * kv_heads * ((most + 16 * qt - 1) / (16 * qt)), tiles = (max_len + (long)TILE - 1) / TILE;
    if (items >= 512 && qt == 2 && tiles <= 32768) return Cut{1, (int)tiles};
    const long longest = items > 512 ? 48 * items / 512 : 48;
    long piece = tiles * items / 512;
    if (piece > longest) piece = longest;
    if (piece < 4 * qt) piece = 4 * qt;
    if (tiles <= piece + 16) return Cut{1, (int)tiles};
    long splits = (tiles + piece - 1) / piece;
    if (splits > MAX_SPLITS) splits = MAX_SPLITS;
    return Cut{(int)splits, (int)((tiles + splits - 1) / splits)};
}

hipError_t launch_cached_attention(const void *q, long ldq, bool bf16, int heads, int D, const KvCache &c, const KvRows &rows, float scale, const uint64_t *tree,
                                   Cut cut, float *partials, void *out, hipStream_t st)
{
    if (D == 128) return bf16 ? cached_attention<true, 128>(q, ldq, heads, c, rows, scale, tree, cut, partials, out, st)
                              : cached_attention<false, 128>(q, ldq, heads, c, rows, scale, tree, cut, partials, out, st);
    return bf16 ? cached_attention<true, 64>(q, ldq, heads, c, rows, scale, tree, cut, partials, out, st)
                : cached_attention<false, 64>(q, ldq, heads, c, rows, scale, tree, cut, partials, out, st);
}

}  // namespace samp

// The bookkeeping of a cache's pages on the device: page tables of sequences that go on (fork), pages moved together (compact), and the copying that both ask for.
//
// Tables and counts are small; what bounds their kernels is the latency of a few dependent steps and the launches.  So where the counts of all pages fit the LDS of one CU, one
// block does a whole call, with barriers between its steps and counters in LDS; larger ones take the same steps as kernels with the counters in the workspace.  Counters
// are sums and minima of whole numbers, so results do not depend on the order in which they are formed.
#include "../../include/samp.h"
#include "decoder.h"
#include "decoder_rules.h"
#include "divisor.h"

namespace samp {
namespace {

constexpr int BLOCK = 1024, NONE = 0x7fffffff;

// the sums of the values of the threads before this one, and of all, N of them at a time; `parts` holds a value for each wave
template <int WAVES, int N>
__device__ __forceinline__ void block_scan(const int (&v)[N], int (*parts)[WAVES], int (&before)[N], int (&all)[N])
{
    static_assert(WAVES <= 16, "a wave's first lanes hold the waves' sums");
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int sum[N];
#pragma unroll
    for (int n = 0; n < N; n++) sum[n] = wave_scan(v[n]);
    lds_barrier();                                                    // (parts may still be read from a scan before)
#pragma unroll
    for (int n = 0; n < N; n++)
        if (lane == 63) parts[n][w] = sum[n];
    lds_barrier();
#pragma unroll
    for (int n = 0; n < N; n++) {
        const int waves = wave_scan(lane < WAVES ? parts[n][lane] : 0);
        all[n] = __builtin_amdgcn_readlane(waves, WAVES - 1);
        before[n] = sum[n] - v[n] + (w ? __builtin_amdgcn_readlane(waves, max(w - 1, 0)) : 0);
    }
}
template <int WAVES> __device__ __forceinline__ int block_scan(int v, int (&parts)[WAVES], int &all)
{
    const int one[1] = {v};
    int before[1], sum[1];
    block_scan<WAVES, 1>(one, &parts, before, sum);
    all = sum[0];
    return before[0];
}

// ---- fork --------------------------------------------------------------------------------------------
// Entries first .. end - 1 of a row are those that its next positions lie in, page what its parent has in the first of them; len: its next length; wide: how many entries the
// table has no room for
struct __attribute__((aligned(16))) RowPlan { int parent, held, first, end, page, len, wide, pad; };
__device__ __forceinline__ RowPlan row_plan(const PageFork &f, int i)
{
    RowPlan r{};
    r.parent = f.parents ? f.parents[i] : i;
    if ((unsigned)r.parent >= (unsigned)f.rows_from) {
        r.parent = -1;
        return r;
    }
    const int held = f.lens[r.parent], next = f.cu ? f.cu[i + 1] - f.cu[i] : f.max_new;
    r.held = held > 0 ? held : 0;
    const long len = (long)r.held + (next > 0 ? next : 0);
    r.len = len > NONE ? NONE : (int)len;
    const long end = (len + (1 << f.page_shift) - 1) >> f.page_shift, first = next > 0 ? r.held >> f.page_shift : end;
    r.end = (int)(end < f.width ? end : f.width);
    r.first = (int)(first < f.width ? first : f.width);
    r.wide = (int)(end - (first > f.width ? first : f.width));
    if (end <= f.width) r.wide = 0;
    return r;
}
__device__ __forceinline__ bool in_cache(const PageFork &f, int page) { return (unsigned)page < (unsigned)f.pages; }

// Counters of pages: `rest` is what names a page in the new tables and does not write it, `first` the place of the first entry that does
struct Counters { int *rest, *first; };
__device__ __forceinline__ int child_page(const PageFork &f, const RowPlan &r, int j)
{
    const int page = j < r.end ? f.table[(long)r.parent * f.width + j] : -1;
    return in_cache(f, page) ? page : -1;
}
// the entry's page stays where nothing else names the page but entries that write it too, later ones
__device__ __forceinline__ bool stays(const Counters &c, int page, int place) { return page >= 0 && c.rest[page] == 0 && c.first[page] == place; }

// One block.  A thread has every BLOCK-th row (neighbours in different waves) and its first written entry, which is all there is to a row that goes on by a token;
// f(its number or -1, its plan) for each round of them.
template <class Plan, class F> __device__ __forceinline__ void each_row(const PageFork &f, Plan &&plan, F &&do_row)
{
    constexpr int WAVES = BLOCK / 64;
    for (int i0 = 0; i0 < f.rows; i0 += BLOCK) {
        const int row = i0 + (int)(threadIdx.x & 63) * WAVES + (int)(threadIdx.x >> 6);
        RowPlan r{};
        if (row < f.rows) r = plan(row);
        do_row(row < f.rows ? row : -1, r);
    }
}
// The written entries behind the first of the wave's rows that have any: entry(whose they are, whether there is one, its place, its page).  All lanes of a wave call it together.
// A round takes four entries of every row, each by the row's own lane (OWN), or 256 entries of one row, by all lanes: whichever ends in fewer rounds, as each waits for its reads
// (248 rows that go on by 20 tokens over pages of 16: 13.8 us by their own lanes, 33.5 us row by row; 64 rows by 300: 19.1 in one loop for both, 14.6 in two).
constexpr int OWN = -1;
template <class Entry> __device__ __forceinline__ void later_entries(const PageFork &f, int row, const RowPlan &r, Entry &&entry)
{
    const int lane = threadIdx.x & 63, later = row >= 0 ? r.end - r.first - 1 : 0;
    unsigned long long many = __ballot(later > 0);
    if (!__ballot(later > 4 * __popcll(many))) {
        const int *const from = f.table + (long)max(r.parent, 0) * f.width;
        for (int j0 = r.first + 1; __ballot(row >= 0 && j0 < r.end); j0 += 4) {
            int page[4];
#pragma unroll
            for (int u = 0; u < 4; u++) page[u] = later > 0 ? from[min(j0 + u, r.end - 1)] : -1;
#pragma unroll
            for (int u = 0; u < 4; u++) entry(OWN, later > 0 && j0 + u < r.end, row * f.width + j0 + u, in_cache(f, page[u]) ? page[u] : -1);
        }
        return;
    }
    for (; many; many &= many - 1) {
        const int owner = __builtin_ctzll(many), first = __builtin_amdgcn_readlane(r.first, owner), end = __builtin_amdgcn_readlane(r.end, owner);
        const int at = __builtin_amdgcn_readlane(row, owner) * f.width;
        const int *const from = f.table + (long)__builtin_amdgcn_readlane(r.parent, owner) * f.width;
        for (int j0 = first + 1; j0 < end; j0 += 256) {
            int page[4];
#pragma unroll
            for (int u = 0; u < 4; u++) page[u] = from[min(j0 + 64 * u + lane, end - 1)];
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const int j = j0 + 64 * u + lane;
                if (j0 + 64 * u < end) entry(owner, j < end, at + j, in_cache(f, page[u]) ? page[u] : -1);
            }
        }
    }
}

__device__ __forceinline__ void count_writers(const PageFork &f, const Counters &c, int row, const RowPlan &r)
{
    if (row >= 0 && r.first < r.end && r.page >= 0) atomicMin(&c.first[r.page], row * f.width + r.first);
    later_entries(f, row, r, [&](int, bool there, int place, int page) __attribute__((always_inline)) {
        if (there && page >= 0) atomicMin(&c.first[page], place);
    });
}

// One block, everything in LDS.  Needs of the rows (in `needs`, which becomes their ranks), free pages in order, counts, entries.  plan(row): its RowPlan; list: the free pages, as many as
// were asked for or as there are.
template <class Plan>
__device__ __forceinline__ void assign(const PageFork &f, const Counters &c, Plan &&plan, int *needs, unsigned short *list, int (*parts)[BLOCK / 64])
{
    const int tid = threadIdx.x, lane = tid & 63;
    int wide = 0, wide_high = 0;                                      // (8192 rows lack up to 2^28 each)
    each_row(f, plan, [&](int row, const RowPlan &r) {
        int n = row >= 0 && r.first < r.end && !stays(c, r.page, row * f.width + r.first);
        later_entries(f, row, r, [&](int owner, bool there, int place, int page) __attribute__((always_inline)) {
            const bool need = there && !stays(c, page, place);
            const int more = owner == OWN ? need : __popcll(__ballot(need));
            n += owner == OWN || lane == owner ? more : 0;
        });
        if (row >= 0) {
            needs[row] = n;
            wide += r.wide & 0xffff;
            wide_high += r.wide >> 16;
        }
    });
    // (a thread has some neighbouring pages, at most PAGES, whose counters it keeps, and some neighbouring rows)
    constexpr int PAGES = 16;
    const int per = ((f.pages + BLOCK - 1) / BLOCK + 3) & ~3;
    const int at = tid * per, end = min(at + per, f.pages);
    int rest[PAGES];
    unsigned is_free = 0, written = 0;                                // bits of the pages
#pragma unroll
    for (int q = 0; q < PAGES; q += 4)
        if (q < per && at + q < end) {                                // (the counters of four pages at a time, some of them behind the last page's)
            const v4i r = *reinterpret_cast<const v4i *>(&c.rest[at + q]), w = *reinterpret_cast<const v4i *>(&c.first[at + q]);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                rest[q + e] = r[e];
                written |= (unsigned)(w[e] != NONE) << (q + e);
                is_free |= (unsigned)(r[e] == 0 && w[e] == NONE && at + q + e < end) << (q + e);
            }
        }
    lds_barrier();
    const int rows_per = (f.rows + BLOCK - 1) / BLOCK, row0 = tid * rows_per, row1 = min(row0 + rows_per, f.rows);
    int sum = 0;
    for (int i = row0; i < row1; i++) sum += needs[i];
    const int v[4] = {sum, (int)__popc(is_free), wide, wide_high};
    int before[4], all[4];
    block_scan<BLOCK / 64, 4>(v, parts, before, all);
    const int wanted = all[0], free_pages = all[1];
    int rank = before[0];
    for (int i = row0; i < row1; i++) {
        const int n = needs[i];
        needs[i] = rank;
        rank += n;
    }
    rank = before[1];
#pragma unroll
    for (int q = 0; q < PAGES; q += 4) {
        if (q >= per) break;
#pragma unroll
        for (int e = q; e < q + 4; e++) {
            if (at + e >= end) continue;
            int n = rest[e];
            if (is_free >> e & 1) {
                if (rank < wanted) {
                    list[rank] = (unsigned short)(at + e);
                    n = 1;
                }
                rank++;
            } else if (n == 0 && (written >> e & 1)) n = 1;           // the first of its writers
            f.refs_out[at + e] = n;
        }
    }
    if (tid == 0) f.lacking[0] = (int)min(max(wanted - free_pages, 0) + all[2] + ((long)all[3] << 16), (long)NONE);
    lds_barrier();
    each_row(f, plan, [&](int row, const RowPlan &r) {
        int rank = row >= 0 ? needs[row] : 0;
        if (row >= 0) {
            int from = -1, to = -1;
            const int part = r.held & ((1 << f.page_shift) - 1), place = row * f.width + r.first;
            if (r.first < r.end) {
                const bool need = !stays(c, r.page, place);
                const int fresh = need && rank < free_pages ? list[rank] : -1;
                f.table_out[place] = need ? fresh : r.page;
                rank += need;
                if (fresh >= 0 && r.page >= 0 && part) {
                    from = r.page;
                    to = fresh;
                }
            }
            f.copies[row] = from;
            f.copies[f.rows + row] = to;
            f.copies[2 * f.rows + row] = from >= 0 ? part : 0;
            f.lens_out[row] = r.len;
        }
        later_entries(f, row, r, [&](int owner, bool there, int place, int page) __attribute__((always_inline)) {
            const bool need = there && !stays(c, page, place);
            const unsigned long long mask = __ballot(need);
            const int at = owner == OWN ? rank : __builtin_amdgcn_readlane(rank, owner) + __popcll(mask & ((1ull << lane) - 1));
            if (there) f.table_out[place] = !need ? page : at < free_pages ? list[at] : -1;
            rank += owner == OWN ? need : lane == owner ? __popcll(mask) : 0;
        });
    });
}

// What a row of the old tables becomes: how many rows continue it, and how many of those have no next position; pages that it fills, and whether it has begun another
struct __attribute__((aligned(16))) Children { int all, idle, whole, part; };

// the entries of a new row that nothing is written to, by a wave
__device__ __forceinline__ void copy_row(const PageFork &f, int row, int lane)
{
    const RowPlan r = row_plan(f, row);
    const int *const from = f.table + (long)max(r.parent, 0) * f.width;
    int *const to = f.table_out + (long)row * f.width;
    for (int j0 = 0; j0 < f.width; j0 += 256) {
        int page[4];
#pragma unroll
        for (int u = 0; u < 4; u++) page[u] = from[min(j0 + 64 * u + lane, f.width - 1)];
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int j = j0 + 64 * u + lane;
            if (j < f.width && (j < r.first || j >= r.end)) to[j] = j < r.end && in_cache(f, page[u]) ? page[u] : -1;
        }
    }
}

// The first block does the bookkeeping, the others copy what does not depend on it, sixteen rows each.  What bounds it is the one block's instructions and dependent reads: 256 beams over
// 2610 pages 8.7 us, 4 over 31 5.0.  by: divisor() of the width
__global__ __launch_bounds__(BLOCK) void fork_block_kernel(PageFork f, unsigned by)
{
    extern __shared__ __attribute__((aligned(16))) char shared[];
    __shared__ int parts[4][BLOCK / 64];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    constexpr int WAVES = BLOCK / 64;
    if (blockIdx.x) {
        const int row = ((int)blockIdx.x - 1) * WAVES + w;
        if (row < f.rows) copy_row(f, row, lane);
        return;
    }
    RowPlan *const plans = reinterpret_cast<RowPlan *>(shared);
    Children *const children = reinterpret_cast<Children *>(plans + f.rows);
    const int padded = (f.pages + 3) & ~3;
    int *const counters = reinterpret_cast<int *>(children + f.rows_from), *const needs = counters + 2 * padded;
    unsigned short *const list = reinterpret_cast<unsigned short *>(needs + f.rows);
    const Counters c{counters, counters + padded};
    for (int i = tid; i < f.rows_from; i += BLOCK) {
        const int held = max(f.lens[i], 0);
        children[i] = Children{0, 0, held >> f.page_shift, held & ((1 << f.page_shift) - 1)};
    }
    for (int i0 = 0; i0 < f.pages; i0 += 4 * BLOCK) {
        int n[4];
#pragma unroll
        for (int u = 0; u < 4; u++) n[u] = f.refs[min(i0 + u * BLOCK + tid, f.pages - 1)];
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int i = i0 + u * BLOCK + tid;
            if (i < f.pages) {
                c.rest[i] = n[u];
                c.first[i] = NONE;
            }
        }
    }
    lds_barrier();
    auto plan = [&](int row) {
        RowPlan r = row_plan(f, row);
        r.page = r.first < r.end ? child_page(f, r, r.first) : -1;
        return r;
    };
    each_row(f, plan, [&](int row, const RowPlan &r) {
        if (row >= 0) plans[row] = r;
        if (row >= 0 && r.parent >= 0) {
            atomicAdd(&children[r.parent].all, 1);
            if (r.len == r.held) atomicAdd(&children[r.parent].idle, 1);
        }
        count_writers(f, c, row, r);
    });
    lds_barrier();
    // The old tables' names leave as often as no row takes them on (rows that go on write from the page that their next position lies in), eight entries of a thread requested at a time
    constexpr int AT_ONCE = 8;
    const int entries = f.rows_from * f.width;
    for (int i0 = 0; i0 < entries; i0 += AT_ONCE * BLOCK) {
        int old[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) old[u] = f.table[min(i0 + u * BLOCK + tid, entries - 1)];
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) {
            if (i0 + u * BLOCK >= entries) break;
            const int i = min(i0 + u * BLOCK + tid, entries - 1), row = (int)over((unsigned)i, by, (unsigned)f.width), j = i - row * f.width;
            const Children n = children[row];
            const int more = (j < n.whole ? n.all : j == n.whole && n.part ? n.idle : 0) - 1;
            if (more && i0 + u * BLOCK + tid < entries && in_cache(f, old[u])) atomicAdd(&c.rest[old[u]], more);
        }
    }
    lds_barrier();
    assign(f, c, [&](int row) { return plans[row]; }, needs, list, parts);
}

// The same in five launches over all of the chip, which bound it up to a million pages: 20000 pages and 64 rows of 128 entries 15.6 us, 250000 and 256 of 256 17.2, 8 million 54 (160 MB).
__global__ __launch_bounds__(256) void fork_clear_kernel(PageFork f, Counters c)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < f.pages) {
        c.rest[i] = f.refs[i];
        c.first[i] = NONE;
    }
}
// a wave a row
__global__ __launch_bounds__(256) void fork_count_kernel(PageFork f, Counters c)
{
    const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    RowPlan r{};
    if (row < f.rows) r = row_plan(f, row);
    for (int j = blockIdx.y * 64 + lane; j < f.width; j += 64 * gridDim.y) {
        const int old = row < f.rows_from ? f.table[(long)row * f.width + j] : -1, child = row < f.rows ? child_page(f, r, j) : -1;
        if (in_cache(f, old)) atomicAdd(&c.rest[old], -1);
        if (row >= f.rows) continue;
        if (j < r.first || j >= r.end) {
            if (child >= 0) atomicAdd(&c.rest[child], 1);
            f.table_out[(long)row * f.width + j] = child;
        } else if (child >= 0) atomicMin(&c.first[child], row * f.width + j);
    }
}
// Blocks in front: the free pages of FORK_CHUNK pages each; behind them: what a row needs.  A block looks at AT_ONCE rounds of 256 pages or entries together.
constexpr int AT_ONCE = 16, FORK_CHUNK = 256 * AT_ONCE;
struct Needs { int *of_row, *wide, *in_chunk, *total; };              // pages, entries that the table lacks; free pages; of all chunks
__global__ __launch_bounds__(256) void fork_needs_kernel(PageFork f, Counters c, Needs needs, int chunks)
{
    __shared__ int parts[4];
    const int tid = threadIdx.x;
    int n = 0, all;
    if ((int)blockIdx.x < chunks) {
        const long first = (long)blockIdx.x * FORK_CHUNK + tid;
        int rest[AT_ONCE], written[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) {
            const long page = min(first + u * 256, (long)f.pages - 1);
            rest[u] = c.rest[page];
            written[u] = c.first[page];
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) n += first + u * 256 < f.pages && rest[u] == 0 && written[u] == NONE;
        block_scan(n, parts, all);
        if (tid == 0) needs.in_chunk[blockIdx.x] = all;
        return;
    }
    const int row = blockIdx.x - chunks;
    const RowPlan r = row_plan(f, row);
    for (int j0 = r.first; j0 < r.end; j0 += 1024) {
        int page[4];
#pragma unroll
        for (int u = 0; u < 4; u++) page[u] = child_page(f, r, j0 + u * 256 + tid);
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int j = j0 + u * 256 + tid;
            n += j < r.end && !stays(c, page[u], row * f.width + j);
        }
    }
    block_scan(n, parts, all);
    if (tid == 0) {
        needs.of_row[row] = all;
        needs.wide[row] = r.wide;
    }
}
// The free pages that are asked for, in order, and the counts; a block behind the last chunk's ranks the rows.
__global__ __launch_bounds__(256) void fork_free_kernel(PageFork f, Counters c, Needs needs, int *__restrict__ rank_of, int chunks, int *__restrict__ list)
{
    __shared__ int parts[4][4], count[64];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool of_rows = (int)blockIdx.x == chunks;
    const long first = (long)blockIdx.x * FORK_CHUNK + tid;
    int rest[AT_ONCE], written[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; u++) {
        const long page = min(first + u * 256, (long)f.pages - 1);
        rest[u] = c.rest[page];
        written[u] = c.first[page];
    }
    int v[4] = {}, before[4], all[4];                                 // free pages (in front of this chunk's), needs, wide
    for (int i = tid; i < (of_rows ? chunks : min((int)blockIdx.x, chunks)); i += 256) v[0] += needs.in_chunk[i];
    // (of the block behind the chunks a thread has neighbouring rows)
    const int per = (f.rows + 255) / 256;
    for (int u = 0; u < per; u++) {
        const int i = tid * per + u;
        if (i >= f.rows) break;
        v[1] += needs.of_row[i];
        if (of_rows) {
            v[2] += needs.wide[i] & 0xffff;                           // (8192 rows lack up to 2^28 each)
            v[3] += needs.wide[i] >> 16;
        }
    }
    block_scan<4, 4>(v, parts, before, all);
    const int wanted = all[1];
    if (of_rows) {
        int rank = before[1];
        for (int u = 0; u < per; u++) {
            const int i = tid * per + u;
            if (i >= f.rows) break;
            rank_of[i] = rank;
            rank += needs.of_row[i];
        }
        if (tid == 0) {
            needs.total[0] = all[0];
            f.lacking[0] = (int)min(max(wanted - all[0], 0) + all[2] + ((long)all[3] << 16), (long)NONE);
        }
        return;
    }
    unsigned is_free = 0;
#pragma unroll
    for (int u = 0; u < AT_ONCE; u++) {
        const bool one = first + u * 256 < f.pages && rest[u] == 0 && written[u] == NONE;
        is_free |= (unsigned)one << u;
        const int n = __popcll(__ballot(one));
        if (lane == 0) count[4 * u + w] = n;
    }
    lds_barrier();
    const int mine = count[lane], in_front = wave_scan(mine) - mine;  // of the chunk's 64 pages number `lane`
#pragma unroll
    for (int u = 0; u < AT_ONCE; u++) {
        const long page = first + u * 256;
        const bool one = is_free >> u & 1;
        const int rank = all[0] + __builtin_amdgcn_readlane(in_front, 4 * u + w) + __popcll(__ballot(one) & ((1ull << lane) - 1));
        int n = rest[u];
        if (one) {
            if (rank < wanted) {
                list[rank] = (int)page;
                n = 1;
            }
        } else if (n == 0 && written[u] != NONE) n = 1;               // the first of its writers
        if (page < f.pages) f.refs_out[page] = n;
    }
}
// a block a row: the entries that its next positions lie in
__global__ __launch_bounds__(256) void fork_entries_kernel(PageFork f, Counters c, Needs needs, const int *__restrict__ rank_of, const int *__restrict__ list)
{
    __shared__ int count[16];
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int free_pages = needs.total[0];
    int rank = rank_of[row];
    const RowPlan r = row_plan(f, row);
    const int part = r.held & ((1 << f.page_shift) - 1);
    if (tid == 0) {
        f.lens_out[row] = r.len;
        if (r.first >= r.end) {
            f.copies[row] = f.copies[f.rows + row] = -1;
            f.copies[2 * f.rows + row] = 0;
        }
    }
    for (int j0 = r.first; j0 < r.end; j0 += 1024) {
        int page[4];
        bool need[4];
#pragma unroll
        for (int u = 0; u < 4; u++) page[u] = child_page(f, r, j0 + u * 256 + tid);
        if (j0 > r.first) lds_barrier();
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int j = j0 + u * 256 + tid;
            need[u] = j < r.end && !stays(c, page[u], row * f.width + j);
            const int n = __popcll(__ballot(need[u]));
            if (lane == 0) count[4 * u + w] = n;
        }
        lds_barrier();
        const int mine = lane < 16 ? count[lane] : 0, upto = wave_scan(mine), in_front = upto - mine;
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int j = j0 + u * 256 + tid, at = rank + __builtin_amdgcn_readlane(in_front, 4 * u + w) + __popcll(__ballot(need[u]) & ((1ull << lane) - 1));
            const int to = !need[u] ? page[u] : at < free_pages ? list[at] : -1;
            if (j < r.end) f.table_out[(long)row * f.width + j] = to;
            if (j == r.first) {
                const bool copied = need[u] && to >= 0 && page[u] >= 0 && part;
                f.copies[row] = copied ? page[u] : -1;
                f.copies[f.rows + row] = copied ? to : -1;
                f.copies[2 * f.rows + row] = copied ? part : 0;
            }
        }
        rank += __builtin_amdgcn_readlane(upto, 63);
    }
}

// ---- compact -----------------------------------------------------------------------------------------
// Where a page goes follows from how many pages in use lie in front of it: `word` of 64 pages' bits and the number in front of each word.
struct UsedPages { const unsigned long long *word; const int *before; };
__device__ __forceinline__ int used_before(const UsedPages &u, int page)
{
    return u.before[page >> 6] + __popcll(u.word[page >> 6] & ((1ull << (page & 63)) - 1));
}
struct Compact { const int *refs, *table; int pages, entries, page_len; int *refs_out, *table_out, *copies, *used; };

// copies' rows of the pages that move and of the places that they move to, in order
__device__ __forceinline__ void list_moves(const Compact &a, const UsedPages &u, int used, int page)
{
    const bool in_use = u.word[page >> 6] >> (page & 63) & 1;
    if (in_use != (page >= used)) return;
    const int n = max(1, a.pages / 2), before = used_before(u, page);
    if (in_use) a.copies[before - used_before(u, used)] = page;
    else a.copies[n + page - before] = page;
}
__device__ __forceinline__ void finish_moves(const Compact &a, const UsedPages &u, int used, long at, long step)
{
    const int n = max(1, a.pages / 2), moved = used < a.pages ? used - used_before(u, used) : 0;
    for (long i = at; i < n; i += step) {
        if (i >= moved) a.copies[i] = a.copies[n + i] = -1;
        a.copies[2 * (long)n + i] = i < moved ? a.page_len : 0;
    }
    for (long i = at; i < a.pages; i += step) {
        const int page = (int)i;
        const bool in_use = u.word[page >> 6] >> (page & 63) & 1;
        a.refs_out[page] = page >= used ? 0 : a.refs[in_use ? page : a.copies[page - used_before(u, page)]];
    }
    for (long i = at; i < a.entries; i += step) {
        const int page = a.table[i];
        int to = -1;
        if ((unsigned)page < (unsigned)a.pages && (u.word[page >> 6] >> (page & 63) & 1))
            to = page < used ? page : a.copies[n + used_before(u, page) - used_before(u, used)];
        a.table_out[i] = to;
    }
    if (at == 0) a.used[0] = used;
}

// One block: the new number of every page in LDS (`where`), and the free ones in front of `used`.  A thread has PER neighbouring pages.  Bound by its three dependent steps: 301
// pages 2.6 us, 4096 5.4.
template <int PER>
__global__ __launch_bounds__(BLOCK) void compact_block_kernel(Compact a)
{
    extern __shared__ __attribute__((aligned(16))) int where[];       // [pages]
    __shared__ int parts[BLOCK / 64], in_front;
    unsigned short *const holes = reinterpret_cast<unsigned short *>(where + a.pages);         // [pages / 2]
    const int tid = threadIdx.x, n = max(1, a.pages / 2), first = tid * PER;
    constexpr int AT_ONCE = 4;
    int entry[AT_ONCE], refs[PER];
#pragma unroll
    for (int i = 0; i < PER; i++) refs[i] = first + i < a.pages ? a.refs[first + i] : 0;
#pragma unroll
    for (int u = 0; u < AT_ONCE; u++) entry[u] = tid + u * BLOCK < a.entries ? a.table[tid + u * BLOCK] : -1;
    int count = 0, used;
#pragma unroll
    for (int i = 0; i < PER; i++) count += refs[i] > 0;
    const int before = block_scan(count, parts, used);
    int rank = before;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int page = first + i;
        if (page == used) in_front = rank;                            // pages in use that stay
        if (page < used && refs[i] <= 0) holes[page - rank] = (unsigned short)page;
        rank += refs[i] > 0;
    }
    if (used >= a.pages && tid == 0) in_front = used;
    __syncthreads();
    const int stay = in_front, moved = used - stay;
    rank = before;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int page = first + i;
        if (page >= a.pages) continue;
        int to = -1;
        if (refs[i] > 0) {
            to = page < used ? page : holes[rank - stay];
            a.refs_out[to] = refs[i];
            if (page >= used) {
                a.copies[rank - stay] = page;
                a.copies[n + rank - stay] = to;
            }
        }
        if (page >= used) a.refs_out[page] = 0;
        where[page] = to;
        rank += refs[i] > 0;
    }
    for (int i = tid; i < n; i += BLOCK) {
        if (i >= moved) a.copies[i] = a.copies[n + i] = -1;
        a.copies[2 * n + i] = i < moved ? a.page_len : 0;
    }
    if (tid == 0) a.used[0] = used;
    __syncthreads();
    for (int i0 = 0; i0 < a.entries; i0 += AT_ONCE * BLOCK) {
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) {
            const int i = i0 + u * BLOCK + tid;
            if (i0) entry[u] = i < a.entries ? a.table[i] : -1;
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) {
            const int i = i0 + u * BLOCK + tid;
            if (i < a.entries) a.table_out[i] = (unsigned)entry[u] < (unsigned)a.pages ? where[entry[u]] : -1;
        }
    }
}

// The same in four launches, which is what bounds them: 13071 pages 13.8 us, a million 23.0 (8 MB).
constexpr int CHUNK = 64 * 256;                                       // pages of a block
__global__ __launch_bounds__(256) void compact_bits_kernel(Compact a, unsigned long long *words, int *before, int *chunk_used)
{
    __shared__ int parts[4];
    const long first = (long)blockIdx.x * CHUNK;
    const int tid = threadIdx.x;
    constexpr int AT_ONCE = 16;                                       // a thread's reads, requested together
    for (int i0 = 0; i0 < CHUNK && first + i0 < a.pages; i0 += 256 * AT_ONCE) {
        int refs[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) refs[u] = a.refs[min(first + i0 + u * 256 + tid, (long)a.pages - 1)];
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) {
            const long page = first + i0 + u * 256 + tid;
            const unsigned long long bits = __ballot(page < a.pages && refs[u] > 0);
            if ((tid & 63) == 0 && page < a.pages) words[page >> 6] = bits;
        }
    }
    __syncthreads();
    const long w = (first >> 6) + tid;
    const bool there = w << 6 < a.pages;
    int all;
    const int in_front = block_scan(there ? __popcll(words[w]) : 0, parts, all);
    if (there) before[w] = in_front;
    if (tid == 0) chunk_used[blockIdx.x] = all;
}
__global__ __launch_bounds__(256) void compact_before_kernel(Compact a, int chunks, int *before, const int *chunk_used, int *total)
{
    __shared__ int parts[4];
    int mine = 0, all_before, sum = 0, all;
    for (int i = threadIdx.x; i < chunks; i += 256) {
        const int n = chunk_used[i];
        mine += i < (int)blockIdx.x ? n : 0;
        sum += n;
    }
    block_scan(mine, parts, all_before);
    block_scan(sum, parts, all);
    const long w = (long)blockIdx.x * (CHUNK / 64) + threadIdx.x;
    if (w << 6 < a.pages) before[w] += all_before;
    if (blockIdx.x == 0 && threadIdx.x == 0) total[0] = all;
}
__global__ __launch_bounds__(256) void compact_list_kernel(Compact a, UsedPages u, const int *total)
{
    const long page = (long)blockIdx.x * 256 + threadIdx.x;
    if (page < a.pages) list_moves(a, u, total[0], (int)page);
}
__global__ __launch_bounds__(256) void compact_finish_kernel(Compact a, UsedPages u, const int *total)
{
    finish_moves(a, u, total[0], (long)blockIdx.x * 256 + threadIdx.x, (long)gridDim.x * 256);
}

// ---- copies ------------------------------------------------------------------------------------------
template <int D> __device__ __forceinline__ void copy_part(const KvCache &c, const KeyBounds &bounds, int from, int to, int rows, int head, bool is_v, int lane)
{
    const size_t src = ((size_t)from * c.kv_heads + head) << c.page_shift, dst = ((size_t)to * c.kv_heads + head) << c.page_shift;
    int8_t *const codes = is_v ? c.v : c.k;
    float *const steps = is_v ? c.v_step : c.k_step;
    const v4i *const read = reinterpret_cast<const v4i *>(codes + src * D);
    v4i *const write = reinterpret_cast<v4i *>(codes + dst * D);
    const int chunks = rows * (D / 16);
    for (int at = lane; at < rows; at += 64) steps[dst + at] = steps[src + at];
    constexpr int BATCH = 8;
    for (int at = lane; at < chunks; at += 64 * BATCH) {
        v4i held[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; i++) held[i] = read[min(at + 64 * i, chunks - 1)];
#pragma unroll
        for (int i = 0; i < BATCH; i++)
            if (at + 64 * i < chunks) write[at + 64 * i] = held[i];
    }
    if (bounds.codes && !is_v) {
        const size_t a = (size_t)from * c.kv_heads + head, b = (size_t)to * c.kv_heads + head;
        if (lane < 2 * D / 16) reinterpret_cast<v4i *>(bounds.codes + b * 2 * D)[lane] = reinterpret_cast<const v4i *>(bounds.codes + a * 2 * D)[lane];
        if (lane == 0) bounds.steps[b] = bounds.steps[a];
    }
}

// A wave copies the keys or the values of one key head of one page at a time, all of what it reads requested before the first of it is written (up to 8 KB; in turns, more).
// It has every so-manieth entry of the list, looked up 64 at a time, as a list may be long and hold few copies (20 among 50000 of 8 key heads 6.6 us, each looked up by itself 41).
// Bound by HBM: 980 pages of 64 positions, 8 key heads of 128 (265 MB read and written) 53.9 us, 4.9 TB/s, near a large copy's 5.0; the begun pages of 256 beams (11 MB) 4.3 us.
template <int D>
__global__ __launch_bounds__(256) void cache_copy_kernel(KvCache c, KeyBounds bounds, const int *__restrict__ copies, int n)
{
    const int lane = threadIdx.x & 63, parts = 2 * c.kv_heads, group = blockIdx.x / parts, part = blockIdx.x - group * parts, head = part >> 1, waves = gridDim.x / parts * 4;
    const bool is_v = part & 1;
    for (int e0 = 4 * group + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); e0 < n; e0 += 64 * waves) {
        const int mine = e0 + lane * waves;
        int from_of = -1, to_of = -1, rows_of = 0;
        if (mine < n) {
            from_of = copies[mine];
            to_of = copies[n + mine];
            rows_of = min(copies[2 * (long)n + mine], 1 << c.page_shift);
        }
        const bool copied = (unsigned)from_of < (unsigned)c.pages && (unsigned)to_of < (unsigned)c.pages && rows_of > 0 && from_of != to_of;
        for (unsigned long long left = __ballot(copied); left; left &= left - 1) {
            const int owner = __builtin_ctzll(left);
            copy_part<D>(c, bounds, __builtin_amdgcn_readlane(from_of, owner), __builtin_amdgcn_readlane(to_of, owner), __builtin_amdgcn_readlane(rows_of, owner), head, is_v, lane);
        }
    }
}

unsigned blocks_for(long items, long most) { return (unsigned)(items < 1 ? 1 : items < most ? items : most); }
template <class T> T *take(char *&at, size_t n)
{
    T *p = reinterpret_cast<T *>(at);
    at += (n * sizeof(T) + 255) / 256 * 256;
    return p;
}
size_t room(size_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

size_t pages_fork_workspace(int pages, int rows_from, int width, int rows)
{
    const size_t chunks = ((size_t)pages + FORK_CHUNK - 1) / FORK_CHUNK;
    return fork_in_block(pages, rows_from, width, rows) ? 0 : 3 * room(4 * (size_t)pages) + 3 * room(4 * (size_t)rows) + room(4 * chunks) + room(4);
}

hipError_t launch_pages_fork(const PageFork &f, void *ws, hipStream_t st)
{
    if (fork_in_block(f.pages, f.rows_from, f.width, f.rows)) {
        const size_t lds = fork_block_lds(f.pages, f.rows_from, f.rows);
        if (lds > 60 << 10)
            if (hipError_t e = hipFuncSetAttribute((const void *)fork_block_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) return e;
        hipLaunchKernelGGL(fork_block_kernel, dim3((unsigned)(1 + (f.rows + BLOCK / 64 - 1) / (BLOCK / 64))), dim3(BLOCK), lds, st, f,
                           divisor((unsigned long long)f.rows_from * f.width, f.width));
        return hipGetLastError();
    }
    char *at = static_cast<char *>(ws);
    int *const list = take<int>(at, f.pages);
    Counters c;
    c.rest = take<int>(at, f.pages);
    c.first = take<int>(at, f.pages);
    const int most = f.rows > f.rows_from ? f.rows : f.rows_from, chunks = (int)(((size_t)f.pages + FORK_CHUNK - 1) / FORK_CHUNK);
    int *const rank_of = take<int>(at, f.rows);
    Needs needs;
    needs.of_row = take<int>(at, f.rows);
    needs.wide = take<int>(at, f.rows);
    needs.in_chunk = take<int>(at, chunks);
    needs.total = take<int>(at, 1);
    hipLaunchKernelGGL(fork_clear_kernel, dim3((unsigned)((f.pages + 255) / 256)), dim3(256), 0, st, f, c);
    hipLaunchKernelGGL(fork_count_kernel, dim3((unsigned)((most + 3) / 4), blocks_for((f.width + 63) / 64, 64)), dim3(256), 0, st, f, c);
    hipLaunchKernelGGL(fork_needs_kernel, dim3((unsigned)(chunks + f.rows)), dim3(256), 0, st, f, c, needs, chunks);
    hipLaunchKernelGGL(fork_free_kernel, dim3((unsigned)(chunks + 1)), dim3(256), 0, st, f, c, needs, rank_of, chunks, list);
    hipLaunchKernelGGL(fork_entries_kernel, dim3((unsigned)f.rows), dim3(256), 0, st, f, c, needs, rank_of, list);
    return hipGetLastError();
}

size_t pages_compact_workspace(int pages, int entries)
{
    if (compact_in_block(pages, entries)) return 0;
    const size_t words = ((size_t)pages + 63) / 64, chunks = ((size_t)pages + CHUNK - 1) / CHUNK;
    return room(8 * words) + room(4 * words) + room(4 * chunks) + room(4);
}

hipError_t launch_pages_compact(const int *refs, int pages, const int *table, int entries, int page_len, int *refs_out, int *table_out, int *copies, int *used, void *ws,
                                hipStream_t st)
{
    const Compact a{refs, table, pages, entries, page_len, refs_out, table_out, copies, used};
    const size_t count = ((size_t)pages + 63) / 64;
    if (compact_in_block(pages, entries)) {
        const size_t lds = compact_block_lds(pages);
        auto kern = pages <= 4 * BLOCK ? compact_block_kernel<4> : compact_block_kernel<8>;
        hipLaunchKernelGGL(kern, dim3(1), dim3(BLOCK), lds, st, a);
        return hipGetLastError();
    }
    const int chunks = (int)(((size_t)pages + CHUNK - 1) / CHUNK);
    char *at = static_cast<char *>(ws);
    unsigned long long *const words = take<unsigned long long>(at, count);
    int *const before = take<int>(at, count), *const chunk_used = take<int>(at, chunks), *const total = take<int>(at, 1);
    const UsedPages u{words, before};
    hipLaunchKernelGGL(compact_bits_kernel, dim3(chunks), dim3(256), 0, st, a, words, before, chunk_used);
    hipLaunchKernelGGL(compact_before_kernel, dim3(chunks), dim3(256), 0, st, a, chunks, before, chunk_used, total);
    hipLaunchKernelGGL(compact_list_kernel, dim3((unsigned)(((long)pages + 255) / 256)), dim3(256), 0, st, a, u, total);
    const long most = pages > entries ? pages : entries;
    hipLaunchKernelGGL(compact_finish_kernel, dim3(blocks_for((most + 255) / 256, 4096)), dim3(256), 0, st, a, u, total);
    return hipGetLastError();
}

hipError_t launch_cache_copy(const KvCache &c, int D, const KeyBounds &bounds, const int *copies, int n, hipStream_t st)
{
    const int parts = 2 * c.kv_heads;
    // no more blocks than 8192, a list longer than their waves is gone through.  us, 1024 / 4096 / 8192 / 16384, copies of pages x heads x channels: 2000 of 16 x 12 x 64 21.1 / 18.6 / 19.6 / 21.1,
    // 20000 of 16 x 8 x 128 290 / 284 / 281 / 278, of one head of 64 18.1 / 16.8 / 17.8 / 18.5; 20 among 50000 8.6 / 7.8 / 7.4 / 9.9; fewer than 1000 copies within 2 % of each other
    const unsigned blocks = parts * blocks_for((n + 3l) / 4, max(1, 8192 / parts));
    auto kern = D == 128 ? cache_copy_kernel<128> : cache_copy_kernel<64>;
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), 0, st, c, bounds, copies, n);
    return hipGetLastError();
}

}  // namespace samp

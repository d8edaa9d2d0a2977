// The bookkeeping of a cache's pages on the device: page tables of sequences that go on (fork), pages moved together (compact), and the copying that both ask for.
//
// Tables and counts are small; what bounds their kernels is the latency of a few dependent steps and the launches.  So where the counts of all pages fit the LDS of one CU, one
// block does a whole call, with barriers between its steps and counters in LDS; larger ones take the same steps as kernels with the counters in the workspace.  Counters
// are sums and minima of whole numbers, so results do not depend on the order in which they are formed.
#include "../../include/samp.h"
#include "decoder.h"
#include "decoder_rules.h"

namespace samp {
namespace {

constexpr int BLOCK = 1024, NONE = 0x7fffffff;

// the sum of the values of the threads before this one, and of all; `parts` holds a value for each wave
__device__ __forceinline__ int block_scan(int v, int *parts, int &all)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int sum = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int other = __shfl_up(sum, o, 64);
        if (lane >= o) sum += other;
    }
    __syncthreads();
    if (lane == 63) parts[w] = sum;
    __syncthreads();
    int before = 0;
    all = 0;
    for (int i = 0; i < (int)blockDim.x >> 6; i++) {
        const int p = parts[i];
        before += i < w ? p : 0;
        all += p;
    }
    return before + sum - v;
}

// ---- fork --------------------------------------------------------------------------------------------
// Entries first .. end - 1 of a row are those that its next positions lie in; wide: how many of them the table has no room for
struct RowPlan { int parent, held, first, end; long len; int wide; };
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
    r.len = (long)r.held + (next > 0 ? next : 0);
    const long end = (r.len + (1 << f.page_shift) - 1) >> f.page_shift, first = next > 0 ? r.held >> f.page_shift : end;
    r.end = (int)(end < f.width ? end : f.width);
    r.first = (int)(first < f.width ? first : f.width);
    r.wide = (int)(end - (first > f.width ? first : f.width));
    if (end <= f.width) r.wide = 0;
    return r;
}
__device__ __forceinline__ bool in_cache(const PageFork &f, int page) { return (unsigned)page < (unsigned)f.pages; }

// Counters of pages: `rest` is what names a page in the new tables and does not write it, `first` the place of the first entry that does
struct Counters { int *rest, *first; };

// The old tables' names leave, the new ones' come; entries that nothing is written to are done with.  Threads `at`, at + step .. of all
__device__ __forceinline__ void count_names(const PageFork &f, const Counters &c, long at, long step)
{
    const long old = (long)f.rows_from * f.width;
    for (long i = at; i < old; i += step) {
        const int page = f.table[i];
        if (in_cache(f, page)) atomicAdd(&c.rest[page], -1);
    }
    const long all = (long)f.rows * f.width;
    for (long i = at; i < all; i += step) {
        const int row = (int)(i / f.width), j = (int)(i - (long)row * f.width);
        const RowPlan r = row_plan(f, row);
        int page = j < r.end && r.parent >= 0 ? f.table[(long)r.parent * f.width + j] : -1;
        if (!in_cache(f, page)) page = -1;
        if (j < r.first || j >= r.end) {
            if (page >= 0) atomicAdd(&c.rest[page], 1);
            f.table_out[i] = page;
        }
    }
}

// Eight lanes a row: which of its entries first + lane, + 8 .. are written
__device__ __forceinline__ int child_page(const PageFork &f, const RowPlan &r, int j)
{
    const int page = j < r.end ? f.table[(long)r.parent * f.width + j] : -1;
    return in_cache(f, page) ? page : -1;
}
__device__ __forceinline__ void count_writers(const PageFork &f, const Counters &c, int row, int lane)
{
    const RowPlan r = row_plan(f, row);
    for (int j = r.first + lane; j < r.end; j += 8) {
        const int page = child_page(f, r, j);
        if (page >= 0) atomicMin(&c.first[page], row * f.width + j);
    }
}
// the entry's page stays where nothing else names the page but entries that write it too, later ones
__device__ __forceinline__ bool stays(const Counters &c, int page, int place) { return page >= 0 && c.rest[page] == 0 && c.first[page] == place; }
__device__ __forceinline__ unsigned of_eight(bool b) { return (unsigned)(__ballot(b) >> (threadIdx.x & 56)) & 0xffu; }

__device__ __forceinline__ int count_needs(const PageFork &f, const Counters &c, int row, int lane)
{
    const RowPlan r = row_plan(f, row);
    int needs = 0;
    for (int j0 = r.first; j0 < r.end; j0 += 8) {
        const int j = j0 + lane;
        needs += __popc(of_eight(j < r.end && !stays(c, child_page(f, r, j), row * f.width + j)));
    }
    return needs;
}
// list: the free pages in order, as many as were asked for or as there are
__device__ __forceinline__ void give_pages(const PageFork &f, const Counters &c, const int *list, int free_pages, int row, int lane, int rank)
{
    const RowPlan r = row_plan(f, row);
    int from = -1, to = -1;
    for (int j0 = r.first; j0 < r.end; j0 += 8) {
        const int j = j0 + lane, page = child_page(f, r, j);
        const bool need = j < r.end && !stays(c, page, row * f.width + j);
        const unsigned mask = of_eight(need);
        const int at = rank + __popc(mask & ((1u << lane) - 1));
        const int fresh = need && at < free_pages ? list[at] : -1;
        if (j < r.end) f.table_out[(long)row * f.width + j] = need ? fresh : page;
        if (j == r.first && fresh >= 0 && page >= 0 && (r.held & ((1 << f.page_shift) - 1))) {
            from = page;
            to = fresh;
        }
        rank += __popc(mask);
    }
    if (lane == 0) {
        f.copies[row] = from;
        f.copies[f.rows + row] = to;
        f.copies[2 * f.rows + row] = from >= 0 ? r.held & ((1 << f.page_shift) - 1) : 0;
        f.lens_out[row] = r.len > NONE ? NONE : (int)r.len;
    }
}

// One block: needs of the rows (in `needs`, which becomes their ranks), free pages in order, counts, entries
__device__ __forceinline__ void assign(const PageFork &f, const Counters &c, int *needs, int *list, int *parts)
{
    const int tid = threadIdx.x, eighth = tid >> 3, lane = tid & 7;
    int wide = 0;
    for (int row = eighth; row < f.rows; row += BLOCK / 8) {
        const int n = count_needs(f, c, row, lane);
        if (lane == 0) {
            needs[row] = n;
            wide += row_plan(f, row).wide;
        }
    }
    __syncthreads();
    int wanted, free_pages, all_wide;
    {
        const int per = (f.rows + BLOCK - 1) / BLOCK, at = tid * per;
        int sum = 0;
        for (int i = at; i < min(at + per, f.rows); i++) sum += needs[i];
        int rank = block_scan(sum, parts, wanted);
        for (int i = at; i < min(at + per, f.rows); i++) {
            const int n = needs[i];
            needs[i] = rank;
            rank += n;
        }
    }
    block_scan(wide, parts, all_wide);
    {
        const int per = (f.pages + BLOCK - 1) / BLOCK;
        const long at = (long)tid * per, end = min(at + per, (long)f.pages);
        int sum = 0;
        for (long i = at; i < end; i++) sum += c.rest[i] == 0 && c.first[i] == NONE;
        int rank = block_scan(sum, parts, free_pages);
        for (long i = at; i < end; i++) {
            int n = c.rest[i];
            if (n == 0 && c.first[i] == NONE) {
                if (rank < wanted) {
                    list[rank] = (int)i;
                    n = 1;
                }
                rank++;
            } else if (n == 0) n = 1;                                 // the first of its writers
            f.refs_out[i] = n;
        }
    }
    if (tid == 0) f.lacking[0] = max(wanted - free_pages, 0) + all_wide;
    __syncthreads();
    for (int row = eighth; row < f.rows; row += BLOCK / 8) give_pages(f, c, list, free_pages, row, lane, needs[row]);
}

__global__ __launch_bounds__(BLOCK) void fork_block_kernel(PageFork f, int *__restrict__ list)
{
    extern __shared__ __attribute__((aligned(16))) int shared[];
    __shared__ int parts[BLOCK / 64];
    const Counters c{shared, shared + f.pages};
    int *const needs = shared + 2 * f.pages;
    for (int i = threadIdx.x; i < f.pages; i += BLOCK) {
        c.rest[i] = f.refs[i];
        c.first[i] = NONE;
    }
    __syncthreads();
    count_names(f, c, threadIdx.x, BLOCK);
    for (int row = threadIdx.x >> 3; row < f.rows; row += BLOCK / 8) count_writers(f, c, row, threadIdx.x & 7);
    __syncthreads();
    assign(f, c, needs, list, parts);
}

__global__ __launch_bounds__(256) void fork_clear_kernel(PageFork f, Counters c)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < f.pages) {
        c.rest[i] = f.refs[i];
        c.first[i] = NONE;
    }
}
__global__ __launch_bounds__(256) void fork_count_kernel(PageFork f, Counters c)
{
    const long at = (long)blockIdx.x * 256 + threadIdx.x, step = (long)gridDim.x * 256;
    count_names(f, c, at, step);
    for (long row = at >> 3; row < f.rows; row += step >> 3) count_writers(f, c, (int)row, threadIdx.x & 7);
}
__global__ __launch_bounds__(BLOCK) void fork_assign_kernel(PageFork f, Counters c, int *needs, int *list)
{
    __shared__ int parts[BLOCK / 64];
    assign(f, c, needs, list, parts);
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

__global__ __launch_bounds__(BLOCK) void compact_block_kernel(Compact a)
{
    extern __shared__ __attribute__((aligned(16))) unsigned long long words[];
    __shared__ int parts[BLOCK / 64];
    const int tid = threadIdx.x, count = (a.pages + 63) >> 6;
    int *const before = reinterpret_cast<int *>(words + count);
    for (int i = tid; i < count << 6; i += BLOCK) {
        const unsigned long long bits = __ballot(i < a.pages && a.refs[min(i, a.pages - 1)] > 0);
        if ((i & 63) == 0) words[i >> 6] = bits;
    }
    __syncthreads();
    int used, base = 0;
    for (int i0 = 0; i0 < count; i0 += BLOCK) {
        const int i = i0 + tid;
        const int in_front = block_scan(i < count ? __popcll(words[i]) : 0, parts, used);
        if (i < count) before[i] = base + in_front;
        base += used;
    }
    used = base;
    __syncthreads();
    const UsedPages u{words, before};
    for (int i = tid; i < a.pages; i += BLOCK) list_moves(a, u, used, i);
    __syncthreads();
    finish_moves(a, u, used, tid, BLOCK);
}

constexpr int CHUNK = 64 * 256;                                       // pages of a block
__global__ __launch_bounds__(256) void compact_bits_kernel(Compact a, unsigned long long *words, int *before, int *chunk_used)
{
    __shared__ int parts[4];
    const long first = (long)blockIdx.x * CHUNK;
    const int tid = threadIdx.x;
    for (int i = tid; i < CHUNK; i += 256) {
        const long page = first + i;
        const unsigned long long bits = __ballot(page < a.pages && a.refs[min(page, (long)a.pages - 1)] > 0);
        if ((i & 63) == 0 && page < a.pages) words[page >> 6] = bits;
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
// A wave copies the keys or the values of one key head of one page at a time, all of what it reads requested before the first of it is written (up to 8 KB; in turns, more).
template <int D>
__global__ __launch_bounds__(256) void cache_copy_kernel(KvCache c, KeyBounds bounds, const int *__restrict__ copies, int n)
{
    const int lane = threadIdx.x & 63;
    const long step = (long)gridDim.x * 4, units = 2l * n * c.kv_heads;
    for (long u = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); u < units; u += step) {
        const int entry = (int)(u / (2 * c.kv_heads)), part = (int)(u - (long)entry * 2 * c.kv_heads), head = part >> 1;
        const bool is_v = part & 1;
        const int from = copies[entry], to = copies[n + entry], rows = min(copies[2 * (long)n + entry], 1 << c.page_shift);
        if ((unsigned)from >= (unsigned)c.pages || (unsigned)to >= (unsigned)c.pages || rows <= 0 || from == to) continue;
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

size_t pages_fork_workspace(int pages, int rows)
{
    const size_t list = room(4 * (size_t)pages);
    return fork_in_block(pages, rows) ? list : 3 * list + room(4 * (size_t)rows);
}

hipError_t launch_pages_fork(const PageFork &f, void *ws, hipStream_t st)
{
    char *at = static_cast<char *>(ws);
    int *const list = take<int>(at, f.pages);
    if (fork_in_block(f.pages, f.rows)) {
        const size_t lds = fork_block_lds(f.pages, f.rows);
        if (lds > 64 << 10)
            if (hipError_t e = hipFuncSetAttribute((const void *)fork_block_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) return e;
        hipLaunchKernelGGL(fork_block_kernel, dim3(1), dim3(BLOCK), lds, st, f, list);
        return hipGetLastError();
    }
    Counters c;
    c.rest = take<int>(at, f.pages);
    c.first = take<int>(at, f.pages);
    int *const needs = take<int>(at, f.rows);
    const long entries = (long)f.width * (f.rows > f.rows_from ? f.rows : f.rows_from);
    hipLaunchKernelGGL(fork_clear_kernel, dim3((unsigned)((f.pages + 255) / 256)), dim3(256), 0, st, f, c);
    hipLaunchKernelGGL(fork_count_kernel, dim3(blocks_for((entries + 255) / 256, 4096)), dim3(256), 0, st, f, c);
    hipLaunchKernelGGL(fork_assign_kernel, dim3(1), dim3(BLOCK), 0, st, f, c, needs, list);
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
        hipLaunchKernelGGL(compact_block_kernel, dim3(1), dim3(BLOCK), 12 * count, st, a);
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
    const unsigned blocks = blocks_for((2l * n * c.kv_heads + 3) / 4, 8192);
    auto kern = D == 128 ? cache_copy_kernel<128> : cache_copy_kernel<64>;
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), 0, st, c, bounds, copies, n);
    return hipGetLastError();
}

}  // namespace samp

// C ABI of the 8-bit decoder's operators: argument checking in front of the launchers of decoder.h.
#include "../../include/samp.h"
#include "api_common.h"
#include "decoder.h"
#include "decoder_rules.h"

#include <cmath>

using namespace samp;

namespace {

constexpr size_t ALIGN = 256;
size_t up(size_t v) { return (v + ALIGN - 1) / ALIGN * ALIGN; }

int check_type(int32_t type)
{
    return type == SAMP_TYPE_F16 || type == SAMP_TYPE_BF16 ? SAMP_OK : fail(SAMP_ERR_ARG, "unknown type %d", (int)type);
}

// 16-bit rows that are read 16 bytes at a time: `width` values, `ld` from one to the next
int check_rows(const char *what, const void *p, int64_t ld, int64_t width)
{
    if (!p) return fail(SAMP_ERR_ARG, "%s is NULL", what);
    if (!aligned(p, 16) || ld % 8) return fail(SAMP_ERR_ARG, "%s: rows must be 16-byte aligned (leading dimension %lld)", what, (long long)ld);
    if (ld < width || ld > SAMP_MAX_ROW) return fail(SAMP_ERR_SHAPE, "%s: a leading dimension of %lld to %d is needed (%lld)", what, (long long)width,
                                                     SAMP_MAX_ROW, (long long)ld);
    return SAMP_OK;
}

int check_tokens(int32_t M, int32_t N, int32_t K)
{
    if (M < 1 || M > SAMP_MAX_TOKENS) return fail(SAMP_ERR_SHAPE, "1 to %d rows are supported (M=%d)", SAMP_MAX_TOKENS, M);
    // (K: an int32 sum of 127 * 128 each)
    if (N < 16 || N % 16 || K < 64 || K % 64 || K > 131072 || (long long)N * K > INT32_MAX)
        return fail(SAMP_ERR_SHAPE, "N %% 16 == 0, K %% 64 == 0, K <= 131072, N * K < 2^31 needed (N=%d K=%d)", N, K);
    return SAMP_OK;
}

int check_product(const void *Wp, const float *s_w, const float *bias, const void *out)
{
    if (!Wp || !s_w || !out) return fail(SAMP_ERR_ARG, "NULL pointer");
    if (!aligned(Wp, 16) || !aligned(s_w, 16) || !aligned(bias, 16) || !aligned(out, 16)) return fail(SAMP_ERR_ARG, "matrices and tables must be 16-byte aligned");
    return SAMP_OK;
}

int check_page_len(int32_t page_len)
{
    if (page_len < 16 || page_len > 1024 || (page_len & (page_len - 1))) return fail(SAMP_ERR_SHAPE, "page_len must be a power of two, 16 to 1024 (%d)", page_len);
    return SAMP_OK;
}
int shift_of(int32_t page_len)
{
    int shift = 4;
    while (1 << shift < page_len) shift++;
    return shift;
}

int check_cache(const samp_kv_cache_t *c, KvCache *to)
{
    if (!c || !c->k || !c->v || !c->k_step || !c->v_step) return fail(SAMP_ERR_ARG, "NULL pointer in the cache");
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_step, 16) || !aligned(c->v_step, 16)) return fail(SAMP_ERR_ARG, "the cache must be 16-byte aligned");
    if (c->head_dim != 64 && c->head_dim != 128) return fail(SAMP_ERR_SHAPE, "head_dim must be 64 or 128 (%d)", c->head_dim);
    if (int rc = check_page_len(c->page_len)) return rc;
    if (c->pages < 1 || c->kv_heads < 1 || c->kv_heads > SAMP_MAX_HEADS) return fail(SAMP_ERR_SHAPE, "pages >= 1 and 1 to %d key heads needed", SAMP_MAX_HEADS);
    *to = KvCache{c->k, c->v, c->k_step, c->v_step, c->pages, c->kv_heads, shift_of(c->page_len)};
    return SAMP_OK;
}

// (a maximum above the number of rows, as of a program that passes its largest batch, counts as that number)
int check_kv_rows(KvRows &r, const char *most)
{
    if (!r.table || !r.lens) return fail(SAMP_ERR_ARG, "the page table or the lengths are NULL");
    if (r.batch < 1 || r.batch > SAMP_MAX_BATCH) return fail(SAMP_ERR_SHAPE, "1 to %d sequences are supported (%d)", SAMP_MAX_BATCH, r.batch);
    if (r.width < 1 || r.max_rows < 1 || r.rows < 1 || r.rows > SAMP_MAX_TOKENS)
        return fail(SAMP_ERR_SHAPE, "a table width, %s and rows of at least 1 are needed, rows up to %d", most, SAMP_MAX_TOKENS);
    if (!r.cu && (long long)r.batch * r.max_rows != r.rows)
        return fail(SAMP_ERR_SHAPE, "without offsets every sequence has %s rows: %d x %d are not %d", most, r.batch, r.max_rows, r.rows);
    if (r.max_rows > r.rows) r.max_rows = r.rows;
    if (r.max_rows > SAMP_MAX_CACHE_ROWS) return fail(SAMP_ERR_SHAPE, "%s is %d, %d at most are supported", most, r.max_rows, SAMP_MAX_CACHE_ROWS);
    return SAMP_OK;
}

int check_heads(int32_t heads, int32_t kv_heads, float scale)
{
    if (kv_heads < 1 || heads < kv_heads || heads % kv_heads || heads > SAMP_MAX_HEADS)
        return fail(SAMP_ERR_SHAPE, "query heads must be a multiple of the key heads, %d at most (%d, %d)", SAMP_MAX_HEADS, heads, kv_heads);
    // (the kernels' exponentials are of base 2)
    if (!std::isfinite(scale * 1.44269504088896341f) || !(scale > 0.0f)) return fail(SAMP_ERR_SCALE, "the scale is not positive, or log2(e) times it not finite");
    return SAMP_OK;
}

int check_bounds(const samp_key_bounds_t *b, KeyBounds *to)
{
    if (!b || !b->codes || !b->steps) return fail(SAMP_ERR_ARG, "NULL pointer in the bounds");
    if (!aligned(b->codes, 16) || !aligned(b->steps, 16)) return fail(SAMP_ERR_ARG, "the bounds must be 16-byte aligned");
    *to = KeyBounds{b->codes, b->steps};
    return SAMP_OK;
}

int check_workspace(const void *workspace, size_t bytes, size_t need)
{
    if (need && (!workspace || !aligned(workspace, ALIGN) || bytes < need)) return fail(SAMP_ERR_SPACE, "a 256-byte aligned workspace of %zu bytes is needed", need);
    return SAMP_OK;
}

int check_beams(int32_t type, int32_t batch, int32_t beams, int32_t vocab, int32_t keep)
{
    if (type != SAMP_TYPE_F16 && type != SAMP_TYPE_BF16 && type != SAMP_TYPE_F32) return fail(SAMP_ERR_ARG, "unknown type %d", (int)type);
    if (batch < 1 || batch > SAMP_MAX_BATCH || beams < 1 || beams > SAMP_MAX_BEAMS || vocab < 1 || vocab > SAMP_MAX_VOCAB || keep < 1 || keep > SAMP_MAX_KEEP)
        return fail(SAMP_ERR_SHAPE, "1 to %d sequences, 1 to %d beams, a vocabulary of 1 to %d and keep of 1 to %d are supported (%d, %d, %d, %d)", SAMP_MAX_BATCH,
                    SAMP_MAX_BEAMS, SAMP_MAX_VOCAB, SAMP_MAX_KEEP, batch, beams, vocab, keep);
    if (!pieces_fit(type == SAMP_TYPE_F32, (long)batch * beams, vocab)) return fail(SAMP_ERR_SHAPE, "%d sequences x %d beams x %d logits are more threads than a launch has", batch, beams, vocab);
    return SAMP_OK;
}

int check_pages(int32_t pages)
{
    if (pages < 1 || pages > SAMP_MAX_PAGES) return fail(SAMP_ERR_SHAPE, "1 to %d pages are supported (%d)", SAMP_MAX_PAGES, pages);
    return SAMP_OK;
}

int check_choice(int32_t batch, int32_t kv_heads, int32_t width, int32_t page_len, int32_t max_new, int32_t keep, int32_t sinks, int32_t recent)
{
    if (width > SAMP_MAX_TABLE) return fail(SAMP_ERR_SHAPE, "pages are chosen from at most %d of a sequence (width %d)", SAMP_MAX_TABLE, width);
    const long need = ((long)max_new + page_len - 2) / page_len + 1;
    if (sinks < 0 || recent < need || keep < 1 || (long)sinks + recent > keep)
        return fail(SAMP_ERR_SHAPE, "sinks >= 0, recent >= %ld for max_new %d, and sinks + recent <= keep are needed (%d, %d, %d)", need, max_new, sinks, recent, keep);
    if (keep > SAMP_MAX_TABLE) return fail(SAMP_ERR_SHAPE, "keep is at most %d (%d)", SAMP_MAX_TABLE, keep);
    if (!choice_fits(batch, kv_heads, width)) return fail(SAMP_ERR_SHAPE, "%d sequences x %d key heads x %d pages are more threads than a launch has", batch, kv_heads, width);
    return SAMP_OK;
}

}  // namespace

extern "C" {

int samp_quantize_tokens(const uint16_t *x, int64_t ldx, int32_t type, int32_t M, int32_t K, int8_t *codes, float *steps, void *stream)
{
    if (int rc = check_type(type)) return rc;
    if (!codes || !steps) return fail(SAMP_ERR_ARG, "NULL pointer");
    if (M < 1 || M > SAMP_MAX_TOKENS || K < 8 || K % 8) return fail(SAMP_ERR_SHAPE, "1 to %d rows of a multiple of 8 values are supported (M=%d K=%d)", SAMP_MAX_TOKENS, M, K);
    if (int rc = check_rows("x", x, ldx, K)) return rc;
    if (!aligned(codes, 8) || !aligned(steps, 4)) return fail(SAMP_ERR_ARG, "codes must be 8-byte, steps 4-byte aligned");
    HIP_TRY(launch_quantize_tokens(x, ldx, type == SAMP_TYPE_BF16, M, K, codes, steps, (hipStream_t)stream));
    return SAMP_OK;
}

int samp_gemm_i8_tokens_packed(const int8_t *codes, const float *steps, const int8_t *Wp, const float *s_w, const float *bias, int32_t gelu, uint16_t *out,
                               int32_t type, int32_t M, int32_t N, int32_t K, void *stream)
{
    if (int rc = check_type(type)) return rc;
    if (int rc = check_tokens(M, N, K)) return rc;
    if (int rc = check_product(Wp, s_w, bias, out)) return rc;
    if (!codes || !steps) return fail(SAMP_ERR_ARG, "NULL pointer");
    if (!aligned(codes, 16) || !aligned(steps, 4)) return fail(SAMP_ERR_ARG, "codes must be 16-byte, steps 4-byte aligned");
    HIP_TRY(launch_gemm_i8_tokens(codes, steps, Wp, s_w, bias, gelu != 0, out, type == SAMP_TYPE_BF16, M, N, K, (hipStream_t)stream));
    return SAMP_OK;
}

size_t samp_linear_i8_tokens_workspace_bytes(int32_t M, int32_t K)
{
    if (check_tokens(M, 16, K) || tokens_fused_any(M, K)) return 0;
    return up((size_t)M * K) + up((size_t)M * sizeof(float));
}

int samp_linear_i8_tokens(const uint16_t *x, int64_t ldx, int32_t type, const int8_t *Wp, const float *s_w, const float *bias, int32_t gelu, uint16_t *out,
                          int32_t M, int32_t N, int32_t K, void *workspace, size_t workspace_bytes, void *stream)
{
    if (int rc = check_type(type)) return rc;
    if (int rc = check_tokens(M, N, K)) return rc;
    if (int rc = check_product(Wp, s_w, bias, out)) return rc;
    if (int rc = check_rows("x", x, ldx, K)) return rc;
    if (tokens_fused(M, N, K)) {
        HIP_TRY(launch_linear_few(x, ldx, type == SAMP_TYPE_BF16, Wp, s_w, bias, gelu != 0, out, M, N, K, (hipStream_t)stream));
        return SAMP_OK;
    }
    const size_t need = samp_linear_i8_tokens_workspace_bytes(M, K);
    if (!workspace || !aligned(workspace, ALIGN) || workspace_bytes < need) return fail(SAMP_ERR_SPACE, "a 256-byte aligned workspace of %zu bytes is needed", need);
    int8_t *codes = static_cast<int8_t *>(workspace);
    float *steps = reinterpret_cast<float *>(codes + up((size_t)M * K));
    HIP_TRY(launch_quantize_tokens(x, ldx, type == SAMP_TYPE_BF16, M, K, codes, steps, (hipStream_t)stream));
    HIP_TRY(launch_gemm_i8_tokens(codes, steps, Wp, s_w, bias, gelu != 0, out, type == SAMP_TYPE_BF16, M, N, K, (hipStream_t)stream));
    return SAMP_OK;
}

int samp_cache_write(const samp_kv_cache_t *cache, const uint16_t *k, int64_t ldk, const uint16_t *v, int64_t ldv, int32_t type, const int32_t *table,
                     int32_t width, const int32_t *cu, const int32_t *lens, int32_t batch, int32_t max_new, int32_t rows, void *stream)
{
    KvCache c;
    KvRows r{table, width, cu, lens, batch, max_new, rows};
    if (int rc = check_type(type)) return rc;
    if (int rc = check_cache(cache, &c)) return rc;
    if (int rc = check_kv_rows(r, "max_new")) return rc;
    if (int rc = check_rows("k", k, ldk, (int64_t)c.kv_heads * cache->head_dim)) return rc;
    if (int rc = check_rows("v", v, ldv, (int64_t)c.kv_heads * cache->head_dim)) return rc;
    HIP_TRY(launch_cache_write(c, k, ldk, v, ldv, type == SAMP_TYPE_BF16, cache->head_dim, r, (hipStream_t)stream));
    return SAMP_OK;
}

int samp_cache_read(const samp_kv_cache_t *cache, uint16_t *k, uint16_t *v, int32_t type, const int32_t *table, int32_t width, const int32_t *cu,
                    const int32_t *lens, int32_t batch, int32_t max_rows, int32_t rows, void *stream)
{
    KvCache c;
    KvRows r{table, width, cu, lens, batch, max_rows, rows};
    if (int rc = check_type(type)) return rc;
    if (int rc = check_cache(cache, &c)) return rc;
    if (int rc = check_kv_rows(r, "max_rows")) return rc;
    if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) return fail(SAMP_ERR_ARG, "k and v must be 16-byte aligned and not NULL");
    HIP_TRY(launch_cache_read(c, k, v, type == SAMP_TYPE_BF16, cache->head_dim, r, (hipStream_t)stream));
    return SAMP_OK;
}

static int check_cached(int32_t rows, int32_t batch, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t max_new, int32_t max_len, Cut *cut)
{
    if (int rc = check_heads(heads, kv_heads, 1.0f)) return rc;
    if (head_dim != 64 && head_dim != 128) return fail(SAMP_ERR_SHAPE, "head_dim must be 64 or 128 (%d)", head_dim);
    if (batch < 1 || batch > SAMP_MAX_BATCH || max_new < 1 || max_len < 1 || rows < 1 || rows > SAMP_MAX_TOKENS)
        return fail(SAMP_ERR_SHAPE, "1 to %d sequences, 1 to %d rows, max_new >= 1 and max_len >= 1 needed", SAMP_MAX_BATCH, SAMP_MAX_TOKENS);
    if (max_new > rows) max_new = rows;
    *cut = cached_attention_cut(batch, heads, kv_heads, max_new, max_len);
    if ((double)batch * heads * max_new * cut->splits > 2147483647.0) return fail(SAMP_ERR_SHAPE, "batch x heads x max_new, times the pieces of a context, is past 2^31");
    return SAMP_OK;
}

size_t samp_attention_cache_workspace_bytes(int32_t rows, int32_t batch, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t max_new, int32_t max_len)
{
    Cut cut;
    if (check_cached(rows, batch, heads, kv_heads, head_dim, max_new, max_len, &cut)) return 0;
    return cut.splits == 1 ? 0 : up((size_t)rows * heads * cut.splits * (head_dim + 2) * sizeof(float));
}

int samp_attention_cache(const uint16_t *q, int64_t ldq, int32_t type, int32_t heads, const samp_kv_cache_t *cache, const int32_t *table, int32_t width,
                         const int32_t *cu, const int32_t *lens, int32_t batch, int32_t max_new, int32_t max_len, int32_t rows, float scale,
                         const uint64_t *tree, uint16_t *out, void *workspace, size_t workspace_bytes, void *stream)
{
    KvCache c;
    KvRows r{table, width, cu, lens, batch, max_new, rows};
    if (int rc = check_type(type)) return rc;
    if (int rc = check_cache(cache, &c)) return rc;
    if (int rc = check_kv_rows(r, "max_new")) return rc;
    if (int rc = check_heads(heads, c.kv_heads, scale)) return rc;
    Cut cut;
    if (int rc = check_cached(rows, batch, heads, c.kv_heads, cache->head_dim, max_new, max_len, &cut)) return rc;
    if (int rc = check_rows("q", q, ldq, (int64_t)heads * cache->head_dim)) return rc;
    if (!out || !aligned(out, 16)) return fail(SAMP_ERR_ARG, "out must be 16-byte aligned and not NULL");
    if (tree && r.max_rows > 64) return fail(SAMP_ERR_SHAPE, "a tree has at most 64 drafted tokens (max_new %d)", max_new);
    if (tree && !aligned(tree, 8)) return fail(SAMP_ERR_ARG, "tree must be 8-byte aligned");
    const size_t need = samp_attention_cache_workspace_bytes(rows, batch, heads, c.kv_heads, cache->head_dim, max_new, max_len);
    if (need && (!workspace || !aligned(workspace, ALIGN) || workspace_bytes < need))
        return fail(SAMP_ERR_SPACE, "a 256-byte aligned workspace of %zu bytes is needed", need);
    HIP_TRY(launch_cached_attention(q, ldq, type == SAMP_TYPE_BF16, heads, cache->head_dim, c, r, scale, tree, cut, static_cast<float *>(workspace), out,
                                    (hipStream_t)stream));
    return SAMP_OK;
}

int samp_attention_causal(const uint16_t *q, int64_t ldq, const uint16_t *k, int64_t ldk, const uint16_t *v, int64_t ldv, int32_t type, int32_t heads,
                          int32_t kv_heads, int32_t head_dim, const int32_t *cu, int32_t batch, int32_t max_len, int32_t rows, float scale, uint16_t *out,
                          void *stream)
{
    if (int rc = check_type(type)) return rc;
    if (int rc = check_heads(heads, kv_heads, scale)) return rc;
    if (head_dim != 64 && head_dim != 128) return fail(SAMP_ERR_SHAPE, "head_dim must be 64 or 128 (%d)", head_dim);
    if (batch < 1 || batch > SAMP_MAX_BATCH || rows < 1 || rows > SAMP_MAX_TOKENS || max_len < 1)
        return fail(SAMP_ERR_SHAPE, "1 to %d sequences, 1 to %d rows and max_len >= 1 needed", SAMP_MAX_BATCH, SAMP_MAX_TOKENS);
    if (!cu && (long long)batch * max_len != rows) return fail(SAMP_ERR_SHAPE, "without offsets every sequence has max_len rows: %d x %d are not %d", batch, max_len, rows);
    if (max_len > rows) max_len = rows;
    if (int rc = check_rows("q", q, ldq, (int64_t)heads * head_dim)) return rc;
    if (int rc = check_rows("k", k, ldk, (int64_t)kv_heads * head_dim)) return rc;
    if (int rc = check_rows("v", v, ldv, (int64_t)kv_heads * head_dim)) return rc;
    if (!out || !aligned(out, 16)) return fail(SAMP_ERR_ARG, "out must be 16-byte aligned and not NULL");
    if ((double)batch * heads * ((max_len + 127) / 128) > 2147483647.0) return fail(SAMP_ERR_SHAPE, "too many strips of queries");
    HIP_TRY(launch_causal_attention(q, ldq, k, ldk, v, ldv, type == SAMP_TYPE_BF16, heads, kv_heads, head_dim, cu, batch, max_len, rows, scale, out,
                                    (hipStream_t)stream));
    return SAMP_OK;
}

size_t samp_beam_select_workspace_bytes(int32_t type, int32_t batch, int32_t beams, int32_t vocab, int32_t keep)
{
    return check_beams(type, batch, beams, vocab, keep) ? 0 : up(beam_workspace(type, batch, beams, vocab, keep));
}

int samp_beam_select(const void *logits, int64_t ld, int32_t type, const float *scores, const uint8_t *finished, int32_t end, int32_t batch, int32_t beams,
                     int32_t vocab, int32_t keep, float *best, int32_t *parents, int32_t *tokens, void *workspace, size_t workspace_bytes, void *stream)
{
    if (int rc = check_beams(type, batch, beams, vocab, keep)) return rc;
    if (!logits || !scores || !best || !parents || !tokens) return fail(SAMP_ERR_ARG, "NULL pointer");
    if (!aligned(logits, type == SAMP_TYPE_F32 ? 4 : 2) || !aligned(scores, 4) || !aligned(best, 4) || !aligned(parents, 4) || !aligned(tokens, 4))
        return fail(SAMP_ERR_ARG, "logits, scores and results must be aligned to their values");
    if (ld < vocab || ld > SAMP_MAX_ROW) return fail(SAMP_ERR_SHAPE, "logits: a leading dimension of %d to %d is needed (%lld)", vocab, SAMP_MAX_ROW, (long long)ld);
    if (int rc = check_workspace(workspace, workspace_bytes, samp_beam_select_workspace_bytes(type, batch, beams, vocab, keep))) return rc;
    HIP_TRY(launch_beam_select(logits, ld, type, scores, finished, end, batch, beams, vocab, keep, best, parents, tokens, workspace, (hipStream_t)stream));
    return SAMP_OK;
}

size_t samp_pages_fork_workspace_bytes(int32_t pages, int32_t rows_from, int32_t width, int32_t rows)
{
    if (check_pages(pages) || rows < 1 || rows > SAMP_MAX_BATCH || rows_from < 1 || rows_from > SAMP_MAX_BATCH || width < 1) return 0;
    return pages_fork_workspace(pages, rows_from, width, rows);
}

int samp_pages_fork(const int32_t *refs, int32_t pages, const int32_t *table, const int32_t *lens, int32_t rows_from, int32_t width, int32_t page_len,
                    const int32_t *parents, const int32_t *cu, int32_t max_new, int32_t rows, int32_t *refs_out, int32_t *table_out, int32_t *lens_out, int32_t *copies,
                    int32_t *lacking, void *workspace, size_t workspace_bytes, void *stream)
{
    if (int rc = check_pages(pages)) return rc;
    if (int rc = check_page_len(page_len)) return rc;
    if (!refs || !table || !lens || !refs_out || !table_out || !lens_out || !copies || !lacking) return fail(SAMP_ERR_ARG, "NULL pointer");
    if (rows < 1 || rows > SAMP_MAX_BATCH || rows_from < 1 || rows_from > SAMP_MAX_BATCH || width < 1 || (!cu && max_new < 0))
        return fail(SAMP_ERR_SHAPE, "1 to %d rows, a table width of at least 1 and max_new >= 0 are needed (%d, %d, %d, %d)", SAMP_MAX_BATCH, rows, rows_from, width, max_new);
    if ((long long)rows * width > 1 << 30 || (long long)rows_from * width > 1 << 30) return fail(SAMP_ERR_SHAPE, "a table has at most 2^30 entries");
    if (refs == refs_out || table == table_out || lens == lens_out) return fail(SAMP_ERR_ARG, "results must not overlap inputs");
    if (int rc = check_workspace(workspace, workspace_bytes, samp_pages_fork_workspace_bytes(pages, rows_from, width, rows))) return rc;
    const PageFork f{refs, table, lens, parents, cu, pages, rows_from, width, shift_of(page_len), max_new, rows, refs_out, table_out, lens_out, copies, lacking};
    HIP_TRY(launch_pages_fork(f, workspace, (hipStream_t)stream));
    return SAMP_OK;
}

size_t samp_pages_compact_workspace_bytes(int32_t pages, int32_t entries)
{
    return check_pages(pages) || entries < 0 ? 0 : pages_compact_workspace(pages, entries);
}

int samp_pages_compact(const int32_t *refs, int32_t pages, const int32_t *table, int32_t entries, int32_t page_len, int32_t *refs_out, int32_t *table_out,
                       int32_t *copies, int32_t *used, void *workspace, size_t workspace_bytes, void *stream)
{
    if (int rc = check_pages(pages)) return rc;
    if (int rc = check_page_len(page_len)) return rc;
    if (entries < 0) return fail(SAMP_ERR_SHAPE, "entries >= 0 needed (%d)", entries);
    if (!refs || !refs_out || !copies || !used || (entries && (!table || !table_out))) return fail(SAMP_ERR_ARG, "NULL pointer");
    if (refs == refs_out || (entries && table == table_out)) return fail(SAMP_ERR_ARG, "results must not overlap inputs");
    if (int rc = check_workspace(workspace, workspace_bytes, samp_pages_compact_workspace_bytes(pages, entries))) return rc;
    HIP_TRY(launch_pages_compact(refs, pages, table, entries, page_len, refs_out, table_out, copies, used, workspace, (hipStream_t)stream));
    return SAMP_OK;
}

int samp_cache_copy(const samp_kv_cache_t *cache, const samp_key_bounds_t *bounds, const int32_t *copies, int32_t n, void *stream)
{
    KvCache c;
    KeyBounds kb{nullptr, nullptr};
    if (int rc = check_cache(cache, &c)) return rc;
    if (bounds)
        if (int rc = check_bounds(bounds, &kb)) return rc;
    if (!copies) return fail(SAMP_ERR_ARG, "copies is NULL");
    if (n < 1 || n > SAMP_MAX_PAGES) return fail(SAMP_ERR_SHAPE, "1 to %d copies are supported (%d)", SAMP_MAX_PAGES, n);
    HIP_TRY(launch_cache_copy(c, cache->head_dim, kb, copies, n, (hipStream_t)stream));
    return SAMP_OK;
}

int samp_cache_bounds(const samp_kv_cache_t *cache, const samp_key_bounds_t *bounds, const int32_t *table, int32_t width, const int32_t *cu, const int32_t *lens,
                      int32_t batch, int32_t max_new, int32_t rows, void *stream)
{
    KvCache c;
    KeyBounds kb;
    KvRows r{table, width, cu, lens, batch, max_new, rows};
    if (int rc = check_cache(cache, &c)) return rc;
    if (int rc = check_bounds(bounds, &kb)) return rc;
    if (int rc = check_kv_rows(r, "max_new")) return rc;
    HIP_TRY(launch_cache_bounds(c, cache->head_dim, kb, r, (hipStream_t)stream));
    return SAMP_OK;
}

size_t samp_cache_select_workspace_bytes(int32_t batch, int32_t kv_heads, int32_t width)
{
    if (batch < 1 || batch > SAMP_MAX_BATCH || kv_heads < 1 || kv_heads > SAMP_MAX_HEADS || width < 1 || width > SAMP_MAX_TABLE || !choice_fits(batch, kv_heads, width)) return 0;
    return up(cache_select_workspace(batch, kv_heads, width));
}

int samp_cache_select(const uint16_t *q, int64_t ldq, int32_t type, int32_t heads, const samp_kv_cache_t *cache, const samp_key_bounds_t *bounds, const int32_t *table,
                      int32_t width, const int32_t *cu, const int32_t *lens, int32_t batch, int32_t max_new, int32_t rows, int32_t keep, int32_t sinks, int32_t recent,
                      int32_t *tables, int32_t *lens_out, void *workspace, size_t workspace_bytes, void *stream)
{
    KvCache c;
    KeyBounds kb;
    KvRows r{table, width, cu, lens, batch, max_new, rows};
    if (int rc = check_type(type)) return rc;
    if (int rc = check_cache(cache, &c)) return rc;
    if (int rc = check_bounds(bounds, &kb)) return rc;
    if (int rc = check_kv_rows(r, "max_new")) return rc;
    if (int rc = check_heads(heads, c.kv_heads, 1.0f)) return rc;
    if (int rc = check_rows("q", q, ldq, (int64_t)heads * cache->head_dim)) return rc;
    if (int rc = check_choice(batch, c.kv_heads, width, cache->page_len, r.max_rows, keep, sinks, recent)) return rc;
    if (!tables || !lens_out) return fail(SAMP_ERR_ARG, "NULL pointer");
    if (lens == lens_out) return fail(SAMP_ERR_ARG, "results must not overlap inputs");
    if (int rc = check_workspace(workspace, workspace_bytes, samp_cache_select_workspace_bytes(batch, c.kv_heads, width))) return rc;
    HIP_TRY(launch_cache_select(q, ldq, type == SAMP_TYPE_BF16, heads, cache->head_dim, c, kb, r, keep, sinks, recent, tables, lens_out, workspace, (hipStream_t)stream));
    return SAMP_OK;
}

// The tables of the key heads and the lengths; then what the choice needs, and after it, in the same place, the attention
static size_t chosen_bytes(int32_t batch, int32_t kv_heads, int32_t keep) { return up(4 * (size_t)batch * kv_heads * keep) + up(4 * (size_t)batch); }
static int32_t chosen_len(int32_t max_len, int32_t keep, int32_t page_len)
{
    const long long most = (long long)keep * page_len;
    return max_len < most ? max_len : (int32_t)most;
}

size_t samp_attention_sparse_workspace_bytes(int32_t rows, int32_t batch, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t page_len, int32_t width,
                                             int32_t max_new, int32_t max_len, int32_t keep)
{
    Cut cut;
    if (check_page_len(page_len) || keep < 1 || keep > SAMP_MAX_TABLE || width < 1 || width > SAMP_MAX_TABLE) return 0;
    max_len = chosen_len(max_len, keep, page_len);
    if (check_cached(rows, batch, heads, kv_heads, head_dim, max_new, max_len, &cut) || !choice_fits(batch, kv_heads, width)) return 0;
    const size_t choice = samp_cache_select_workspace_bytes(batch, kv_heads, width), attention = samp_attention_cache_workspace_bytes(rows, batch, heads, kv_heads, head_dim, max_new, max_len);
    return chosen_bytes(batch, kv_heads, keep) + (choice > attention ? choice : attention);
}

int samp_attention_sparse(const uint16_t *q, int64_t ldq, int32_t type, int32_t heads, const samp_kv_cache_t *cache, const samp_key_bounds_t *bounds,
                          const int32_t *table, int32_t width, const int32_t *cu, const int32_t *lens, int32_t batch, int32_t max_new, int32_t max_len, int32_t rows,
                          int32_t keep, int32_t sinks, int32_t recent, float scale, const uint64_t *tree, uint16_t *out, void *workspace, size_t workspace_bytes,
                          void *stream)
{
    KvCache c;
    KeyBounds kb;
    KvRows r{table, width, cu, lens, batch, max_new, rows};
    if (int rc = check_type(type)) return rc;
    if (int rc = check_cache(cache, &c)) return rc;
    if (int rc = check_bounds(bounds, &kb)) return rc;
    if (int rc = check_kv_rows(r, "max_new")) return rc;
    if (int rc = check_heads(heads, c.kv_heads, scale)) return rc;
    if (int rc = check_choice(batch, c.kv_heads, width, cache->page_len, r.max_rows, keep, sinks, recent)) return rc;
    max_len = chosen_len(max_len, keep, cache->page_len);
    Cut cut;
    if (int rc = check_cached(rows, batch, heads, c.kv_heads, cache->head_dim, max_new, max_len, &cut)) return rc;
    if (int rc = check_rows("q", q, ldq, (int64_t)heads * cache->head_dim)) return rc;
    if (!out || !aligned(out, 16)) return fail(SAMP_ERR_ARG, "out must be 16-byte aligned and not NULL");
    if (tree && r.max_rows > 64) return fail(SAMP_ERR_SHAPE, "a tree has at most 64 drafted tokens (max_new %d)", max_new);
    if (tree && !aligned(tree, 8)) return fail(SAMP_ERR_ARG, "tree must be 8-byte aligned");
    if (int rc = check_workspace(workspace, workspace_bytes,
                                 samp_attention_sparse_workspace_bytes(rows, batch, heads, c.kv_heads, cache->head_dim, cache->page_len, width, max_new, max_len, keep)))
        return rc;
    int *const tables = static_cast<int *>(workspace), *const chosen_lens = tables + up(4 * (size_t)batch * c.kv_heads * keep) / 4;
    float *const partials = reinterpret_cast<float *>(static_cast<char *>(workspace) + chosen_bytes(batch, c.kv_heads, keep));
    HIP_TRY(launch_cache_select(q, ldq, type == SAMP_TYPE_BF16, heads, cache->head_dim, c, kb, r, keep, sinks, recent, tables, chosen_lens, partials, (hipStream_t)stream));
    const KvRows chosen{tables, keep, cu, chosen_lens, batch, r.max_rows, rows, c.kv_heads};
    HIP_TRY(launch_cached_attention(q, ldq, type == SAMP_TYPE_BF16, heads, cache->head_dim, c, chosen, scale, tree, cut, partials, out, (hipStream_t)stream));
    return SAMP_OK;
}

}  // extern "C"

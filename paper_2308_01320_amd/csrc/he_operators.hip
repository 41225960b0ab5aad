// The operators' C entries (include/he.h): every argument is checked here, before anything is launched.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "operators.h"

using namespace he_op;

namespace {

thread_local char g_text[256] = "";

__attribute__((format(printf, 2, 3))) he_status refuse(he_status s, const char* fmt, ...) {
    va_list a;
    va_start(a, fmt);
    vsnprintf(g_text, sizeof g_text, fmt, a);
    va_end(a);
    return s;
}

constexpr int kMost = 1 << 30;      // positions of a sequence: indexes stay inside an int
constexpr int kMostRows = 1 << 23;  // rows of a packed batch: what a launch of a workgroup to each may have
constexpr int64_t kMostGroups = (1 << 24) - 1;

int elt_bytes(he_dtype t) { return t == HE_F32 ? 4 : 2; }
bool known(he_dtype t) { return t == HE_F32 || t == HE_BF16 || t == HE_F16; }
bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

he_status check_heads(he_dtype t, int n_heads, int n_kv_heads, int d) {
    if (!known(t)) return refuse(HE_ERR_INVALID_ARG, "unknown dtype %d", (int)t);
    if (n_kv_heads < 1 || n_heads < 1 || n_heads % n_kv_heads || n_heads > 65536)
        return refuse(HE_ERR_SHAPE, "%d heads over %d key-value heads: a whole number of heads to each, 65536 at most", n_heads, n_kv_heads);
    if (d < 16 || d > 256 || d % 16) return refuse(HE_ERR_SHAPE, "head_dim %d: a multiple of 16 up to 256", d);
    return HE_OK;
}

// width: elements of a row; out: rows are written, so they may not overlap
he_status check_rows(const he_rows* r, const char* name, he_dtype t, int64_t width, bool out) {
    if (!r || !r->data) return refuse(HE_ERR_INVALID_ARG, "%s is NULL", name);
    if (!aligned(r->data)) return refuse(HE_ERR_SHAPE, "%s does not lie on 16 bytes", name);
    if (r->stride < 0 || r->stride * elt_bytes(t) % 16) return refuse(HE_ERR_SHAPE, "%s: rows %lld elements apart: a multiple of 16 bytes", name, (long long)r->stride);
    if (r->stride > 1 << 22) return refuse(HE_ERR_SHAPE, "%s: rows %lld elements apart: 2^22 at most", name, (long long)r->stride);
    if (out && r->stride < width)
        return refuse(HE_ERR_SHAPE, "%s: rows %lld elements apart, each has %lld", name, (long long)r->stride, (long long)width);
    return HE_OK;
}

int log2_of(int n) { return 31 - __builtin_clz((unsigned)n); }

he_status check_cache(const he_paged_cache* c, int n_heads) {
    if (!c) return refuse(HE_ERR_INVALID_ARG, "cache is NULL");
    if (!c->k || !c->v || !c->pages) return refuse(HE_ERR_INVALID_ARG, "cache: k, v or pages is NULL");
    if (const he_status s = check_heads(c->dtype, n_heads, c->n_kv_heads, c->head_dim)) return s;
    if (c->page_size < 1 || c->page_size > 32768 || (c->page_size & (c->page_size - 1)))
        return refuse(HE_ERR_SHAPE, "page_size %d: a power of two up to 32768", c->page_size);
    if (c->n_pages < 1 || c->pages_per_seq < 1) return refuse(HE_ERR_INVALID_ARG, "cache: n_pages and pages_per_seq are positive");
    if ((int64_t)c->pages_per_seq * c->page_size > kMost) return refuse(HE_ERR_SHAPE, "cache: over 2^30 positions to a sequence");
    if (!aligned(c->k) || !aligned(c->v)) return refuse(HE_ERR_SHAPE, "cache: k or v does not lie on 16 bytes");
    if (c->page_stride < (int64_t)c->n_kv_heads * c->page_size * c->head_dim || c->page_stride * elt_bytes(c->dtype) % 16)
        return refuse(HE_ERR_SHAPE, "page_stride %lld: a page has %lld elements, and pages lie on 16 bytes", (long long)c->page_stride,
                      (long long)c->n_kv_heads * c->page_size * c->head_dim);
    return HE_OK;
}

Cache device_cache(const he_paged_cache& c) {
    return {c.k, c.v, c.pages, c.n_pages, c.pages_per_seq, log2_of(c.page_size), c.n_kv_heads, c.head_dim, c.page_stride};
}
Rows device_rows(const he_rows* r) { return r ? Rows{r->data, r->stride} : Rows{nullptr, 0}; }

he_status check_counts(int n_seqs, int n_tokens) {
    if (n_seqs < 0 || n_tokens < 0) return refuse(HE_ERR_INVALID_ARG, "a negative number of sequences or rows");
    if (n_seqs > 65535) return refuse(HE_ERR_SHAPE, "%d sequences: 65535 at most", n_seqs);
    if (n_tokens > kMostRows) return refuse(HE_ERR_SHAPE, "%d rows: 2^23 at most", n_tokens);
    return HE_OK;
}

he_status launched() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HE_OK : refuse(HE_ERR_DEVICE, "launch: %s", hipGetErrorString(e));
}

int longest_of(const he_paged_cache& c, int max_len) {
    const int all = c.pages_per_seq * c.page_size;
    return max_len < 1 || max_len > all ? all : max_len;
}
size_t split_bytes(int n_seqs, int n_heads, int d, int splits) {
    return splits > 1 ? (size_t)n_seqs * n_heads * splits * (d + 2) * sizeof(float) + 16 : 0;  // (values on 16 bytes behind maxima and sums)
}

}  // namespace

extern "C" {

const char* he_operator_error(void) { return g_text; }

he_status he_paged_append(const he_paged_cache* cache, const he_rope* rope_opt, const he_rows* q_opt, int n_heads, const he_rows* q_out_opt,
                          const he_rows* k, const he_rows* k_out_opt, const he_rows* v, const int32_t* d_seq_starts_opt, const int32_t* d_lens,
                          int n_seqs, int n_tokens, void* stream) {
    if (const he_status s = check_cache(cache, q_opt ? n_heads : cache ? cache->n_kv_heads : 1)) return s;
    const he_dtype t = cache->dtype;
    const int64_t wq = (int64_t)n_heads * cache->head_dim, wk = (int64_t)cache->n_kv_heads * cache->head_dim;
    if (!q_opt != !q_out_opt) return refuse(HE_ERR_INVALID_ARG, "queries come with a place for them (q and q_out), or not at all");
    if (q_opt) {
        if (const he_status s = check_rows(q_opt, "q", t, wq, false)) return s;
        if (const he_status s = check_rows(q_out_opt, "q_out", t, wq, true)) return s;
    }
    if (const he_status s = check_rows(k, "k", t, wk, false)) return s;
    if (const he_status s = check_rows(v, "v", t, wk, false)) return s;
    if (k_out_opt)
        if (const he_status s = check_rows(k_out_opt, "k_out", t, wk, true)) return s;
    Rope rope{};
    if (rope_opt) {
        if (rope_opt->dim < 16 || rope_opt->dim > cache->head_dim || rope_opt->dim % 16)
            return refuse(HE_ERR_SHAPE, "rope.dim %d: a multiple of 16 up to head_dim", rope_opt->dim);
        if (!(rope_opt->base > 0.0) || !std::isfinite(rope_opt->base) || !std::isfinite(rope_opt->scale))
            return refuse(HE_ERR_INVALID_ARG, "rope.base is positive, base and scale are finite");
        if (rope_opt->interleaved != 0 && rope_opt->interleaved != 1) return refuse(HE_ERR_INVALID_ARG, "rope.interleaved must be 0 or 1");
        rope.half = rope_opt->dim / 2;
        rope.interleaved = rope_opt->interleaved;
        for (int i = 0; i < rope.half; ++i)
            rope.turns[i] = rope_opt->scale * std::pow(rope_opt->base, -(double)i / rope.half) * 0.15915494309189533577;  // 1 / 2 pi
    }
    if (!d_lens) return refuse(HE_ERR_INVALID_ARG, "d_lens is NULL");
    if (const he_status s = check_counts(n_seqs, n_tokens)) return s;
    if (!d_seq_starts_opt && n_seqs != n_tokens) return refuse(HE_ERR_INVALID_ARG, "without d_seq_starts a sequence has one row: %d rows, %d sequences", n_tokens, n_seqs);
    if (n_seqs == 0 || n_tokens == 0) return HE_OK;
    append((hipStream_t)stream, t, device_cache(*cache), rope, device_rows(q_opt), n_heads, device_rows(q_out_opt), device_rows(k), device_rows(k_out_opt),
           device_rows(v), d_seq_starts_opt, d_lens, n_seqs, n_tokens);
    return launched();
}

size_t he_paged_attention_workspace(const he_paged_cache* cache, int n_heads, int n_seqs, int max_len) {
    if (check_cache(cache, n_heads) || check_counts(n_seqs, 0)) return 0;
    if (n_seqs == 0) return 0;
    return split_bytes(n_seqs, n_heads, cache->head_dim,
                       paged_splits(cache->dtype, cache->page_size, n_heads, cache->n_kv_heads, n_seqs, longest_of(*cache, max_len)));
}

he_status he_paged_attention(const he_paged_cache* cache, const he_rows* q, int n_heads, const he_rows* out, const int32_t* d_lens, int n_seqs,
                             int max_len, float scale, void* d_workspace, size_t workspace_bytes, void* stream) {
    if (const he_status s = check_cache(cache, n_heads)) return s;
    const int64_t w = (int64_t)n_heads * cache->head_dim;
    if (const he_status s = check_rows(q, "q", cache->dtype, w, false)) return s;
    if (const he_status s = check_rows(out, "out", cache->dtype, w, true)) return s;
    if (!d_lens) return refuse(HE_ERR_INVALID_ARG, "d_lens is NULL");
    if (!std::isfinite(scale)) return refuse(HE_ERR_INVALID_ARG, "scale is not finite");
    if (const he_status s = check_counts(n_seqs, 0)) return s;
    if (n_seqs == 0) return HE_OK;
    const int splits = paged_splits(cache->dtype, cache->page_size, n_heads, cache->n_kv_heads, n_seqs, longest_of(*cache, max_len));
    if ((int64_t)n_seqs * n_heads > kMostGroups) return refuse(HE_ERR_SHAPE, "%d sequences of %d heads: 2^24 in all at most", n_seqs, n_heads);
    const size_t need = split_bytes(n_seqs, n_heads, cache->head_dim, splits);
    if (need > workspace_bytes || (need && !d_workspace))
        return refuse(HE_ERR_CAPACITY, "workspace of %zu bytes, %zu are needed", d_workspace ? workspace_bytes : (size_t)0, need);
    if (need && !aligned(d_workspace)) return refuse(HE_ERR_SHAPE, "workspace does not lie on 16 bytes");
    paged_attention((hipStream_t)stream, cache->dtype, device_cache(*cache), device_rows(q), n_heads, device_rows(out), d_lens, n_seqs, splits, scale,
                    (float*)d_workspace);
    return launched();
}

he_status he_packed_attention(he_dtype dtype, const he_rows* q, int n_heads, const he_rows* k, const he_rows* v, int n_kv_heads, int head_dim,
                              const he_rows* out, const int32_t* d_seq_starts, int n_seqs, int n_tokens, int causal, float scale, void* stream) {
    if (const he_status s = check_heads(dtype, n_heads, n_kv_heads, head_dim)) return s;
    const int64_t wq = (int64_t)n_heads * head_dim, wk = (int64_t)n_kv_heads * head_dim;
    if (const he_status s = check_rows(q, "q", dtype, wq, false)) return s;
    if (const he_status s = check_rows(k, "k", dtype, wk, false)) return s;
    if (const he_status s = check_rows(v, "v", dtype, wk, false)) return s;
    if (const he_status s = check_rows(out, "out", dtype, wq, true)) return s;
    if (!d_seq_starts) return refuse(HE_ERR_INVALID_ARG, "d_seq_starts is NULL");
    if (causal != 0 && causal != 1) return refuse(HE_ERR_INVALID_ARG, "causal must be 0 or 1");
    if (!std::isfinite(scale)) return refuse(HE_ERR_INVALID_ARG, "scale is not finite");
    if (const he_status s = check_counts(n_seqs, n_tokens)) return s;
    if ((int64_t)(n_tokens / 32 + n_seqs) * n_heads > kMostGroups)
        return refuse(HE_ERR_SHAPE, "%d rows, %d sequences, %d heads: (rows / 32 + sequences) heads is 2^24 at most", n_tokens, n_seqs, n_heads);
    if (n_seqs == 0 || n_tokens == 0) return HE_OK;
    packed_attention((hipStream_t)stream, dtype, device_rows(q), n_heads, device_rows(k), device_rows(v), n_kv_heads, head_dim, device_rows(out), d_seq_starts,
                     n_seqs, n_tokens, causal != 0, scale);
    return launched();
}

size_t he_sample_workspace(int rows, int vocab) { return rows < 1 || rows > 65535 || vocab < 1 || vocab > 1 << 20 ? 0 : sample_workspace(rows, vocab); }

he_status he_sample(he_dtype dtype, const he_rows* logits, int rows, int vocab, const he_filters* filters_opt, const float* d_uniform, int32_t* d_ids,
                    float* d_logprobs, void* d_workspace, size_t workspace_bytes, void* stream) {
    if (!known(dtype)) return refuse(HE_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
    if (!logits || !logits->data || !d_uniform || !d_ids || !d_logprobs) return refuse(HE_ERR_INVALID_ARG, "logits, d_uniform, d_ids or d_logprobs is NULL");
    if ((uintptr_t)logits->data % elt_bytes(dtype)) return refuse(HE_ERR_SHAPE, "logits do not lie on whole elements");
    if (rows < 0 || vocab < 1) return refuse(HE_ERR_INVALID_ARG, "%d rows of %d logits", rows, vocab);
    if (vocab > 1 << 20) return refuse(HE_ERR_SHAPE, "vocabulary of %d: 2^20 at most", vocab);
    if (rows > 65535) return refuse(HE_ERR_SHAPE, "%d rows: 65535 at most", rows);
    if (logits->stride < 0) return refuse(HE_ERR_SHAPE, "logits: rows %lld elements apart", (long long)logits->stride);
    if (rows == 0) return HE_OK;
    const size_t need = sample_workspace(rows, vocab);
    if (!d_workspace || workspace_bytes < need) return refuse(HE_ERR_CAPACITY, "workspace of %zu bytes, %zu are needed", d_workspace ? workspace_bytes : (size_t)0, need);
    if (!aligned(d_workspace)) return refuse(HE_ERR_SHAPE, "workspace does not lie on 16 bytes");
    const Filters f = filters_opt ? Filters{filters_opt->d_temperature, filters_opt->d_top_k, filters_opt->d_top_p, filters_opt->d_min_p} : Filters{};
    sample((hipStream_t)stream, dtype, device_rows(logits), rows, vocab, f, d_uniform, d_ids, d_logprobs, d_workspace);
    return launched();
}

}  // extern "C"

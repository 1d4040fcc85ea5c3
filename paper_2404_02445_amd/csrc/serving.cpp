// Entry points of decoding with a paged cache: argument checks and launches.
#include <cmath>
#include <string>

#include "internal.h"

struct mopar_rotary_s {
    mopar::RotaryTable tab;
};

namespace mopar {

namespace {

int bad(const std::string& what) { return set_error(MOPAR_E_ARG, what); }

bool known_dtype(int dtype) { return dtype == MOPAR_F32 || dtype == MOPAR_BF16; }

bool aligned(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Rows of `tokens` x `heads` x `d` elements; `out` rows must not overlap.
int check_rows(const mopar_rows* r, const char* name, int dtype, int64_t tokens, int heads, int d, bool out) {
    const std::string nm(name);
    if (!r || !r->data) return bad(nm + ": null");
    if (!aligned(r->data)) return bad(nm + ": not 16-byte aligned");
    const int64_t epc = 16 / static_cast<int64_t>(dtype_size(dtype)), es = 16 / epc;
    if (r->token_stride < 0 || r->head_stride < 0 || r->token_stride % epc != 0 || r->head_stride % epc != 0)
        return bad(nm + ": strides must be multiples of 16 bytes and not negative");
    const int64_t lim = int64_t(1) << 31;
    if (r->token_stride >= lim / (64 * es)) return set_error(MOPAR_E_UNSUPPORTED, nm + ": 64 token strides reach 2 GiB");
    if (r->head_stride >= (int64_t(1) << 44)) return bad(nm + ": head stride");      // (65536 of them: 2^62 bytes)
    if (out) {
        const bool tokens_outside = (tokens <= 1 || r->token_stride >= (heads - 1) * r->head_stride + d) &&
                                    (heads <= 1 || r->head_stride >= d);
        const bool heads_outside = (heads <= 1 || r->head_stride >= (tokens - 1) * r->token_stride + d) &&
                                   (tokens <= 1 || r->token_stride >= d);
        if (!tokens_outside && !heads_outside) return bad(nm + ": rows overlap");
    }
    return MOPAR_OK;
}

int check_cache(const mopar_cache* c) {
    if (!c) return bad("cache: null");
    if (!known_dtype(c->dtype)) return set_error(MOPAR_E_DTYPE, "cache: dtype must be f32 or bf16");
    if (c->kv_heads < 1 || c->kv_heads > 65536) return bad("cache: kv_heads");
    if (c->head_dim < 1 || c->head_dim > 256 || c->head_dim * dtype_size(c->dtype) % 16 != 0)
        return set_error(MOPAR_E_UNSUPPORTED, "cache: head_dim must be a multiple of 16 bytes and at most 256");
    if (c->page_tokens < 1 || c->page_tokens > 4096 || (c->page_tokens & (c->page_tokens - 1)) != 0)
        return bad("cache: page_tokens must be a power of two, 1 to 4096");
    if (c->pages < 1 || c->pages >= (int64_t(1) << 31)) return bad("cache: pages");
    if (c->n_seq < 0) return bad("cache: n_seq");
    if (c->max_pages < 1 || c->table_stride < c->max_pages) return bad("cache: table_stride must cover max_pages, which is at least 1");
    if (static_cast<int64_t>(c->max_pages) * c->page_tokens >= (int64_t(1) << 31)) return bad("cache: 2^31 slots a sequence");
    if (c->pages > (int64_t(1) << 46) / (static_cast<int64_t>(c->kv_heads) * c->page_tokens * c->head_dim))
        return bad("cache: 2^46 elements and more");
    if (!aligned(c->k) || !aligned(c->v)) return bad("cache: k and v must be 16-byte aligned device pointers");
    if (c->n_seq > 0 && !c->table_dev) return bad("cache: table is null");
    return MOPAR_OK;
}

int check_attention(const mopar_attention* a) {
    if (!a) return bad("attention: null");
    if (!known_dtype(a->dtype)) return set_error(MOPAR_E_DTYPE, "attention: dtype must be f32 or bf16");
    if (a->heads < 1 || a->kv_heads < 1 || a->heads > 65536 || a->heads % a->kv_heads != 0)
        return bad("attention: heads must be a multiple of kv_heads");
    if (a->head_dim != 32 && a->head_dim != 64 && a->head_dim != 96 && a->head_dim != 128)
        return set_error(MOPAR_E_UNSUPPORTED, "attention: head_dim must be 32, 64, 96 or 128");
    if (!(a->scale > 0.0f) || !std::isfinite(a->scale * 1.5f)) return bad("attention: scale must be positive and at most 2^127");
    return MOPAR_OK;
}

int check_cache_attention(const mopar_attention* a, const mopar_cache* c, int64_t tokens, int32_t max_q, int32_t max_len) {
    if (int e = check_attention(a)) return e;
    if (int e = check_cache(c)) return e;
    if (a->dtype != c->dtype || a->kv_heads != c->kv_heads || a->head_dim != c->head_dim)
        return bad("attention: dtype, kv_heads and head_dim must be the cache's");
    if (tokens < 0 || tokens >= (int64_t(1) << 31) || max_q < 0 || max_len < 1) return bad("attention: tokens, max_q or max_len");
    if (static_cast<int64_t>(max_q) * (a->heads / a->kv_heads) >= (int64_t(1) << 20))
        return set_error(MOPAR_E_UNSUPPORTED, "attention: 2^20 query rows a key head and more");
    if (cache_limit(*c, max_len) > 1 << 30) return set_error(MOPAR_E_UNSUPPORTED, "attention: more than 2^30 slots a sequence");
    if (!attention_cache_fits(*a, c->n_seq, max_q, max_len))
        return set_error(MOPAR_E_UNSUPPORTED, "attention: sequences, key heads, max_q and max_len make 2^22 tiles or 2^30 stages and more");
    return MOPAR_OK;
}

// ... of a launch that may need more threads than a grid has
int launched(hipError_t e, const char* who) {
    if (e == hipErrorInvalidConfiguration) return set_error(MOPAR_E_UNSUPPORTED, std::string(who) + ": more than 2^32 threads");
    return hip_check(e, who);
}

}  // namespace

static int rotary_create_impl(const mopar_rotary_desc* desc, mopar_rotary_t* out) {
    if (!out) return bad("rotary: null out");
    *out = nullptr;
    if (!desc) return bad("rotary: null");
    RotaryTable tab;
    if (int e = rotary_table(*desc, &tab)) return e;
    *out = new mopar_rotary_s{tab};
    return MOPAR_OK;
}

static int rotary_apply_impl(const mopar_rotary_s* rot, int32_t dtype, int64_t tokens, int32_t heads, const int32_t* pos, const mopar_rows* x,
                      const mopar_rows* y, void* stream) {
    if (!rot) return bad("rotary: null");
    if (!known_dtype(dtype)) return set_error(MOPAR_E_DTYPE, "rotary: dtype must be f32 or bf16");
    const int d = rot->tab.d;
    if (d * dtype_size(dtype) % 16 != 0) return set_error(MOPAR_E_UNSUPPORTED, "rotary: head_dim must be a multiple of 16 bytes");
    if (tokens < 0 || heads < 0 || heads > 65536) return bad("rotary: tokens or heads");
    if (tokens == 0 || heads == 0) return MOPAR_OK;
    if (tokens >= (int64_t(1) << 31) / heads) return set_error(MOPAR_E_UNSUPPORTED, "rotary: 2^31 heads of tokens and more");
    if (!pos) return bad("rotary: positions are null");
    if (int e = check_rows(x, "rotary: x", dtype, tokens, heads, d, false)) return e;
    if (int e = check_rows(y, "rotary: y", dtype, tokens, heads, d, true)) return e;
    return launched(launch_rotary(rot->tab, dtype, tokens, heads, heads, pos, 1, x, y, static_cast<hipStream_t>(stream)), "mopar_rotary_apply");
}

static int cache_append_impl(const mopar_cache* c, const mopar_rotary_s* rot, int64_t tokens, int32_t heads, const int32_t* pos,
                      const int32_t* seq, const int32_t* slot, const mopar_rows* q, const mopar_rows* q_out, const mopar_rows* k,
                      const mopar_rows* v, void* stream) {
    if (int e = check_cache(c)) return e;
    if (tokens < 0 || heads < 0 || heads > 65536) return bad("append: tokens or heads");
    if (!rot) heads = 0;
    if (rot && rot->tab.d != c->head_dim) return bad("append: the rotary's head_dim is not the cache's");
    if (tokens == 0) return MOPAR_OK;
    if (tokens >= (int64_t(1) << 31) / (heads + 2 * static_cast<int64_t>(c->kv_heads)))
        return set_error(MOPAR_E_UNSUPPORTED, "append: 2^31 heads of tokens and more");
    if (!seq || !slot || (rot && !pos)) return bad("append: positions, sequences or slots are null");
    if (heads > 0) {
        if (int e = check_rows(q, "append: q", c->dtype, tokens, heads, c->head_dim, false)) return e;
        if (int e = check_rows(q_out, "append: q_out", c->dtype, tokens, heads, c->head_dim, true)) return e;
    }
    if (int e = check_rows(k, "append: k", c->dtype, tokens, c->kv_heads, c->head_dim, false)) return e;
    if (int e = check_rows(v, "append: v", c->dtype, tokens, c->kv_heads, c->head_dim, false)) return e;
    return launched(launch_cache_append(*c, rot ? &rot->tab : nullptr, tokens, heads, pos, seq, slot, q, q_out, k, v,
                                        static_cast<hipStream_t>(stream)),
                    "mopar_cache_append");
}

static int cache_keep_impl(const mopar_cache* c, int32_t layers, int64_t layer_stride, const int32_t* len, const int32_t* offsets,
                    int64_t entries, const int32_t* path, int32_t max_path, void* stream) {
    if (int e = check_cache(c)) return e;
    const int64_t epc = 16 / static_cast<int64_t>(dtype_size(c->dtype));
    if (layers < 0 || entries < 0 || max_path < 0) return bad("keep: layers, entries or max_path");
    if (layers > 1 && (layer_stride % epc != 0 || layer_stride < c->pages * c->kv_heads * c->page_tokens * c->head_dim))
        return bad("keep: layer_stride must cover a layer's pages and be a multiple of 16 bytes");
    if (layers > 1 && layer_stride > (int64_t(1) << 58) / layers) return bad("keep: 2^58 elements of layers and more");   // (2^60 bytes)
    if (c->n_seq == 0 || layers == 0 || entries == 0 || max_path == 0) return MOPAR_OK;
    if (!len || !offsets || !path) return bad("keep: lengths, offsets or path are null");
    const int64_t blocks = (static_cast<int64_t>(2) * c->kv_heads * c->head_dim / epc + 255) / 256;
    if (blocks * c->n_seq >= kMaxThreads / 256 / layers) return set_error(MOPAR_E_UNSUPPORTED, "keep: too many sequences and layers");
    return hip_check(launch_cache_keep(*c, layers, layer_stride, len, offsets, entries, path, max_path, static_cast<hipStream_t>(stream)),
                     "mopar_cache_keep");
}

static int attention_prompt_impl(const mopar_attention* a, int64_t tokens, int32_t n_seq, const int32_t* offsets, int32_t max_len,
                          const mopar_rows* q, const mopar_rows* k, const mopar_rows* v, const mopar_rows* out, void* stream) {
    if (int e = check_attention(a)) return e;
    if (tokens < 0 || tokens >= (int64_t(1) << 31) || n_seq < 0 || max_len < 0) return bad("attention: tokens, n_seq or max_len");
    if (tokens == 0 || n_seq == 0 || max_len == 0) return MOPAR_OK;
    if (!prompt_fits(tokens, n_seq, max_len, a->heads))
        return set_error(MOPAR_E_UNSUPPORTED, "attention: 2^30 tokens, or 2^24 tiles of 128 tokens of a sequence and head, and more");
    if (!offsets) return bad("attention: offsets are null");
    if (int e = check_rows(q, "attention: q", a->dtype, tokens, a->heads, a->head_dim, false)) return e;
    if (int e = check_rows(k, "attention: k", a->dtype, tokens, a->kv_heads, a->head_dim, false)) return e;
    if (int e = check_rows(v, "attention: v", a->dtype, tokens, a->kv_heads, a->head_dim, false)) return e;
    if (int e = check_rows(out, "attention: out", a->dtype, tokens, a->heads, a->head_dim, true)) return e;
    return hip_check(launch_attention_prompt(*a, tokens, n_seq, offsets, max_len, q, k, v, out, static_cast<hipStream_t>(stream)),
                     "mopar_attention_prompt");
}

static int attention_cache_ws_impl(const mopar_attention* a, const mopar_cache* c, int64_t tokens, int32_t max_q, int32_t max_len, size_t* bytes) {
    if (!bytes) return bad("attention: null bytes");
    if (int e = check_cache_attention(a, c, tokens, max_q, max_len)) return e;
    *bytes = attention_cache_ws_bytes(*a, *c, tokens, max_q, max_len);
    return MOPAR_OK;
}

static int attention_cache_impl(const mopar_attention* a, const mopar_cache* c, int64_t tokens, const int32_t* offsets, int32_t max_q,
                         const int32_t* len, int32_t max_len, const uint64_t* mask, int32_t mask_words, const mopar_rows* q,
                         const mopar_rows* out, void* ws, size_t ws_bytes, void* stream) {
    if (int e = check_cache_attention(a, c, tokens, max_q, max_len)) return e;
    if (mask && mask_words < (static_cast<int64_t>(max_q) + 63) / 64) return bad("attention: the mask has fewer words than max_q needs");
    if (tokens == 0 || c->n_seq == 0 || max_q == 0) return MOPAR_OK;
    if (!offsets || !len) return bad("attention: offsets or lengths are null");
    if (mask && (reinterpret_cast<uintptr_t>(mask) & 7) != 0) return bad("attention: the mask is not 8-byte aligned");
    if (int e = check_rows(q, "attention: q", a->dtype, tokens, a->heads, a->head_dim, false)) return e;
    if (int e = check_rows(out, "attention: out", a->dtype, tokens, a->heads, a->head_dim, true)) return e;
    const size_t need = attention_cache_ws_bytes(*a, *c, tokens, max_q, max_len);
    if (need > 0 && !aligned(ws)) return bad("attention: the workspace is null or not 16-byte aligned");
    if (ws_bytes < need) return set_error(MOPAR_E_WORKSPACE, "attention: the workspace is smaller than mopar_attention_cache_workspace_bytes");
    return hip_check(launch_attention_cache(*a, *c, tokens, offsets, max_q, len, max_len, mask, mask_words, q, out, ws,
                                            static_cast<hipStream_t>(stream)),
                     "mopar_attention_cache");
}

}  // namespace mopar

using namespace mopar;

extern "C" {

int mopar_rotary_create(const mopar_rotary_desc* desc, mopar_rotary_t* out) {
    return guarded("mopar_rotary_create", [&] { return rotary_create_impl(desc, out); });
}

void mopar_rotary_destroy(mopar_rotary_t rotary) { delete rotary; }

int mopar_rotary_apply(mopar_rotary_t rotary, int32_t dtype, int64_t tokens, int32_t heads, const int32_t* pos_dev,
                       const mopar_rows* x, const mopar_rows* y, void* stream) {
    return guarded("mopar_rotary_apply", [&] { return rotary_apply_impl(rotary, dtype, tokens, heads, pos_dev, x, y, stream); });
}

int mopar_cache_append(const mopar_cache* cache, mopar_rotary_t rotary, int64_t tokens, int32_t heads, const int32_t* pos_dev,
                       const int32_t* seq_dev, const int32_t* slot_dev, const mopar_rows* q, const mopar_rows* q_out,
                       const mopar_rows* k, const mopar_rows* v, void* stream) {
    return guarded("mopar_cache_append", [&] {
        return cache_append_impl(cache, rotary, tokens, heads, pos_dev, seq_dev, slot_dev, q, q_out, k, v, stream);
    });
}

int mopar_cache_keep(const mopar_cache* cache, int32_t layers, int64_t layer_stride, const int32_t* len_dev,
                     const int32_t* path_offsets_dev, int64_t entries, const int32_t* path_dev, int32_t max_path, void* stream) {
    return guarded("mopar_cache_keep", [&] {
        return cache_keep_impl(cache, layers, layer_stride, len_dev, path_offsets_dev, entries, path_dev, max_path, stream);
    });
}

int mopar_attention_prompt(const mopar_attention* a, int64_t tokens, int32_t n_seq, const int32_t* offsets_dev, int32_t max_len,
                           const mopar_rows* q, const mopar_rows* k, const mopar_rows* v, const mopar_rows* out, void* stream) {
    return guarded("mopar_attention_prompt",
                   [&] { return attention_prompt_impl(a, tokens, n_seq, offsets_dev, max_len, q, k, v, out, stream); });
}

int mopar_attention_cache_workspace_bytes(const mopar_attention* a, const mopar_cache* cache, int64_t tokens, int32_t max_q,
                                          int32_t max_len, size_t* bytes) {
    return guarded("mopar_attention_cache_workspace_bytes",
                   [&] { return attention_cache_ws_impl(a, cache, tokens, max_q, max_len, bytes); });
}

int mopar_attention_cache(const mopar_attention* a, const mopar_cache* cache, int64_t tokens, const int32_t* offsets_dev,
                          int32_t max_q, const int32_t* len_dev, int32_t max_len, const uint64_t* mask_dev, int32_t mask_words,
                          const mopar_rows* q, const mopar_rows* out, void* ws, size_t ws_bytes, void* stream) {
    return guarded("mopar_attention_cache", [&] {
        return attention_cache_impl(a, cache, tokens, offsets_dev, max_q, len_dev, max_len, mask_dev, mask_words, q, out, ws,
                                    ws_bytes, stream);
    });
}

}  // extern "C"

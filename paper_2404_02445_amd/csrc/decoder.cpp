// Entry points of a decoder's steps in 8 bits: argument checks and launches.
#include <cmath>
#include <string>

#include "internal.h"

namespace mopar {

namespace {

int bad(const std::string& what) { return set_error(MOPAR_E_ARG, what); }
int unsupported(const std::string& what) { return set_error(MOPAR_E_UNSUPPORTED, what); }

int check_dtype(int dtype, const char* who) {
    return dtype == MOPAR_F32 || dtype == MOPAR_BF16 ? MOPAR_OK : set_error(MOPAR_E_DTYPE, std::string(who) + ": dtype must be f32 or bf16");
}

bool on(const void* p, size_t align) { return p && (reinterpret_cast<uintptr_t>(p) & (align - 1)) == 0; }

constexpr int64_t kSpan = int64_t(1) << 46;     // elements from the first to the last row

// Rows of `width` elements; the rows of an output must not overlap.
int check_matrix(const mopar_matrix* m, const char* name, int dtype, int64_t rows, int64_t width, bool out) {
    const std::string nm(name);
    if (!m || !on(m->data, dtype_size(dtype))) return bad(nm + ": null or off its elements' alignment");
    if (m->stride < 0) return bad(nm + ": negative stride");
    if (out && rows > 1 && m->stride < width) return bad(nm + ": rows overlap");
    if (rows > 1 && m->stride >= kSpan / rows) return unsupported(nm + ": 2^46 elements and more");
    return MOPAR_OK;
}

int check_rows8(const mopar_rows8* m, const char* name, int64_t rows, int64_t width, bool out) {
    const std::string nm(name);
    if (!m || !on(m->q, 16)) return bad(nm + ": null or not 16-byte aligned");
    if (!on(m->scale, 4)) return bad(nm + ": scales are null or not 4-byte aligned");
    if (m->stride < 0 || m->stride % 16 != 0) return bad(nm + ": the stride must be a multiple of 16 and not negative");
    if (m->stride >= (int64_t(1) << 23)) return unsupported(nm + ": a stride of 2^23 bytes and more");
    if (out && rows > 1 && m->stride < width) return bad(nm + ": rows overlap");
    return MOPAR_OK;
}

int check_rows(int32_t dtype, int64_t tokens, int32_t width, const char* who) {
    if (int e = check_dtype(dtype, who)) return e;
    if (tokens < 0) return bad(std::string(who) + ": tokens");
    if (tokens >= (int64_t(1) << 31)) return unsupported(std::string(who) + ": 2^31 tokens and more");
    if (width < 1 || width > (1 << 24)) return bad(std::string(who) + ": width must be 1 to 2^24");
    return MOPAR_OK;
}

int rms_norm_impl(int32_t dtype, int64_t tokens, int32_t width, const mopar_matrix* x, const mopar_matrix* residual,
                  const mopar_matrix* total, const void* weight, float eps, const mopar_matrix* out, const mopar_rows8* out8, void* stream) {
    if (int e = check_rows(dtype, tokens, width, "norm")) return e;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return bad("norm: eps must be finite and not negative");
    if (total && !residual) return bad("norm: total goes with a residual");
    if (!out && !out8) return bad("norm: neither out nor out8");
    if (tokens == 0) return MOPAR_OK;
    if (int e = check_matrix(x, "norm: x", dtype, tokens, width, false)) return e;
    RowsJob j{};
    if (residual) {
        if (int e = check_matrix(residual, "norm: residual", dtype, tokens, width, false)) return e;
        j.residual = *residual;
    }
    if (total) {
        if (int e = check_matrix(total, "norm: total", dtype, tokens, width, true)) return e;
        j.total = *total;
    }
    if (!on(weight, dtype_size(dtype))) return bad("norm: weight is null or off its elements' alignment");
    if (out) {
        if (int e = check_matrix(out, "norm: out", dtype, tokens, width, true)) return e;
        if (total && total->data == out->data) return bad("norm: out and total are the same rows");
        j.out = *out;
    }
    if (out8) {
        if (int e = check_rows8(out8, "norm: out8", tokens, width, true)) return e;
        j.out8 = *out8;
    }
    j.dtype = dtype;
    j.tokens = tokens;
    j.width = width;
    j.x = *x;
    j.weight = weight;
    j.eps = eps;
    return hip_check(launch_rows8(j, static_cast<hipStream_t>(stream)), "mopar_rms_norm");
}

int quantize_rows_impl(int32_t dtype, int64_t tokens, int32_t width, const mopar_matrix* x, const mopar_matrix* gate, int32_t act,
                       const mopar_rows8* out8, void* stream) {
    if (int e = check_rows(dtype, tokens, width, "quantize")) return e;
    if (act < MOPAR_GATE_NONE || act > MOPAR_GATE_GELU) return bad("quantize: act");
    if ((act == MOPAR_GATE_NONE) != !gate) return bad("quantize: a gate goes with its activation");
    if (tokens == 0) return MOPAR_OK;
    if (int e = check_matrix(x, "quantize: x", dtype, tokens, width, false)) return e;
    RowsJob j{};
    if (gate) {
        if (int e = check_matrix(gate, "quantize: gate", dtype, tokens, width, false)) return e;
        j.gate = *gate;
    }
    if (int e = check_rows8(out8, "quantize: out8", tokens, width, true)) return e;
    j.dtype = dtype;
    j.tokens = tokens;
    j.width = width;
    j.x = *x;
    j.act = act;
    j.out8 = *out8;
    return hip_check(launch_rows8(j, static_cast<hipStream_t>(stream)), "mopar_quantize_rows");
}

int check_linear8(int64_t tokens, int64_t n_out, int32_t width) {
    if (tokens < 0 || n_out < 0 || width < 1) return bad("linear8: tokens, n_out or width");
    if (tokens >= (int64_t(1) << 31) || n_out >= (int64_t(1) << 31)) return unsupported("linear8: 2^31 rows and more");
    if (width >= 1 << 17) return unsupported("linear8: a width of 2^17 and more");
    if ((tokens + 63) / 64 * ((n_out + 63) / 64) >= (int64_t(1) << 23)) return unsupported("linear8: 2^23 tiles of 64 by 64 results and more");
    return MOPAR_OK;
}

int linear8_ws_impl(int64_t tokens, int64_t n_out, int32_t width, size_t* bytes) {
    if (!bytes) return bad("linear8: null bytes");
    if (int e = check_linear8(tokens, n_out, width)) return e;
    *bytes = linear8_ws_bytes(tokens, n_out, width);
    return MOPAR_OK;
}

int linear8_impl(int32_t dtype, int64_t tokens, int64_t n_out, int32_t width, const mopar_rows8* x, const mopar_rows8* w, const void* bias,
                 const mopar_matrix* out, void* ws, size_t ws_bytes, void* stream) {
    if (int e = check_dtype(dtype, "linear8")) return e;
    if (int e = check_linear8(tokens, n_out, width)) return e;
    if (tokens == 0 || n_out == 0) return MOPAR_OK;
    if (int e = check_rows8(x, "linear8: x", tokens, width, false)) return e;
    if (int e = check_rows8(w, "linear8: w", n_out, width, false)) return e;
    if (bias && !on(bias, dtype_size(dtype))) return bad("linear8: the bias is off its elements' alignment");
    if (int e = check_matrix(out, "linear8: out", dtype, tokens, n_out, true)) return e;
    if (!ws) ws_bytes = 0;
    if (ws && !on(ws, 16)) return bad("linear8: the workspace is not 16-byte aligned");
    if (ws && ws_bytes < linear8_ws_bytes(tokens, n_out, width))
        return set_error(MOPAR_E_WORKSPACE, "linear8: the workspace is smaller than mopar_linear8_workspace_bytes");
    return hip_check(launch_linear8(dtype, tokens, n_out, width, *x, *w, bias, *out, ws, linear8_plan(tokens, n_out, width, ws_bytes),
                                    static_cast<hipStream_t>(stream)),
                     "mopar_linear8");
}

int check_logprobs(int64_t rows, int32_t vocab, int32_t top) {
    if (rows < 0 || vocab < 1) return bad("logprobs: rows or vocab");
    if (rows >= (int64_t(1) << 24) || vocab >= 1 << 28) return unsupported("logprobs: 2^24 rows, or a vocabulary of 2^28, and more");
    if (top < 0 || top > 64 || top > vocab) return bad("logprobs: top must be 0 to 64 and at most vocab");
    return MOPAR_OK;
}

int token_logprobs_ws_impl(int64_t rows, int32_t vocab, int32_t top, size_t* bytes) {
    if (!bytes) return bad("logprobs: null bytes");
    if (int e = check_logprobs(rows, vocab, top)) return e;
    *bytes = logprob_ws_bytes(rows, vocab, top);
    return MOPAR_OK;
}

int token_logprobs_impl(int32_t dtype, int64_t rows, int32_t vocab, const mopar_matrix* logits, float scale, const int32_t* token, int32_t top,
                        float* logprob, float* entropy, int32_t* rank, float* top_logprob, int32_t* top_id, void* ws, size_t ws_bytes,
                        void* stream) {
    if (int e = check_dtype(dtype, "logprobs")) return e;
    if (int e = check_logprobs(rows, vocab, top)) return e;
    if (!(scale > 0.0f) || !std::isfinite(scale * 1.5f)) return bad("logprobs: scale must be positive and at most 2^127");
    if (rows == 0) return MOPAR_OK;
    if (int e = check_matrix(logits, "logprobs: logits", dtype, rows, vocab, false)) return e;
    if (!on(token, 4) || !on(logprob, 4)) return bad("logprobs: tokens or logprob are null or not 4-byte aligned");
    if ((entropy && !on(entropy, 4)) || (rank && !on(rank, 4))) return bad("logprobs: entropy or rank are not 4-byte aligned");
    if (top > 0 && (!on(top_logprob, 4) || !on(top_id, 4))) return bad("logprobs: top_logprob or top_id are null or not 4-byte aligned");
    if (ws && !on(ws, 16)) return bad("logprobs: the workspace is not 16-byte aligned");
    if (ws && ws_bytes < logprob_ws_bytes(rows, vocab, top))
        return set_error(MOPAR_E_WORKSPACE, "logprobs: the workspace is smaller than mopar_token_logprobs_workspace_bytes");
    const LogprobJob j{dtype, rows, vocab, *logits, scale, token, top, logprob, entropy, rank, top_logprob, top_id};
    return hip_check(launch_token_logprobs(j, ws ? logprob_splits(rows, vocab) : 1, ws, static_cast<hipStream_t>(stream)), "mopar_token_logprobs");
}

}  // namespace

}  // namespace mopar

using namespace mopar;

extern "C" {

int mopar_rms_norm(int32_t dtype, int64_t tokens, int32_t width, const mopar_matrix* x, const mopar_matrix* residual,
                   const mopar_matrix* total, const void* weight, float eps, const mopar_matrix* out, const mopar_rows8* out8, void* stream) {
    return guarded("mopar_rms_norm", [&] { return rms_norm_impl(dtype, tokens, width, x, residual, total, weight, eps, out, out8, stream); });
}

int mopar_quantize_rows(int32_t dtype, int64_t tokens, int32_t width, const mopar_matrix* x, const mopar_matrix* gate, int32_t act,
                        const mopar_rows8* out8, void* stream) {
    return guarded("mopar_quantize_rows", [&] { return quantize_rows_impl(dtype, tokens, width, x, gate, act, out8, stream); });
}

int mopar_linear8_workspace_bytes(int64_t tokens, int64_t n_out, int32_t width, size_t* bytes) {
    return guarded("mopar_linear8_workspace_bytes", [&] { return linear8_ws_impl(tokens, n_out, width, bytes); });
}

int mopar_linear8(int32_t dtype, int64_t tokens, int64_t n_out, int32_t width, const mopar_rows8* x, const mopar_rows8* w,
                  const void* bias, const mopar_matrix* out, void* ws, size_t ws_bytes, void* stream) {
    return guarded("mopar_linear8",
                   [&] { return linear8_impl(dtype, tokens, n_out, width, x, w, bias, out, ws, ws_bytes, stream); });
}

int mopar_token_logprobs_workspace_bytes(int64_t rows, int32_t vocab, int32_t top, size_t* bytes) {
    return guarded("mopar_token_logprobs_workspace_bytes", [&] { return token_logprobs_ws_impl(rows, vocab, top, bytes); });
}

int mopar_token_logprobs(int32_t dtype, int64_t rows, int32_t vocab, const mopar_matrix* logits, float scale, const int32_t* token_dev,
                         int32_t top, float* logprob_dev, float* entropy_dev, int32_t* rank_dev, float* top_logprob_dev,
                         int32_t* top_id_dev, void* ws, size_t ws_bytes, void* stream) {
    return guarded("mopar_token_logprobs", [&] {
        return token_logprobs_impl(dtype, rows, vocab, logits, scale, token_dev, top, logprob_dev, entropy_dev, rank_dev, top_logprob_dev,
                                   top_id_dev, ws, ws_bytes, stream);
    });
}

}  // extern "C"

// C-ABI entry points of the token operators: argument validation, then the
// launchers.
#include <cfloat>
#include <cmath>
#include <exception>
#include <string>

#include "attention_share.h"
#include "token_types.h"

using namespace neo;

namespace {

// Nothing thrown below (an allocation of a message or of the workspace's
// table) crosses the C boundary.
template <typename F>
int guarded(const char* fn, F&& body) noexcept {
    try {
        return body();
    } catch (const std::exception&) {
        try {
            return fail(NEO_ERR_OOM, std::string(fn) + ": out of host memory");
        } catch (...) {
            return NEO_ERR_OOM;
        }
    } catch (...) {
        return NEO_ERR_OOM;
    }
}

struct Check {
    const char* fn;
    int rc = NEO_OK;
    bool bad(int code, const std::string& what) {
        if (rc == NEO_OK) rc = fail(code, std::string(fn) + ": " + what);
        return false;
    }
    bool size(int v, const char* name, int least) {
        return v >= least ? rc == NEO_OK : bad(NEO_ERR_INVALID_ARG, std::string(name) + (least ? " must be > 0" : " must be >= 0"));
    }
    bool ptr(const void* p, const char* name) { return p ? rc == NEO_OK : bad(NEO_ERR_INVALID_ARG, std::string(name) + " is NULL"); }
    bool aligned(const void* p, const char* name, size_t to) {
        return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0
                   ? rc == NEO_OK
                   : bad(NEO_ERR_ALIGN, std::string(name) + " not " + std::to_string(to) + "-byte aligned");
    }
    bool stride(int64_t s, int64_t least, const char* name) {
        return s >= least ? rc == NEO_OK : bad(NEO_ERR_SHAPE, std::string(name) + " is less than a row");
    }
    // float data of `dtype`, int8 rows
    bool data(const void* p, int64_t s, int64_t cols, int dtype, const char* name) {
        return ptr(p, name) && aligned(p, name, dtype_size(dtype)) && stride(s, cols, (std::string(name) + "_stride").c_str());
    }
    bool rows8(const void* p, int64_t s, int64_t cols, const char* name) {
        if (!(ptr(p, name) && aligned(p, name, 16) && stride(s, (cols + 15) / 16 * 16, (std::string(name) + "_stride").c_str()))) return false;
        return s % 16 == 0 ? rc == NEO_OK : bad(NEO_ERR_ALIGN, std::string(name) + "_stride is not a multiple of 16");
    }
    bool type(int dtype) { return dtype_valid(dtype) ? rc == NEO_OK : bad(NEO_ERR_INVALID_ARG, "dtype"); }
    int launched(hipError_t e) { return e == hipSuccess ? NEO_OK : hip_fail(e, (std::string(fn) + " launch").c_str()); }
};

bool check_cache(Check& c, const neo_kv_cache* k) {
    if (!c.ptr(k, "cache")) return false;
    c.size(k->pages, "cache.pages", 1);
    c.size(k->kv_heads, "cache.kv_heads", 1);
    c.size(k->page_size, "cache.page_size", 1);
    c.size(k->head_dim, "cache.head_dim", 1);
    if (c.rc == NEO_OK && (k->head_dim % 16 || k->head_dim > 256))
        c.bad(NEO_ERR_UNSUPPORTED, "cache.head_dim must be a multiple of 16 up to 256");
    if (c.rc == NEO_OK && (int64_t)k->kv_heads * k->head_dim > (int64_t)0x7fffffff / k->page_size)
        c.bad(NEO_ERR_UNSUPPORTED, "cache: a page of 2 GiB or more");
    c.ptr(k->k, "cache.k") && c.aligned(k->k, "cache.k", 16);
    c.ptr(k->v, "cache.v") && c.aligned(k->v, "cache.v", 16);
    c.ptr(k->k_scale, "cache.k_scale") && c.aligned(k->k_scale, "cache.k_scale", 4);
    c.ptr(k->v_scale, "cache.v_scale") && c.aligned(k->v_scale, "cache.v_scale", 4);
    return c.rc == NEO_OK;
}

// Rows [tokens][heads][dim] that a call writes: no two of them overlap.
bool check_out(Check& c, const void* p, int64_t ts, int64_t hs, int tokens, int heads, int dim, int dtype, const char* name) {
    if (!(c.ptr(p, name) && c.aligned(p, name, dtype_size(dtype)))) return false;
    const std::string n(name);
    if (tokens > 1) c.stride(ts, dim, (n + "_token_stride").c_str());
    if (heads > 1) c.stride(hs, dim, (n + "_head_stride").c_str());
    // (differences of 64-bit strides are taken in 128 bits)
    const __int128 t = tokens > 1 ? ts : 0, h = heads > 1 ? hs : 0;
    if (c.rc == NEO_OK && tokens > 1 && heads > 1 && t < h * (heads - 1) + dim && h < t * (tokens - 1) + dim)
        c.bad(NEO_ERR_SHAPE, n + ": tokens and heads overlap");
    return c.rc == NEO_OK;
}

// What both rotary calls take; in place, the strides are the input's.
bool check_rotary(Check& c, const void* x, int64_t xts, int64_t xhs, int tokens, int heads, int dim, int rot_dim, int layout, int dtype,
                  const int64_t* positions, const double* freqs, double amplitude, const void* y, int64_t yts, int64_t yhs,
                  const char* in, const char* out) {
    if (c.rc == NEO_OK && (rot_dim < 2 || rot_dim % 2 || rot_dim > dim)) c.bad(NEO_ERR_SHAPE, "rot_dim must be even, 2 .. head_dim");
    if (c.rc == NEO_OK && layout != NEO_ROTARY_HALF && layout != NEO_ROTARY_INTERLEAVED) c.bad(NEO_ERR_INVALID_ARG, "layout");
    if (c.rc == NEO_OK && !(std::fabs(amplitude) <= FLT_MAX)) c.bad(NEO_ERR_INVALID_ARG, "amplitude must be finite in float32");
    if (c.rc != NEO_OK || tokens == 0) return c.rc == NEO_OK;
    c.ptr(x, in) && c.aligned(x, in, dtype_size(dtype));
    if (c.rc == NEO_OK && (xts < 0 || xhs < 0)) c.bad(NEO_ERR_INVALID_ARG, "negative stride");
    c.ptr(positions, "positions") && c.aligned(positions, "positions", 8);
    c.ptr(freqs, "freqs") && c.aligned(freqs, "freqs", 8);
    check_out(c, y, yts, yhs, tokens, heads, dim, dtype, out);
    if (c.rc == NEO_OK && x == y && ((tokens > 1 && xts != yts) || (heads > 1 && xhs != yhs)))
        c.bad(NEO_ERR_SHAPE, std::string(out) + " in place of " + in + " has its strides");
    return c.rc == NEO_OK;
}

// What both attention calls take; false also where there is nothing to do.
bool check_attention(Check& c, const neo_kv_cache* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride, int tokens,
                     int q_heads, int dtype, const int32_t* page_table, int64_t table_stride, const int32_t* context_lens,
                     const int32_t* q_starts, int seqs, int max_chunk, int max_context, float scale, int window, const void* out,
                     int64_t out_token_stride, int64_t out_head_stride) {
    c.type(dtype) && check_cache(c, cache) && c.size(tokens, "tokens", 0) && c.size(q_heads, "q_heads", 1) &&
        c.size(seqs, "seqs", 0) && c.size(max_chunk, "max_chunk", 0) && c.size(max_context, "max_context", 0) &&
        c.size(window, "window", 0);
    if (c.rc == NEO_OK && q_heads % cache->kv_heads) c.bad(NEO_ERR_SHAPE, "q_heads is not a multiple of cache.kv_heads");
    if (c.rc == NEO_OK && !(scale > 0.f && std::isfinite(scale))) c.bad(NEO_ERR_INVALID_ARG, "scale must be finite and > 0");
    if (c.rc != NEO_OK || tokens == 0 || seqs == 0 || max_chunk == 0) return false;
    c.ptr(q, "q") && c.aligned(q, "q", dtype_size(dtype));
    c.ptr(out, "out") && c.aligned(out, "out", dtype_size(dtype));
    if (q_token_stride < 0 || q_head_stride < 0) c.bad(NEO_ERR_INVALID_ARG, "negative stride");
    c.stride(out_head_stride, cache->head_dim, "out_head_stride") && c.stride(out_token_stride, cache->head_dim, "out_token_stride");
    c.ptr(page_table, "page_table") && c.aligned(page_table, "page_table", 4);
    c.ptr(context_lens, "context_lens") && c.aligned(context_lens, "context_lens", 4);
    c.ptr(q_starts, "q_starts") && c.aligned(q_starts, "q_starts", 4);
    if (c.rc == NEO_OK && max_context > 0x7fff0000) c.bad(NEO_ERR_UNSUPPORTED, "max_context above 2^31 - 2^16");
    if (c.rc == NEO_OK && (table_stride < 0 || ((int64_t)max_context + cache->page_size - 1) / cache->page_size > table_stride))
        c.bad(NEO_ERR_SHAPE, "max_context does not fit table_stride pages");
    return c.rc == NEO_OK;
}

bool check_layers(Check& c, const neo_kv_cache* k, int layers, int64_t layer_stride) {
    check_cache(c, k) && c.size(layers, "layers", 0);
    if (c.rc == NEO_OK && layers > 1 && layer_stride / k->page_size / k->kv_heads < k->pages)
        c.bad(NEO_ERR_SHAPE, "layer_stride is less than a layer");
    if (c.rc == NEO_OK && layers > 1 && (layers > 1 << 16 || layer_stride > 1ll << 38))
        c.bad(NEO_ERR_UNSUPPORTED, "layers above 2^16 or layer_stride above 2^38");
    return c.rc == NEO_OK;
}

int compact(const char* fn, const neo_kv_cache* cache, int layers, int64_t layer_stride, const int32_t* page_table, int64_t table_stride,
            int64_t table_pages, const int32_t* bases, const int32_t* keep, const int32_t* keep_starts, int kept, int seqs, int max_keep,
            neo_stream_t stream) {
    Check c{fn};
    check_layers(c, cache, layers, layer_stride) && c.size(kept, "kept", 0) && c.size(seqs, "seqs", 0) && c.size(max_keep, "max_keep", 0);
    if (c.rc == NEO_OK && (table_pages < 0 || table_stride < 0 || (seqs > 1 && table_stride < table_pages)))
        c.bad(NEO_ERR_SHAPE, "table_stride is less than a row");
    if (c.rc == NEO_OK && (table_stride > 0x7fffffff || table_pages > 0x7fffffff))
        c.bad(NEO_ERR_UNSUPPORTED, "table_stride or table_pages above 2^31 - 1");
    if (c.rc != NEO_OK || layers == 0 || kept == 0 || seqs == 0 || max_keep == 0 || table_pages == 0) return c.rc;
    c.ptr(page_table, "page_table") && c.aligned(page_table, "page_table", 4);
    c.ptr(bases, "bases") && c.aligned(bases, "bases", 4);
    c.ptr(keep, "keep") && c.aligned(keep, "keep", 4);
    c.ptr(keep_starts, "keep_starts") && c.aligned(keep_starts, "keep_starts", 4);
    if (c.rc != NEO_OK) return c.rc;
    CompactArgs a{*cache, layers > 1 ? layer_stride : 0, layers, page_table, bases, keep, keep_starts, table_stride, table_pages, kept, seqs,
                  std::min(max_keep, kept)};
    return c.launched(launch_kv_compact(a, (hipStream_t)stream));
}

// Both calls over shared prefixes; `saved` null: by the bounds.
int shared_attention(const char* fn, const neo_kv_cache* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride, int tokens,
                     int q_heads, int dtype, const int32_t* page_table, int64_t table_stride, const int32_t* context_lens,
                     const int32_t* q_starts, int seqs, const int32_t* group_starts, const int32_t* prefix_lens, int groups,
                     int max_chunk, int max_group, int max_context, int max_own, const int64_t* saved, float scale, int window, void* out,
                     int64_t out_token_stride, int64_t out_head_stride, neo_stream_t stream) {
    Check c{fn};
    c.size(groups, "groups", 0) && c.size(max_group, "max_group", 0) && c.size(max_own, "max_own", 0);
    if (c.rc != NEO_OK || !check_attention(c, cache, q, q_token_stride, q_head_stride, tokens, q_heads, dtype, page_table, table_stride,
                                           context_lens, q_starts, seqs, max_chunk, max_context, scale, window, out,
                                           out_token_stride, out_head_stride))
        return c.rc;
    if (groups == 0 || groups > seqs) c.bad(NEO_ERR_SHAPE, "groups must be 1 .. seqs");
    c.ptr(group_starts, "group_starts") && c.aligned(group_starts, "group_starts", 4);
    c.ptr(prefix_lens, "prefix_lens") && c.aligned(prefix_lens, "prefix_lens", 4);
    if (c.rc != NEO_OK) return c.rc;
    AttnArgs own{*cache, q, out, q_token_stride, q_head_stride, out_token_stride, out_head_stride, table_stride,
                 page_table, context_lens, q_starts, tokens, q_heads, seqs, std::min(max_chunk, tokens), max_context,
                 window, scale};
    own.group_starts = group_starts, own.prefix_lens = prefix_lens, own.all_seqs = seqs;
    own.max_own = max_own ? std::min(max_own, max_context) : max_context;
    AttnArgs shared = own;
    shared.seqs = groups, shared.max_chunk = std::max(1, std::min(max_group, tokens));
    if ((int64_t)own.max_chunk * q_heads > (1 << 28) / seqs || (int64_t)shared.max_chunk * q_heads > (1 << 28) / groups)
        return c.bad(NEO_ERR_UNSUPPORTED, "max_chunk * q_heads * seqs or max_group * q_heads * groups above 2^28"), c.rc;
    Workspace ws;
    const double less = saved ? (double)*saved
                              : saved_by_bounds(seqs, groups, (int64_t)tokens * (q_heads / cache->kv_heads), own.max_chunk, max_context,
                                                max_own, window);
    if (!worth_sharing(less, cache->kv_heads, cache->head_dim)) {
        if (const size_t need = attention_workspace(own)) {
            const int rc = stream_workspace(c.fn, (hipStream_t)stream, need, &ws);
            if (rc != NEO_OK) return rc;
        }
        return c.launched(launch_attention(dtype, own, ws.ptr, (hipStream_t)stream));
    }
    // the rows' parts of the shared tokens, how many each sequence shares, and behind them the shares' parts, of one launch
    // at a time
    const size_t rows = (size_t)tokens * q_heads, o = rows * cache->head_dim, lens = o + 2 * rows, parts = (lens + seqs + 3) / 4 * 4;
    const int rc = stream_workspace(c.fn, (hipStream_t)stream,
                                    (parts + std::max(attention_shared_floats(shared), attention_own_floats(own))) * sizeof(float), &ws);
    if (rc != NEO_OK) return rc;
    for (AttnArgs* a : {&shared, &own}) {
        a->part_o = ws.ptr;
        a->part_ml = reinterpret_cast<float2*>(ws.ptr + o);
        a->shared = reinterpret_cast<int32_t*>(ws.ptr + lens);
    }
    if (const int failed = c.launched(launch_attention_shared(dtype, shared, ws.ptr + parts, (hipStream_t)stream))) return failed;
    return c.launched(launch_attention_own(dtype, own, ws.ptr + parts, (hipStream_t)stream));
}

}  // namespace

int neo_rmsnorm_int8(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                     const float* gamma, float eps, int rows, int cols, int dtype, void* h, int64_t h_stride, void* y,
                     int64_t y_stride, int8_t* yq, int64_t yq_stride, float* y_scale, neo_stream_t stream) {
    return guarded("neo_rmsnorm_int8", [&] {
        Check c{"neo_rmsnorm_int8"};
        c.type(dtype) && c.size(rows, "rows", 0) && c.size(cols, "cols", 1);
        if (c.rc == NEO_OK && cols > kRowsMaxCols) c.bad(NEO_ERR_UNSUPPORTED, "cols above 65,536");
        if (c.rc == NEO_OK && !(eps >= 0.f && std::isfinite(eps))) c.bad(NEO_ERR_INVALID_ARG, "eps must be finite and >= 0");
        if (c.rc != NEO_OK || rows == 0) return c.rc;
        if (!h && !y && !yq) c.bad(NEO_ERR_INVALID_ARG, "none of h, y and yq given");
        if (!yq != !y_scale) c.bad(NEO_ERR_INVALID_ARG, "yq and y_scale: both or neither");
        c.data(x, x_stride, cols, dtype, "x");
        if (residual) c.data(residual, residual_stride, cols, dtype, "residual");
        if (gamma) c.aligned(gamma, "gamma", 4);
        if (h) c.data(h, h_stride, cols, dtype, "h");
        if (y) c.data(y, y_stride, cols, dtype, "y");
        if (yq) c.rows8(yq, yq_stride, cols, "yq") && c.aligned(y_scale, "y_scale", 4);
        if (h && ((h == x && h_stride != x_stride) || (h == residual && h_stride != residual_stride)))
            c.bad(NEO_ERR_SHAPE, "h in place of an input has that input's stride");
        if (c.rc != NEO_OK) return c.rc;
        RowsArgs a{x, residual, gamma, h, y, yq, y_scale, x_stride, residual_stride, h_stride, y_stride, yq_stride, eps, rows, cols};
        return c.launched(launch_rmsnorm(dtype, a, (hipStream_t)stream));
    });
}

int neo_quantize_tokens_int8(const void* x, int64_t x_stride, const void* gate, int64_t gate_stride, int rows, int cols,
                             int dtype, int8_t* xq, int64_t xq_stride, float* x_scale, neo_stream_t stream) {
    return guarded("neo_quantize_tokens_int8", [&] {
        Check c{"neo_quantize_tokens_int8"};
        c.type(dtype) && c.size(rows, "rows", 0) && c.size(cols, "cols", 1);
        if (c.rc == NEO_OK && cols > kRowsMaxCols) c.bad(NEO_ERR_UNSUPPORTED, "cols above 65,536");
        if (c.rc != NEO_OK || rows == 0) return c.rc;
        c.data(x, x_stride, cols, dtype, "x");
        if (gate) c.data(gate, gate_stride, cols, dtype, "gate");
        c.rows8(xq, xq_stride, cols, "xq");
        c.ptr(x_scale, "x_scale") && c.aligned(x_scale, "x_scale", 4);
        if (c.rc != NEO_OK) return c.rc;
        RowsArgs a{x, gate, nullptr, nullptr, nullptr, xq, x_scale, x_stride, gate_stride, 0, 0, xq_stride, 0.f, rows, cols};
        return c.launched(launch_quantize_tokens(dtype, a, (hipStream_t)stream));
    });
}

int neo_dequantize_tokens_int8(const int8_t* xq, int64_t xq_stride, const float* x_scale, int rows, int cols, int dtype,
                               void* y, int64_t y_stride, neo_stream_t stream) {
    return guarded("neo_dequantize_tokens_int8", [&] {
        Check c{"neo_dequantize_tokens_int8"};
        c.type(dtype) && c.size(rows, "rows", 0) && c.size(cols, "cols", 1);
        if (c.rc != NEO_OK || rows == 0) return c.rc;
        c.rows8(xq, xq_stride, cols, "xq");
        c.ptr(x_scale, "x_scale") && c.aligned(x_scale, "x_scale", 4);
        c.data(y, y_stride, cols, dtype, "y");
        if (c.rc != NEO_OK) return c.rc;
        return c.launched(launch_dequantize_tokens(dtype, xq, xq_stride, x_scale, rows, cols, y, y_stride, (hipStream_t)stream));
    });
}

int neo_matmul_int8(const int8_t* xq, int64_t xq_stride, const float* x_scale, int M, int in_features,
                    const int8_t* w_rows, const float* w_scale, int out_features, const float* bias, int act, int dtype,
                    void* y, int64_t y_stride, neo_stream_t stream) {
    return guarded("neo_matmul_int8", [&] {
        Check c{"neo_matmul_int8"};
        c.type(dtype) && c.size(M, "M", 0) && c.size(in_features, "in_features", 1) && c.size(out_features, "out_features", 1);
        if (c.rc == NEO_OK && act != NEO_ACT_NONE && act != NEO_ACT_RELU) c.bad(NEO_ERR_INVALID_ARG, "act");
        if (c.rc == NEO_OK && (int64_t)in_features * 127 * 127 >= (1LL << 31))
            c.bad(NEO_ERR_UNSUPPORTED, "in_features above 133,144 could overflow int32");
        if (c.rc != NEO_OK || M == 0) return c.rc;
        c.rows8(xq, xq_stride, in_features, "xq");
        c.ptr(x_scale, "x_scale") && c.aligned(x_scale, "x_scale", 4);
        if (M > 1 << 30 || out_features > 1 << 26) c.bad(NEO_ERR_UNSUPPORTED, "M above 2^30 or out_features above 2^26");
        c.ptr(w_rows, "w_rows") && c.aligned(w_rows, "w_rows", 16);
        c.ptr(w_scale, "w_scale") && c.aligned(w_scale, "w_scale", 4);
        if (bias) c.aligned(bias, "bias", 4);
        c.data(y, y_stride, out_features, dtype, "y");
        if (c.rc != NEO_OK) return c.rc;
        MatmulArgs a{xq, w_rows, x_scale, w_scale, bias, y, xq_stride, y_stride, M, out_features, cdiv(in_features, 16) * 16, act, dtype};
        Workspace ws;
        if (const size_t need = matmul_int8_workspace(a)) {
            const int rc = stream_workspace(c.fn, (hipStream_t)stream, need, &ws);
            if (rc != NEO_OK) return rc;
        }
        return c.launched(launch_matmul_int8(a, ws.ptr, (hipStream_t)stream));
    });
}

int neo_kv_write_int8(const neo_kv_cache* cache, const void* k, int64_t k_token_stride, int64_t k_head_stride,
                      const void* v, int64_t v_token_stride, int64_t v_head_stride, int tokens, int dtype,
                      const int64_t* slots, neo_stream_t stream) {
    return guarded("neo_kv_write_int8", [&] {
        Check c{"neo_kv_write_int8"};
        c.type(dtype) && check_cache(c, cache) && c.size(tokens, "tokens", 0);
        if (c.rc != NEO_OK || tokens == 0) return c.rc;
        c.ptr(k, "k") && c.aligned(k, "k", dtype_size(dtype));
        c.ptr(v, "v") && c.aligned(v, "v", dtype_size(dtype));
        if (k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 || v_head_stride < 0)
            c.bad(NEO_ERR_INVALID_ARG, "negative stride");
        c.ptr(slots, "slots") && c.aligned(slots, "slots", 8);
        if (c.rc != NEO_OK) return c.rc;
        KvArgs a{*cache, k, v, nullptr, nullptr, k_token_stride, k_head_stride, v_token_stride, v_head_stride, slots, tokens};
        return c.launched(launch_kv_write(dtype, a, (hipStream_t)stream));
    });
}

int neo_kv_read_int8(const neo_kv_cache* cache, const int64_t* slots, int tokens, int dtype, void* k_out, void* v_out,
                     neo_stream_t stream) {
    return guarded("neo_kv_read_int8", [&] {
        Check c{"neo_kv_read_int8"};
        c.type(dtype) && check_cache(c, cache) && c.size(tokens, "tokens", 0);
        if (c.rc != NEO_OK || tokens == 0) return c.rc;
        if (!k_out && !v_out) c.bad(NEO_ERR_INVALID_ARG, "neither k_out nor v_out given");
        c.aligned(k_out, "k_out", dtype_size(dtype));
        c.aligned(v_out, "v_out", dtype_size(dtype));
        c.ptr(slots, "slots") && c.aligned(slots, "slots", 8);
        if (c.rc != NEO_OK) return c.rc;
        KvArgs a{*cache, nullptr, nullptr, k_out, v_out, 0, 0, 0, 0, slots, tokens};
        return c.launched(launch_kv_read(dtype, a, (hipStream_t)stream));
    });
}

int neo_rotary_frequencies(int rot_dim, double base, int scaling, double factor, double context, double low, double high,
                           double* freqs) {
    return guarded("neo_rotary_frequencies", [&] {
        Check c{"neo_rotary_frequencies"};
        if (rot_dim < 2 || rot_dim % 2) c.bad(NEO_ERR_INVALID_ARG, "rot_dim must be even and > 0");
        if (!(base >= 1 && std::isfinite(base))) c.bad(NEO_ERR_INVALID_ARG, "base must be finite and >= 1");
        if (scaling < NEO_ROTARY_NONE || scaling > NEO_ROTARY_TURNS) c.bad(NEO_ERR_INVALID_ARG, "scaling");
        if (scaling != NEO_ROTARY_NONE && !(factor >= 1 && std::isfinite(factor))) c.bad(NEO_ERR_INVALID_ARG, "factor must be finite and >= 1");
        if (scaling == NEO_ROTARY_TURNS && !(context > 0 && std::isfinite(context) && low >= 0 && low < high && std::isfinite(high)))
            c.bad(NEO_ERR_INVALID_ARG, "context must be > 0 and 0 <= low < high, finite");
        c.ptr(freqs, "freqs");
        if (c.rc != NEO_OK) return c.rc;
        if (scaling == NEO_ROTARY_BASE && rot_dim > 2) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
        for (int i = 0; i < rot_dim / 2; ++i) {
            double f = std::pow(base, -2.0 * i / rot_dim);
            if (scaling == NEO_ROTARY_LINEAR) f /= factor;
            if (scaling == NEO_ROTARY_TURNS) {
                const double turns = context * f / 6.283185307179586;
                const double w = std::min(1.0, std::max(0.0, (turns - low) / (high - low)));
                f *= w + (1 - w) / factor;
            }
            freqs[i] = f;
        }
        return (int)NEO_OK;
    });
}

int neo_rotary(const void* x, int64_t x_token_stride, int64_t x_head_stride, int tokens, int heads, int head_dim, int rot_dim,
               int layout, int dtype, const int64_t* positions, const double* freqs, double amplitude, void* y,
               int64_t y_token_stride, int64_t y_head_stride, neo_stream_t stream) {
    return guarded("neo_rotary", [&] {
        Check c{"neo_rotary"};
        c.type(dtype) && c.size(tokens, "tokens", 0) && c.size(heads, "heads", 1) && c.size(head_dim, "head_dim", 1);
        if (c.rc == NEO_OK && (head_dim > 1024 || (int64_t)heads * head_dim > 1 << 28))
            c.bad(NEO_ERR_UNSUPPORTED, "head_dim above 1024, or heads * head_dim above 2^28");
        check_rotary(c, x, x_token_stride, x_head_stride, tokens, heads, head_dim, rot_dim, layout, dtype, positions, freqs, amplitude, y,
                     y_token_stride, y_head_stride, "x", "y");
        if (c.rc != NEO_OK || tokens == 0) return c.rc;
        RotaryArgs a{x, y, x_token_stride, x_head_stride, y_token_stride, y_head_stride, heads, positions, freqs, amplitude, tokens,
                     head_dim, rot_dim, layout, {}};
        return c.launched(launch_rotary(dtype, a, false, (hipStream_t)stream));
    });
}

int neo_rotary_kv_write_int8(const neo_kv_cache* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride, int q_heads,
                             const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                             int64_t v_head_stride, int tokens, int rot_dim, int layout, int dtype, const int64_t* positions,
                             const double* freqs, double amplitude, const int64_t* slots, void* q_out, int64_t out_token_stride,
                             int64_t out_head_stride, neo_stream_t stream) {
    return guarded("neo_rotary_kv_write_int8", [&] {
        Check c{"neo_rotary_kv_write_int8"};
        c.type(dtype) && check_cache(c, cache) && c.size(tokens, "tokens", 0) && c.size(q_heads, "q_heads", 1);
        if (c.rc == NEO_OK && ((int64_t)q_heads * cache->head_dim > 1 << 28 || cache->kv_heads > 1 << 23))
            c.bad(NEO_ERR_UNSUPPORTED, "q_heads * head_dim above 2^28, or kv_heads above 2^23");
        if (c.rc != NEO_OK) return c.rc;
        check_rotary(c, q, q_token_stride, q_head_stride, tokens, q_heads, cache->head_dim, rot_dim, layout, dtype, positions, freqs,
                     amplitude, q_out, out_token_stride, out_head_stride, "q", "q_out");
        if (c.rc != NEO_OK || tokens == 0) return c.rc;
        c.ptr(k, "k") && c.aligned(k, "k", dtype_size(dtype));
        c.ptr(v, "v") && c.aligned(v, "v", dtype_size(dtype));
        if (k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 || v_head_stride < 0)
            c.bad(NEO_ERR_INVALID_ARG, "negative stride");
        c.ptr(slots, "slots") && c.aligned(slots, "slots", 8);
        if (c.rc != NEO_OK) return c.rc;
        RotaryArgs a{q, q_out, q_token_stride, q_head_stride, out_token_stride, out_head_stride, q_heads, positions, freqs, amplitude,
                     tokens, cache->head_dim, rot_dim, layout,
                     {*cache, k, v, nullptr, nullptr, k_token_stride, k_head_stride, v_token_stride, v_head_stride, slots, tokens}};
        return c.launched(launch_rotary(dtype, a, true, (hipStream_t)stream));
    });
}

int neo_kv_copy_pages(const neo_kv_cache* cache, int layers, int64_t layer_stride, const int32_t* src, const int32_t* dst,
                      const int32_t* entries, int pairs, neo_stream_t stream) {
    return guarded("neo_kv_copy_pages", [&] {
        Check c{"neo_kv_copy_pages"};
        check_layers(c, cache, layers, layer_stride) && c.size(pairs, "pairs", 0);
        if (c.rc != NEO_OK || layers == 0 || pairs == 0) return c.rc;
        c.ptr(src, "src") && c.aligned(src, "src", 4);
        c.ptr(dst, "dst") && c.aligned(dst, "dst", 4);
        c.aligned(entries, "entries", 4);
        if (c.rc != NEO_OK) return c.rc;
        CopyArgs a{*cache, layers > 1 ? layer_stride : 0, layers, src, dst, entries, pairs};
        return c.launched(launch_kv_copy(a, (hipStream_t)stream));
    });
}

int neo_kv_compact(const neo_kv_cache* cache, int layers, int64_t layer_stride, const int32_t* page_table, int64_t table_stride,
                   const int32_t* bases, const int32_t* keep, const int32_t* keep_starts, int kept, int seqs, int max_keep,
                   neo_stream_t stream) {
    return guarded("neo_kv_compact", [&] {
        return compact("neo_kv_compact", cache, layers, layer_stride, page_table, table_stride, table_stride, bases, keep, keep_starts,
                       kept, seqs, max_keep, stream);
    });
}

int neo_kv_compact_columns(const neo_kv_cache* cache, int layers, int64_t layer_stride, const int32_t* page_table, int64_t table_stride,
                           int64_t table_pages, const int32_t* bases, const int32_t* keep, const int32_t* keep_starts, int kept,
                           int seqs, int max_keep, neo_stream_t stream) {
    return guarded("neo_kv_compact_columns", [&] {
        return compact("neo_kv_compact_columns", cache, layers, layer_stride, page_table, table_stride, table_pages, bases, keep,
                       keep_starts, kept, seqs, max_keep, stream);
    });
}

int neo_attention_paged_int8(const neo_kv_cache* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                             int tokens, int q_heads, int dtype, const int32_t* page_table, int64_t table_stride,
                             const int32_t* context_lens, const int32_t* q_starts, int seqs, int max_chunk,
                             int max_context, float scale, int window, void* out, int64_t out_token_stride,
                             int64_t out_head_stride, neo_stream_t stream) {
    return guarded("neo_attention_paged_int8", [&] {
        Check c{"neo_attention_paged_int8"};
        if (!check_attention(c, cache, q, q_token_stride, q_head_stride, tokens, q_heads, dtype, page_table, table_stride, context_lens,
                             q_starts, seqs, max_chunk, max_context, scale, window, out, out_token_stride, out_head_stride))
            return c.rc;
        AttnArgs a{*cache, q, out, q_token_stride, q_head_stride, out_token_stride, out_head_stride, table_stride,
                   page_table, context_lens, q_starts, tokens, q_heads, seqs, std::min(max_chunk, tokens), max_context,
                   window, scale};
        if ((int64_t)a.max_chunk * q_heads > (1 << 28) / seqs)
            return c.bad(NEO_ERR_UNSUPPORTED, "max_chunk * q_heads * seqs above 2^28"), c.rc;
        Workspace ws;
        if (const size_t need = attention_workspace(a)) {
            const int rc = stream_workspace(c.fn, (hipStream_t)stream, need, &ws);
            if (rc != NEO_OK) return rc;
        }
        return c.launched(launch_attention(dtype, a, ws.ptr, (hipStream_t)stream));
    });
}

int neo_attention_shared_int8(const neo_kv_cache* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride, int tokens,
                              int q_heads, int dtype, const int32_t* page_table, int64_t table_stride, const int32_t* context_lens,
                              const int32_t* q_starts, int seqs, const int32_t* group_starts, const int32_t* prefix_lens, int groups,
                              int max_chunk, int max_group, int max_context, int max_own, float scale, int window, void* out,
                              int64_t out_token_stride, int64_t out_head_stride, neo_stream_t stream) {
    return guarded("neo_attention_shared_int8", [&] {
        return shared_attention("neo_attention_shared_int8", cache, q, q_token_stride, q_head_stride, tokens, q_heads, dtype, page_table,
                                table_stride, context_lens, q_starts, seqs, group_starts, prefix_lens, groups, max_chunk, max_group,
                                max_context, max_own, nullptr, scale, window, out, out_token_stride, out_head_stride, stream);
    });
}

int neo_attention_shared_saving_int8(const neo_kv_cache* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                                     int tokens, int q_heads, int dtype, const int32_t* page_table, int64_t table_stride,
                                     const int32_t* context_lens, const int32_t* q_starts, int seqs, const int32_t* group_starts,
                                     const int32_t* prefix_lens, int groups, int max_chunk, int max_group, int max_context,
                                     int max_own, int64_t saved, float scale, int window, void* out, int64_t out_token_stride,
                                     int64_t out_head_stride, neo_stream_t stream) {
    return guarded("neo_attention_shared_saving_int8", [&] {
        return shared_attention("neo_attention_shared_saving_int8", cache, q, q_token_stride, q_head_stride, tokens, q_heads, dtype,
                                page_table, table_stride, context_lens, q_starts, seqs, group_starts, prefix_lens, groups, max_chunk,
                                max_group, max_context, max_own, &saved, scale, window, out, out_token_stride, out_head_stride, stream);
    });
}

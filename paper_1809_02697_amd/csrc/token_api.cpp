// C-ABI entry points of the token operators: argument validation, then the
// launchers.
#include <cmath>
#include <exception>
#include <string>

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

int neo_attention_paged_int8(const neo_kv_cache* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                             int tokens, int q_heads, int dtype, const int32_t* page_table, int64_t table_stride,
                             const int32_t* context_lens, const int32_t* q_starts, int seqs, int max_chunk,
                             int max_context, float scale, int window, void* out, int64_t out_token_stride,
                             int64_t out_head_stride, neo_stream_t stream) {
    return guarded("neo_attention_paged_int8", [&] {
        Check c{"neo_attention_paged_int8"};
        c.type(dtype) && check_cache(c, cache) && c.size(tokens, "tokens", 0) && c.size(q_heads, "q_heads", 1) &&
            c.size(seqs, "seqs", 0) && c.size(max_chunk, "max_chunk", 0) && c.size(max_context, "max_context", 0) &&
            c.size(window, "window", 0);
        if (c.rc == NEO_OK && q_heads % cache->kv_heads) c.bad(NEO_ERR_SHAPE, "q_heads is not a multiple of cache.kv_heads");
        if (c.rc == NEO_OK && !(scale > 0.f && std::isfinite(scale))) c.bad(NEO_ERR_INVALID_ARG, "scale must be finite and > 0");
        if (c.rc != NEO_OK || tokens == 0 || seqs == 0 || max_chunk == 0) return c.rc;
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
        if (c.rc != NEO_OK) return c.rc;
        AttnArgs a{*cache, q, out, q_token_stride, q_head_stride, out_token_stride, out_head_stride, table_stride,
                   page_table, context_lens, q_starts, tokens, q_heads, seqs, std::min(max_chunk, tokens), max_context,
                   window, scale};
        if ((int64_t)a.max_chunk * q_heads > (1 << 28) / seqs)
            return c.bad(NEO_ERR_UNSUPPORTED, "max_chunk * q_heads * seqs above 2^28"), c.rc;
        Workspace ws;
        if (const size_t need = attention_workspace(dtype, a)) {
            const int rc = stream_workspace(c.fn, (hipStream_t)stream, need, &ws);
            if (rc != NEO_OK) return rc;
        }
        return c.launched(launch_attention(dtype, a, ws.ptr, (hipStream_t)stream));
    });
}

// Checks of arguments that the context operators' entry points share.
#pragma once
#include "../../include/w2v_shard.h"

#include <cmath>
#include <cstdlib>

#include "common.h"
#include "context.h"
#include "elem.h"

namespace w2v {

inline int launched() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? W2V_OK : fail(W2V_ERR_HIP, "a launch failed: %s", hipGetErrorString(e));
}

inline bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

inline int check_type(int type) {
    return (unsigned)type < ELEM_TYPES ? W2V_OK : fail(W2V_ERR_ARG, "type %d is none of W2V_T_*", type);
}

constexpr uint64_t ROWS_MAX = 1ull << 40, STRIDE_MAX = 1ull << 40;      // elements; rows times stride stays below 2^64 bytes

inline int check_spec(const w2v_attend_spec* s) {
    if (!s) return fail(W2V_ERR_NULL, "spec is NULL");
    if (int rc = check_type(s->type)) return rc;
    if (s->width == 0 || s->width > W2V_HEAD_MAX) return fail(W2V_ERR_ARG, "width = %u outside 1..%d", s->width, W2V_HEAD_MAX);
    if (s->heads == 0 || s->kv_heads == 0 || s->heads > 1024 || s->heads % s->kv_heads)
        return fail(W2V_ERR_ARG, "%u heads do not share %u", s->heads, s->kv_heads);
    if (s->sinks > W2V_SINKS_MAX) return fail(W2V_ERR_ARG, "sinks = %u above %d", s->sinks, W2V_SINKS_MAX);
    if (!(s->scale > 0.f) || !std::isfinite(s->scale)) return fail(W2V_ERR_ARG, "scale must be finite and positive");
    if (s->bias_dev) {
        if (!s->bucket_dev) return fail(W2V_ERR_NULL, "bucket_dev is NULL");
        if (s->span == 0 || s->span > W2V_SPAN_MAX) return fail(W2V_ERR_ARG, "span = %u outside 1..%d", s->span, W2V_SPAN_MAX);
        if (s->n_buckets == 0 || s->n_buckets > W2V_BUCKETS_MAX)
            return fail(W2V_ERR_ARG, "n_buckets = %u outside 1..%d", s->n_buckets, W2V_BUCKETS_MAX);
    }
    return W2V_OK;
}

inline int check_heads(const w2v_heads* x, const w2v_attend_spec* s, uint32_t heads, uint32_t rows, bool output, const char* name) {
    if (!x || !x->p) return fail(W2V_ERR_NULL, "%s is NULL", name);
    if (!aligned(x->p, elem_bytes(s->type))) return fail(W2V_ERR_ARG, "%s is not aligned to its elements", name);
    if (x->token_stride >= STRIDE_MAX || x->head_stride >= STRIDE_MAX ||
        (rows > 1 && x->token_stride > (1ull << 60) / rows))
        return fail(W2V_ERR_ARG, "%s reaches too far", name);
    if (!output) return W2V_OK;
    // rows of one head, heads of one row: the nearer ones must not touch, nor the farther ones what lies between
    const uint64_t by_row = rows > 1 ? x->token_stride : ~0ull, by_head = heads > 1 ? x->head_stride : ~0ull;
    const uint64_t near = by_row < by_head ? by_row : by_head, far = by_row < by_head ? by_head : by_row;
    const uint64_t count = by_row < by_head ? rows : heads;
    if (near < s->width || (far != ~0ull && far < near * (count - 1) + s->width))
        return fail(W2V_ERR_ARG, "rows of %s overlap", name);
    return W2V_OK;
}

// Whether an output's heads and another array's touch.  Arrays apart from each other are told by their ends; others, as q, k and v of a
// word side by side, have to have one stride from word to word, where a head of one meets a head of the other or does not.
inline int check_apart(const w2v_heads* out, uint32_t out_heads, const char* out_name, const w2v_heads* in, uint32_t in_heads,
                const char* in_name, const w2v_attend_spec* s, uint32_t rows) {
    const uint64_t size = elem_bytes(s->type), a = (uint64_t)(uintptr_t)out->p / size, b = (uint64_t)(uintptr_t)in->p / size;
    const auto reach = [&](const w2v_heads* x, uint32_t heads) {
        return (uint64_t)(rows - 1) * x->token_stride + (uint64_t)(heads - 1) * x->head_stride + s->width;
    };
    if (a + reach(out, out_heads) <= b || b + reach(in, in_heads) <= a) return W2V_OK;
    const int64_t step = rows > 1 ? (int64_t)out->token_stride : 0, width = s->width;
    // words w of the input on either side of an output's head that lies `far` elements on from one of the input's
    const auto touches = [&](int64_t far) {
        const int64_t from = step ? far / step : 0;
        bool meet = false;
        for (int64_t w = from - 1; w <= from + 1; ++w) meet |= std::llabs(far - w * step) < width && std::llabs(w) < (int64_t)rows;
        return meet;
    };
    bool meet = rows > 1 && out->token_stride != in->token_stride;
    if (out->head_stride == in->head_stride) {        // what counts is how many heads apart two are
        for (int64_t d = 1 - (int64_t)in_heads; d < (int64_t)out_heads && !meet; ++d)
            meet = touches((int64_t)(a - b) + d * (int64_t)out->head_stride);
    } else {
        for (uint32_t h = 0; h < out_heads && !meet; ++h)
            for (uint32_t g = 0; g < in_heads && !meet; ++g)
                meet = touches((int64_t)(a + h * out->head_stride) - (int64_t)(b + g * in->head_stride));
    }
    return meet ? fail(W2V_ERR_ARG, "%s overlaps %s", out_name, in_name) : W2V_OK;
}

inline Heads heads_of(const w2v_heads* x) { return Heads{x->p, x->token_stride, x->head_stride}; }
inline HeadsOut heads_out(const w2v_heads* x) { return HeadsOut{x->p, x->token_stride, x->head_stride}; }

}  // namespace w2v

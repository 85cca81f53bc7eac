// C ABI of the context operators: argument checks and the order in which their kernels are queued.  They belong to no
// shard and keep nothing between calls.  See include/w2v_shard.h for the contract of every entry point.
#include "../../include/w2v_shard.h"

#include <cmath>
#include <cstdlib>

#include "common.h"
#include "context.h"
#include "elem.h"

using namespace w2v;
static_assert(W2V_HEAD_MAX == HEAD_MAX && W2V_SINKS_MAX == SINKS_MAX && W2V_SPAN_MAX == SPAN_MAX, "limits");
static_assert(W2V_T_F32 == ELEM_F32 && W2V_T_F16 == ELEM_F16 && W2V_T_BF16 == ELEM_BF16, "element types");

namespace {

int launched() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? W2V_OK : fail(W2V_ERR_HIP, "a launch failed: %s", hipGetErrorString(e));
}

bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

int check_type(int type) {
    return (unsigned)type < ELEM_TYPES ? W2V_OK : fail(W2V_ERR_ARG, "type %d is none of W2V_T_*", type);
}

constexpr uint64_t ROWS_MAX = 1ull << 40, STRIDE_MAX = 1ull << 40;      // elements; rows times stride stays below 2^64 bytes

int check_norm(int type, uint64_t rows, uint32_t d) {
    if (int rc = check_type(type)) return rc;
    if (d == 0 || d > W2V_NORM_D_MAX) return fail(W2V_ERR_ARG, "d = %u outside 1..%d", d, W2V_NORM_D_MAX);
    if (rows >= ROWS_MAX) return fail(W2V_ERR_ARG, "too many rows");
    return W2V_OK;
}
int check_rows(const void* p, uint64_t stride, uint64_t least, uint64_t rows, int type, const char* name) {
    if (!p) return fail(W2V_ERR_NULL, "%s is NULL", name);
    if (!aligned(p, elem_bytes(type))) return fail(W2V_ERR_ARG, "%s is not aligned to its elements", name);
    if (rows > 1 && stride < least) return fail(W2V_ERR_ARG, "rows of %s overlap", name);
    if (rows > 1 && (stride >= STRIDE_MAX || rows > (1ull << 60) / (stride ? stride : 1)))
        return fail(W2V_ERR_ARG, "%s reaches too far", name);
    return W2V_OK;
}

}  // namespace

extern "C" int w2v_layer_norm(int type, const void* x, uint64_t x_stride, uint64_t rows, uint32_t d, const float* gain,
                              const float* offset, float eps, void* y, uint64_t y_stride, float* mean, float* rstd,
                              void* stream) {
    if (int rc = check_norm(type, rows, d)) return rc;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(W2V_ERR_ARG, "eps must be finite and not negative");
    if (rows == 0) return W2V_OK;
    if (int rc = check_rows(x, x_stride, 0, rows, type, "x")) return rc;
    if (int rc = check_rows(y, y_stride, d, rows, type, "y")) return rc;
    if (x == y && rows > 1 && x_stride != y_stride) return fail(W2V_ERR_ARG, "y is x, but its rows lie elsewhere");
    launch_norm(NormArgs{x, x_stride, rows, d, eps, gain, offset, y, y_stride, mean, rstd}, (uint32_t)type,
                (hipStream_t)stream);
    return launched();
}

extern "C" size_t w2v_layer_norm_backward_workspace(int type, uint64_t rows, uint32_t d) {
    if ((unsigned)type >= ELEM_TYPES || rows >= ROWS_MAX || d == 0 || d > W2V_NORM_D_MAX) return 0;
    return (size_t)norm_backward_parts(rows, d, (uint32_t)type) * 2 * d * sizeof(float);
}

extern "C" int w2v_layer_norm_backward(int type, const void* dy, uint64_t dy_stride, const void* x, uint64_t x_stride,
                                       uint64_t rows, uint32_t d, const float* gain, const float* mean,
                                       const float* rstd, void* dx, uint64_t dx_stride, float* dgain, float* doffset,
                                       void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_norm(type, rows, d)) return rc;
    const bool columns = dgain || doffset;
    if (rows) {
        if (int rc = check_rows(dy, dy_stride, 0, rows, type, "dy")) return rc;
        if (int rc = check_rows(x, x_stride, 0, rows, type, "x")) return rc;
        if (int rc = check_rows(dx, dx_stride, d, rows, type, "dx")) return rc;
        if (!mean || !rstd) return fail(W2V_ERR_NULL, "the rows' statistics are NULL");
        if (rows > 1 && ((dx == x && dx_stride != x_stride) || (dx == dy && dx_stride != dy_stride)))
            return fail(W2V_ERR_ARG, "dx is an input, but its rows lie elsewhere");
        if (columns) {
            const size_t need = w2v_layer_norm_backward_workspace(type, rows, d);
            if (!workspace) return fail(W2V_ERR_NULL, "workspace is NULL");
            if (!aligned(workspace, 256)) return fail(W2V_ERR_ARG, "workspace must be 256-byte aligned");
            if (workspace_bytes < need)
                return fail(W2V_ERR_ARG, "workspace of %zu bytes is too small: %zu are needed", workspace_bytes, need);
        }
    }
    if (!rows && !columns) return W2V_OK;
    launch_norm_backward(NormBackwardArgs{dy, dy_stride, x, x_stride, rows, d, gain, mean, rstd, dx, dx_stride,
                                          columns ? (float*)workspace : nullptr},
                         (uint32_t)type, dgain, doffset, (hipStream_t)stream);
    return launched();
}

// ---------------------------------------------------------------------------------------------
// attention over texts
// ---------------------------------------------------------------------------------------------
namespace {

int check_spec(const w2v_attend_spec* s) {
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

int check_tokens(const w2v_attend_spec* s, const uint64_t* off, uint32_t n_sent, uint32_t n_tokens) {
    if (n_tokens > 0x7FFFFFFFu - 4095u || (uint64_t)n_tokens * s->heads > 1ull << 29)      // (threads of a launch: below 2^32)
        return fail(W2V_ERR_ARG, "too many tokens; pass the texts in blocks");
    if (n_tokens && n_sent == 0) return fail(W2V_ERR_ARG, "tokens without texts");
    if (n_sent > 0x7FFFFFFFu) return fail(W2V_ERR_ARG, "too many texts");
    if (n_tokens && !off) return fail(W2V_ERR_NULL, "sent_off_dev is NULL");
    return W2V_OK;
}

int check_heads(const w2v_heads* x, const w2v_attend_spec* s, uint32_t heads, uint32_t rows, bool output, const char* name) {
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
int check_apart(const w2v_heads* out, uint32_t out_heads, const char* out_name, const w2v_heads* in, uint32_t in_heads,
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

Heads heads_of(const w2v_heads* x) { return Heads{x->p, x->token_stride, x->head_stride}; }
HeadsOut heads_out(const w2v_heads* x) { return HeadsOut{x->p, x->token_stride, x->head_stride}; }

AttendArgs attend_args(const w2v_attend_spec* s, const w2v_heads* q, const w2v_heads* k, const w2v_heads* v,
                       const uint64_t* off, uint32_t n_sent, uint32_t T, const uint8_t* keep, const w2v_heads* out,
                       float* lse) {
    AttendArgs a;
    a.q = heads_of(q); a.k = heads_of(k); a.v = heads_of(v);
    a.off = off; a.n_sent = n_sent; a.T = T;
    a.heads = s->heads; a.kv_heads = s->kv_heads; a.group = s->heads / s->kv_heads; a.width = s->width;
    a.left = s->left < T ? s->left : T; a.right = s->right < T ? s->right : T;
    a.sinks = s->sinks; a.skip_self = s->skip_self != 0;
    a.scale = s->scale; a.scale2 = s->scale * 1.4426950408889634f;
    a.keep = keep;
    a.bias = s->bias_dev; a.buckets = s->bucket_dev; a.n_buckets = s->n_buckets; a.span = s->span;
    a.o = heads_out(out); a.lse = lse;
    return a;
}

}  // namespace

extern "C" int w2v_relative_buckets(uint32_t n_buckets, uint32_t span, uint32_t* map) {
    if (!map) return fail(W2V_ERR_NULL, "map is NULL");
    if (n_buckets < 2 || n_buckets > W2V_BUCKETS_MAX)
        return fail(W2V_ERR_ARG, "n_buckets = %u outside 2..%d", n_buckets, W2V_BUCKETS_MAX);
    if (span == 0 || span > W2V_SPAN_MAX) return fail(W2V_ERR_ARG, "span = %u outside 1..%d", span, W2V_SPAN_MAX);
    const uint32_t half = n_buckets / 2, near = half / 2 ? half / 2 : 1, far = half - near;
    uint32_t t = 0;                           // distances near (span / near)^(t / far) are where bucket near + t begins
    for (uint32_t r = 0; r <= span; ++r) {
        uint32_t b = r < half - 1 ? r : half - 1;
        if (r >= near && far) {
            // a distance that meets a border in exact arithmetic is past it.  Of all maps within the limits, the one whose
            // distance comes nearest to a border without meeting it is 42 buckets over 1006 (435: 5.03e-11 past it); the logarithms'
            // rounding is below 1e-12
            while (t + 1 < far && far * std::log((double)r / near) >= (t + 1) * std::log((double)span / near) - 1e-11) ++t;
            b = near + t;
        }
        map[span - r] = b;
        if (r) map[span + r] = half + b;
    }
    return W2V_OK;
}

extern "C" int w2v_attend(const w2v_attend_spec* spec, const w2v_heads* q, const w2v_heads* k, const w2v_heads* v,
                          const uint64_t* sent_off, uint32_t n_sent, uint32_t n_tokens, const uint8_t* keep,
                          const w2v_heads* out, float* lse, void* stream) {
    if (int rc = check_spec(spec)) return rc;
    if (int rc = check_tokens(spec, sent_off, n_sent, n_tokens)) return rc;
    if (n_tokens == 0) return W2V_OK;
    if (int rc = check_heads(q, spec, spec->heads, n_tokens, false, "q")) return rc;
    if (int rc = check_heads(k, spec, spec->kv_heads, n_tokens, false, "k")) return rc;
    if (int rc = check_heads(v, spec, spec->kv_heads, n_tokens, false, "v")) return rc;
    if (int rc = check_heads(out, spec, spec->heads, n_tokens, true, "out")) return rc;
    if (int rc = check_apart(out, spec->heads, "out", q, spec->heads, "q", spec, n_tokens)) return rc;
    if (int rc = check_apart(out, spec->heads, "out", k, spec->kv_heads, "k", spec, n_tokens)) return rc;
    if (int rc = check_apart(out, spec->heads, "out", v, spec->kv_heads, "v", spec, n_tokens)) return rc;
    launch_attend(attend_args(spec, q, k, v, sent_off, n_sent, n_tokens, keep, out, lse), (uint32_t)spec->type,
                  (hipStream_t)stream);
    return launched();
}

namespace {
// The parts of the backward pass's workspace, each from a 256-byte border on.
struct BackwardSpace {
    size_t high, low, delta, by_distance, distance_sums, late_sums, own_sums, bytes;
    BackwardSpace(const w2v_attend_spec* s, uint32_t T) {
        size_t at = 0;
        const auto part = [&](size_t count) {
            const size_t from = at;
            at += (count * sizeof(float) + 255) / 256 * 256;
            return from;
        };
        high = part((size_t)s->heads * T);
        low = part((size_t)s->heads * T);
        delta = part((size_t)s->heads * T);
        by_distance = part(s->bias_dev ? (size_t)s->heads * attend_bias_parts(T) * (2 * s->span + 1) : 0);
        distance_sums = part(s->bias_dev ? (size_t)s->heads * (2 * s->span + 1) : 0);
        const size_t late = (size_t)attend_late_pieces(T, s->left < T ? s->left : T, s->sinks).count * s->kv_heads * s->sinks * 2 * s->width;
        late_sums = part(late);
        own_sums = part(late);
        bytes = at;
    }
};
}  // namespace

extern "C" size_t w2v_attend_backward_workspace(const w2v_attend_spec* spec, uint32_t n_tokens) {
    if (check_spec(spec) || n_tokens > 0x7FFFFFFFu - 4095u) return 0;
    return BackwardSpace(spec, n_tokens).bytes;
}

extern "C" int w2v_attend_backward(const w2v_attend_spec* spec, const w2v_heads* dout, const w2v_heads* q, const w2v_heads* k,
                                   const w2v_heads* v, const w2v_heads* out, const float* lse, const uint64_t* sent_off,
                                   uint32_t n_sent, uint32_t n_tokens, const uint8_t* keep, const w2v_heads* dq,
                                   const w2v_heads* dk, const w2v_heads* dv, float* dbias, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    if (int rc = check_spec(spec)) return rc;
    if (int rc = check_tokens(spec, sent_off, n_sent, n_tokens)) return rc;
    if (dbias && !spec->bias_dev) return fail(W2V_ERR_ARG, "the gradient of a bias that was not given");
    BackwardArgs b{};
    if (n_tokens) {
        const w2v_heads* of_query[] = {dout, q, out};
        const w2v_heads* of_key[] = {k, v};
        const char* names[] = {"dout", "q", "out", "k", "v"};
        for (int n = 0; n < 3; ++n)
            if (int rc = check_heads(of_query[n], spec, spec->heads, n_tokens, false, names[n])) return rc;
        for (int n = 0; n < 2; ++n)
            if (int rc = check_heads(of_key[n], spec, spec->kv_heads, n_tokens, false, names[3 + n])) return rc;
        if (int rc = check_heads(dq, spec, spec->heads, n_tokens, true, "dq")) return rc;
        if (int rc = check_heads(dk, spec, spec->kv_heads, n_tokens, true, "dk")) return rc;
        if (int rc = check_heads(dv, spec, spec->kv_heads, n_tokens, true, "dv")) return rc;
        if (!lse) return fail(W2V_ERR_NULL, "lse_dev is NULL");
        const BackwardSpace space(spec, n_tokens);
        if (!workspace) return fail(W2V_ERR_NULL, "workspace is NULL");
        if (!aligned(workspace, 256)) return fail(W2V_ERR_ARG, "workspace must be 256-byte aligned");
        if (workspace_bytes < space.bytes)
            return fail(W2V_ERR_ARG, "workspace of %zu bytes is too small: %zu are needed", workspace_bytes, space.bytes);
        struct { const w2v_heads* x; uint32_t heads; const char* name; } arrays[] = {
            {dq, spec->heads, "dq"}, {dk, spec->kv_heads, "dk"}, {dv, spec->kv_heads, "dv"}, {dout, spec->heads, "dout"},
            {q, spec->heads, "q"}, {k, spec->kv_heads, "k"}, {v, spec->kv_heads, "v"}, {out, spec->heads, "out"}};
        for (int n = 0; n < 3; ++n)
            for (int m = n + 1; m < 8; ++m)
                if (int rc = check_apart(arrays[n].x, arrays[n].heads, arrays[n].name, arrays[m].x, arrays[m].heads,
                                         arrays[m].name, spec, n_tokens)) return rc;
        b.a = attend_args(spec, q, k, v, sent_off, n_sent, n_tokens, keep, out, const_cast<float*>(lse));
        b.dout = heads_of(dout);
        b.dq = heads_out(dq); b.dk = heads_out(dk); b.dv = heads_out(dv);
        b.high = (float*)((char*)workspace + space.high);
        b.low = (float*)((char*)workspace + space.low);
        b.delta = (float*)((char*)workspace + space.delta);
        b.by_distance = (float*)((char*)workspace + space.by_distance);
        b.distance_sums = (float*)((char*)workspace + space.distance_sums);
        const LatePieces late = attend_late_pieces(n_tokens, b.a.left, b.a.sinks);
        b.late = late.count; b.late_words = late.words; b.reach = late.reach;
        b.late_sums = (float*)((char*)workspace + space.late_sums);
        b.own_sums = (float*)((char*)workspace + space.own_sums);
    } else if (dbias) {
        b.a.heads = spec->heads; b.a.buckets = spec->bucket_dev; b.a.n_buckets = spec->n_buckets; b.a.span = spec->span;
    } else {
        return W2V_OK;
    }
    b.dbias = dbias;
    launch_attend_backward(b, (uint32_t)spec->type, (hipStream_t)stream);
    return launched();
}

namespace {

int check_step(const w2v_attend_spec* s, uint32_t batch, uint32_t room) {
    if (int rc = check_spec(s)) return rc;
    if (room == 0 || room > 0x7FFFFFFFu - 4095u) return fail(W2V_ERR_ARG, "room = %u outside 1..2^31 - 2^12", room);
    if ((uint64_t)batch * s->heads > 1u << 23) return fail(W2V_ERR_ARG, "too many texts at once");
    return W2V_OK;
}

int check_cache(const w2v_cache* x, const w2v_attend_spec* s, uint32_t batch, uint32_t room, const char* name) {
    if (!x || !x->p) return fail(W2V_ERR_NULL, "%s is NULL", name);
    if (!aligned(x->p, elem_bytes(s->type))) return fail(W2V_ERR_ARG, "%s is not aligned to its elements", name);
    if (x->text_stride >= STRIDE_MAX || x->token_stride >= STRIDE_MAX || x->head_stride >= STRIDE_MAX ||
        x->token_stride > (1ull << 59) / room || x->text_stride > (1ull << 59) / batch)
        return fail(W2V_ERR_ARG, "%s reaches too far", name);
    return W2V_OK;
}

// The workspace: partial results where a cache is read by several blocks.
size_t step_bytes(const w2v_attend_spec* s, uint32_t batch, const StepSplits& p) {
    return p.splits > 1 ? (size_t)batch * s->heads * p.splits * (s->width + 2) * sizeof(float) : 0;
}

}  // namespace

extern "C" size_t w2v_attend_step_workspace(const w2v_attend_spec* spec, uint32_t batch, uint32_t room) {
    if (batch == 0 || check_step(spec, batch, room)) return 0;
    return step_bytes(spec, batch, step_splits(batch, spec->kv_heads, room, spec->left, spec->sinks));
}

extern "C" int w2v_attend_step(const w2v_attend_spec* spec, const w2v_heads* q, const w2v_cache* k, const w2v_cache* v,
                               const uint32_t* n, uint32_t batch, uint32_t room, const uint8_t* keep, const w2v_heads* out,
                               void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_spec(spec)) return rc;
    if (batch == 0) return W2V_OK;
    if (int rc = check_step(spec, batch, room)) return rc;
    if (int rc = check_heads(q, spec, spec->heads, batch, false, "q")) return rc;
    if (int rc = check_cache(k, spec, batch, room, "k")) return rc;
    if (int rc = check_cache(v, spec, batch, room, "v")) return rc;
    if (int rc = check_heads(out, spec, spec->heads, batch, true, "out")) return rc;
    if (!n) return fail(W2V_ERR_NULL, "n_dev is NULL");
    const StepSplits p = step_splits(batch, spec->kv_heads, room, spec->left, spec->sinks);
    const size_t need = step_bytes(spec, batch, p);
    if (need) {
        if (!workspace) return fail(W2V_ERR_NULL, "workspace is NULL");
        if (!aligned(workspace, 256)) return fail(W2V_ERR_ARG, "workspace must be 256-byte aligned");
        if (workspace_bytes < need)
            return fail(W2V_ERR_ARG, "workspace of %zu bytes is too small: %zu are needed", workspace_bytes, need);
    }
    StepArgs a;
    a.q = heads_of(q); a.o = heads_out(out);
    a.k = Cache{k->p, k->text_stride, k->token_stride, k->head_stride};
    a.v = Cache{v->p, v->text_stride, v->token_stride, v->head_stride};
    a.n = n; a.batch = batch; a.room = room;
    a.heads = spec->heads; a.kv_heads = spec->kv_heads; a.group = spec->heads / spec->kv_heads; a.width = spec->width;
    a.left = spec->left; a.sinks = spec->sinks; a.skip_self = spec->skip_self != 0;
    a.scale2 = spec->scale * 1.4426950408889634f;
    a.keep = keep;
    a.bias = spec->bias_dev; a.buckets = spec->bucket_dev; a.n_buckets = spec->n_buckets; a.span = spec->span;
    a.splits = p.splits; a.per_split = p.per_split; a.parts = (float*)workspace;
    launch_step(a, (uint32_t)spec->type, (hipStream_t)stream);
    return launched();
}

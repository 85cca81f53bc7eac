// C ABI of the context operators: argument checks and the order in which their kernels are queued.  They belong to no
// shard and keep nothing between calls.  See include/w2v_shard.h for the contract of every entry point.
#include "checks.h"

using namespace w2v;
static_assert(W2V_HEAD_MAX == HEAD_MAX && W2V_SINKS_MAX == SINKS_MAX && W2V_SPAN_MAX == SPAN_MAX, "limits");
static_assert(W2V_T_F32 == ELEM_F32 && W2V_T_F16 == ELEM_F16 && W2V_T_BF16 == ELEM_BF16, "element types");

namespace {

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

int check_tokens(const w2v_attend_spec* s, const uint64_t* off, uint32_t n_sent, uint32_t n_tokens) {
    if (n_tokens > 0x7FFFFFFFu - 4095u || (uint64_t)n_tokens * s->heads > 1ull << 29)      // (threads of a launch: below 2^32)
        return fail(W2V_ERR_ARG, "too many tokens; pass the texts in blocks");
    if (n_tokens && n_sent == 0) return fail(W2V_ERR_ARG, "tokens without texts");
    if (n_sent > 0x7FFFFFFFu) return fail(W2V_ERR_ARG, "too many texts");
    if (n_tokens && !off) return fail(W2V_ERR_NULL, "sent_off_dev is NULL");
    return W2V_OK;
}

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
    StepArgs a{};
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

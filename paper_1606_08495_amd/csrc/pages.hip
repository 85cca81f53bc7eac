// C ABI of positions that turn and of the cache in pages: argument checks and the order in which their kernels are queued.  They
// belong to no shard and keep nothing between calls.  See include/w2v_shard.h for the contract of every entry point.
#include "checks.h"

#include <initializer_list>

using namespace w2v;

namespace {

// ---- arrays of three axes -------------------------------------------------------------------------------
// Rows of `width` elements at the sums of multiples of three strides: pages, tokens, heads.
struct Lattice {
    uint64_t p, width, stride[3], count[3];           // p in elements
    uint64_t reach() const {
        uint64_t r = width;
        for (int n = 0; n < 3; ++n) r += (count[n] - 1) * stride[n];
        return r;
    }
};
// Axes of two arrays (or of one, with itself), the larger strides first.  An axis of one entry has no stride that counts.
struct Axis2 { uint64_t stride, a, b; };
bool axes_of(const Lattice& a, const Lattice& b, Axis2 (&axes)[3], int& used) {
    used = 0;
    for (int n = 0; n < 3; ++n) {
        if (a.count[n] <= 1 && b.count[n] <= 1) continue;
        if (a.count[n] > 1 && b.count[n] > 1 && a.stride[n] != b.stride[n]) return false;
        const Axis2 x{a.count[n] > 1 ? a.stride[n] : b.stride[n], a.count[n], b.count[n]};
        int at = used++;
        for (; at > 0 && axes[at - 1].stride < x.stride; --at) axes[at] = axes[at - 1];
        axes[at] = x;
    }
    // each stride leads past all that the smaller ones reach
    uint64_t reach = a.width;
    for (int n = used - 1; n >= 0; --n) {
        if (axes[n].stride < reach) return false;
        reach += ((axes[n].a > axes[n].b ? axes[n].a : axes[n].b) - 1) * axes[n].stride;
    }
    return true;
}
// Whether a row of one meets a row of the other: rows `far` elements apart, brought nearer by multiples of each stride, of
// which only those next to the quotient can bring them near enough.
bool rows_meet(const Axis2* axes, int used, uint64_t width, int64_t far) {
    if (used == 0) return std::llabs(far) < (int64_t)width;
    const int64_t step = (int64_t)axes->stride, from = far / step;
    for (int64_t m = from - 1; m <= from + 1; ++m)
        if (m > -(int64_t)axes->b && m < (int64_t)axes->a && rows_meet(axes + 1, used - 1, width, far - m * step)) return true;
    return false;
}
// Whether an output and another array touch.  Where they lie among each other they have to have the same strides.
bool touch(const Lattice& a, const Lattice& b) {
    if (a.p + a.reach() <= b.p || b.p + b.reach() <= a.p) return false;
    Axis2 axes[3];
    int used;
    return !axes_of(a, b, axes, used) || rows_meet(axes, used, a.width, (int64_t)(b.p - a.p));
}
bool apart_from_itself(const Lattice& l) {
    Axis2 axes[3];
    int used;
    return axes_of(l, l, axes, used);
}

Lattice lattice_of(const w2v_heads* x, const w2v_attend_spec* s, uint32_t heads, uint32_t rows) {
    return Lattice{(uint64_t)(uintptr_t)x->p / elem_bytes(s->type), s->width, {0, x->token_stride, x->head_stride}, {1, rows, heads}};
}
Lattice lattice_of(const w2v_pages* x, const w2v_attend_spec* s, const w2v_page_table* t) {
    return Lattice{(uint64_t)(uintptr_t)x->p / elem_bytes(s->type), s->width, {x->page_stride, x->token_stride, x->head_stride},
                   {t->n_pages, t->page_words, s->kv_heads}};
}

// ---- checks -----------------------------------------------------------------------------------------------
int check_rotary(const w2v_rotary* r, uint32_t width) {
    if (!r) return fail(W2V_ERR_NULL, "rotary is NULL");
    if (!r->turns_dev) return fail(W2V_ERR_NULL, "turns_dev is NULL");
    if (!aligned(r->turns_dev, 8)) return fail(W2V_ERR_ARG, "turns_dev is not aligned to its elements");
    if (r->rotated < 2 || r->rotated % 2 || r->rotated > width)
        return fail(W2V_ERR_ARG, "rotated = %u is not even and 2..%u", r->rotated, width);
    if (!std::isfinite(r->gain)) return fail(W2V_ERR_ARG, "gain must be finite");
    return W2V_OK;
}

// The type, width and heads of a call that has no w2v_attend_spec, for the checks that want one.
int check_shape(int type, uint32_t width, uint32_t heads, uint32_t kv_heads, uint32_t tokens, w2v_attend_spec* s) {
    if (int rc = check_type(type)) return rc;
    if (width == 0 || width > W2V_HEAD_MAX) return fail(W2V_ERR_ARG, "width = %u outside 1..%d", width, W2V_HEAD_MAX);
    if (heads > 1024 || kv_heads > 1024) return fail(W2V_ERR_ARG, "more than 1024 heads");
    if (tokens > 0x7FFFFFFFu - 4095u) return fail(W2V_ERR_ARG, "too many tokens; pass the texts in blocks");
    *s = w2v_attend_spec{};
    s->type = type;
    s->width = width;
    s->heads = heads;
    s->kv_heads = kv_heads;
    return W2V_OK;
}

int check_offsets(const uint64_t* off, uint32_t n_sent) {
    if (!off) return fail(W2V_ERR_NULL, "sent_off_dev is NULL");
    if (n_sent == 0) return fail(W2V_ERR_ARG, "tokens without texts");
    if (n_sent > 0x7FFFFFFFu) return fail(W2V_ERR_ARG, "too many texts");
    return W2V_OK;
}

int check_table(const w2v_page_table* t) {
    if (!t) return fail(W2V_ERR_NULL, "table is NULL");
    if (!t->page_dev) return fail(W2V_ERR_NULL, "page_dev is NULL");
    if (!aligned(t->page_dev, 4)) return fail(W2V_ERR_ARG, "page_dev is not aligned to its elements");
    if (t->page_words == 0 || t->page_words > W2V_PAGE_WORDS_MAX || (t->page_words & (t->page_words - 1)))
        return fail(W2V_ERR_ARG, "page_words = %u is no power of two up to %d", t->page_words, W2V_PAGE_WORDS_MAX);
    if (t->slots == 0 || (uint64_t)t->slots * t->page_words > 0x7FFFFFFFu - 4095u)
        return fail(W2V_ERR_ARG, "slots * page_words outside 1..2^31 - 2^12");
    if (t->n_pages == 0) return fail(W2V_ERR_ARG, "a pool of no pages");
    if (t->stride >= STRIDE_MAX) return fail(W2V_ERR_ARG, "the table reaches too far");
    return W2V_OK;
}
uint32_t shift_of(const w2v_page_table* t) { return (uint32_t)__builtin_ctz(t->page_words); }

int check_pages(const w2v_pages* x, const w2v_attend_spec* s, const w2v_page_table* t, const char* name) {
    if (!x || !x->p) return fail(W2V_ERR_NULL, "%s is NULL", name);
    if (!aligned(x->p, elem_bytes(s->type))) return fail(W2V_ERR_ARG, "%s is not aligned to its elements", name);
    if (x->page_stride >= STRIDE_MAX || x->token_stride >= STRIDE_MAX || x->head_stride >= STRIDE_MAX ||
        x->page_stride > (1ull << 59) / t->n_pages)
        return fail(W2V_ERR_ARG, "%s reaches too far", name);
    return W2V_OK;
}

// Outputs against everything else that a call reads or writes.
struct Span { Lattice l; const char* name; bool output; };
int check_spans(std::initializer_list<Span> spans) {
    for (auto a = spans.begin(); a != spans.end(); ++a)
        for (auto b = spans.begin(); b != spans.end(); ++b) {
            if (a == b || !a->output || (b->output && b < a)) continue;
            if (touch(a->l, b->l)) return fail(W2V_ERR_ARG, "%s overlaps %s", a->name, b->name);
        }
    return W2V_OK;
}

TurnArray turn_array(const w2v_heads* in, void* out, uint64_t out_token, uint64_t out_head, uint32_t heads) {
    return TurnArray{heads_of(in), out, out_token, out_head, heads};
}
bool same(const w2v_heads* a, const w2v_heads* b, uint32_t heads, uint32_t rows) {
    return a->p == b->p && (rows <= 1 || a->token_stride == b->token_stride) && (heads <= 1 || a->head_stride == b->head_stride);
}

}  // namespace

extern "C" int w2v_rotary_turns(uint32_t rotated, double base, int scaling, double factor, uint32_t trained, double low,
                                double high, uint64_t* turns) {
    if (!turns) return fail(W2V_ERR_NULL, "turns is NULL");
    if (rotated < 2 || rotated % 2 || rotated > W2V_HEAD_MAX)
        return fail(W2V_ERR_ARG, "rotated = %u is not even and 2..%d", rotated, W2V_HEAD_MAX);
    if (!(base > 1) || !std::isfinite(base)) return fail(W2V_ERR_ARG, "base must be finite and above 1");
    if (scaling < W2V_ROTARY_PLAIN || scaling > W2V_ROTARY_PARTS) return fail(W2V_ERR_ARG, "scaling %d is none of W2V_ROTARY_*", scaling);
    if (scaling != W2V_ROTARY_PLAIN && (!(factor >= 1) || !std::isfinite(factor)))
        return fail(W2V_ERR_ARG, "factor must be finite and at least 1");
    if (scaling == W2V_ROTARY_PARTS && (!(low >= 0) || !(high > low) || !std::isfinite(high) || trained == 0))
        return fail(W2V_ERR_ARG, "trained must be positive, and 0 <= low < high");
    constexpr long double TAU = 6.283185307179586476925286766559L;
    for (uint32_t c = 0; c < rotated / 2; ++c) {
        long double f = std::pow((long double)base, -2.0L * c / rotated);
        if (scaling == W2V_ROTARY_LINEAR) f /= factor;
        if (scaling == W2V_ROTARY_BASE && c) f *= std::pow((long double)factor, -2.0L * c / (rotated - 2));
        if (scaling == W2V_ROTARY_PARTS) {
            const long double t = trained * f / TAU, w = (t - low) / ((long double)high - low);
            const long double held = w < 0 ? 0 : w > 1 ? 1 : w;
            f *= held + (1 - held) / factor;
        }
        turns[c] = (uint64_t)(f / TAU * 18446744073709551616.0L + 0.5L);
    }
    return W2V_OK;
}

extern "C" int w2v_rotate(int type, uint32_t width, const w2v_rotary* rotary, int back, const w2v_heads* x, uint32_t heads,
                          const w2v_heads* y, uint32_t y_heads, const uint64_t* sent_off, uint32_t n_sent, uint32_t n_tokens,
                          const int32_t* position, const w2v_heads* x_out, const w2v_heads* y_out, void* stream) {
    w2v_attend_spec s;
    if (int rc = check_shape(type, width, heads, y ? y_heads : 0, n_tokens, &s)) return rc;
    if (int rc = check_rotary(rotary, width)) return rc;
    if (heads == 0 || (y && y_heads == 0)) return fail(W2V_ERR_ARG, "no heads");
    if (n_tokens == 0) return W2V_OK;
    if (!position)
        if (int rc = check_offsets(sent_off, n_sent)) return rc;
    if (int rc = check_heads(x, &s, heads, n_tokens, false, "x")) return rc;
    if (int rc = check_heads(x_out, &s, heads, n_tokens, true, "x_out")) return rc;
    const Lattice in = lattice_of(x, &s, heads, n_tokens), out = lattice_of(x_out, &s, heads, n_tokens);
    if (!same(x, x_out, heads, n_tokens) && touch(out, in)) return fail(W2V_ERR_ARG, "x_out overlaps x");
    TurnArgs a{};
    a.x = turn_array(x, x_out->p, x_out->token_stride, x_out->head_stride, heads);
    if (y) {
        if (int rc = check_heads(y, &s, y_heads, n_tokens, false, "y")) return rc;
        if (int rc = check_heads(y_out, &s, y_heads, n_tokens, true, "y_out")) return rc;
        const Lattice y_in = lattice_of(y, &s, y_heads, n_tokens), y_to = lattice_of(y_out, &s, y_heads, n_tokens);
        if (!same(y, y_out, y_heads, n_tokens) && touch(y_to, y_in)) return fail(W2V_ERR_ARG, "y_out overlaps y");
        if (touch(out, y_in) || touch(y_to, in) || touch(out, y_to)) return fail(W2V_ERR_ARG, "x_out and y_out overlap, or each other's input");
        a.y = turn_array(y, y_out->p, y_out->token_stride, y_out->head_stride, y_heads);
    }
    a.width = width; a.rotated = rotary->rotated; a.halves = rotary->halves != 0; a.back = back != 0; a.gain = rotary->gain;
    a.turns = rotary->turns_dev;
    a.off = position ? nullptr : sent_off; a.n_sent = n_sent; a.T = n_tokens; a.position = position;
    launch_rotate(a, (uint32_t)type, (hipStream_t)stream);
    return launched();
}

extern "C" int w2v_pages_append(int type, uint32_t width, const w2v_rotary* rotary, const w2v_heads* k, const w2v_heads* v,
                                uint32_t kv_heads, const w2v_heads* q, uint32_t heads, const w2v_heads* q_out,
                                const uint64_t* sent_off, uint32_t n_sent, uint32_t n_tokens, const uint32_t* n,
                                const int32_t* position, const w2v_page_table* table, const w2v_pages* k_pages,
                                const w2v_pages* v_pages, void* stream) {
    w2v_attend_spec s;
    if (int rc = check_shape(type, width, q ? heads : 0, kv_heads, n_tokens, &s)) return rc;
    if (kv_heads == 0 || (q && heads == 0)) return fail(W2V_ERR_ARG, "no heads");
    if (rotary)
        if (int rc = check_rotary(rotary, width)) return rc;
    if (q && !rotary) return fail(W2V_ERR_ARG, "q is given, but nothing to turn it by");
    if (n_tokens == 0) return W2V_OK;
    if (sent_off) {
        if (int rc = check_offsets(sent_off, n_sent)) return rc;
    } else if (n_sent != n_tokens) {
        return fail(W2V_ERR_ARG, "one word each of %u texts are not %u words", n_sent, n_tokens);
    }
    if (!n) return fail(W2V_ERR_NULL, "n_dev is NULL");
    if (int rc = check_table(table)) return rc;
    if (int rc = check_heads(k, &s, kv_heads, n_tokens, false, "k")) return rc;
    if (int rc = check_heads(v, &s, kv_heads, n_tokens, false, "v")) return rc;
    if (int rc = check_pages(k_pages, &s, table, "k_pages")) return rc;
    if (int rc = check_pages(v_pages, &s, table, "v_pages")) return rc;
    const Lattice k_in = lattice_of(k, &s, kv_heads, n_tokens), v_in = lattice_of(v, &s, kv_heads, n_tokens);
    const Lattice k_to = lattice_of(k_pages, &s, table), v_to = lattice_of(v_pages, &s, table);
    if (!apart_from_itself(k_to) || !apart_from_itself(v_to)) return fail(W2V_ERR_ARG, "places of a pool overlap");
    if (int rc = check_spans({{k_to, "k_pages", true}, {v_to, "v_pages", true}, {k_in, "k", false}, {v_in, "v", false}})) return rc;
    TurnArgs a{};
    if (q) {
        if (int rc = check_heads(q, &s, heads, n_tokens, false, "q")) return rc;
        if (int rc = check_heads(q_out, &s, heads, n_tokens, true, "q_out")) return rc;
        const Lattice in = lattice_of(q, &s, heads, n_tokens), out = lattice_of(q_out, &s, heads, n_tokens);
        if (!same(q, q_out, heads, n_tokens) && touch(out, in)) return fail(W2V_ERR_ARG, "q_out overlaps q");
        if (int rc = check_spans({{out, "q_out", true}, {k_to, "k_pages", true}, {v_to, "v_pages", true}, {k_in, "k", false}, {v_in, "v", false}}))
            return rc;
        if (touch(k_to, in) || touch(v_to, in)) return fail(W2V_ERR_ARG, "a pool overlaps q");
        a.x = turn_array(q, q_out->p, q_out->token_stride, q_out->head_stride, heads);
    }
    a.y = turn_array(k, k_pages->p, k_pages->token_stride, k_pages->head_stride, kv_heads);
    a.z = turn_array(v, v_pages->p, v_pages->token_stride, v_pages->head_stride, kv_heads);
    a.y_page = k_pages->page_stride; a.z_page = v_pages->page_stride;
    a.width = width;
    if (rotary) {
        a.rotated = rotary->rotated; a.halves = rotary->halves != 0; a.gain = rotary->gain;
        a.turns = rotary->turns_dev;
    }
    a.off = sent_off; a.n_sent = n_sent; a.T = n_tokens; a.position = position;
    a.n = n; a.table = table->page_dev; a.table_stride = table->stride; a.room = table->slots * table->page_words;
    a.shift = shift_of(table); a.n_pages = table->n_pages;
    launch_append(a, (uint32_t)type, (hipStream_t)stream);
    return launched();
}

namespace {

int check_attend_pages(const w2v_attend_spec* s, uint32_t batch, const w2v_page_table* t, uint32_t shared) {
    if (int rc = check_spec(s)) return rc;
    if (int rc = check_table(t)) return rc;
    if ((uint64_t)batch * s->heads > 1u << 23) return fail(W2V_ERR_ARG, "too many texts at once");
    if (shared % t->page_words || shared > t->slots * t->page_words)
        return fail(W2V_ERR_ARG, "shared = %u is no number of whole pages within the room", shared);
    return W2V_OK;
}

// The workspace: partial results where a text's words are read by several blocks.
PageSplits pages_splits(const w2v_attend_spec* s, uint32_t batch, const w2v_page_table* t, uint32_t shared) {
    return page_splits((uint32_t)s->type, batch, s->heads, s->kv_heads, s->width, t->slots * t->page_words, shared, s->left, s->sinks);
}
size_t pages_bytes(const w2v_attend_spec* s, uint32_t batch, const PageSplits& p) {
    const uint32_t parts = p.front + p.own.splits;
    return parts > 1 ? (size_t)batch * s->heads * parts * (s->width + 2) * sizeof(float) : 0;
}

}  // namespace

extern "C" size_t w2v_attend_pages_workspace(const w2v_attend_spec* spec, uint32_t batch, const w2v_page_table* table,
                                             uint32_t shared) {
    if (batch == 0 || check_attend_pages(spec, batch, table, shared)) return 0;
    return pages_bytes(spec, batch, pages_splits(spec, batch, table, shared));
}

extern "C" int w2v_attend_pages(const w2v_attend_spec* spec, const w2v_heads* q, const w2v_pages* k, const w2v_pages* v,
                                const w2v_page_table* table, uint32_t shared, const uint32_t* n, uint32_t batch,
                                const uint8_t* keep, const w2v_heads* out, void* workspace, size_t workspace_bytes,
                                void* stream) {
    if (int rc = check_spec(spec)) return rc;
    if (batch == 0) return W2V_OK;
    if (int rc = check_attend_pages(spec, batch, table, shared)) return rc;
    if (int rc = check_heads(q, spec, spec->heads, batch, false, "q")) return rc;
    if (int rc = check_pages(k, spec, table, "k_pages")) return rc;
    if (int rc = check_pages(v, spec, table, "v_pages")) return rc;
    if (int rc = check_heads(out, spec, spec->heads, batch, true, "out")) return rc;
    if (!n) return fail(W2V_ERR_NULL, "n_dev is NULL");
    const Lattice to = lattice_of(out, spec, spec->heads, batch);
    if (!same(q, out, spec->heads, batch) && touch(to, lattice_of(q, spec, spec->heads, batch)))
        return fail(W2V_ERR_ARG, "out overlaps q");
    if (touch(to, lattice_of(k, spec, table)) || touch(to, lattice_of(v, spec, table)))
        return fail(W2V_ERR_ARG, "out overlaps a pool");
    const PageSplits p = pages_splits(spec, batch, table, shared);
    const size_t need = pages_bytes(spec, batch, p);
    if (need) {
        if (!workspace) return fail(W2V_ERR_NULL, "workspace is NULL");
        if (!aligned(workspace, 256)) return fail(W2V_ERR_ARG, "workspace must be 256-byte aligned");
        if (workspace_bytes < need)
            return fail(W2V_ERR_ARG, "workspace of %zu bytes is too small: %zu are needed", workspace_bytes, need);
    }
    StepArgs a{};
    a.q = heads_of(q); a.o = heads_out(out);
    a.k = Cache{k->p, k->page_stride, k->token_stride, k->head_stride};
    a.v = Cache{v->p, v->page_stride, v->token_stride, v->head_stride};
    a.n = n; a.batch = batch; a.room = table->slots * table->page_words;
    a.heads = spec->heads; a.kv_heads = spec->kv_heads; a.group = spec->heads / spec->kv_heads; a.width = spec->width;
    a.left = spec->left; a.sinks = spec->sinks; a.skip_self = spec->skip_self != 0;
    a.scale2 = spec->scale * 1.4426950408889634f;
    a.keep = keep;
    a.bias = spec->bias_dev; a.buckets = spec->bucket_dev; a.n_buckets = spec->n_buckets; a.span = spec->span;
    a.splits = p.own.splits; a.per_split = p.own.per_split; a.parts = (float*)workspace;
    a.begin = p.begin; a.front = p.front;
    a.table = table->page_dev; a.table_stride = table->stride; a.shift = shift_of(table); a.n_pages = table->n_pages;
    a.shared = shared;
    launch_pages(a, (uint32_t)spec->type, (hipStream_t)stream);
    return launched();
}

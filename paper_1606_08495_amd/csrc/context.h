// Launches of the context operators (layer norm, attention over texts, positions, pages) for context.hip and pages.hip, which
// check what callers pass.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace w2v {

// ---- layer norm ------------------------------------------------------------------------------------
struct NormArgs {
    const void* x; uint64_t x_stride; uint64_t rows; uint32_t d; float eps;
    const float* gain; const float* offset;              // either may be null
    void* y; uint64_t y_stride; float* mean; float* rstd;     // the statistics may be null
};
void launch_norm(const NormArgs& a, uint32_t type, hipStream_t st);

struct NormBackwardArgs {
    const void* dy; uint64_t dy_stride; const void* x; uint64_t x_stride; uint64_t rows; uint32_t d;
    const float* gain; const float* mean; const float* rstd;
    void* dx; uint64_t dx_stride;
    float* parts;            // [norm_backward_parts][2][d], or null where neither column gradient is wanted
};
uint32_t norm_backward_parts(uint64_t rows, uint32_t d, uint32_t type);
void launch_norm_backward(const NormBackwardArgs& a, uint32_t type, float* dgain, float* doffset, hipStream_t st);

// ---- attention over texts --------------------------------------------------------------------------
constexpr uint32_t HEAD_MAX = 128, SINKS_MAX = 64, SPAN_MAX = 1023;

// Rows of heads: element c of head h of token i at p[i token + h head + c].
struct Heads { const void* p; uint64_t token, head; };
struct HeadsOut { void* p; uint64_t token, head; };

struct AttendArgs {
    Heads q, k, v;
    const uint64_t* off; uint32_t n_sent, T;             // texts, tokens
    uint32_t heads, kv_heads, group, width;              // group = heads / kv_heads
    uint32_t left, right, sinks; bool skip_self;         // left, right <= T
    float scale, scale2;                                 // scale2 = scale log2 e
    const uint8_t* keep;                                 // or null
    const float* bias; const uint32_t* buckets; uint32_t n_buckets, span;      // bias may be null
    HeadsOut o; float* lse;                              // lse [heads][T], may be null in the forward pass
};
void launch_attend(const AttendArgs& a, uint32_t type, hipStream_t st);

struct BackwardArgs {
    AttendArgs a;                                        // a.o and a.lse as the forward pass left them
    Heads dout;
    HeadsOut dq, dk, dv; float* dbias;                   // dbias [heads][n_buckets], may be null
    float *high, *low, *delta;                           // workspace, [heads][T]: weights are 2^(x - high - low); sums of dout o
    float* by_distance; float* distance_sums;            // workspace: [heads][bias_parts][2 span + 1], [heads][2 span + 1]
    // first words that stay visible: queries further than `reach` behind their block are taken in `late` pieces of
    // late_words queries, whose sums (and those of the text's own block) lie in workspace: [late][kv_heads][sinks][2][width]
    uint32_t late, late_words, reach;
    float* late_sums; float* own_sums;
};
struct LatePieces { uint32_t count, words, reach; };
LatePieces attend_late_pieces(uint32_t T, uint32_t left, uint32_t sinks);
uint32_t attend_bias_parts(uint32_t T);
void launch_attend_backward(const BackwardArgs& b, uint32_t type, hipStream_t st);

// ---- one new word per text over a cache --------------------------------------------------------------
struct Cache { const void* p; uint64_t text, token, head; };
struct StepArgs {
    Heads q; Cache k, v; HeadsOut o;                     // q, o: token = text
    const uint32_t* n; uint32_t batch, room;             // words of each text, the new one last
    uint32_t heads, kv_heads, group, width, left, sinks; bool skip_self;
    float scale2;
    const uint8_t* keep;                                 // [batch][room] or null
    const float* bias; const uint32_t* buckets; uint32_t n_buckets, span;
    uint32_t splits, per_split; float* parts;            // workspace: [batch][heads][splits][width + 2]
    // over pages: k.text and v.text lead from page to page, word j of a text is on page table[text table_stride + (j >> shift)] (row 0
    // for j < shared); room is the table's
    const uint32_t* table; uint64_t table_stride; uint32_t shift, n_pages, shared;
    // the first `begin` words are the common prefix's blocks' (0: there are none), which leave `front` parts of each row before the others;
    // parts: [batch][heads][front + splits][width + 2]
    uint32_t begin, front;
};
struct StepSplits { uint32_t splits, per_split; };
StepSplits step_splits(uint32_t batch, uint32_t kv_heads, uint32_t room, uint32_t left, uint32_t sinks);
void launch_step(const StepArgs& a, uint32_t type, hipStream_t st);

// Over pages.  What a call splits into, by sizes alone.
uint32_t prefix_splits(uint32_t type, uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t words);
struct PageSplits { uint32_t begin, front; StepSplits own; };
PageSplits page_splits(uint32_t type, uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t width, uint32_t room, uint32_t shared,
                       uint32_t left, uint32_t sinks);
void launch_pages(const StepArgs& a, uint32_t type, hipStream_t st);
// of k_page_tiles.hip, for k_pages.hip
void launch_prefix(const StepArgs& a, uint32_t type, hipStream_t st);
void launch_own_tiles(const StepArgs& a, uint32_t type, hipStream_t st);      // (16 bits)

// ---- positions that turn, and words on their way into pages ------------------------------------------
struct TurnArray { Heads in; void* out; uint64_t out_token, out_head; uint32_t heads; };      // heads = 0: none
struct TurnArgs {
    // rotate: x, y turned.  append: q, k turned, v as it is; k and v go into pages, out_token leading from place to place there
    TurnArray x, y, z;
    uint32_t width, rotated; bool halves, back; float gain;
    const uint64_t* turns;                               // [rotated / 2]
    const uint64_t* off; uint32_t n_sent, T;             // off null: token i is of text i, or positions are given
    const int32_t* position;                             // or null
    uint32_t tokens;                                     // of a block
    // append
    const uint32_t* n; const uint32_t* table; uint64_t table_stride, y_page, z_page; uint32_t room, shift, n_pages;
};
void launch_rotate(TurnArgs a, uint32_t type, hipStream_t st);
void launch_append(TurnArgs a, uint32_t type, hipStream_t st);

}  // namespace w2v

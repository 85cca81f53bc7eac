// Launches of the context operators (layer norm, attention over texts) for context.hip, which checks what callers pass.
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
};
struct StepSplits { uint32_t splits, per_split; };
StepSplits step_splits(uint32_t batch, uint32_t kv_heads, uint32_t room, uint32_t left, uint32_t sinks);
void launch_step(const StepArgs& a, uint32_t type, hipStream_t st);

}  // namespace w2v

// Attention of one new word per text over cached keys and values: step.h over a cache of one stride from word to word.
// Measured: 32 texts of up to 32768 words (574335 in all), 32 heads of 128 over 8, 16 bits: 590 us (4.0 TB/s; a large copy moves
// 4.8).  One text of 500 words, 5 heads of 60: 8 us and 4 us for the join.
#include "step.h"

namespace w2v {

// Blocks enough to fill the device several times over where the caches are long, parts of at least 256 keys.
StepSplits step_splits(uint32_t batch, uint32_t kv_heads, uint32_t room, uint32_t left, uint32_t sinks) {
    const uint64_t most = (uint64_t)left + 1 + sinks < room ? (uint64_t)left + 1 + sinks : room;
    const uint64_t rows = (uint64_t)batch * kv_heads, want = 4096 / rows > 1 ? 4096 / rows : 1;
    uint64_t per = (most + want - 1) / want;
    per = per < 256 ? 256 : (per + 63) / 64 * 64;
    return StepSplits{(uint32_t)((most + per - 1) / per), (uint32_t)per};
}

void launch_step(const StepArgs& a, uint32_t type, hipStream_t st) {
    if (type == ELEM_F32) step_any<float, false>(a, st);
    else if (type == ELEM_F16) step_any<_Float16, false>(a, st);
    else step_any<__bf16, false>(a, st);
}

}  // namespace w2v

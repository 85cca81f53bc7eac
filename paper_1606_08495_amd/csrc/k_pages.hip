// Attention of one new word per text over a cache in pages: step.h with a look into the table of pages a step ahead of the rows.
#include "step.h"

namespace w2v {

// A prefix that several texts have is taken by its own blocks (k_prefix.hip); what is left of the texts as for a cache of one stride.
PageSplits page_splits(uint32_t type, uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t room, uint32_t shared, uint32_t left, uint32_t sinks) {
    PageSplits p{};
    if (shared && batch > 1) {
        p.begin = shared;
        p.front = prefix_splits(type, batch, heads, kv_heads, shared);
    }
    const uint32_t rest = room > p.begin ? room - p.begin : 1;
    p.own = step_splits(batch, kv_heads, rest, left, sinks);
    return p;
}

namespace {
// 16 bits: the texts' own words on the matrix cores too, whose 32 rows of queries cost less than converting every element on the
// vector units.
template <typename T> void pages_any(const StepArgs& a, uint32_t type, hipStream_t st) {
    if (a.front || sizeof(T) == 2) launch_tiles(a, type, st);
    if constexpr (sizeof(T) == 4) step_any<T, true>(a, st);
    pages_join<T>(a, st);
}
}  // namespace

void launch_pages(const StepArgs& a, uint32_t type, hipStream_t st) {
    if (type == ELEM_F32) pages_any<float>(a, type, st);
    else if (type == ELEM_F16) pages_any<_Float16>(a, type, st);
    else pages_any<__bf16>(a, type, st);
}

}  // namespace w2v

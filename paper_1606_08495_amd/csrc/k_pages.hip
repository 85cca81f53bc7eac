// Attention of one new word per text over a cache in pages: what a call is split into.  step.h with a look into the table of pages a
// step ahead of the rows, or the tiles of k_page_tiles.hip.
#include "step.h"

namespace w2v {
namespace {

// In 16 bits and with heads that share keys the texts' own words go through the matrix cores: 32 rows of queries, however few are
// real, cost less than the conversions and multiply-adds of each head on the vector units (four heads of 128 over 574335 words: 456 us,
// 505).  A key head of one query head is taken by the vector units (48 windows of 1024, six heads of 100: 37 us, 51), and so are 32 bits.
bool own_tiles(uint32_t type, uint32_t group) { return type != ELEM_F32 && group > 1; }

template <typename T> void pages_any(const StepArgs& a, uint32_t type, hipStream_t st) {
    if (a.front) launch_prefix(a, type, st);
    if (own_tiles(type, a.group)) launch_own_tiles(a, type, st);
    else step_any<T, true>(a, st);
    pages_join<T>(a, st);
}

// A prefix is taken by blocks of its own where reading it once for each text would move this many bytes more: below, their launch and
// the join cost more than reading it from the caches.
constexpr uint64_t PREFIX_BYTES = 64 << 20;

}  // namespace

// Of the texts' own words a block has 512 at least (fewer cost a join that is longer than what they save), or 1024 of the vector units' where
// there is a block for every compute unit without a split; and blocks are enough to fill the device several times over.
PageSplits page_splits(uint32_t type, uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t width, uint32_t room, uint32_t shared,
                       uint32_t left, uint32_t sinks) {
    PageSplits p{};
    if (batch > 1 && (uint64_t)(batch - 1) * shared * kv_heads * width * 2 * elem_bytes(type) >= PREFIX_BYTES) {
        p.begin = shared;
        p.front = prefix_splits(type, batch, heads, kv_heads, shared);
    }
    const uint64_t rest = room > p.begin ? room - p.begin : 1, rows = (uint64_t)batch * kv_heads;
    const uint64_t shown = (uint64_t)left + 1 + sinks < rest ? (uint64_t)left + 1 + sinks : rest;
    const bool tiles = own_tiles(type, heads / kv_heads);
    const uint64_t least = !tiles && rows >= 256 ? 1024 : 512;
    uint64_t want = (tiles ? 8192 : 4096) / rows;
    if (want > shown / least) want = shown / least;
    if (want < 1) want = 1;
    const uint64_t per = ((shown + want - 1) / want + 63) / 64 * 64;
    p.own = StepSplits{(uint32_t)((shown + per - 1) / per), (uint32_t)per};
    return p;
}

void launch_pages(const StepArgs& a, uint32_t type, hipStream_t st) {
    if (type == ELEM_F32) pages_any<float>(a, type, st);
    else if (type == ELEM_F16) pages_any<_Float16>(a, type, st);
    else pages_any<__bf16>(a, type, st);
}

}  // namespace w2v

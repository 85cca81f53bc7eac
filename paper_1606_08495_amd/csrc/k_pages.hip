// Attention of one new word per text over a cache in pages: what a call is split into.  step.h with a look into the table of pages a
// step ahead of the rows, or the tiles of k_page_tiles.hip.
#include "step.h"

namespace w2v {
namespace {

// In 16 bits the texts' own words go through the matrix cores where three query heads or more share a key head: their 32 rows of
// queries, however few are real, then cost less than the conversions and multiply-adds of each head on the vector units.  32 texts
// of up to 8192 words, 8 key heads of 128: 140, 150, 175 and 305 us for one, two, three and eight query heads each on the vector units,
// 138 to 155 on the matrix cores; 48 texts of up to 1000, 6 of 100: 25, 30, 40 and 68, and 35 to 37.
bool own_tiles(uint32_t type, uint32_t group) { return type != ELEM_F32 && group > 2; }

template <typename T> void pages_any(const StepArgs& a, uint32_t type, hipStream_t st) {
    if (a.front) launch_prefix(a, type, st);
    if (own_tiles(type, a.group)) launch_own_tiles(a, type, st);
    else step_any<T, true>(a, st);
    pages_join<T>(a, st);
}

// A prefix is taken by blocks of its own where reading it once for each text would move this many bytes more: below, their launch and
// the join cost more than reading it from the caches.  24 texts with up to 900 words behind it in 32 bits, 8 heads of 64: 126 MB more
// (1408 words) 23 us with blocks of its own and 23 without, 368 MB 27 and 38.  In 16 bits both are level at 250 MB: 64 texts, 32 heads of 128
// over 8, 130 MB 54 and 47, 252 MB 56 and 57, 504 MB 63 and 77; 8 texts, 128 MB 39 and 30, 427 MB 42 and 63.
// Of a window only so much is in the prefix as the texts have not moved on behind it, and texts of unequal length are shown different
// words of it: windows that are shorter than the prefix have to be four times as large.  64 texts with up to 900 words behind 32768,
// 16 bits, 8 key heads of 128: windows of 1040 words (256 MB) 63 us with blocks of the prefix's own and 41 without, 2080 (512 MB) 64 and
// 62, 6241 82 and 175; 6 heads of 100 behind 16384: 887 words (128 MB) 49 and 27, 3550 (512 MB) 51 and 73.
constexpr uint64_t PREFIX_BYTES = 128 << 20, PREFIX_BYTES_WINDOW = 512 << 20;

}  // namespace

// How many parts a text's own words are taken in.  The vector units' blocks have 512 words at least, or 1024 where there is a block for
// every compute unit without a split (48 texts behind windows of 1028, 6 heads of 100: 33 us in one part, 33 and 4.5 for the join in two
// or four), and are enough to fill the device several times over.  The matrix cores' have 128 at least and fill it once, but of long texts, which may
// be of unequal length, 1024 (16 texts of up to 3000 words, 4 key heads of 96: 23 us in parts of 128 to 192, 32 of 512).
// Up to 512 words are not split: the join's launch costs more (500 words: 14 us, 17 in parts).  Behind a prefix with blocks of its own, where
// there is a join in any case, parts are shorter.
PageSplits page_splits(uint32_t type, uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t width, uint32_t room, uint32_t shared,
                       uint32_t left, uint32_t sinks) {
    PageSplits p{};
    const bool windowed = (uint64_t)left + 1 + sinks < shared;
    const uint32_t seen = windowed ? left + 1 + sinks : shared;      // words of the prefix that a text is shown at most
    if (batch > 1 && (uint64_t)(batch - 1) * seen * kv_heads * width * 2 * elem_bytes(type) >= (windowed ? PREFIX_BYTES_WINDOW : PREFIX_BYTES)) {
        p.begin = shared;
        p.front = prefix_splits(type, batch, heads, kv_heads, seen);
    }
    const uint64_t rest = room > p.begin ? room - p.begin : 1, rows = (uint64_t)batch * kv_heads;
    const uint64_t shown = (uint64_t)left + 1 + sinks < rest ? (uint64_t)left + 1 + sinks : rest;
    const bool tiles = own_tiles(type, heads / kv_heads);
    uint64_t want;
    if (tiles) {
        const uint64_t whole = 1024 / rows, longer = 8192 / rows < shown / 1024 ? 8192 / rows : shown / 1024;
        want = whole > longer ? whole : longer;
        if (want > shown / 128) want = shown / 128;
        if (shown <= 512 && !p.front) want = 1;
    } else {
        const uint64_t least = p.front ? 256 : rows >= 256 ? 1024 : 512;
        want = 4096 / rows < shown / least ? 4096 / rows : shown / least;
    }
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

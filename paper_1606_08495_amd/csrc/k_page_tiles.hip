// Attention of the newest words of texts over pages on the matrix cores: over the words that all texts begin with, which lie in pages
// once, and in 16 bits over a text's own words.
//
// For a key head the queries of all texts and of the heads that share it are the rows of one product with the prefix's keys,
// and their weights those of one with its values: the prefix is read once for 32 WR rows and not once for each.  Of a text's own words the
// rows are the few heads that share a key head; the rest of the 32 is padding, which costs less than the vector units' work.
// Rows are staged in LDS by tiles of 64 words, whose places a thread each looks up in the table of pages two tiles ahead.  As in attention
// over texts scores are transposed (keys are rows, a query is a lane), the maximum and sum of a query lie in its two lanes, and weights
// feed the second product from the registers they are in.  WR wavefronts have 32 queries each; with WK = 2 two of them share
// queries and take a half of every tile each.  A block has a part of the words and leaves (maximum, sum, output) of its queries over it in
// the workspace, where the join finds them (step.h).
//
// Scores, maxima, sums and outputs are fp32; weights are rounded to the type of v for the second product, relative to the row's maximum
// (fp16: lifted by a power of two, so that small ones keep their bits), and summed before that.  What the rounding left is multiplied too,
// so that a weight has twice the type's bits and one rounding at the end is what results are off by, whatever the number of queries.  It
// costs little where memory is what the matrix cores wait for: over a text's own words 458 us for 455 below, for up to 64 queries of a
// prefix's key head 39 and 41 us for 37 and 39 (16384 words, 32 and 64 queries), and more for many: 84 us for 74 below.  Left out there,
// results were 1.4 times as far off.
//
// What bounds it: a text's own words memory (32 texts of 574335 words, 32 heads of 128 over 8, 16 bits: 452 us, 5.2 TB/s; two wavefronts a
// block, four blocks a CU take turns).  The prefix, where many queries share it, its two products and the exponentials, with
// two wavefronts a SIMD: 64 texts behind 32768 words, the same heads, 84 us (51 GFLOP with the weights' second product, 610 TFLOP/s), and
// 45 us for their own 33000 words.  24 texts behind 4096 words in 32 bits, 8 heads of 64, bias: 15 us.
#include <type_traits>

#include "attend.h"
#include "tiles.h"

namespace w2v {
namespace {

constexpr uint64_t NOWHERE = ~0ull;
template <typename T> constexpr float RISE = std::is_same<T, _Float16>::value ? 2.f : 8.f;
template <typename T> constexpr float LIFT = std::is_same<T, _Float16>::value ? 13.f : 0.f;

__device__ __forceinline__ uint32_t lanes_least(uint32_t x) {
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t y = (uint32_t)__shfl_xor((int)x, d, 64);
        x = y < x ? y : x;
    }
    return __builtin_amdgcn_readfirstlane(x);
}

// A query: its text, head, and the words it is shown, lo .. hi and those before `sinks`.
struct Query { uint32_t text, head, lo, hi; };
__device__ __forceinline__ Query query_of(const StepArgs& a, uint32_t text, uint32_t head) {
    Query q;
    q.text = text;
    q.head = head;
    const uint32_t n = a.n[text];
    q.hi = n < a.room ? n : a.room;
    q.lo = q.hi && q.hi - 1 > a.left ? q.hi - 1 - a.left : 0;
    return q;
}
__device__ __forceinline__ bool shows(const StepArgs& a, const Query& q, uint32_t j) {
    return j < q.hi && (j >= q.lo || j < a.sinks) && !(a.skip_self && j + 1 == q.hi) && (!a.keep || a.keep[(uint64_t)q.text * a.room + j]);
}
// What a block's queries are shown between them, of the prefix or of their text's own words: `sunk` words from `first` on, then those
// from lo on.  Words lie in the pages of row `pages` of the table (those before `shared` in row 0's).
struct Axis {
    uint32_t first, sunk, lo, count, shared;
    const uint32_t *row0, *pages;
    __device__ __forceinline__ uint32_t word(uint32_t at) const { return at < sunk ? first + at : lo + at - sunk; }
    __device__ __forceinline__ uint32_t page(uint32_t j, uint32_t shift) const { return (j < shared ? row0 : pages)[j >> shift]; }
};

__device__ __forceinline__ float query_bias(const StepArgs& a, const Query& q, uint32_t j) {
    const uint32_t back = q.hi - 1 - j < a.span ? q.hi - 1 - j : a.span;
    return scaled_bias(a.bias, a.buckets, a.n_buckets, a.span, q.head, -(int32_t)back);
}

// A query's part [from, to) of the axis, word by word and nothing touched that it is not shown: for rows whose result is not finite.
template <typename T>
__device__ void careful_row(const StepArgs& a, const Axis& x, uint32_t kv_head, const Query& q, uint32_t from, uint32_t to, uint32_t lane,
                            float& m, float& total, float (&o)[2]) {
    const T* row = head_row<T>(a.q, q.text, q.head);
    const auto place = [&](const Cache& c, uint32_t j) {
        return (const T*)c.p + (uint64_t)x.page(j, a.shift) * c.text + (uint64_t)(j & ((1u << a.shift) - 1)) * c.token + (uint64_t)kv_head * c.head;
    };
    const auto score = [&](uint32_t j) {
        const float s = dot_rows(row, place(a.k, j), a.width) * a.scale2;
        return a.bias ? s + query_bias(a, q, j) : s;
    };
    const auto in = [&](uint32_t at) {
        const uint32_t j = x.word(at < to ? at : to - 1);
        return at < to && shows(a, q, j) && x.page(j, a.shift) < a.n_pages;
    };
    m = -__builtin_inff();
    bool nan = false;
    for (uint32_t at = from + lane; at < to; at += WAVE) {
        if (!in(at)) continue;
        const float s = score(x.word(at));
        nan |= s != s;
        m = fmaxf(m, s);
    }
    m = wave_max(m);
    o[0] = o[1] = total = 0.f;
    if (__any(nan) || m == __builtin_inff()) {        // every weight is not a number, and so is every column
        o[0] = o[1] = total = __builtin_nanf("");
        m = -__builtin_inff();
        return;
    }
    if (m == -__builtin_inff()) return;
    for (uint32_t at0 = from; at0 < to; at0 += WAVE) {
        const uint32_t at = at0 + lane, j = x.word(at < to ? at : to - 1);
        const float p = in(at) ? exp2f(score(j) - m) : 0.f;
        total += p;
        for (uint64_t left = __ballot(p != 0.f); left; left &= left - 1) {
            const int l = __builtin_ctzll(left);
            const T* v = place(a.v, (uint32_t)__shfl((int)j, l, 64));
            const float pl = __shfl(p, l, 64);
            if (lane < a.width) o[0] = fmaf(pl, (float)v[lane], o[0]);
            if (lane + WAVE < a.width) o[1] = fmaf(pl, (float)v[lane + WAVE], o[1]);
        }
    }
    total = lanes_sum<64>(total);
}

constexpr int KEYS = 64;                              // of a tile

// One block, of the prefix (PREFIX) or of one text's own words.
template <typename T, int DB, int WR, int WK, bool BIAS, bool PREFIX>
__device__ __forceinline__ void tile_block(const StepArgs& a, uint32_t block) {
    constexpr int THREADS = 64 * WR * WK, KEEP = DB * 16 + 2;
    constexpr bool JOINT = DB <= (sizeof(T) == 2 ? 2 : 1);      // both pieces of a tile at a time, where registers allow
    typedef Tile<T, DB, KEYS> Tl;
    // Blocks of the prefix have two of each tile, and one barrier a tile; the others' many small blocks a CU take turns by themselves.
    constexpr int BUFFERS = WR > 1 ? 2 : 1;
    __shared__ __align__(16) char tiles[BUFFERS][2 * Tl::BYTES];
    __shared__ uint64_t places[3][2][KEYS];
    __shared__ uint32_t bounds[2 * WR];
    extern __shared__ uint32_t buckets[];             // of distances 0 .. -span
    static_assert(WK == 1 || WR * KEEP * 64 * 4 <= (int)sizeof(tiles), "room to join the parts");
    const uint32_t lane = threadIdx.x % WAVE, h = lane / 32, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const uint32_t wr = wave % WR, wk = wave / WR;
    uint32_t kv_head, split, row_tile, text = 0;
    const uint32_t rows = PREFIX ? a.batch * a.group : a.group, row_tiles = (rows + 32 * WR - 1) / (32 * WR);
    if constexpr (PREFIX) {
        // blocks of the same words and key head lie eight apart: they run on one die and share its cache
        const uint32_t unit = block / (8 * row_tiles) * 8 + block % 8;
        row_tile = block / 8 % row_tiles;
        if (unit >= a.kv_heads * a.front) return;
        kv_head = unit % a.kv_heads;
        split = unit / a.kv_heads;
    } else {
        // the heads of the same words, which lie side by side in memory, follow each other
        kv_head = block % a.kv_heads; block /= a.kv_heads;
        row_tile = block % row_tiles; block /= row_tiles;
        split = block % a.splits;
        text = block / a.splits;
    }
    const bool whole = !PREFIX && a.front + a.splits == 1;
    const uint32_t first = row_tile * 32 * WR + wr * 32;
    const bool some = first < rows, real = first + lane % 32 < rows;
    const uint32_t row = real ? first + lane % 32 : rows - 1;
    Axis x;
    x.row0 = a.table;
    x.shared = PREFIX ? ~0u : a.shared;
    x.pages = a.table + (uint64_t)text * a.table_stride;
    // Without a window the first words are known before the texts' lengths are: their pages are asked for at once.
    const bool bounded = a.left < a.room;
    uint32_t from = split * a.per_split, to, early_page = 0;
    if (!PREFIX && !bounded) {
        const uint32_t j = a.begin + from + threadIdx.x;
        early_page = x.page(j < a.room ? j : a.room - 1, a.shift);
    }
    const Query own = PREFIX ? query_of(a, row / a.group, kv_head * a.group + row % a.group) : query_of(a, text, kv_head * a.group + row);
    if constexpr (!PREFIX) {
        x.sunk = own.lo < a.sinks ? own.lo : a.sinks;
        x.first = x.sunk < a.begin ? x.sunk : a.begin;
        x.sunk -= x.first;
        x.lo = own.lo < a.begin ? a.begin : own.lo;
        x.count = x.sunk + (own.hi > x.lo ? own.hi - x.lo : 0);
        x.first = __builtin_amdgcn_readfirstlane(x.first);
        x.sunk = __builtin_amdgcn_readfirstlane(x.sunk);
        x.lo = __builtin_amdgcn_readfirstlane(x.lo);
        x.count = __builtin_amdgcn_readfirstlane(x.count);
        to = x.count < from + a.per_split ? x.count : from + a.per_split;
        if (from >= to && !whole) return;
    }

    typename Frag<T>::vec q[2 * DB];
#pragma unroll
    for (int s = 0; s < 2 * DB; ++s) q[s] = load_operand<T, DB>(head_row<T>(a.q, own.text, own.head), s, h, a.width);
    uint32_t lo_least = 0, lo_most = 0, hi_least = own.hi, hi_most = own.hi;
    if constexpr (BIAS)
        for (uint32_t c = threadIdx.x; c <= a.span; c += THREADS) buckets[c] = a.buckets[a.span - c];
    if constexpr (PREFIX) {
        x.first = x.lo = x.sunk = 0;
        x.count = a.begin;
        if (bounded) {
            lo_least = lanes_least(own.lo), lo_most = ~lanes_least(~own.lo), hi_most = ~lanes_least(~own.hi);
            if (lane == 0) {
                bounds[wr] = lo_least;
                bounds[WR + wr] = hi_most;
            }
            __syncthreads();
            uint32_t lo = ~0u, end = 0;
#pragma unroll
            for (int w = 0; w < WR; ++w) {
                lo = bounds[w] < lo ? bounds[w] : lo;
                end = bounds[WR + w] > end ? bounds[WR + w] : end;
            }
            end = __builtin_amdgcn_readfirstlane(end < a.begin ? end : a.begin);
            x.lo = __builtin_amdgcn_readfirstlane(lo < end ? lo : end);
            x.sunk = x.lo < a.sinks ? x.lo : a.sinks;
            x.count = x.sunk + end - x.lo;
        }
        const uint32_t per = ((x.count + KEYS - 1) / KEYS + a.front - 1) / a.front * KEYS;
        from = split * per < x.count ? split * per : x.count;
        to = x.count - from < per ? x.count : from + per;
    }
    const uint32_t shift = x.lo - x.sunk;             // word of key n >= sunk: n + shift

    Acc o[DB];
#pragma unroll
    for (int b = 0; b < DB; ++b) o[b] = Acc{};
    float m = -__builtin_inff(), total = 0.f;
    const float unit_scale = BIAS ? 1.f : a.scale2;   // of the scores once masked
    float far = 0.f;
    if constexpr (BIAS) far = scaled_bias(a.bias, a.buckets, a.n_buckets, a.span, own.head, -(int32_t)a.span);
    const uint32_t at_along = Tl::base_along(lane), at_across = Tl::base_across(lane);


    Transit<T, DB, KEYS, THREADS> k, v;
    k.start(Heads{a.k.p, a.k.token, a.k.head}, kv_head, 0);
    v.start(Heads{a.v.p, a.v.token, a.v.head}, kv_head, 0);
    // Where the tiles' rows lie, found by a thread each two tiles ahead: elements from the pools' starts, NOWHERE for keys that are not to be
    // shown (past the end, on no page, dropped).
    uint64_t k_next = 0, v_next = 0;
    const auto look = [&](uint32_t at, bool known) __attribute__((always_inline)) {
        const uint32_t j = x.word(at < to ? at : to - 1), page = known ? early_page : x.page(j, a.shift);
        bool in = at < to && page < a.n_pages;
        if (!PREFIX) in &= !(a.skip_self && j + 1 == own.hi) && (!a.keep || a.keep[(uint64_t)text * a.room + j]);
        const uint32_t place = j & ((1u << a.shift) - 1);
        k_next = in ? page * a.k.text + place * a.k.token : NOWHERE;
        v_next = in ? page * a.v.text + place * a.v.token : NOWHERE;
    };
    const auto tell = [&](uint32_t turn, uint32_t r) __attribute__((always_inline)) {
        places[turn][0][r] = k_next;
        places[turn][1][r] = v_next;
    };
    const auto fetch = [&](uint32_t turn) __attribute__((always_inline)) {
        uint32_t gone = 0;
#pragma unroll
        for (uint32_t n = 0; n < decltype(k)::PER; ++n) {
            const uint32_t r = k.r0 + n * decltype(k)::RS;
            const uint64_t at = places[turn][0][r], v_at = places[turn][1][r];
            gone |= (at == NOWHERE ? 1u : 0u) << n;
            k.at[n] = k.base + (at == NOWHERE ? 0 : at);
            v.at[n] = v.base + (at == NOWHERE ? 0 : v_at);
        }
        k.load(a.width);
        v.load(a.width);
        return gone;
    };
    const auto store = [&](char* to_tile, uint32_t gone) __attribute__((always_inline)) {
        k.store(to_tile, a.width);
        if (!rare(__any(gone != 0))) v.store(to_tile + Tl::BYTES, a.width);
        else v.store_rows(to_tile + Tl::BYTES, a.width, gone);
    };
    uint32_t turn = 0, buffer = 0;                    // of the tile in work
    const auto after = [](uint32_t turn) __attribute__((always_inline)) { return turn == 2 ? 0 : turn + 1; };
    if (from < to && threadIdx.x < 2 * KEYS) {        // the first two tiles'
        look(from + threadIdx.x, !PREFIX && !bounded);
        tell(threadIdx.x / KEYS, threadIdx.x % KEYS);
    }
    if (PREFIX) {
        hi_least = lanes_least(own.hi);
        if (!bounded) {
            hi_most = ~lanes_least(~own.hi);
            if (lane == 0) bounds[wr] = hi_most;
        }
    }
    __syncthreads();
    if (PREFIX && !bounded) {                         // where all texts end within the prefix, so does the block: nothing is known of later places
        uint32_t end = 0;
#pragma unroll
        for (int w = 0; w < WR; ++w) end = bounds[w] > end ? bounds[w] : end;
        end = __builtin_amdgcn_readfirstlane(end);
        if (end < to) {
            to = end > from ? end : from;
            if (threadIdx.x < 2 * KEYS && from + threadIdx.x >= to) {
                k_next = v_next = NOWHERE;
                tell(threadIdx.x / KEYS, threadIdx.x % KEYS);
            }
            __syncthreads();
        }
    }
    if (from < to) store(tiles[0], fetch(0));
    __syncthreads();
    for (uint32_t n0 = from; n0 < to; n0 += KEYS) {
        const bool more = n0 + KEYS < to;
        uint32_t gone = 0;
        if (more) {
            gone = fetch(after(turn));
            if (n0 + 2 * KEYS < to && threadIdx.x < KEYS) look(n0 + 2 * KEYS + threadIdx.x, false);
        }
        const char *const k_tile = tiles[buffer], *const v_tile = k_tile + Tl::BYTES;
        // P pieces of 32 keys from piece p0 on, together: their products do not wait for each other
        const auto pieces = [&](auto P, int p0) __attribute__((always_inline)) {
            Acc s[P.value];
#pragma unroll
            for (int p = 0; p < P.value; ++p) s[p] = Acc{};
            // Operands are read from LDS all at once, the values' while the scores are in work: left to itself the compiler has each
            // product wait for the read before it.
            constexpr bool EARLY = sizeof(T) == 2 && WR > 1;
            typename Frag<T>::vec rows[EARLY ? 2 * DB : 1][P.value], columns[EARLY ? 2 * P.value : 1][DB];
            if constexpr (EARLY) {
#pragma unroll
                for (int c = 0; c < 2 * DB; ++c)
#pragma unroll
                    for (int p = 0; p < P.value; ++p) rows[c][p] = Tl::along(k_tile, at_along + (p0 + p) * (32 / 4 * Tl::STRIDE), 0, c);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int c = 0; c < 2 * DB; ++c)
#pragma unroll
                for (int p = 0; p < P.value; ++p)
                    mma(EARLY ? rows[EARLY ? c : 0][p] : Tl::along(k_tile, at_along + (p0 + p) * (32 / 4 * Tl::STRIDE), 0, c), q[c], s[p]);
            if constexpr (EARLY) {
#pragma unroll
                for (int g = 0; g < 2 * P.value; ++g)
#pragma unroll
                    for (int b = 0; b < DB; ++b) columns[g][b] = Tl::across(v_tile, at_across + (p0 + g / 2) * (32 / 4 * Tl::STRIDE), 0, g % 2, b);
                __builtin_amdgcn_sched_barrier(0);
            }
            float most = -__builtin_inff();
#pragma unroll
            for (int p = 0; p < P.value; ++p) {
                const uint32_t n = n0 + (p0 + p) * 32, j0 = n + shift;
                const uint32_t kept32 = (uint32_t)__ballot(places[turn][0][(p0 + p) * 32 + lane % 32] != NOWHERE);
                const bool linear = n >= x.sunk;
                const auto word = [&](int r) __attribute__((always_inline)) { return x.word(n + 4 * h + acc_row(r, 0)); };
                if constexpr (BIAS) {
                    if (linear && hi_least > a.span && j0 + 31 <= hi_least - 1 - a.span) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[p][r] = fmaf(s[p][r], a.scale2, far);
                    } else {
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const uint32_t back = own.hi - 1 - word(r), b = buckets[back < a.span ? back : a.span];      // (words behind the text: masked)
                            const float w = b < a.n_buckets ? a.bias[(uint64_t)own.head * a.n_buckets + b] : 0.f;
                            s[p][r] = fmaf(s[p][r], a.scale2, fabsf(w) < __builtin_inff() ? fminf(fmaxf(w, -BIAS_HELD), BIAS_HELD) * LOG2E : w);
                        }
                    }
                }
                bool all = kept32 == 0xFFFFFFFFu;
                if (PREFIX) all &= linear && j0 >= lo_most && j0 + 32 <= hi_least && !a.keep && !(a.skip_self && j0 + 32 >= hi_least);
                if (!all) {
                    // a bit for each of the lane's keys, formed one by one: sixteen at a time would take their registers from the walk
                    uint32_t in = kept32 >> 4 * h;    // key 8 (r / 4) + r % 4 of the lane's half
                    if (PREFIX) {
                        uint32_t shown = 0;
#pragma clang loop unroll(disable)
                        for (uint32_t r = 0; r < 32; ++r)
                            if (!(r & 4) && shows(a, own, x.word(n + 4 * h + r))) shown |= 1u << r;
                        in &= shown;
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[p][r] = in >> acc_row(r, 0) & 1 ? s[p][r] : -__builtin_inff();
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, s[p][r]);
            }
            most = halves_max(most) * unit_scale;
            if (__any(most > m + RISE<T>)) {
                const float up = fmaxf(m, most);
                const float factor = up == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m - up);
                m = up;
                total *= factor;
#pragma unroll
                for (int b = 0; b < DB; ++b) o[b] *= factor;
            }
            const float base = m == -__builtin_inff() ? 0.f : m - LIFT<T>;
            float sum = 0.f;
            constexpr bool PARTS = sizeof(T) == 4, REST = sizeof(T) == 2;
            Acc part[PARTS ? DB : 1] = {};            // 32 bits: the pieces' sums first, then the whole's: one long chain would lose bits
#pragma unroll
            for (int g = 0; g < 2 * P.value; ++g) {   // 16 keys
                const int p = g / 2;
#pragma unroll
                for (int c = 8 * (g % 2); c < 8 * (g % 2) + 8; ++c) {
                    s[p][c] = __builtin_amdgcn_exp2f(fmaf(s[p][c], unit_scale, -base));
                    sum += s[p][c];
                }
                const auto w = acc_operand<T>(s[p], g % 2);
                typename Frag<T>::vec rest;           // what the rounding left of the weights
                if constexpr (REST)
#pragma unroll
                    for (int c = 0; c < 8; ++c) rest[c] = (T)(s[p][8 * (g % 2) + c] - (float)w[c]);
#pragma unroll
                for (int b = 0; b < DB; ++b) {
                    Acc& into = PARTS ? part[PARTS ? b : 0] : o[b];
                    const auto column = EARLY ? columns[EARLY ? g : 0][b] : Tl::across(v_tile, at_across + (p0 + p) * (32 / 4 * Tl::STRIDE), 0, g % 2, b);
                    mma(column, w, into);
                    if constexpr (REST) mma(column, rest, into);
                }
            }
            total += sum;
            if constexpr (PARTS)
#pragma unroll
                for (int b = 0; b < DB; ++b) o[b] += part[b];
        };
        // whether any of the wavefront's queries is shown any of a piece
        const auto needs = [&](int p) __attribute__((always_inline)) {
            const uint32_t n = n0 + p * 32, j0 = n + shift;
            return some && n < to && (!PREFIX || n < x.sunk || (j0 < hi_most && (j0 + 32 > lo_least || j0 < a.sinks)));
        };
        if constexpr (WK == 2) {
            if (needs(wk)) pieces(std::integral_constant<int, 1>{}, wk);
        } else {
            const bool joint = JOINT && needs(0) && needs(1);
            if (joint) pieces(std::integral_constant<int, JOINT ? 2 : 1>{}, 0);
            else {
#pragma clang loop unroll(disable)
                for (int p = 0; p < 2; ++p)
                    if (needs(p)) pieces(std::integral_constant<int, 1>{}, p);
            }
        }
        if (more) {
            if constexpr (BUFFERS == 1) __syncthreads();
            else buffer ^= 1;
            store(tiles[buffer], gone);
            if (n0 + 2 * KEYS < to && threadIdx.x < KEYS) tell(after(after(turn)), threadIdx.x);
            turn = after(turn);
            __syncthreads();
        }
    }
    if constexpr (WK == 2) {                          // the second half's sums through LDS to the first
        float* const other = (float*)tiles + wr * KEEP * WAVE + lane;
        __syncthreads();
        if (wk) {
            other[0] = m;
            other[WAVE] = total;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) other[(2 + b * 16 + r) * WAVE] = o[b][r];
        }
        __syncthreads();
        if (wk) return;
        const float m1 = other[0], up = fmaxf(m, m1);
        const float f0 = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m - up);
        const float f1 = m1 == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m1 - up);
        // (a maximum is -infinity where a half has seen nothing: its sums are zero; not a number stays where it is)
        total = total * (total == 0.f ? 1.f : f0) + other[WAVE] * (other[WAVE] == 0.f ? 1.f : f1);
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[b][r] = o[b][r] * f0 + other[(2 + b * 16 + r) * WAVE] * f1;
        m = up;
    }
    if (!some) return;
    total = halves_sum(total);
    float worst = total * 0.f;                        // not a number, if any sum is not finite
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) worst = fmaf(o[b][r], 0.f, worst);
    worst = halves_sum(worst);
    const bool redo = worst != 0.f;
    const uint32_t place = PREFIX ? split : a.front + split;
    const auto part_of = [&](uint32_t text, uint32_t head) __attribute__((always_inline)) {
        return a.parts + (((uint64_t)text * a.heads + head) * (a.front + a.splits) + place) * (a.width + 2);
    };
    if (real && !redo) {
        const float inv = !whole ? 1.f : total == 0.f ? 0.f : 1.f / total;
        float* p = whole ? nullptr : part_of(own.text, own.head);
        T* out = head_row<T>(a.o, own.text, own.head);
        if (!whole && h == 0) {
            p[0] = total == 0.f ? -__builtin_inff() : m - LIFT<T>;
            p[1] = total;
        }
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const uint32_t c = 32 * b + acc_row(r, h);
                if (whole) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) if (c + e < a.width) out[c + e] = (T)(o[b][r + e] * inv);
                } else if (c + 4 <= a.width) {
                    *(Pack<float, 4>::mem*)(p + 2 + c) = Pack<float, 4>::vec{o[b][r], o[b][r + 1], o[b][r + 2], o[b][r + 3]};
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) if (c + e < a.width) p[2 + c + e] = o[b][r + e];
                }
            }
    }
    // what a query is not shown must not show: rows that are not finite are formed from their words alone
    uint64_t again = __ballot(redo && real && h == 0);
    if (rare(again)) for (; again; again &= again - 1) {
        const int l = __builtin_ctzll(again);
        const Query one{(uint32_t)__shfl((int)own.text, l, 64), (uint32_t)__shfl((int)own.head, l, 64), (uint32_t)__shfl((int)own.lo, l, 64),
                        (uint32_t)__shfl((int)own.hi, l, 64)};
        float most, sum, row[2];
        careful_row<T>(a, x, kv_head, one, from, to, lane, most, sum, row);
        if (whole) {
            T* out = head_row<T>(a.o, one.text, one.head);
#pragma unroll
            for (int c = 0; c < 2; ++c) if (lane + c * WAVE < a.width) out[lane + c * WAVE] = (T)(sum == 0.f ? 0.f : row[c] / sum);
            continue;
        }
        float* p = part_of(one.text, one.head);
        if (lane == 0) {
            p[0] = most;
            p[1] = sum;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) if (lane + c * WAVE < a.width) p[2 + lane + c * WAVE] = row[c];
    }
}

template <typename T, int DB, int WR, int WK, bool BIAS, bool PREFIX>
__global__ __launch_bounds__(64 * WR * WK, (sizeof(T) == 2 || DB <= 2 ? 2 : 1)) void tile_kernel(const StepArgs a) {
    tile_block<T, DB, WR, WK, BIAS, PREFIX>(a, blockIdx.x);
}

// Queries of a prefix's block: as many as there are for one key head, up to 128.  (32 bits: 64 at least, whose four wavefronts' registers
// hold a tile on its way.)
uint32_t prefix_rows(uint32_t type, uint32_t rows) { return rows <= 32 && type != ELEM_F32 ? 32 : rows <= 64 ? 64 : 128; }

template <typename T, int DB, int WR, int WK, bool PREFIX> void tiles_bias(const StepArgs& a, hipStream_t st) {
    const uint32_t rows = PREFIX ? a.batch * a.group : a.group, row_tiles = (rows + 32 * WR - 1) / (32 * WR);
    const uint32_t blocks = PREFIX ? (a.kv_heads * a.front + 7) / 8 * 8 * row_tiles : a.batch * a.kv_heads * row_tiles * a.splits;
    if (a.bias) tile_kernel<T, DB, WR, WK, true, PREFIX><<<blocks, 64 * WR * WK, (a.span + 1) * sizeof(uint32_t), st>>>(a);
    else tile_kernel<T, DB, WR, WK, false, PREFIX><<<blocks, 64 * WR * WK, 0, st>>>(a);
}
template <typename T, int DB> void tiles_run(const StepArgs& a, uint32_t type, bool prefix, hipStream_t st) {
    if (prefix) {
        switch (prefix_rows(type, a.batch * a.group)) {
            case 128: return tiles_bias<T, DB, 4, 1, true>(a, st);
            case 64: return tiles_bias<T, DB, 2, 2, true>(a, st);
        }
        if constexpr (sizeof(T) == 2) tiles_bias<T, DB, 1, 2, true>(a, st);
    } else if constexpr (sizeof(T) == 2) {
        tiles_bias<T, DB, 1, 2, false>(a, st);
    }
}
template <typename T> void tiles_any(const StepArgs& a, uint32_t type, bool prefix, hipStream_t st) {
    switch ((a.width + 31) / 32) {
        case 1: return tiles_run<T, 1>(a, type, prefix, st);
        case 2: return tiles_run<T, 2>(a, type, prefix, st);
        case 3: return tiles_run<T, 3>(a, type, prefix, st);
        default: return tiles_run<T, 4>(a, type, prefix, st);
    }
}

}  // namespace

// Parts of a prefix of which a text is shown so many words: blocks enough to fill the device twice over, of at least a tile each.
uint32_t prefix_splits(uint32_t type, uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t words) {
    const uint32_t rows = batch * (heads / kv_heads), per_block = prefix_rows(type, rows);
    const uint32_t blocks = (rows + per_block - 1) / per_block * kv_heads, most = (words + KEYS - 1) / KEYS;
    const uint32_t want = blocks < 512 ? (512 + blocks - 1) / blocks : 1;
    return want < most ? want : most;
}

namespace {
void launch(const StepArgs& a, uint32_t type, bool prefix, hipStream_t st) {
    if (type == ELEM_F32) tiles_any<float>(a, type, prefix, st);
    else if (type == ELEM_F16) tiles_any<_Float16>(a, type, prefix, st);
    else tiles_any<__bf16>(a, type, prefix, st);
}
}  // namespace

void launch_prefix(const StepArgs& a, uint32_t type, hipStream_t st) { launch(a, type, true, st); }
void launch_own_tiles(const StepArgs& a, uint32_t type, hipStream_t st) { launch(a, type, false, st); }

}  // namespace w2v

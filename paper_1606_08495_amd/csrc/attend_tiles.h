// What the tiled attention kernels share: the words of a wavefront, the axis of keys they walk over, scores with bias and mask.
#pragma once
#include <type_traits>

#include "attend.h"
#include "tiles.h"

namespace w2v {

constexpr int BLOCK_WORDS = 128, WAVE_WORDS = 32, KEYS = 64, THREADS = 256, GROUPS = BLOCK_WORDS / WAVE_WORDS;

// Where there are fewer blocks than this, a block has twice the wavefronts, and each takes one of a tile's two pieces.
constexpr uint32_t SPLIT_BELOW = 512;
// (Not for wide heads in 32 bits, whose registers would not hold for the second wavefront on a SIMD.)
template <typename T, int DB> constexpr bool splits = sizeof(T) == 2 || DB <= 2;
constexpr size_t LDS_BYTES = 160 * 1024;              // a block's most

// A block's wavefront: which group of 32 words it has, and which half of a tile where it has one.
struct Place {
    uint32_t lane, h, wave, half;
    __device__ __forceinline__ Place() {
        const uint32_t n = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
        lane = threadIdx.x % WAVE;
        h = lane / 32;
        wave = n % GROUPS;
        half = n / GROUPS;
    }
};

// The texts of a block's first and last token and of a wavefront's.
struct Texts {
    uint32_t block_first, block_last, wave_first, wave_last;
    __device__ __forceinline__ Texts(const AttendArgs& a, uint32_t b0, uint32_t b1, uint32_t w0, uint32_t w1, uint32_t lane) {
        const uint32_t s = texts_of(a.off, a.n_sent, lane < 32 ? (lane < 16 ? b0 : b1) : (lane < 48 ? w0 : w1), lane);
        block_first = __builtin_amdgcn_readlane(s, 0);
        block_last = __builtin_amdgcn_readlane(s, 16);
        wave_first = __builtin_amdgcn_readlane(s, 32);
        wave_last = __builtin_amdgcn_readlane(s, 48);
    }
};

// A word and what it is shown, for the lanes of a wavefront; and over the wavefront's words, in scalar registers.
// (A wavefront past the last token takes that token, without weight.)
struct Words {
    uint32_t i; Shown s;
    uint32_t lo_least, lo_most, hi_least, hi_most, i_first, i_last, first_least, sunk_least;
    __device__ __forceinline__ Words(const AttendArgs& a, uint32_t first, uint32_t lane) {
        i_first = first < a.T ? first : a.T - 1;
        i_last = first + WAVE_WORDS - 1 < a.T ? first + WAVE_WORDS - 1 : a.T - 1;
        i = first + lane % WAVE_WORDS < i_last ? first + lane % WAVE_WORDS : i_last;
    }
    __device__ __forceinline__ void find(const AttendArgs& a, const Texts& t, uint32_t lane) {
        s = shown_to(a, i, text_between(a.off, t.wave_first, t.wave_last, i, a.T, lane));
        lo_least = __builtin_amdgcn_readfirstlane(s.lo);
        hi_least = __builtin_amdgcn_readfirstlane(s.hi);
        first_least = __builtin_amdgcn_readfirstlane(s.first);
        sunk_least = __builtin_amdgcn_readfirstlane(s.sunk);
        lo_most = __builtin_amdgcn_readlane(s.lo, WAVE_WORDS - 1);
        hi_most = __builtin_amdgcn_readlane(s.hi, WAVE_WORDS - 1);
    }
    // Whether any of the words is shown any of the tokens j0 .. j0 + 31.  (First words that stay visible lie before all
    // windows only for the first word's text: later texts begin at or after the first word.)
    __device__ __forceinline__ bool shown_any(uint32_t j0) const {
        return j0 < hi_most && (j0 + 32 > lo_least || (j0 < sunk_least && j0 + 32 > first_least));
    }
};

// The axis of keys of a block: `sunk` words from `first` on, then those from `lo` to the end.
struct Axis {
    uint32_t first, sunk, shift, count;
    __device__ __forceinline__ Axis(const AttendArgs& a, uint32_t word0, uint32_t last, const Texts& t) {
        const uint32_t s0 = t.block_first, s1 = t.block_last;
        const Shown from = shown_to(a, word0, text_bounds(a.off, s0, word0, a.T));
        const Shown to = shown_to(a, last, text_bounds(a.off, s1, last, a.T));
        first = from.first;
        sunk = from.sunk - from.first;
        shift = from.lo - sunk;                       // token of key n >= sunk: n + shift
        count = sunk + (to.hi > from.lo ? to.hi - from.lo : 0);
        first = __builtin_amdgcn_readfirstlane(first);
        sunk = __builtin_amdgcn_readfirstlane(sunk);
        shift = __builtin_amdgcn_readfirstlane(shift);
        count = __builtin_amdgcn_readfirstlane(count);
    }
    __device__ __forceinline__ uint32_t token(uint32_t n) const { return n < sunk ? first + n : shift + n; }
};

// Tiles [from, to) of a block's axis.
struct Tiles { uint32_t from, to; };
// Keys [from, to) of the axis that those of a wavefront's words are shown which need something: words follow each other, so do
// what they are shown.  The same in all lanes; none where from >= to.
__device__ __forceinline__ Tiles keys_of(const Words& w, const Axis& x, bool need) {
    const uint32_t who = (uint32_t)__ballot(need);
    if (!who) return Tiles{~0u, 0};
    const int one = __builtin_ctz(who), last = 31 - __builtin_clz(who);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane(w.s.lo, one), hi = (uint32_t)__builtin_amdgcn_readlane(w.s.hi, last);
    const uint32_t first = (uint32_t)__builtin_amdgcn_readlane(w.s.first, one), sunk = (uint32_t)__builtin_amdgcn_readlane(w.s.sunk, one);
    const uint32_t j = sunk > first ? first : lo;
    const uint32_t from = j - x.first < x.sunk ? j - x.first : j - x.shift, to = hi - x.shift;
    return Tiles{from < x.count ? from : x.count, to < x.count ? to : x.count};
}
// The tiles of the block's, from those of its four groups of words (behind a barrier).
__device__ __forceinline__ Tiles tiles_of(const Tiles (&groups)[GROUPS]) {
    Tiles t{~0u, 0};
#pragma unroll
    for (int n = 0; n < GROUPS; ++n) {
        t.from = groups[n].from < t.from ? groups[n].from : t.from;
        t.to = groups[n].to > t.to ? groups[n].to : t.to;
    }
    if (t.from >= t.to) return Tiles{0, 0};
    return Tiles{(uint32_t)__builtin_amdgcn_readfirstlane(t.from / KEYS), (uint32_t)__builtin_amdgcn_readfirstlane((t.to + KEYS - 1) / KEYS)};
}

// Bias by distance, times log2 e, with the outermost values repeated on both sides so that every distance within a
// 32 x 32 piece that is not wholly past the span is in the table.
constexpr int BIAS_SIDE = 64;
__host__ __device__ constexpr uint32_t bias_table(uint32_t span) { return (2 * (span + BIAS_SIDE) + 1 + 3) / 4 * 4; }
__device__ __forceinline__ void fill_bias(const AttendArgs& a, uint32_t head, float* table) {
    const int32_t reach = (int32_t)a.span + BIAS_SIDE;
    for (int32_t at = threadIdx.x; at <= 2 * reach; at += (int32_t)blockDim.x) table[at] = scaled_bias(a, head, at - reach);
}

// A value that is computed where it is used, piece by piece: what sixteen rows derive from it is not kept in registers of
// its own over the whole walk.
__device__ __forceinline__ uint32_t per_piece(uint32_t x) {
    asm volatile("" : "+v"(x));
    return x;
}

// Scores of a piece of 32 keys, masked: s on the way in holds the products.  With a bias they are to base two, without one
// they still lack the scale, which is positive.
template <bool BIAS>
__device__ __forceinline__ void piece_scores(const AttendArgs& a, const Words& w, const Axis& x, uint32_t n0, uint64_t kept, bool linear,
                                    const float* table, uint32_t h, Acc& s) {
    const uint32_t j0 = n0 + x.shift;                 // of the piece's first key where the axis is linear
    const uint32_t kept32 = (uint32_t)kept;
    const bool all = linear && j0 >= w.lo_most && j0 + 32 <= w.hi_least && kept32 == 0xFFFFFFFFu &&
                     !(a.skip_self && j0 <= w.i_last && j0 + 32 > w.i_first);
    const int32_t span = (int32_t)a.span;
    if constexpr (BIAS) {
        const int32_t reach = span + BIAS_SIDE;
        if (linear) {
            const int32_t far = (int32_t)j0 - (int32_t)w.i_first + 31, near = (int32_t)j0 - (int32_t)w.i_last;
            if (far <= -span || near >= span) {
                const float b = table[far <= -span ? 0 : 2 * reach];
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.scale2, b);
            } else {
                const float* at = table + ((int32_t)j0 - (int32_t)w.i + reach + 4 * (int32_t)h);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.scale2, at[acc_row(r, 0)]);
            }
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int32_t dist = (int32_t)x.token(per_piece(n0 + 4 * h) + acc_row(r, 0)) - (int32_t)w.i;
                s[r] = fmaf(s[r], a.scale2, table[(dist < -reach ? -reach : dist > reach ? reach : dist) + reach]);
            }
        }
    }
    if (all) return;
    const auto mask = [&](auto LINEAR) __attribute__((always_inline)) {
        const uint32_t base = per_piece((LINEAR.value ? j0 : n0) + 4 * h);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const uint32_t j = LINEAR.value ? base + acc_row(r, 0) : x.token(base + acc_row(r, 0));
            bool in = (j - w.s.lo < w.s.hi - w.s.lo) | (j - w.s.first < w.s.sunk - w.s.first);
            in &= (kept32 >> acc_row(r, h) & 1) != 0;
            in &= !(a.skip_self & (j == w.i));
            s[r] = in ? s[r] : -__builtin_inff();
        }
    };
    if (linear) mask(std::true_type{});
    else mask(std::false_type{});
}

// Keys and values of a block, tile by tile from memory to LDS, and which of the next tile's words are kept.
template <typename T, int DB, int SPLIT> struct KeyTiles {
    Transit<T, DB, KEYS, SPLIT * THREADS> k, v;
    uint8_t keep;
    // the tile that is fetched first is tile t
    __device__ __forceinline__ void start(const AttendArgs& a, uint32_t kv_head, const Axis& x, uint32_t t) {
        k.start(a.k, kv_head, (int64_t)(int32_t)x.shift + (int64_t)t * KEYS);
        v.start(a.v, kv_head, (int64_t)(int32_t)x.shift + (int64_t)t * KEYS);
        keep = 1;
    }
    __device__ __forceinline__ void fetch(const AttendArgs& a, uint32_t kv_head, const Axis& x, uint32_t t, uint32_t lane) {
        const uint32_t n0 = t * KEYS, last = x.count - 1;
        if (n0 >= x.sunk && n0 + KEYS <= x.count) {
            k.aim();
            v.aim();
        } else {
            const auto token = [&](uint32_t r) __attribute__((always_inline)) { return x.token(n0 + r < last ? n0 + r : last); };
            k.aim(token);
            v.aim(token);
        }
        k.load(a.width);
        v.load(a.width);
        if (a.keep) keep = a.keep[x.token(n0 + lane < last ? n0 + lane : last)];
    }
};

}  // namespace w2v

// Attention over texts, forward.
//
// Four products and two exponentials' worth of work per pair of words and head: for a long window the matrix cores and the
// vector units bound it, for short texts its way through memory does.  A block holds 128 consecutive words of
// the whole token stream, whichever texts they belong to -- short texts share a block instead of filling one
// each -- and walks over the words that any of them is shown: the text's first words that stay visible, then the span of
// the windows, as one axis of keys in tiles of 64 that go through LDS.  A wavefront holds 32 of the words with its
// scores transposed (keys are rows, its words are lanes): maximum and sum of a word are kept by its two lanes, and the
// weights feed the second product from the registers they are in.  Pieces of 32 keys that none of
// its words is shown are skipped, those that all of them are shown take no mask.
//
// Scores, maxima, sums and outputs are fp32.  Weights are rounded to the type of v for the second product, relative to the
// row's maximum (or to one at most 2^8 below it: outputs are rescaled only when the maximum has risen by more), which
// leaves them the relative rounding that v has; their sum is taken before the rounding.  Heads of up to 32 columns add
// what the rounding left in a second product: the gradient's dout . out is then a sum of few terms, which
// may cancel down to the weights' rounding, and the matrix cores wait for the exponentials there anyway.
#include "attend.h"
#include "tiles.h"

namespace w2v {
namespace {

constexpr int BLOCK_WORDS = 128, WAVE_WORDS = 32, KEYS = 64, THREADS = 256;
constexpr float RISE = 8.f;           // how far (to base two) a maximum may rise before outputs are rescaled

// A word and what it is shown, for the lanes of a wavefront; and over the wavefront's words, in scalar registers.
struct Words {
    uint32_t i; Shown s;
    uint32_t lo_least, lo_most, hi_least, hi_most, i_first, i_last, first_least, sunk_least;
    __device__ Words(const AttendArgs& a, uint32_t first, uint32_t lane) {
        const uint32_t last = first + WAVE_WORDS - 1 < a.T ? first + WAVE_WORDS - 1 : a.T - 1;
        i = first + lane % WAVE_WORDS < last ? first + lane % WAVE_WORDS : last;
        i_first = first < last ? first : last;
        i_last = last;
        const uint32_t s0 = text_of(a.off, a.n_sent, i_first, lane), s1 = text_of(a.off, a.n_sent, i_last, lane);
        s = shown_to(a, i, text_between(a.off, s0, s1, i, a.T));
        lo_least = __builtin_amdgcn_readfirstlane(s.lo);
        hi_least = __builtin_amdgcn_readfirstlane(s.hi);
        first_least = __builtin_amdgcn_readfirstlane(s.first);
        sunk_least = __builtin_amdgcn_readfirstlane(s.sunk);
        lo_most = __builtin_amdgcn_readlane(s.lo, WAVE_WORDS - 1);
        hi_most = __builtin_amdgcn_readlane(s.hi, WAVE_WORDS - 1);
    }
    // Whether any of the words is shown any of the tokens j0 .. j0 + 31.  (First words that stay visible lie before all
    // windows only for the first word's text: later texts begin at or after the first word.)
    __device__ bool shown_any(uint32_t j0) const {
        return j0 < hi_most && (j0 + 32 > lo_least || (j0 < sunk_least && j0 + 32 > first_least));
    }
};

// The axis of keys of a block: `sunk` words from `first` on, then those from `lo` to the end.
struct Axis {
    uint32_t first, sunk, shift, count;
    __device__ Axis(const AttendArgs& a, uint32_t word0, uint32_t lane) {
        const uint32_t last = word0 + BLOCK_WORDS - 1 < a.T ? word0 + BLOCK_WORDS - 1 : a.T - 1;
        const uint32_t s0 = text_of(a.off, a.n_sent, word0, lane), s1 = text_of(a.off, a.n_sent, last, lane);
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
    __device__ uint32_t token(uint32_t n) const { return n < sunk ? first + n : shift + n; }
};

// Bias by distance, times log2 e, with the outermost values repeated on both sides so that every distance within a
// 32 x 32 piece that is not wholly past the span is in the table.
constexpr int BIAS_SIDE = 64, BIAS_TABLE = 2 * SPAN_MAX + 1 + 2 * BIAS_SIDE;
__device__ inline void fill_bias(const AttendArgs& a, uint32_t head, float* table) {
    const int32_t reach = (int32_t)a.span + BIAS_SIDE;
    for (int32_t at = threadIdx.x; at <= 2 * reach; at += THREADS) table[at] = scaled_bias(a, head, at - reach);
}

// Scores of a piece of 32 keys, with bias and mask: s on the way in holds the products.
template <bool BIAS>
__device__ inline void piece_scores(const AttendArgs& a, const Words& w, const Axis& x, uint32_t n0, uint64_t kept, bool linear,
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
                const int32_t dist = (int32_t)x.token(n0 + acc_row(r, h)) - (int32_t)w.i;
                s[r] = fmaf(s[r], a.scale2, table[(dist < -reach ? -reach : dist > reach ? reach : dist) + reach]);
            }
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= a.scale2;
    }
    if (all) return;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const uint32_t row = acc_row(r, h), j = linear ? j0 + row : x.token(n0 + row);
        bool in = (j - w.s.lo < w.s.hi - w.s.lo) | (j - w.s.first < w.s.sunk - w.s.first);
        in &= (kept32 >> row & 1) != 0;
        in &= !(a.skip_self && j == w.i);
        s[r] = in ? s[r] : -__builtin_inff();
    }
}

template <typename T, int DB, bool BIAS>
__global__ __launch_bounds__(THREADS) void attend_kernel(const AttendArgs a) {
    typedef Tile<T, DB, KEYS> Tl;
    constexpr int BUFFERS = 2 * 2 * Tl::BYTES <= 128 * 1024 ? 2 : 1;
    __shared__ __align__(16) char tiles[BUFFERS][2][Tl::BYTES];
    __shared__ float table[BIAS ? BIAS_TABLE : 1];
    const uint32_t lane = threadIdx.x % WAVE, h = lane / 32, wave = threadIdx.x / WAVE;
    const uint32_t head = blockIdx.x % a.heads, kv_head = head / a.group;
    const uint32_t words = (a.T + BLOCK_WORDS - 1) / BLOCK_WORDS;
    const uint32_t word0 = (words - 1 - blockIdx.x / a.heads) * BLOCK_WORDS;      // those that may see most first
    const Axis x(a, word0, lane);
    const uint32_t first = word0 + wave * WAVE_WORDS;
    const Words w(a, first < a.T ? first : a.T - 1, lane);
    const bool some = first < a.T;                    // the block's last wavefronts may have no word
    if (BIAS) fill_bias(a, head, table);

    typename Frag<T>::vec q[2 * DB];
#pragma unroll
    for (int s = 0; s < 2 * DB; ++s) q[s] = load_operand(head_row<T>(a.q, w.i, head), s, h, a.width);
    Acc o[DB];
#pragma unroll
    for (int b = 0; b < DB; ++b) o[b] = Acc{};
    float m = -__builtin_inff(), total = 0.f;

    Transit<T, DB, KEYS, THREADS> tk, tv;
    uint8_t keep = 1;
    const uint32_t count = (x.count + KEYS - 1) / KEYS;
    const auto fetch = [&](uint32_t t) {
        const auto row = [&](const Heads& p, uint32_t r) -> const T* {
            const uint32_t n = t * KEYS + r;
            if (n >= x.count) return nullptr;
            const uint32_t j = x.token(n);
            return a.keep && !a.keep[j] ? nullptr : head_row<T>(p, j, kv_head);
        };
        tk.load([&](uint32_t r) { return row(a.k, r); }, a.width);
        tv.load([&](uint32_t r) { return row(a.v, r); }, a.width);
        if (a.keep) keep = t * KEYS + lane < x.count ? a.keep[x.token(t * KEYS + lane)] : 0;
    };
    uint64_t kept = ~0ull;
    if (count) {
        fetch(0);
        tk.store(tiles[0][0]);
        tv.store(tiles[0][1]);
        kept = __ballot(keep != 0);
    }
    __syncthreads();
    for (uint32_t t = 0; t < count; ++t) {
        if (t + 1 < count) fetch(t + 1);
        const char *kt = tiles[t % BUFFERS][0], *vt = tiles[t % BUFFERS][1];
#pragma unroll
        for (uint32_t piece = 0; piece < KEYS / 32; ++piece) {
            const uint32_t n0 = t * KEYS + piece * 32;
            const bool linear = n0 >= x.sunk;
            if (!some || n0 >= x.count || (linear && !w.shown_any(n0 + x.shift))) continue;
            Acc s = {};
#pragma unroll
            for (int k = 0; k < 2 * DB; ++k) mma(Tl::along(kt, piece * 32 + lane % 32, k, h), q[k], s);
            piece_scores<BIAS>(a, w, x, n0, kept >> (piece * 32), linear, table, h, s);
            float most = s[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) most = fmaxf(most, s[r]);
            most = halves_max(most);
            if (__any(most > m + RISE)) {
                const float to = fmaxf(m, most);
                const float factor = to == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m - to);
                m = to;
                total *= factor;
#pragma unroll
                for (int b = 0; b < DB; ++b) o[b] *= factor;
            }
            const float base = m == -__builtin_inff() ? 0.f : m;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = __builtin_amdgcn_exp2f(s[r] - base);
                total += s[r];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const auto p = acc_operand<T>(s, k);
                typename Frag<T>::vec v[DB];
#pragma unroll
                for (int b = 0; b < DB; ++b) {
                    v[b] = Tl::across(vt, piece * 32, k, b, lane);
                    mma(v[b], p, o[b]);
                }
                if constexpr (sizeof(T) == 2 && DB == 1) {      // what the rounding left of the weights
                    typename Frag<T>::vec rest;
#pragma unroll
                    for (int t = 0; t < 8; ++t) rest[t] = (T)(s[8 * k + t] - (float)p[t]);
                    mma(v[0], rest, o[0]);
                }
            }
        }
        if (t + 1 < count) {
            if (BUFFERS == 1) __syncthreads();
            tk.store(tiles[(t + 1) % BUFFERS][0]);
            tv.store(tiles[(t + 1) % BUFFERS][1]);
            kept = __ballot(keep != 0);
            __syncthreads();
        }
    }
    if (!some) return;

    total = halves_sum(total);
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const bool real = first + lane % WAVE_WORDS < a.T;
    float worst = 0.f;                                // not a number, if any result is not finite
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            o[b][r] *= inv;
            worst = fmaf(o[b][r], 0.f, worst);
        }
    worst = halves_sum(worst);
    const bool redo = worst != 0.f;
    if (real && !redo) {
        T* out = head_row<T>(a.o, w.i, head);
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const uint32_t c = 32 * b + acc_row(r, h);
                typename Pack<T, 4>::vec four;
#pragma unroll
                for (int e = 0; e < 4; ++e) four[e] = (T)o[b][r + e];
                if (c + 4 <= a.width) *(typename Pack<T, 4>::mem*)(out + c) = four;
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e) if (c + e < a.width) out[c + e] = four[e];
            }
        if (h == 0 && a.lse)
            a.lse[(size_t)head * a.T + w.i] = total == 0.f ? -__builtin_inff() : (m + __builtin_log2f(total)) * LN2;
    }
    // what a word is not shown must not show: rows that are not finite are formed from their words alone
    for (uint64_t rows = __ballot(redo && real && h == 0); rows; rows &= rows - 1) {
        const int l = __builtin_ctzll(rows);
        Shown s;
        s.lo = __shfl(w.s.lo, l, 64); s.hi = __shfl(w.s.hi, l, 64);
        s.first = __shfl(w.s.first, l, 64); s.sunk = __shfl(w.s.sunk, l, 64);
        const uint32_t i = __shfl(w.i, l, 64);
        float row[2], lse;
        attend_row<T>(a, head, i, s, lane, row, lse);
        T* out = head_row<T>(a.o, i, head);
#pragma unroll
        for (int c = 0; c < 2; ++c) if (lane + c * WAVE < a.width) out[lane + c * WAVE] = (T)row[c];
        if (lane == 0 && a.lse) a.lse[(size_t)head * a.T + i] = lse;
    }
}

template <typename T, int DB> void attend_run(const AttendArgs& a, hipStream_t st) {
    const uint32_t blocks = (a.T + BLOCK_WORDS - 1) / BLOCK_WORDS * a.heads;
    if (a.bias) attend_kernel<T, DB, true><<<blocks, THREADS, 0, st>>>(a);
    else attend_kernel<T, DB, false><<<blocks, THREADS, 0, st>>>(a);
}
template <typename T> void attend_any(const AttendArgs& a, hipStream_t st) {
    switch ((a.width + 31) / 32) {
        case 1: return attend_run<T, 1>(a, st);
        case 2: return attend_run<T, 2>(a, st);
        case 3: return attend_run<T, 3>(a, st);
        default: return attend_run<T, 4>(a, st);
    }
}

}  // namespace

void launch_attend(const AttendArgs& a, uint32_t type, hipStream_t st) {
    if (type == ELEM_F32) attend_any<float>(a, st);
    else if (type == ELEM_F16) attend_any<_Float16>(a, st);
    else attend_any<__bf16>(a, st);
}

}  // namespace w2v

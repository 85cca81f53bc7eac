// Attention over texts, forward.
//
// Two products (four operations a column) and an exponential per pair of words and head: for a long window the matrix cores and the
// vector units bound it, for short texts its way through memory does.  A block holds 128 consecutive words of
// the whole token stream, whichever texts they belong to -- short texts share a block instead of filling one
// each -- and walks over the words that any of them is shown: the text's first words that stay visible, then the span of
// the windows, as one axis of keys in tiles of 64 that go through LDS.  A wavefront holds 32 of the words with its
// scores transposed (keys are rows, its words are lanes): maximum and sum of a word are kept by its two lanes, and the
// weights feed the second product from the registers they are in.  Pieces of 32 keys that none of
// its words is shown are skipped, those that all of them are shown take no mask.
//
// Scores, maxima, sums and outputs are fp32.  Weights are rounded to the type of v for the second product, relative to the
// row's maximum (or to one a little below it: outputs are rescaled only when the maximum has risen by more, see RISE), which
// leaves them the relative rounding that v has; their sum is taken before the rounding.  Heads of up to 32 columns add
// what the rounding left in a second product: the gradient's dout . out is then a sum of few terms, which
// may cancel down to the weights' rounding, and the matrix cores wait for the exponentials there anyway.
//
// Measured: 32768 words, 16 heads of 128 over 4, 16 bits, window of 1024: 480 us (567 TFLOP/s of the pairs shown; products
// and exponentials take turns in the two wavefronts of a SIMD).  131333 words in texts of 10 to 40, 5 heads of 60, 32 bits, window
// of 10 on either side: 370 us (633 MB; a block's chain of dependent accesses).
#include "attend_tiles.h"

namespace w2v {
namespace {

// How far (to base two) a maximum may rise before outputs are rescaled, and what weights are lifted by before they are rounded.
// fp16 would lose weights below 2^-25 of the row's maximum altogether, of which a long text may hold 10^5, and round those below 2^-14
// coarsely; lifted, these are 2^-38 and 2^-27, and none is above 2^15.
template <typename T> constexpr float RISE = std::is_same<T, _Float16>::value ? 2.f : 8.f;
template <typename T> constexpr float LIFT = std::is_same<T, _Float16>::value ? 13.f : 0.f;

template <typename T, int DB, bool BIAS, int SPLIT>
__global__ __launch_bounds__(SPLIT * THREADS, ((splits<T, DB>) ? 2 : 1)) void attend_kernel(const AttendArgs a) {
    typedef Tile<T, DB, KEYS> Tl;
    constexpr int BUFFERS = 2 * 2 * Tl::BYTES <= 72 * 1024 ? 2 : 1, KEEP = DB * 16 + 2;
    constexpr bool JOINT = DB <= 2;      // both pieces of a tile at a time, where registers allow
    __shared__ __align__(16) char tiles[BUFFERS][2][Tl::BYTES];
    static_assert(SPLIT == 1 || GROUPS * KEEP * WAVE * 4 <= (int)sizeof(tiles), "room to join the halves");
    extern __shared__ float table[];
    const Place place;
    const uint32_t lane = place.lane, h = place.h, wave = place.wave, half = place.half;
    const uint32_t head = blockIdx.x % a.heads, kv_head = head / a.group;
    const uint32_t words = (a.T + BLOCK_WORDS - 1) / BLOCK_WORDS;
    const uint32_t word0 = (words - 1 - blockIdx.x / a.heads) * BLOCK_WORDS;      // those that may see most first
    const uint32_t first = word0 + wave * WAVE_WORDS, last = word0 + BLOCK_WORDS - 1 < a.T ? word0 + BLOCK_WORDS - 1 : a.T - 1;
    Words w(a, first, lane);
    const bool some = first < a.T;                    // the block's last wavefronts may have no word

    typename Frag<T>::vec q[2 * DB];
#pragma unroll
    for (int s = 0; s < 2 * DB; ++s) q[s] = load_operand<T, DB>(head_row<T>(a.q, w.i, head), s, h, a.width);
    const Texts texts(a, word0, last, w.i_first, w.i_last, lane);
    const Axis x(a, word0, last, texts);
    w.find(a, texts, lane);
    if (BIAS) fill_bias(a, head, table);
    Acc o[DB];
#pragma unroll
    for (int b = 0; b < DB; ++b) o[b] = Acc{};
    float m = -__builtin_inff(), total = 0.f;
    const float unit = BIAS ? 1.f : a.scale2;         // of the scores as piece_scores leaves them
    // a half's piece of every tile is the same one: its rows are part of the lane's bases
    const uint32_t own_rows = SPLIT == 2 ? half * 32 : 0;
    const uint32_t at_along = Tl::base_along(lane) + own_rows / 4 * Tl::STRIDE, at_across = Tl::base_across(lane) + own_rows / 4 * Tl::STRIDE;

    KeyTiles<T, DB, SPLIT> next;
    const uint32_t count = (x.count + KEYS - 1) / KEYS;
    next.start(a, kv_head, x, 0);
    uint64_t kept = ~0ull;
    if (count) {
        next.fetch(a, kv_head, x, 0, lane);
        kept = __ballot(next.keep != 0);
        next.k.store(tiles[0][0], a.width);
        next.v.store(tiles[0][1], a.width, kept);
    }
    __syncthreads();
    for (uint32_t t = 0; t < count; ++t) {
        if (t + 1 < count) next.fetch(a, kv_head, x, t + 1, lane);
        const char *kt = tiles[t % BUFFERS][0], *vt = tiles[t % BUFFERS][1];
        // P pieces of 32 keys from piece p0 on
        const auto pieces = [&](auto P, int p0) __attribute__((always_inline)) {
            Acc s[P.value];
#pragma unroll
            for (int p = 0; p < P.value; ++p) s[p] = Acc{};
#pragma unroll
            for (int k = 0; k < 2 * DB; ++k)
#pragma unroll
                for (int p = 0; p < P.value; ++p) mma(Tl::along(kt, at_along, (p0 + p) * 32, k), q[k], s[p]);
            float most = -__builtin_inff();
#pragma unroll
            for (int p = 0; p < P.value; ++p) {
                const uint32_t n0 = t * KEYS + (p0 + p) * 32 + own_rows;
                piece_scores<BIAS>(a, w, x, n0, kept >> ((p0 + p) * 32 + own_rows), n0 >= x.sunk, table, h, s[p]);
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, s[p][r]);
            }
            most = halves_max(most) * unit;
            if (__any(most > m + RISE<T>)) {
                const float to = fmaxf(m, most);
                const float factor = to == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m - to);
                m = to;
                total *= factor;
#pragma unroll
                for (int b = 0; b < DB; ++b) o[b] *= factor;
            }
            const float base = m == -__builtin_inff() ? 0.f : m - LIFT<T>;
            // What is summed here is the pieces' first, then the whole row's: a long row would make one long chain of roundings.
            // (In 16 bits that of the weights hides the chain of o.)
            float sum = 0.f;
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int p = 0; p < P.value; ++p)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        s[p][r] = __builtin_amdgcn_exp2f(fmaf(s[p][r], unit, -base));
                        sum += s[p][r];
                    }
#pragma unroll
                for (int b = 0; b < DB; ++b) {
                    Acc part = {};
#pragma unroll
                    for (int g = 0; g < 2 * P.value; ++g)
                        mma(Tl::across(vt, at_across, (p0 + g / 2) * 32, g % 2, b), acc_operand<T>(s[g / 2], g % 2), part);
                    o[b] += part;
                }
                total += sum;
                return;
            }
#pragma unroll
            for (int g = 0; g < 2 * P.value; ++g) {   // 16 keys
                const int p = g / 2;
                typename Frag<T>::vec e;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const float y = __builtin_amdgcn_exp2f(fmaf(s[p][8 * (g % 2) + c], unit, -base));
                    sum += y;
                    e[c] = (T)y;
                    s[p][8 * (g % 2) + c] = y;
                }
                typename Frag<T>::vec v[DB];
#pragma unroll
                for (int b = 0; b < DB; ++b) {
                    v[b] = Tl::across(vt, at_across, (p0 + p) * 32, g % 2, b);
                    mma(v[b], e, o[b]);
                }
                if constexpr (sizeof(T) == 2 && DB == 1) {      // what the rounding left of the weights
                    typename Frag<T>::vec rest;
#pragma unroll
                    for (int c = 0; c < 8; ++c) rest[c] = (T)(s[p][8 * (g % 2) + c] - (float)e[c]);
                    mma(v[0], rest, o[0]);
                }
            }
            total += sum;
        };
        const auto needs = [&](uint32_t piece) __attribute__((always_inline)) {
            const uint32_t n0 = t * KEYS + piece * 32 + own_rows;
            return some && n0 < x.count && (n0 < x.sunk || w.shown_any(n0 + x.shift));
        };
        if constexpr (SPLIT == 2) {
            if (needs(0)) pieces(std::integral_constant<int, 1>{}, 0);
        } else {
            const bool n0 = needs(0), n1 = needs(1);
            if (JOINT && n0 && n1) pieces(std::integral_constant<int, JOINT ? 2 : 1>{}, 0);
            else {
                if (n0) pieces(std::integral_constant<int, 1>{}, 0);
                if (n1) pieces(std::integral_constant<int, 1>{}, 1);
            }
        }
        if (t + 1 < count) {
            if (BUFFERS == 1) __syncthreads();
            kept = __ballot(next.keep != 0);
            next.k.store(tiles[(t + 1) % BUFFERS][0], a.width);
            next.v.store(tiles[(t + 1) % BUFFERS][1], a.width, kept);
            __syncthreads();
        }
    }
    if constexpr (SPLIT == 2) {                       // the second half's sums through LDS to the first
        float* const other = (float*)&tiles[0][0][0] + wave * KEEP * WAVE + lane;
        __syncthreads();
        if (half) {
            other[0] = m;
            other[WAVE] = total;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) other[(2 + b * 16 + r) * WAVE] = o[b][r];
        }
        __syncthreads();
        if (half) return;
        const float m1 = other[0], to = fmaxf(m, m1);
        const float f0 = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m - to);
        const float f1 = m1 == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m1 - to);
        // (a maximum is -infinity where a half has seen nothing: its sums are zero; not a number stays where it is)
        total = total * (total == 0.f ? 1.f : f0) + other[WAVE] * (other[WAVE] == 0.f ? 1.f : f1);
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[b][r] = o[b][r] * f0 + other[(2 + b * 16 + r) * WAVE] * f1;
        m = to;
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
    const bool redo = worst != 0.f || (BIAS && total != 0.f && fabsf(m) >= HELD);
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
            a.lse[(size_t)head * a.T + w.i] = total == 0.f ? -__builtin_inff() : (m - LIFT<T> + __builtin_log2f(total)) * LN2;
    }
    // what a word is not shown must not show: rows that are not finite are formed from their words alone
    uint64_t rows = __ballot(redo && real && h == 0);
    if (rare(rows)) for (; rows; rows &= rows - 1) {
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

template <typename T, int DB, bool BIAS> void attend_bias(const AttendArgs& a, hipStream_t st) {
    const uint32_t blocks = (a.T + BLOCK_WORDS - 1) / BLOCK_WORDS * a.heads, table = BIAS ? bias_table(a.span) * sizeof(float) : 0;
    if constexpr (splits<T, DB>)
        if (blocks < SPLIT_BELOW) return attend_kernel<T, DB, BIAS, 2><<<blocks, 2 * THREADS, table, st>>>(a);
    attend_kernel<T, DB, BIAS, 1><<<blocks, THREADS, table, st>>>(a);
}
template <typename T, int DB> void attend_run(const AttendArgs& a, hipStream_t st) {
    if (a.bias) attend_bias<T, DB, true>(a, st);
    else attend_bias<T, DB, false>(a, st);
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

// Attention over texts, backward.
//
//   dS = p (dP - delta),  dP = dout v^T,  delta = rowsum(dout out)
//   dq = scale dS k,  dk = scale dS^T q,  dv = p^T dout,  dbias[b] = sum of dS over the pairs of bucket b
// Weights are formed anew from q, k and the rows' logarithms, or what these are made of where they are large (attend.h).
// No sum is shared between blocks, so no atomics and the same bits every time: one kernel holds 128 words as queries and walks over their keys (dq, and the bias' sums; three
// products a pair), another holds 128 words as keys and walks over the queries they are shown to (dk, dv; four products a
// pair).  That is seven products instead of the five of a kernel that adds dq up in memory.  In both a
// wavefront's own 32 words are the lanes, their rows feed the B operands from registers, and p and dS feed the last
// products from the registers they are formed in; p and dS are rounded to the rows' type there (in fp16 behind a power of two, see lift_piece), all sums are fp32.
//
// A text's first words that stay visible are seen by every later word.  The keys' kernel takes the queries up to a
// border behind its block; those behind go in pieces to blocks of their own (late), whose sums are joined in
// order at the end.
//
// Measured, forward and backward: 9139 words in whole texts, 6 heads of 100, fp16 603 us (in a profile: forward 176, queries' kernel
// 219, keys' 256); 17676 words, 8 heads of 64 over 2, window of 512, bias and its gradient, bf16 471 us; 65135 words in texts of
// 10 to 40, 5 heads of 60, 32 bits, bias 884 us.  Vector work and latency bound them.
// In 16 bits the queries' kernel of heads wider than 96 keeps 48 to 108 bytes a lane in scratch, the keys' up to 60.
#include "attend_tiles.h"

namespace w2v {
namespace {

// What is stored of a lane's column of results: row `to` of `width` elements, c[b] rows 32 b + acc_row.
template <typename T, int DB> __device__ inline void store_column(T* to, uint32_t width, const Acc (&c)[DB], float factor, uint32_t h) {
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const uint32_t at = 32 * b + acc_row(r, h);
            typename Pack<T, 4>::vec four;
#pragma unroll
            for (int e = 0; e < 4; ++e) four[e] = (T)(c[b][r + e] * factor);
            if (at + 4 <= width) *(typename Pack<T, 4>::mem*)(to + at) = four;
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) if (at + e < width) to[at + e] = four[e];
        }
}
// Whether a lane's column, both halves of it, holds a value that is not finite.
template <int DB> __device__ inline bool not_finite(const Acc (&c)[DB]) {
    float worst = 0.f;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) worst = fmaf(c[b][r], 0.f, worst);
    return halves_sum(worst) != 0.f;
}

// fp16 holds 2^-24 .. 2^16, and dS = p (dP - delta) is as small as the outputs' gradient over the number of words: rounded as it
// is, a mean's gradient over some thousand words would lose most of its bits.  Before it is rounded, a word's dS (a lane's column)
// is therefore multiplied by a power of two, `lift`, which its sums carry too: as high as its largest value so far allows, so
// that this one lies at 2^9 or above, terms down to 2^-23 of it keep all bits, and none overflows.  Weights as they enter dv's products
// are lifted by 2^14 from the start: none is above one.  (bf16 and fp32 have fp32's range and need neither.)
template <typename T> constexpr bool lifts = std::is_same<T, _Float16>::value;
template <typename T> constexpr float WEIGHT_LIFT = lifts<T> ? 14.f : 0.f;      // to base two
constexpr float FIRST_LIFT = 0x1p100f, LIFTED_MOST = 0x1p15f;
template <int N> __device__ __forceinline__ void lift_piece(Acc& ds, Acc (&sum)[N], float& lift) {
    float most = fabsf(ds[0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) most = fmaxf(most, fabsf(ds[r]));
    most = halves_max(most);
    if (rare(__any(most * lift >= LIFTED_MOST))) {
        const float to = most * lift >= LIFTED_MOST ? __builtin_amdgcn_ldexpf(1.f, 10 - __builtin_amdgcn_frexp_expf(most)) : lift;
        const float factor = to / lift;
#pragma unroll
        for (int n = 0; n < N; ++n) sum[n] *= factor;
        lift = to;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) ds[r] *= lift;
}

// Joins what two halves of a block have summed for the same words: the second's through LDS to the first.  True for the half
// that goes on with the sums.  A place for each of the block's four groups of words.
template <int N> __device__ __forceinline__ bool join_halves(float* room, Acc (&c)[N], uint32_t wave, uint32_t half, uint32_t lane) {
    float* const other = room + wave * N * 16 * WAVE + lane;
    __syncthreads();
    if (half)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) other[(n * 16 + r) * WAVE] = c[n][r];
    __syncthreads();
    if (half) return false;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) c[n][r] += other[(n * 16 + r) * WAVE];
    return true;
}

// ---- queries: dq, delta, the bias' sums -----------------------------------------------------------------
// delta is taken from out as it was rounded, or, where that would show, formed from the scores in a pass of its own before the
// others (sum of p dP, which needs neither out nor its rounding): for the bias' gradient, an fp32 sum over all pairs, and for
// words that are shown few others (kept or not), whose out is large.  Which it is depends on the word alone, not on
// those that share its block.  With normal inputs, out's rounding adds to the error of dq, whose own rounding and dS' make most of
// it: 56 % of it at 2 words, 10 % at 8, 3 % at 32, 2 % at 64, below 1.5 % from 128 on.
constexpr uint32_t EXACT_WORDS = 128;

// Sums of dS by distance.  A piece's 32 x 32 values have 63 distances.  They go through LDS, each row moved by its number so that a
// distance is a column (SKEW floats a row; what a row does not fill stays zero), and a lane adds up one column.
// (Atomic adds in LDS take a cycle a lane: sixteen times that.)
constexpr int SKEW = 64, SKEW_FLOATS = 32 * SKEW;

// LDS of a block beside what depends on the span: tiles, in whose place the halves are joined, and what its wavefronts exchange.
template <typename T, int DB, bool BIAS, int SPLIT> struct QueryRoom {
    static constexpr int PAIR = 2 * Tile<T, DB, KEYS>::BYTES, BUFFERS = 2 * PAIR <= (BIAS ? 40 : 72) * 1024 ? 2 : 1;
    static constexpr int JOINED = SPLIT == 2 ? GROUPS * DB * 16 * WAVE * 4 : 0;
    __attribute__((aligned(16))) char tiles[BUFFERS * PAIR > JOINED ? BUFFERS * PAIR : JOINED];
    typedef float OfWords[SPLIT][SPLIT == 2 ? GROUPS : 1][SPLIT == 2 ? WAVE_WORDS : 1];      // (nothing to exchange in one half)
    OfWords deltas, largest;
    Tiles far_keys[GROUPS], delta_keys[GROUPS];
};

template <typename T, int DB, bool BIAS, int SPLIT>
__global__ __launch_bounds__(SPLIT * THREADS, ((splits<T, DB>) ? 2 : 1)) void query_kernel(const BackwardArgs b) {
    const AttendArgs& a = b.a;
    typedef Tile<T, DB, KEYS> Tl;
    typedef QueryRoom<T, DB, BIAS, SPLIT> Room;
    constexpr int BUFFERS = Room::BUFFERS;
    __shared__ Room room;
    auto& tiles = room.tiles;
    auto &deltas = room.deltas, &largest = room.largest;
    auto &far_keys = room.far_keys, &delta_keys = room.delta_keys;
    extern __shared__ float dynamic[];
    const int32_t span = (int32_t)a.span, reach = span + BIAS_SIDE;
    const Place place;
    const uint32_t lane = place.lane, h = place.h, wave = place.wave, half = place.half;
    const uint32_t head = blockIdx.x % a.heads, kv_head = head / a.group;
    const uint32_t words = (a.T + BLOCK_WORDS - 1) / BLOCK_WORDS;
    const uint32_t part = words - 1 - blockIdx.x / a.heads, word0 = part * BLOCK_WORDS;
    const uint32_t first = word0 + wave * WAVE_WORDS, last = word0 + BLOCK_WORDS - 1 < a.T ? word0 + BLOCK_WORDS - 1 : a.T - 1;
    Words w(a, first, lane);
    const bool some = first < a.T, real = first + lane % WAVE_WORDS < a.T;

    typename Frag<T>::vec q[2 * DB], g[2 * DB];
    float delta = 0.f;
#pragma unroll
    for (int s = 0; s < 2 * DB; ++s) {
        q[s] = load_operand<T, DB>(head_row<T>(a.q, w.i, head), s, h, a.width);
        g[s] = load_operand<T, DB>(head_row<T>(b.dout, w.i, head), s, h, a.width);
        const auto o = load_operand<T, DB>((const T*)head_row<T>(a.o, w.i, head), s, h, a.width);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            delta = fmaf((float)g[s][t], (float)o[t], delta);
            if (!real) g[s][t] = (T)0.f;              // lanes past the last word repeat it, without weight
        }
    }
    delta = real ? halves_sum(delta) : 0.f;
    const float lse = a.lse[(size_t)head * a.T + w.i];
    const bool far = real && is_far(lse);
    float high = lse == -__builtin_inff() ? 0.f : lse * LOG2E, low = 0.f;      // (0: of a word that is shown nothing, every score is masked)
    const Texts texts(a, word0, last, w.i_first, w.i_last, lane);
    const Axis x(a, word0, last, texts);
    w.find(a, texts, lane);
    float* const table = dynamic;
    float* const skew = dynamic + bias_table(a.span) + (half * GROUPS + wave) * (SKEW_FLOATS + bias_table(a.span));
    float* const sums = skew + SKEW_FLOATS;
    if (BIAS) {
        fill_bias(a, head, table);
        if (b.dbias) for (int32_t c = lane; c < SKEW_FLOATS + (int32_t)bias_table(a.span); c += WAVE) skew[c] = 0.f;
    }
    const float unit = BIAS ? 1.f : a.scale2;
    // a half's piece of every tile is the same one: its rows are part of the lane's bases
    const uint32_t own_rows = SPLIT == 2 ? half * 32 : 0;
    const uint32_t at_along = Tl::base_along(lane) + own_rows / 4 * Tl::STRIDE, at_across = Tl::base_across(lane) + own_rows / 4 * Tl::STRIDE;

    KeyTiles<T, DB, SPLIT> next;
    const uint32_t count = (x.count + KEYS - 1) / KEYS;
    const bool exact = sizeof(T) == 2 && real &&
                       ((BIAS && b.dbias) || w.s.hi - w.s.lo + w.s.sunk - w.s.first <= EXACT_WORDS);
    const bool some_exact = __any(exact);
    // Passes over tiles [from, to): LOGARITHMS are formed anew where they are far, then DELTA, then the GRADIENTS.
    constexpr int LOGARITHMS = 0, DELTA = 1, GRADIENTS = 2;
    bool walked = false;
    float formed = 0.f, most = -__builtin_inff(), total = 0.f, before = 0.f, after = 0.f;
    float share = 1.f;                                // 2^-low
    float lift = lifts<T> ? FIRST_LIFT : 1.f;
    Acc dq[DB];
#pragma unroll
    for (int n = 0; n < DB; ++n) dq[n] = Acc{};
    const auto walk = [&](auto PASS, const Tiles range) __attribute__((always_inline)) {
        constexpr int pass = PASS.value;
        if (range.from >= range.to) return;
        next.start(a, kv_head, x, range.from);
        next.fetch(a, kv_head, x, range.from, lane);
        if (walked) __syncthreads();                  // the last tiles of the pass before
        walked = true;
        uint64_t kept = __ballot(next.keep != 0);
        next.k.store(tiles + range.from % BUFFERS * 2 * Tl::BYTES, a.width, kept);
        next.v.store(tiles + range.from % BUFFERS * 2 * Tl::BYTES + Tl::BYTES, a.width, kept);
        __syncthreads();
        for (uint32_t t = range.from; t < range.to; ++t) {
            if (t + 1 < range.to) next.fetch(a, kv_head, x, t + 1, lane);
            const char *kt = tiles + t % BUFFERS * 2 * Tl::BYTES, *vt = kt + Tl::BYTES;
            const auto one = [&](uint32_t piece) __attribute__((always_inline)) {
                const uint32_t row0 = piece * 32 + own_rows, n0 = t * KEYS + row0, j0 = n0 + x.shift;
                const char *kp = kt + piece * (32 / 4) * Tl::STRIDE, *vp = vt + piece * (32 / 4) * Tl::STRIDE;
                const bool linear = n0 >= x.sunk;
                if (!some || n0 >= x.count || (linear && !w.shown_any(j0))) return;
                if (pass == DELTA && !some_exact) return;
                Acc s = {}, dp = {};
#pragma unroll
                for (int k = 0; k < 2 * DB; ++k) {
                    mma(Tl::along(kp, at_along, 0, k), q[k], s);
                    if constexpr (pass != LOGARITHMS) mma(Tl::along(vp, at_along, 0, k), g[k], dp);
                }
                piece_scores<BIAS>(a, w, x, n0, kept >> row0, linear, table, h, s);
                if constexpr (pass == LOGARITHMS) {
                    float to = s[0];
#pragma unroll
                    for (int r = 1; r < 16; ++r) to = fmaxf(to, s[r]);
                    to = fmaxf(most, halves_max(to) * unit);
                    if (to == -__builtin_inff()) return;      // (the same in a word's two lanes)
                    total *= __builtin_amdgcn_exp2f(most - to);
                    most = to;
                    float sum = 0.f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(fmaf(s[r], unit, -most));
                    total += sum;
                    return;
                }
                if constexpr (pass == DELTA) {
                    float sum = 0.f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(s[r], unit, -high));
                        sum = fmaf(p, p == 0.f ? 0.f : dp[r], sum);
                    }
                    formed += sum;
                    return;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[r], unit, -high));      // 2^low times the weight
                    s[r] = p * fmaf(dp[r], share, -delta);
                    if (BIAS && p == 0.f) s[r] = 0.f;     // the sums by distance are not formed anew
                }
                if constexpr (BIAS) {
                    if (b.dbias) {
                        const int32_t distant = (int32_t)j0 - (int32_t)w.i_first + 31, near = (int32_t)j0 - (int32_t)w.i_last;
                        if (linear && (distant <= -span || near >= span)) {
                            float all = 0.f;
#pragma unroll
                            for (int r = 0; r < 16; ++r) all += s[r];
                            if (distant <= -span) before += all; else after += all;
                        } else if (linear) {
                            float* const to = skew + 4 * h * (SKEW + 1) + 31 - lane % 32;
#pragma unroll
                            for (int r = 0; r < 16; ++r) to[acc_row(r, 0) * (SKEW + 1)] = s[r];
                            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                            float all = 0.f;
#pragma unroll
                            for (int n = 0; n < 32; ++n) all += skew[n * SKEW + lane];
                            // column c: distance j0 - i_first - 31 + c
                            if (lane < 63) sums[(int32_t)j0 - (int32_t)w.i_first - 31 + (int32_t)lane + reach] += all;
                            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                        } else {
// the piece where the first words and the window meet: one half after the other, no place twice at a time
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const int32_t dist = (int32_t)x.token(per_piece(n0 + 4 * h) + acc_row(r, 0)) - (int32_t)w.i;
                                const bool inside = dist > -span && dist < span;
                                before += dist <= -span ? s[r] : 0.f;
                                after += dist >= span ? s[r] : 0.f;
                                float* const to = sums + (inside ? dist + reach : 0);
                                if (inside && h == 0) __hip_atomic_fetch_add(to, s[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
                                if (inside && h == 1) __hip_atomic_fetch_add(to, s[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
                            }
                        }
                    }
                }
                if constexpr (lifts<T>) lift_piece(s, dq, lift);
                if constexpr (sizeof(T) == 4) {
                    // a piece's sum first, then to the whole: a long row would make one long chain of roundings
#pragma unroll
                    for (int n = 0; n < DB; ++n) {
                        Acc part = {};
#pragma unroll
                        for (int k = 0; k < 2; ++k) mma(Tl::across(kp, at_across, 0, k, n), acc_operand<T>(s, k), part);
                        dq[n] += part;
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const auto ds = acc_operand<T>(s, k);
#pragma unroll
                        for (int n = 0; n < DB; ++n) mma(Tl::across(kp, at_across, 0, k, n), ds, dq[n]);
                    }
                }
            };
            if constexpr (SPLIT == 2) one(0);
            else
#pragma unroll 1
                for (uint32_t piece = 0; piece < KEYS / 32; ++piece) one(piece);
            if (t + 1 < range.to) {
                if (BUFFERS == 1) __syncthreads();
                char* const to = tiles + (t + 1) % BUFFERS * 2 * Tl::BYTES;
                kept = __ballot(next.keep != 0);
                next.k.store(to, a.width, kept);
                next.v.store(to + Tl::BYTES, a.width, kept);
                __syncthreads();
            }
        }
    };
    {
        const Tiles keys = keys_of(w, x, far), more = keys_of(w, x, exact);
        if (half == 0 && lane == 0) {
            far_keys[wave] = keys;
            delta_keys[wave] = more;
        }
        __syncthreads();
        const Tiles range = tiles_of(far_keys);
        if (rare(range.to)) {
            walk(std::integral_constant<int, LOGARITHMS>{}, range);
            total = halves_sum(total);
            if constexpr (SPLIT == 2) {
                if (h == 0) { deltas[half][wave][lane] = total; largest[half][wave][lane] = most; }
                __syncthreads();
                const float m0 = largest[0][wave][lane % 32], m1 = largest[1][wave][lane % 32];
                const float t0 = deltas[0][wave][lane % 32], t1 = deltas[1][wave][lane % 32];
                most = fmaxf(m0, m1);
                total = (t0 == 0.f ? 0.f : t0 * __builtin_amdgcn_exp2f(m0 - most)) + (t1 == 0.f ? 0.f : t1 * __builtin_amdgcn_exp2f(m1 - most));
            }
            if (far && total != 0.f) {
                high = most;
                low = __builtin_log2f(total);
            }
            share = __builtin_amdgcn_exp2f(-low);
        }
    }
    const Tiles whole{0, count};
    if constexpr (sizeof(T) == 2) {
        const Tiles range = tiles_of(delta_keys);
        if (range.to) {
            walk(std::integral_constant<int, DELTA>{}, range);
            formed = halves_sum(formed) * share;
            if constexpr (SPLIT == 2) {
                if (h == 0) deltas[half][wave][lane] = formed;
                __syncthreads();
                formed = deltas[0][wave][lane % 32] + deltas[1][wave][lane % 32];
            }
            delta = exact ? formed : delta;
        }
    }
    if (real && h == 0 && half == 0) {
        const size_t at = (size_t)head * a.T + w.i;
        b.high[at] = high;
        b.low[at] = low;
        b.delta[at] = delta;
    }
    delta *= share;                                   // as the walk takes it
    walk(std::integral_constant<int, GRADIENTS>{}, whole);
    if constexpr (lifts<T>)
#pragma unroll
        for (int n = 0; n < DB; ++n) dq[n] *= 1.f / lift;
    bool mine = true;
    if constexpr (SPLIT == 2) mine = join_halves((float*)tiles, dq, wave, half, lane);
    if (some && mine) {
        const bool redo = not_finite(dq);
        if (real && !redo) store_column<T>(head_row<T>(b.dq, w.i, head), a.width, dq, a.scale, h);
        uint64_t rows = __ballot(redo && real && h == 0);
        if (rare(rows)) for (; rows; rows &= rows - 1) {
            const int l = __builtin_ctzll(rows);
            Shown s;
            s.lo = __shfl(w.s.lo, l, 64); s.hi = __shfl(w.s.hi, l, 64);
            s.first = __shfl(w.s.first, l, 64); s.sunk = __shfl(w.s.sunk, l, 64);
            const uint32_t i = __shfl(w.i, l, 64);
            float row[2];
            const size_t at = (size_t)head * a.T + i;
            query_row<T>(b, head, i, s, RowSum{b.high[at], b.low[at], b.delta[at]}, lane, row);
            T* to = head_row<T>(b.dq, i, head);
#pragma unroll
            for (int c = 0; c < 2; ++c) if (lane + c * WAVE < a.width) to[lane + c * WAVE] = (T)row[c];
        }
    }
    if constexpr (BIAS) {
        if (!b.dbias) return;
        // the outermost distances: what lies past the span in the array, and what went by registers
        __syncthreads();
        static_assert(BIAS_SIDE == 64, "one place a lane on either side");
        before = lanes_sum<64>(before + sums[lane]);
        after = lanes_sum<64>(after + sums[2 * reach - lane]);
        if (lane == 0) { sums[BIAS_SIDE] += before; sums[2 * reach - BIAS_SIDE] += after; }
        __syncthreads();
        float* to = b.by_distance + ((size_t)head * words + part) * (2 * span + 1);
        for (int32_t c = threadIdx.x; c <= 2 * span; c += SPLIT * THREADS) {
            float all = 0.f;
#pragma unroll
            for (int n = 0; n < SPLIT * GROUPS; ++n)
                all += dynamic[bias_table(a.span) + n * (SKEW_FLOATS + bias_table(a.span)) + SKEW_FLOATS + BIAS_SIDE + c];
            to[c] = all;
        }
    }
}

// ---- keys: dk, dv ---------------------------------------------------------------------------------------
// The border behind which queries of the block's first words that stay visible are late.
__device__ inline uint32_t late_border(const BackwardArgs& b, uint32_t j) {
    return j / BLOCK_WORDS * BLOCK_WORDS + BLOCK_WORDS + b.reach;
}

// Heads whose rows as keys, beside the sums for dk and dv, leave no registers for a second wavefront on a SIMD: their blocks always
// have both halves and read those rows from LDS (16384 words of 16 heads of 96 in a window of 1024, 16 bits: the backward pass
// takes 635 us instead of 706; of 128: 872 instead of 904).
template <typename T, int DB> constexpr bool own_rows_in_lds = DB * sizeof(T) >= 6;

template <typename T, int DB, bool BIAS, int SPLIT>
__global__ __launch_bounds__(SPLIT * THREADS, SPLIT == 2 || DB * sizeof(T) <= 4 ? 2 : 1) void key_kernel(const BackwardArgs b) {
    const AttendArgs& a = b.a;
    typedef Tile<T, DB, KEYS> Tl;
    constexpr int BUFFERS = 2 * 2 * Tl::BYTES <= 72 * 1024 ? 2 : 1;
    constexpr int ROOM = SPLIT == 2 ? GROUPS * DB * 16 * WAVE * 4 : 0;
    __shared__ __align__(16) char tiles[BUFFERS * 2 * Tl::BYTES > ROOM ? BUFFERS * 2 * Tl::BYTES : ROOM];
    // wide heads: the block's own keys and values as operands from LDS, registers do not hold them beside the sums
    constexpr bool OWN = SPLIT == 2 && own_rows_in_lds<T, DB>;
    typedef Tile<T, DB, BLOCK_WORDS> Ow;
    __shared__ __align__(16) char own[OWN ? 2 * Ow::BYTES : 16];
    __shared__ float rows[BUFFERS][3][KEYS];          // of the queries: high, delta, low
    extern __shared__ float table[];
    const Place place;
    const uint32_t lane = place.lane, h = place.h, wave = place.wave, half = place.half;
    const uint32_t kv_head = blockIdx.x % a.kv_heads, block = blockIdx.x / a.kv_heads;
    const bool late = block < b.late;
    const int32_t reach = (int32_t)a.span + BIAS_SIDE;

    // the block's keys k0 .. k1, the queries q0 .. q1 that any of them is shown to, and a lane's own [lo, hi) of them
    uint32_t k0, k1, q0, q1;
    if (late) {
        q0 = block * b.late_words;
        const Text t = text_bounds(a.off, text_of(a.off, a.n_sent, q0, lane), q0, a.T);
        k0 = t.first;
        k1 = t.end - t.first < a.sinks ? t.end : t.first + a.sinks;
        q1 = t.end < q0 + b.late_words ? t.end : q0 + b.late_words;
        if (late_border(b, k0) >= q1) return;         // none of this piece's queries are late
    } else {
        k0 = (block - b.late) * BLOCK_WORDS;
        k1 = k0 + BLOCK_WORDS < a.T ? k0 + BLOCK_WORDS : a.T;
    }
    k0 = __builtin_amdgcn_readfirstlane(k0);
    k1 = __builtin_amdgcn_readfirstlane(k1);
    const uint32_t wave0 = k0 + wave * WAVE_WORDS;
    const bool some = wave0 < k1, real = wave0 + lane % WAVE_WORDS < k1;
    const uint32_t j_first = some ? wave0 : k1 - 1, j_last = wave0 + WAVE_WORDS - 1 < k1 ? wave0 + WAVE_WORDS - 1 : k1 - 1;
    const uint32_t j = real ? wave0 + lane % WAVE_WORDS : k1 - 1;
    typename Frag<T>::vec kf[OWN ? 1 : 2 * DB], vf[OWN ? 1 : 2 * DB];
    if constexpr (OWN) {
        Transit<T, DB, BLOCK_WORDS, SPLIT * THREADS> t;
        const auto token = [&](uint32_t r) __attribute__((always_inline)) { return k0 + r < k1 ? k0 + r : k1 - 1; };
        t.start(a.k, kv_head, k0);
        t.aim(token);
        t.load(a.width);
        t.template store<true>(own, a.width);
        t.start(a.v, kv_head, k0);
        t.aim(token);
        t.load(a.width);
        t.template store<true>(own + Ow::BYTES, a.width);
    } else {
#pragma unroll
        for (int s = 0; s < 2 * DB; ++s) {
            kf[s] = load_operand<T, DB>(head_row<T>(a.k, j, kv_head), s, h, a.width);
            vf[s] = load_operand<T, DB>(head_row<T>(a.v, j, kv_head), s, h, a.width);
        }
    }
    const uint32_t own_base = Ow::base_along(lane) + wave * (WAVE_WORDS / 4) * Ow::STRIDE;
    const bool keep = !(a.keep && !a.keep[j]);
    const Texts texts(a, k0, k1 - 1, j_first, j_last, lane);
    const Text text = text_between(a.off, texts.wave_first, texts.wave_last, j, a.T, lane);
    uint32_t lo = 0, hi = 0;
    const uint32_t border = late_border(b, j);
    if (late) {
        lo = border > q0 ? border : q0;
        hi = q1;
    } else {
        q0 = sees(a, k0, text_bounds(a.off, texts.block_first, k0, a.T)).lo;
        const Text t = text_bounds(a.off, texts.block_last, k1 - 1, a.T);
        q1 = sees(a, k1 - 1, t).hi;
        if (a.sinks && t.first + a.sinks > k0) {
            const uint32_t last = late_border(b, k0), to = t.end < last ? t.end : last;
            q1 = q1 < to ? to : q1;
        }
        const Shown s = sees(a, j, text);
        lo = s.lo;
        hi = s.sunk < border ? s.sunk : border;
        hi = hi < s.hi ? s.hi : hi;
    }
    q0 = __builtin_amdgcn_readfirstlane(q0);
    q1 = __builtin_amdgcn_readfirstlane(q1);
    if (!real || !keep || lo >= hi) lo = hi = 0;
    uint32_t lo_least = lo < hi ? lo : ~0u, lo_most = lo_least, hi_most = hi, hi_least = hi;
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
        lo_least = min(lo_least, (uint32_t)__shfl_xor((int)lo_least, m, 64));
        lo_most = max(lo_most, (uint32_t)__shfl_xor((int)lo_most, m, 64));
        hi_least = min(hi_least, (uint32_t)__shfl_xor((int)hi_least, m, 64));
        hi_most = max(hi_most, (uint32_t)__shfl_xor((int)hi_most, m, 64));
    }
    lo_least = __builtin_amdgcn_readfirstlane(lo_least);
    lo_most = __builtin_amdgcn_readfirstlane(lo_most);
    hi_least = __builtin_amdgcn_readfirstlane(hi_least);
    hi_most = __builtin_amdgcn_readfirstlane(hi_most);
    Acc dk[DB], dv[DB];
#pragma unroll
    for (int n = 0; n < DB; ++n) dk[n] = dv[n] = Acc{};

    Transit<T, DB, KEYS, SPLIT * THREADS> tq, tg;
    // a half's piece of every tile is the same one: its rows are part of the lane's bases
    const uint32_t own_rows = SPLIT == 2 ? half * 32 : 0;
    const uint32_t at_along = Tl::base_along(lane) + own_rows / 4 * Tl::STRIDE, at_across = Tl::base_across(lane) + own_rows / 4 * Tl::STRIDE;
    float high = 0.f, low = 0.f, delta = 0.f;
    bool lowered = false;                             // whether any of a tile's queries has a low part
    float lift = lifts<T> ? FIRST_LIFT : 1.f;
    const uint32_t per_head = q1 > q0 ? (q1 - q0 + KEYS - 1) / KEYS : 0, count = per_head * a.group;
    const auto fetch = [&](uint32_t t) __attribute__((always_inline)) {
        const uint32_t head = kv_head * a.group + t / per_head, i0 = q0 + t % per_head * KEYS;
        if (t % per_head == 0) {
            tq.start(a.q, head, q0);
            tg.start(b.dout, head, q0);
        }
        if (i0 + KEYS <= q1) {
            tq.aim();
            tg.aim();
        } else {
            const auto token = [&](uint32_t r) __attribute__((always_inline)) { return i0 + r < q1 ? i0 + r : q1 - 1; };
            tq.aim(token);
            tg.aim(token);
        }
        tq.load(a.width);
        tg.load(a.width);
        const uint32_t i = i0 + threadIdx.x % KEYS < q1 ? i0 + threadIdx.x % KEYS : q1 - 1;
        high = b.high[(size_t)head * a.T + i];
        low = b.low[(size_t)head * a.T + i];
        delta = b.delta[(size_t)head * a.T + i];
    };
    const auto put = [&](uint32_t t) __attribute__((always_inline)) {
        tq.store(tiles + t % BUFFERS * 2 * Tl::BYTES, a.width);
        tg.store(tiles + t % BUFFERS * 2 * Tl::BYTES + Tl::BYTES, a.width);
        if constexpr (lifts<T>) {                     // 2^14 p: from high, unless that is so large that it would be lost there
            const bool far = fabsf(high) > FAR;
            high -= far ? 0.f : WEIGHT_LIFT<T>;
            low -= far ? WEIGHT_LIFT<T> : 0.f;
        }
        if (threadIdx.x < KEYS) {
            rows[t % BUFFERS][0][threadIdx.x] = high;
            rows[t % BUFFERS][1][threadIdx.x] = delta;
            rows[t % BUFFERS][2][threadIdx.x] = low;
        }
        lowered = __any(low != 0.f);                  // (a wavefront's lanes hold all of the tile's queries)
    };
    if (count) {
        fetch(0);
        put(0);
    }
    for (uint32_t t = 0; t < count; ++t) {
        if (BIAS && t % per_head == 0) {
            __syncthreads();
            fill_bias(a, kv_head * a.group + t / per_head, table);
        }
        if (BUFFERS == 1 || t == 0 || (BIAS && t % per_head == 0)) __syncthreads();
        if (t + 1 < count) fetch(t + 1);
        const char *qt = tiles + t % BUFFERS * 2 * Tl::BYTES, *gt = qt + Tl::BYTES;
        const auto one = [&](uint32_t piece) __attribute__((always_inline)) {
            const uint32_t row0 = piece * 32 + own_rows, i0 = q0 + t % per_head * KEYS + row0;
            const char *qp = qt + piece * (32 / 4) * Tl::STRIDE, *gp = gt + piece * (32 / 4) * Tl::STRIDE;
            if (!some || i0 >= hi_most || i0 + 32 <= lo_least) return;
            Acc s = {}, dp = {};
            const uint32_t at_own = per_piece(own_base);      // (what does not change is not kept in registers)
#pragma unroll
            for (int k = 0; k < 2 * DB; ++k) {
                if constexpr (OWN) {
                    mma(Tl::along(qp, at_along, 0, k), Ow::along(own, at_own, 0, k), s);
                    mma(Tl::along(gp, at_along, 0, k), Ow::along(own + Ow::BYTES, at_own, 0, k), dp);
                } else {
                    mma(Tl::along(qp, at_along, 0, k), kf[k], s);
                    mma(Tl::along(gp, at_along, 0, k), vf[k], dp);
                }
            }
            __builtin_amdgcn_sched_barrier(0);        // (what the next products read is not asked for before: registers)
            const float *l2 = &rows[t % BUFFERS][0][row0 + 4 * h], *dl = l2 + KEYS, *ll = dl + KEYS;
            if constexpr (BIAS) {
                const int32_t far = (int32_t)j_last - (int32_t)i0, near = (int32_t)j_first - (int32_t)i0 - 31;
                if (far <= -(int32_t)a.span || near >= (int32_t)a.span) {
                    const float c = table[far <= -(int32_t)a.span ? 0 : 2 * reach];
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.scale2, c) - l2[acc_row(r, 0)];
                } else {
                    const float* at = table + ((int32_t)j - (int32_t)i0 + reach - 4 * (int32_t)h);
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.scale2, at[-acc_row(r, 0)]) - l2[acc_row(r, 0)];
                }
            } else {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.scale2, -l2[acc_row(r, 0)]);
            }
            if (rare(lowered) || !(i0 >= lo_most && i0 + 32 <= hi_least && !(a.skip_self && i0 <= j_last && i0 + 32 > j_first))) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] -= ll[acc_row(r, 0)];      // (zero nearly always)
                const uint32_t base = per_piece(i0 + 4 * h);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const uint32_t i = base + acc_row(r, 0);
                    const bool in = (i - lo < hi - lo) & !(a.skip_self & (i == j));
                    s[r] = in ? s[r] : -__builtin_inff();
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = __builtin_amdgcn_exp2f(s[r]);
                dp[r] = s[r] * (dp[r] - dl[acc_row(r, 0)]);
            }
            if constexpr (lifts<T>) lift_piece(dp, dk, lift);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (sizeof(T) == 4) {
                // the same for a text's queries and heads
#pragma unroll
                for (int n = 0; n < DB; ++n) {
                    Acc v = {}, x = {};
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        mma(Tl::across(gp, at_across, 0, k, n), acc_operand<T>(s, k), v);
                        mma(Tl::across(qp, at_across, 0, k, n), acc_operand<T>(dp, k), x);
                    }
                    dv[n] += v;
                    dk[n] += x;
                }
            } else {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const auto p = acc_operand<T>(s, k), ds = acc_operand<T>(dp, k);
#pragma unroll
                    for (int n = 0; n < DB; ++n) {
                        mma(Tl::across(gp, at_across, 0, k, n), p, dv[n]);
                        mma(Tl::across(qp, at_across, 0, k, n), ds, dk[n]);
                    }
                }
            }
        };
        if constexpr (SPLIT == 2) one(0);
        else
#pragma unroll 1
            for (uint32_t piece = 0; piece < KEYS / 32; ++piece) one(piece);
        if (t + 1 < count) {
            if (BUFFERS == 1) __syncthreads();
            put(t + 1);
            if (BUFFERS == 2) __syncthreads();
        }
    }
    if constexpr (lifts<T>)
#pragma unroll
        for (int n = 0; n < DB; ++n) {
            dk[n] *= 0x1p-14f / lift;
            dv[n] *= 0x1p-14f;
        }
    if constexpr (SPLIT == 2) {
        const bool mine = join_halves((float*)tiles, dk, wave, half, lane);
        join_halves((float*)tiles, dv, wave, half, lane);
        if (!mine) return;
    }
    if (!some) return;

    // rows that later pieces add to are left in fp32, the others are finished
    const uint32_t at = late ? j - k0 : j - text.first;      // among the text's first words
    const uint32_t last = (text.end - 1) / (b.late_words ? b.late_words : 1);
    const bool joined = b.late && at < a.sinks && text.end > border;
    const bool redo = not_finite(dk) | not_finite(dv);
    float* const kept = late || joined
        ? (late ? b.late_sums + ((size_t)block * a.kv_heads + kv_head) * a.sinks * 2 * a.width
                : b.own_sums + ((size_t)last * a.kv_heads + kv_head) * a.sinks * 2 * a.width) + (size_t)at * 2 * a.width
        : nullptr;
    if (real && !redo) {
        if (kept) {
            store_column<float>(kept, a.width, dk, 1.f, h);
            store_column<float>(kept + a.width, a.width, dv, 1.f, h);
        } else {
            store_column<T>(head_row<T>(b.dk, j, kv_head), a.width, dk, a.scale, h);
            store_column<T>(head_row<T>(b.dv, j, kv_head), a.width, dv, 1.f, h);
        }
    }
    uint64_t again = __ballot(redo && real && h == 0);
    if (rare(again)) for (; again; again &= again - 1) {
        const int l = __builtin_ctzll(again);
        const uint32_t jl = __shfl(j, l, 64);
        float ck[2] = {0.f, 0.f}, cv[2] = {0.f, 0.f};
        key_row<T>(b, kv_head, jl, __shfl(lo, l, 64), __shfl(hi, l, 64), lane, ck, cv);
        float* const at = (float*)__shfl((unsigned long long)kept, l, 64);
        T *to_k = head_row<T>(b.dk, jl, kv_head), *to_v = head_row<T>(b.dv, jl, kv_head);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const uint32_t col = lane + c * WAVE;
            if (col >= a.width) continue;
            if (at) { at[col] = ck[c]; at[a.width + col] = cv[c]; }
            else { to_k[col] = (T)(ck[c] * a.scale); to_v[col] = (T)cv[c]; }
        }
    }
}

// ---- the end: late pieces joined, the bias' gradient -----------------------------------------------------
constexpr uint32_t END_THREADS = 1024, FEW_PARTS = 16;      // blocks whose sums the last kernel joins by itself: a launch less
template <typename T> __global__ __launch_bounds__(END_THREADS) void end_kernel(const BackwardArgs b, uint32_t parts) {
    const AttendArgs& a = b.a;
    const uint32_t lane = threadIdx.x % WAVE;
    const uint32_t joins = b.late * a.kv_heads;
    if (blockIdx.x < joins) {
        // the piece that holds a text's last word joins that text's rows
        const uint32_t piece = blockIdx.x / a.kv_heads, kv_head = blockIdx.x % a.kv_heads, i0 = piece * b.late_words;
        const Text t = text_bounds(a.off, text_of(a.off, a.n_sent, i0, lane), i0, a.T);
        if ((t.end - 1) / b.late_words != piece) return;
        for (uint32_t at = threadIdx.x; at < a.sinks * 2 * a.width; at += END_THREADS) {
            const uint32_t place = at / (2 * a.width), j = t.first + place;
            if (j >= t.end || t.end <= late_border(b, j)) continue;
            const size_t step = (size_t)a.kv_heads * a.sinks * 2 * a.width;
            const size_t from = (size_t)kv_head * a.sinks * 2 * a.width + at;
            float s = b.own_sums[piece * step + from];
            for (uint32_t p = late_border(b, j) / b.late_words; p <= piece; ++p) s += b.late_sums[p * step + from];
            const uint32_t c = at % (2 * a.width);
            if (c < a.width) head_row<T>(b.dk, j, kv_head)[c] = (T)(s * a.scale);
            else head_row<T>(b.dv, j, kv_head)[c - a.width] = (T)s;
        }
        return;
    }
    // 32 distances of a head: 32 shares of the blocks' sums, joined in order
    const uint32_t distances = 2 * a.span + 1, groups = (distances + 31) / 32;
    const uint32_t head = (blockIdx.x - joins) / groups, c = (blockIdx.x - joins) % groups * 32 + threadIdx.x % 32;
    __shared__ float shares[END_THREADS / 32][32];
    const float* from = b.by_distance + (size_t)head * parts * distances;
    float s = 0.f;
    if (c < distances) {
#pragma unroll 4
        for (uint32_t p = threadIdx.x / 32; p < parts; p += END_THREADS / 32) s += from[(size_t)p * distances + c];
    }
    shares[threadIdx.x / 32][threadIdx.x % 32] = s;
    __syncthreads();
    if (threadIdx.x >= 32 || c >= distances) return;
    for (uint32_t n = 1; n < END_THREADS / 32; ++n) s += shares[n][threadIdx.x];
    b.distance_sums[(size_t)head * distances + c] = s;
}

// dbias of a head: its sums by distance -- joined already, or here from a few blocks' -- then the distances of each bucket, both
// in order: a wavefront for a bucket, its lanes' shares of the distances joined.
__global__ __launch_bounds__(END_THREADS) void buckets_kernel(const BackwardArgs b, const float* by_distance, uint32_t parts) {
    const AttendArgs& a = b.a;
    __shared__ float sums[2 * SPAN_MAX + 1];
    __shared__ uint32_t bucket[2 * SPAN_MAX + 1];
    const uint32_t head = blockIdx.x, distances = 2 * a.span + 1;
    for (uint32_t c = threadIdx.x; c < distances; c += END_THREADS) {
        float s = 0.f;
        for (uint32_t p = 0; p < parts; ++p) s += by_distance[((size_t)head * parts + p) * distances + c];
        sums[c] = s;
        bucket[c] = a.buckets[c];
    }
    __syncthreads();
    for (uint32_t k = threadIdx.x / WAVE; k < a.n_buckets; k += END_THREADS / WAVE) {
        float s = 0.f;
        for (uint32_t c = threadIdx.x % WAVE; c < distances; c += WAVE) s += bucket[c] == k ? sums[c] : 0.f;
        s = lanes_sum<64>(s);
        if (threadIdx.x % WAVE == 0) b.dbias[(size_t)head * a.n_buckets + k] = s;
    }
}

// LDS of a block of the queries' kernel that depends on the span: the bias' table and, where its gradient is wanted, room for it.
template <bool BIAS, int SPLIT> size_t query_room(const BackwardArgs& b) {
    const uint32_t table = BIAS ? bias_table(b.a.span) : 0;
    return (table + (BIAS && b.dbias ? SPLIT * GROUPS * (SKEW_FLOATS + table) : 0)) * sizeof(float);
}
template <typename T, int DB, bool BIAS> bool query_split(const BackwardArgs& b, uint32_t blocks) {
    return blocks < SPLIT_BELOW && query_room<BIAS, 2>(b) + sizeof(QueryRoom<T, DB, BIAS, 2>) <= LDS_BYTES;
}
template <typename T, int DB, bool BIAS> void backward_run(const BackwardArgs& b, hipStream_t st) {
    const AttendArgs& a = b.a;
    static_assert(sizeof(QueryRoom<T, DB, BIAS, 1>) + (BIAS ? (5 * bias_table(SPAN_MAX) + 4 * SKEW_FLOATS) * sizeof(float) : 0) <= LDS_BYTES,
                  "blocks of one half have room at every span");
    const uint32_t words = attend_bias_parts(a.T), table = BIAS ? bias_table(a.span) * sizeof(float) : 0;
    uint32_t blocks = words * a.heads;
    bool split = splits<T, DB> && query_split<T, DB, BIAS>(b, blocks);
    if constexpr (splits<T, DB>)
        if (split) query_kernel<T, DB, BIAS, 2><<<blocks, 2 * THREADS, query_room<BIAS, 2>(b), st>>>(b);
    if (!split) query_kernel<T, DB, BIAS, 1><<<blocks, THREADS, query_room<BIAS, 1>(b), st>>>(b);
    blocks = (b.late + words) * a.kv_heads;
    if constexpr (splits<T, DB> && own_rows_in_lds<T, DB>) {
        key_kernel<T, DB, BIAS, 2><<<blocks, 2 * THREADS, table, st>>>(b);
    } else {
        if constexpr (splits<T, DB>)
            if (blocks < SPLIT_BELOW) return key_kernel<T, DB, BIAS, 2><<<blocks, 2 * THREADS, table, st>>>(b);
        key_kernel<T, DB, BIAS, 1><<<blocks, THREADS, table, st>>>(b);
    }
}
template <typename T, int DB> void backward_bias(const BackwardArgs& b, hipStream_t st) {
    if (b.a.bias) backward_run<T, DB, true>(b, st);
    else backward_run<T, DB, false>(b, st);
}
template <typename T> void backward_any(const BackwardArgs& b, hipStream_t st) {
    if (b.a.T)
        switch ((b.a.width + 31) / 32) {
            case 1: backward_bias<T, 1>(b, st); break;
            case 2: backward_bias<T, 2>(b, st); break;
            case 3: backward_bias<T, 3>(b, st); break;
            default: backward_bias<T, 4>(b, st);
        }
    const uint32_t parts = attend_bias_parts(b.a.T);
    const bool joined = b.dbias && parts > FEW_PARTS;
    const uint32_t blocks = b.late * b.a.kv_heads + (joined ? b.a.heads * ((2 * b.a.span + 32) / 32) : 0);
    if (blocks) end_kernel<T><<<blocks, END_THREADS, 0, st>>>(b, parts);
    if (b.dbias) buckets_kernel<<<b.a.heads, END_THREADS, 0, st>>>(b, joined ? b.distance_sums : b.by_distance, joined ? 1 : parts);
}

}  // namespace

uint32_t attend_bias_parts(uint32_t T) { return (T + BLOCK_WORDS - 1) / BLOCK_WORDS; }

// Pieces of at least 512 queries, at most 256 of them; none where no word outlives its window.
LatePieces attend_late_pieces(uint32_t T, uint32_t left, uint32_t sinks) {
    const uint32_t size = (T + 255) / 256 > 512 ? ((T + 255) / 256 + KEYS - 1) / KEYS * KEYS : 512;
    const uint32_t reach = left > size ? left : size;
    if (sinks == 0 || T <= BLOCK_WORDS + reach) return LatePieces{0, size, T};
    return LatePieces{(T + size - 1) / size, size, reach};
}

void launch_attend_backward(const BackwardArgs& b, uint32_t type, hipStream_t st) {
    if (type == ELEM_F32) backward_any<float>(b, st);
    else if (type == ELEM_F16) backward_any<_Float16>(b, st);
    else backward_any<__bf16>(b, st);
}

}  // namespace w2v

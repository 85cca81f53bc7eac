// Attention over texts: what its kernels share -- which words a word is shown, element access, and a row at a time.
//
//   x_ij = scale q_i . k_j + bias[head][bucket(j - i)] over the words j shown to word i
//   p_ij = exp(x_ij) / sum_j exp(x_ij),  o_i = sum_j p_ij v_j,  lse_i = log sum_j exp(x_ij)
// Exponentials are taken to base two; logarithms are kept natural in memory.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "context.h"
#include "elem.h"

namespace w2v {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr uint32_t WAVE = 64;

template <typename T> __device__ inline const T* head_row(const Heads& x, uint32_t token, uint32_t head) {
    return (const T*)x.p + (uint64_t)token * x.token + (uint64_t)head * x.head;
}
template <typename T> __device__ inline T* head_row(const HeadsOut& x, uint32_t token, uint32_t head) {
    return (T*)x.p + (uint64_t)token * x.token + (uint64_t)head * x.head;
}

// ---- texts ------------------------------------------------------------------------------------------
// The last text that starts at or before a token, for four tokens at a time: lanes 16 g .. 16 g + 15 look for their token i
// together, 64 offsets a round, and all end with its text.  Whatever the offsets hold, the result is below n_sent and the search
// ends.
__device__ inline uint32_t texts_of(const uint64_t* off, uint32_t n_sent, uint32_t i, uint32_t lane) {
    uint32_t lo = 0, hi = n_sent;
    while (__any(hi - lo > 1)) {
        const uint32_t step = (hi - lo + 63) / 64;
        uint32_t c = 0;
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            const uint32_t at = lo + (lane % 16 * 4 + u + 1) * step;       // n_sent < 2^31: no overflow
            const uint64_t before = __ballot(at < hi && off[at < hi ? at : lo] <= (uint64_t)i);
            c += __popc((uint32_t)(before >> (lane / 16 * 16)) & 0xFFFFu);
        }
        lo += c * step;
        hi = hi - lo < step ? hi : lo + step;
    }
    return lo;
}
__device__ inline uint32_t text_of(const uint64_t* off, uint32_t n_sent, uint32_t i, uint32_t lane) {
    return __builtin_amdgcn_readfirstlane(texts_of(off, n_sent, i, lane));
}

// Tokens [first, end) of the text of token i, always first <= i < end <= T.
struct Text { uint32_t first, end; };
__device__ inline Text text_bounds(const uint64_t* off, uint32_t text, uint32_t i, uint32_t T) {
    const uint64_t a = off[text], b = off[text + 1];
    Text t;
    t.first = a < (uint64_t)i ? (uint32_t)a : i;
    t.end = b < (uint64_t)T ? (uint32_t)b : T;
    if (t.end <= i) t.end = i + 1;
    return t;
}
// The same for the tokens of a wavefront's lanes, which lie between those of texts s0 and s1 (the same in all lanes).
__device__ inline Text text_between(const uint64_t* off, uint32_t s0, uint32_t s1, uint32_t i, uint32_t T, uint32_t lane) {
    Text t;
    if (s1 - s0 < 63) {                               // their offsets side by side in the lanes
        const uint64_t mine = off[lane <= s1 - s0 ? s0 + lane : s1 + 1];
        const uint32_t o = mine < (uint64_t)T ? (uint32_t)mine : T;
        uint32_t at = 0;
#pragma unroll
        for (uint32_t b = 32; b; b /= 2) {
            const uint32_t there = (uint32_t)__shfl((int)o, (int)((at + b) & 63), 64);
            if (at + b <= s1 - s0 && there <= i) at += b;
        }
        t.first = (uint32_t)__shfl((int)o, (int)at, 64);
        t.end = (uint32_t)__shfl((int)o, (int)at + 1, 64);
        t.first = t.first < i ? t.first : i;
        if (t.end <= i) t.end = i + 1;
        return t;
    }
    uint32_t lo = s0, hi = s1 + 1;                    // many texts without a word
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (off[mid] <= (uint64_t)i) lo = mid; else hi = mid;
    }
    return text_bounds(off, lo, i, T);
}

// Tokens shown to token i: [lo, hi) of its window and [first, sunk) of the words that stay visible, which end where the
// window begins.  left and right are at most T.
struct Shown { uint32_t lo, hi, first, sunk; };
__device__ inline Shown shown_to(const AttendArgs& a, uint32_t i, Text t) {
    Shown s;
    s.first = t.first;
    s.lo = i - t.first > a.left ? i - a.left : t.first;
    s.hi = t.end - i > a.right ? i + a.right + 1 : t.end;
    const uint32_t sunk = s.lo - t.first > a.sinks ? t.first + a.sinks : s.lo;
    s.sunk = sunk;
    return s;
}
// Tokens that token j is shown to: [lo, hi) through their windows and [hi, late) because it stays visible.
__device__ inline Shown sees(const AttendArgs& a, uint32_t j, Text t) {
    Shown s;
    s.first = t.first;
    s.lo = j - t.first > a.right ? j - a.right : t.first;
    s.hi = t.end - j > a.left ? j + a.left + 1 : t.end;
    s.sunk = j - t.first < a.sinks ? t.end : s.hi;
    return s;
}

// ---- bias --------------------------------------------------------------------------------------------
// The bias of a distance; a bucket past the last adds nothing.
__device__ inline float plain_bias(const float* bias, const uint32_t* buckets, uint32_t n_buckets, uint32_t reach, uint32_t head,
                                   int32_t dist) {
    const int32_t span = (int32_t)reach;
    const int32_t at = (dist < -span ? -span : dist > span ? span : dist) + span;
    const uint32_t b = buckets[at];
    return b < n_buckets ? bias[(size_t)head * n_buckets + b] : 0.f;
}
// The same times log2 e.  Values that would leave fp32 with that factor are held where they do not; infinities are kept.  A row
// whose largest score is about as large as a held value is formed a word at a time, without the factor.
constexpr float BIAS_HELD = 2.3e38f, HELD = 3.2e38f;
__device__ inline float scaled_bias(const float* bias, const uint32_t* buckets, uint32_t n_buckets, uint32_t reach, uint32_t head,
                                    int32_t dist) {
    const float x = plain_bias(bias, buckets, n_buckets, reach, head, dist);
    if (!(fabsf(x) < __builtin_inff())) return x;
    return fminf(fmaxf(x, -BIAS_HELD), BIAS_HELD) * LOG2E;
}
__device__ inline float scaled_bias(const AttendArgs& a, uint32_t head, int32_t dist) {
    return scaled_bias(a.bias, a.buckets, a.n_buckets, a.span, head, dist);
}

// ---- a row at a time ---------------------------------------------------------------------------------
// One wavefront, one query and head (or one key and key head), nothing rounded on the way and nothing touched that the
// word is not shown.  The tiled kernels come back to these for rows whose result is not finite: there a
// masked word's infinity or NaN, which a matrix product multiplies by zero, must not show.  That costs a thousand times a tile's
// share of a row.  It is paid where infinities or NaN are shown, and for words within a tile's reach of a text or
// window that holds them; not for words that `keep` leaves out, whose rows enter the tiles as zeros.
template <typename T> __device__ inline float dot_rows(const T* x, const T* y, uint32_t d) {
    constexpr uint32_t N = pack16<T>;
    typedef typename Pack<T, N>::mem mem;
    float s = 0.f;
    uint32_t c = 0;
    for (; c + N <= d; c += N) {
        const typename Pack<T, N>::vec a = *(const mem*)(x + c), b = *(const mem*)(y + c);
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) s = fmaf((float)a[e], (float)b[e], s);
    }
    for (; c < d; ++c) s = fmaf((float)x[c], (float)y[c], s);
    return s;
}

// The score of (i, j), as it is and to base two; whether j is kept is the caller's to ask.
template <typename T>
__device__ inline float row_plain_score(const AttendArgs& a, uint32_t head, uint32_t i, uint32_t j) {
    const float s = dot_rows(head_row<T>(a.q, i, head), head_row<T>(a.k, j, head / a.group), a.width) * a.scale;
    return a.bias ? s + plain_bias(a.bias, a.buckets, a.n_buckets, a.span, head, (int32_t)j - (int32_t)i) : s;
}
template <typename T>
__device__ inline float row_score(const AttendArgs& a, uint32_t head, uint32_t i, uint32_t j) {
    const float s = dot_rows(head_row<T>(a.q, i, head), head_row<T>(a.k, j, head / a.group), a.width) * a.scale2;
    return a.bias ? s + scaled_bias(a, head, (int32_t)j - (int32_t)i) : s;
}
__device__ inline bool row_keeps(const AttendArgs& a, uint32_t i, uint32_t j) {
    return (!a.keep || a.keep[j]) && !(a.skip_self && i == j);
}

__device__ inline float wave_max(float x) {
    return lanes_join<64>(x, [](float a, float b) __attribute__((always_inline)) { return fmaxf(a, b); });
}

// o_i and lse_i (lane l holds columns l and l + 64 of o).
template <typename T>
__device__ void attend_row(const AttendArgs& a, uint32_t head, uint32_t i, const Shown& s, uint32_t lane, float (&o)[2],
                           float& lse) {
    const uint32_t sunk = s.sunk - s.first, n = sunk + s.hi - s.lo;
    float m = -__builtin_inff();
    bool nan = false;
    for (uint32_t at = lane; at < n; at += WAVE) {
        const uint32_t j = at < sunk ? s.first + at : s.lo + at - sunk;
        if (!row_keeps(a, i, j)) continue;
        const float x = row_plain_score<T>(a, head, i, j);
        nan |= x != x;
        m = fmaxf(m, x);
    }
    m = wave_max(m);
    if (__any(nan) || m == __builtin_inff()) {        // every weight is not a number, and so is every column
        o[0] = o[1] = lse = __builtin_nanf("");
        return;
    }
    const float base = m == -__builtin_inff() ? 0.f : m;
    float total = 0.f;
    o[0] = o[1] = 0.f;
    for (uint32_t at0 = 0; at0 < n; at0 += WAVE) {
        const uint32_t at = at0 + lane;
        const uint32_t j = at < sunk ? s.first + at : s.lo + at - sunk;
        const bool in = at < n && row_keeps(a, i, j);
        const float p = in ? exp2f((row_plain_score<T>(a, head, i, j) - base) * LOG2E) : 0.f;
        total += p;
        for (uint64_t left = __ballot(in && p != 0.f); left; left &= left - 1) {
            const int l = __builtin_ctzll(left);
            const uint32_t jl = (uint32_t)__shfl((int)j, l, 64);
            const float pl = __shfl(p, l, 64);
            const T* v = head_row<T>(a.v, jl, head / a.group);
            if (lane < a.width) o[0] = fmaf(pl, (float)v[lane], o[0]);
            if (lane + WAVE < a.width) o[1] = fmaf(pl, (float)v[lane + WAVE], o[1]);
        }
    }
    total = lanes_sum<64>(total);
    const float inv = total == 0.f ? 0.f : 1.f / total;
    o[0] *= inv;
    o[1] *= inv;
    lse = total == 0.f ? -__builtin_inff() : base + log2f(total) * LN2;
}

// Weights are formed anew as 2^(x - high - low), x to base two.  high is the row's logarithm and low zero, but where the logarithm
// is so large that its own rounding would show (every shown word is masked by a large finite value, or scores are huge):
// there high is the row's largest x and low the logarithm of its sum beside it, both found anew from the scores.
constexpr float FAR = 1024.f;         // of a logarithm: its rounding, a few 2^-13, is the relative error of the row's weights
__device__ inline bool is_far(float lse) { return fabsf(lse) > FAR && fabsf(lse) < __builtin_inff(); }
struct RowSum { float high, low, delta; };

// p and dS of (i, j).  (A word that is shown nothing, or only scores of -infinity, has high = 0: each of its weights is zero.)
template <typename T>
__device__ inline float2 row_gradient(const BackwardArgs& b, uint32_t head, uint32_t i, uint32_t j, const RowSum& r) {
    const AttendArgs& a = b.a;
    const float p = exp2f(row_score<T>(a, head, i, j) - r.high - r.low);
    const float dp = dot_rows(head_row<T>(b.dout, i, head), head_row<T>(a.v, j, head / a.group), a.width);
    return make_float2(p, p == 0.f ? 0.f : p * (dp - r.delta));
}

// dq_i.
template <typename T>
__device__ void query_row(const BackwardArgs& b, uint32_t head, uint32_t i, const Shown& s, const RowSum& r, uint32_t lane,
                          float (&dq)[2]) {
    const AttendArgs& a = b.a;
    const uint32_t sunk = s.sunk - s.first, n = sunk + s.hi - s.lo;
    dq[0] = dq[1] = r.high != r.high ? __builtin_nanf("") : 0.f;
    if (r.high != r.high) return;                     // its weights are not numbers, and so is every column
    for (uint32_t at0 = 0; at0 < n; at0 += WAVE) {
        const uint32_t at = at0 + lane;
        const uint32_t j = at < sunk ? s.first + at : s.lo + at - sunk;
        const bool in = at < n && row_keeps(a, i, j);
        const float ds = in ? row_gradient<T>(b, head, i, j, r).y : 0.f;
        for (uint64_t left = __ballot(in && ds != 0.f); left; left &= left - 1) {
            const int l = __builtin_ctzll(left);
            const uint32_t jl = (uint32_t)__shfl((int)j, l, 64);
            const float x = __shfl(ds, l, 64);
            const T* k = head_row<T>(a.k, jl, head / a.group);
            if (lane < a.width) dq[0] = fmaf(x, (float)k[lane], dq[0]);
            if (lane + WAVE < a.width) dq[1] = fmaf(x, (float)k[lane + WAVE], dq[1]);
        }
    }
    dq[0] *= a.scale;
    dq[1] *= a.scale;
}

// dk_j and dv_j of a key head, over queries [lo, hi) of all heads that share it, added to dk and dv (dk without the scale).
template <typename T>
__device__ void key_row(const BackwardArgs& b, uint32_t kv_head, uint32_t j, uint32_t lo, uint32_t hi, uint32_t lane,
                        float (&dk)[2], float (&dv)[2]) {
    const AttendArgs& a = b.a;
    for (uint32_t head = kv_head * a.group; head < (kv_head + 1) * a.group; ++head)
        for (uint32_t i0 = lo; i0 < hi; i0 += WAVE) {
            const uint32_t i = i0 + lane;
            const bool in = i < hi && row_keeps(a, i, j);
            float2 g = make_float2(0.f, 0.f);
            const size_t at = (size_t)head * a.T + i;
            if (__any(in && b.high[at] != b.high[at])) {      // one such query is enough
                dk[0] = dk[1] = dv[0] = dv[1] = __builtin_nanf("");
                return;
            }
            if (in) g = row_gradient<T>(b, head, i, j, RowSum{b.high[at], b.low[at], b.delta[at]});
            for (uint64_t left = __ballot(in && g.x != 0.f); left; left &= left - 1) {
                const int l = __builtin_ctzll(left);
                const uint32_t il = (uint32_t)__shfl((int)i, l, 64);
                const float p = __shfl(g.x, l, 64), ds = __shfl(g.y, l, 64);
                const T *q = head_row<T>(a.q, il, head), *o = head_row<T>(b.dout, il, head);
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (lane + c * WAVE < a.width) {
                        dk[c] = fmaf(ds, (float)q[lane + c * WAVE], dk[c]);
                        dv[c] = fmaf(p, (float)o[lane + c * WAVE], dv[c]);
                    }
            }
        }
}

}  // namespace w2v

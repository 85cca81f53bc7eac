// The kernels of one new word's attention over cached keys and values, for k_step.hip (rows one stride apart) and k_pages.hip (rows
// in pages).
//
// Every shown row of k and v is read once and used for the few query heads that share it: the way through memory
// bounds it.  A row lies in L lanes of 16 bytes each, so a wavefront reads 64 / L rows at a time and asks for four of each before it
// works on any; a group of lanes keeps maximum, sum and output of its own keys for HEADS query heads in registers, and
// groups, wavefronts and, for long caches, blocks are joined at the end in a fixed order.  Rows that
// `keep` leaves out are read but not used.  All arithmetic is fp32.
#pragma once
#include <type_traits>

#include "attend.h"
#include "tiles.h"

namespace w2v {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / (int)WAVE, AHEAD = 4;

// The keys of a text on one axis: `sunk` first words, then the window up to the new word.  Over pages those from `begin` on.
struct Keys {
    uint32_t first, sunk, lo, count, last;
    __device__ __forceinline__ uint32_t word(uint32_t at) const { return at < sunk ? first + at : lo + at - sunk; }
};
template <bool PAGED> __device__ inline Keys step_keys(const StepArgs& a, uint32_t text) {
    const uint32_t n = a.n[text] < a.room ? a.n[text] : a.room;
    Keys k{0, 0, 0, 0, 0};
    if (n == 0) return k;
    k.last = n - 1;
    k.lo = k.last > a.left ? k.last - a.left : 0;
    k.sunk = k.lo < a.sinks ? k.lo : a.sinks;
    if constexpr (PAGED) {
        k.first = k.sunk < a.begin ? k.sunk : a.begin;
        k.sunk -= k.first;
        k.lo = k.lo < a.begin ? a.begin : k.lo;
        k.count = k.sunk + (n > k.lo ? n - k.lo : 0);
    } else {
        k.count = k.sunk + n - k.lo;
    }
    return k;
}

// Wavefronts a SIMD that the registers are held to: what the plain walk needs by itself.
template <typename T, int HEADS> constexpr int step_waves = (HEADS == 1 ? 5 : HEADS == 2 ? 4 : HEADS == 4 ? 3 : 2) + (sizeof(T) == 4);

// PAGED: where a row lies is looked up in the table of pages, one step ahead of the rows.  WAVES wavefronts a block.
template <typename T, int L, int HEADS, bool PAGED, int WAVES>
__global__ __launch_bounds__(64 * WAVES, (step_waves<T, HEADS>)) void step_kernel(const StepArgs a) {
    constexpr int N = pack16<T>, GROUPS = WAVE / L, THREADS = 64 * WAVES;
    typedef typename Pack<T, N>::vec vec;
    extern __shared__ float dynamic[];                // bias by distance 0 .. -span for each head, times log2 e
    __shared__ float joined[WAVES][HEADS][L * N + 2];
    const uint32_t lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, part = lane % L, group = lane / L;
    const uint32_t rounds = (a.group + HEADS - 1) / HEADS;
    uint32_t at = blockIdx.x;
    // (over pages the heads of the same words follow each other, whose rows lie side by side in memory)
    const uint32_t paged_head = at % a.kv_heads;
    if (PAGED) at /= a.kv_heads;
    const uint32_t split = at % a.splits; at /= a.splits;
    const uint32_t round = at % rounds; at /= rounds;
    const uint32_t kv_head = PAGED ? paged_head : at % a.kv_heads, text = PAGED ? at : at / a.kv_heads;
    const uint32_t head0 = kv_head * a.group + round * HEADS;
    const uint32_t heads = a.group - round * HEADS < HEADS ? a.group - round * HEADS : HEADS;
    const Keys keys = step_keys<PAGED>(a, text);
    const uint32_t from = split * a.per_split, to = keys.count < from + a.per_split ? keys.count : from + a.per_split;
    const bool whole = a.splits == 1 && !(PAGED && a.front);
    if (from >= to && !(split == 0 && whole)) return;

    if (a.bias) {
        for (uint32_t c = threadIdx.x; c < (a.span + 1) * heads; c += THREADS)
            dynamic[c] = scaled_bias(a.bias, a.buckets, a.n_buckets, a.span, head0 + c % heads, -(int32_t)(c / heads));
        __syncthreads();
    }
    // a lane's columns: start .. start + N, of which those before c0 are its neighbour's (the row's last 16 bytes are read whole)
    const uint32_t c0 = part * N, start = a.width < N ? 0 : c0 < a.width - N ? c0 : a.width - N;
    float q[HEADS][N], acc[HEADS][N], m[HEADS], total[HEADS];
#pragma unroll
    for (int g = 0; g < HEADS; ++g)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const uint32_t c = start + e;
            q[g][e] = g < (int)heads && c >= c0 && c < a.width ? (float)head_row<T>(a.q, text, head0 + g)[c] * a.scale2 : 0.f;
        }
    const T* const k0 = (const T*)a.k.p + (PAGED ? 0 : (uint64_t)text * a.k.text) + (uint64_t)kv_head * a.k.head;
    const T* const v0 = (const T*)a.v.p + (PAGED ? 0 : (uint64_t)text * a.v.text) + (uint64_t)kv_head * a.v.head;

    constexpr uint32_t STEP = GROUPS * AHEAD;         // keys of a wavefront's step
    const bool masked = a.keep || a.skip_self;
    vec kx[AHEAD], vx[AHEAD];
    uint32_t j[AHEAD];
    uint8_t keep[AHEAD];
    uint32_t page[AHEAD], next_page[AHEAD];
    const auto ask = [&](uint32_t n0) __attribute__((always_inline)) {
        if (n0 >= to) return;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const uint32_t n = n0 + u * GROUPS + group, at = n < to ? n : to - 1;
            const uint32_t word = keys.word(at);
            next_page[u] = a.table[(word < a.shared ? 0 : (uint64_t)text * a.table_stride) + (word >> a.shift)];
        }
    };
    const auto fetch = [&](uint32_t n0) __attribute__((always_inline)) {      // (past the end: the last key again, without weight)
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const uint32_t n = n0 + u * GROUPS + group, at = n < to ? n : to - 1;
            j[u] = PAGED ? keys.word(at) : at < keys.sunk ? at : keys.lo + at - keys.sunk;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if constexpr (PAGED) {
                const uint32_t at = page[u] < a.n_pages ? page[u] : 0, place = j[u] & ((1u << a.shift) - 1);
                kx[u] = chunk_read<T, L == 8>(k0 + at * a.k.text + place * a.k.token, c0, a.width);
                vx[u] = chunk_read<T, L == 8>(v0 + at * a.v.text + place * a.v.token, c0, a.width);
            } else {
                kx[u] = chunk_read<T, L == 8>(k0 + (uint64_t)j[u] * a.k.token, c0, a.width);
                vx[u] = chunk_read<T, L == 8>(v0 + (uint64_t)j[u] * a.v.token, c0, a.width);
            }
            keep[u] = 1;
        }
        if (a.keep)
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) keep[u] = a.keep[(uint64_t)text * a.room + j[u]];
    };
    // CAREFUL: what has no part in a sum is left out of it, not multiplied by zero -- a neighbour's columns, and values of weight
    // zero, which may be infinite.  Taken where the plain walk, whose finite sums are the same, meets a value that is not finite.
    const auto walk = [&](auto CAREFUL) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < HEADS; ++g) {
            m[g] = -__builtin_inff();
            total[g] = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) acc[g][e] = 0.f;
        }
        if constexpr (PAGED) ask(from + wave * STEP);
        for (uint32_t n0 = from + wave * STEP; n0 < to; n0 += WAVES * STEP) {
            if constexpr (PAGED)
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) page[u] = next_page[u];
            fetch(n0);
            if constexpr (PAGED) ask(n0 + WAVES * STEP);
            if constexpr (CAREFUL.value)
#pragma unroll
                for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                    for (int e = 0; e < N; ++e) if (!(start + e >= c0 && start + e < a.width)) kx[u][e] = (T)0.f;
            bool in[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                in[u] = n0 + u * GROUPS + group < to && keep[u] && !(a.skip_self && j[u] == keys.last);
                if constexpr (PAGED) in[u] &= page[u] < a.n_pages;
            }
            if (PAGED || masked || n0 + STEP > to)                 // what is not shown must not show, whatever it holds
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) vx[u] = in[u] ? vx[u] : vec{};
#pragma unroll
            for (int g = 0; g < HEADS; ++g) {
                float x[AHEAD], most = m[g];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    float s = 0.f;
#pragma unroll
                    for (int e = 0; e < N; ++e) s = fmaf((float)kx[u][e], q[g][e], s);
                    s = lanes_sum<L>(s);
                    if (a.bias && g < (int)heads) {
                        const uint32_t back = keys.last - j[u] < a.span ? keys.last - j[u] : a.span;
                        s += dynamic[(in[u] ? back : 0) * heads + g];
                    }
                    x[u] = in[u] ? s : -__builtin_inff();
                    most = fmaxf(most, x[u]);
                }
                const float base = most == -__builtin_inff() ? 0.f : most;
                const float factor = __builtin_amdgcn_exp2f(m[g] - base);
                m[g] = most;
                total[g] *= factor;
#pragma unroll
                for (int e = 0; e < N; ++e) acc[g][e] *= factor;
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const float p = __builtin_amdgcn_exp2f(x[u] - base);
                    total[g] += p;
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        acc[g][e] = CAREFUL.value && p == 0.f ? acc[g][e] : fmaf(p, (float)vx[u][e], acc[g][e]);
                }
            }
        }
    };
    walk(std::false_type{});
    float worst = 0.f;                                // not a number, if any sum is not finite
#pragma unroll
    for (int g = 0; g < HEADS; ++g) {
        worst = fmaf(total[g], 0.f, worst);
#pragma unroll
        for (int e = 0; e < N; ++e) worst = fmaf(acc[g][e], 0.f, worst);
    }
    if (__any(worst != 0.f)) walk(std::true_type{});
    // the groups of a wavefront, then the wavefronts
#pragma unroll
    for (int g = 0; g < HEADS; ++g) {
        float most = m[g];
#pragma unroll
        for (int d = L; d < (int)WAVE; d *= 2) most = fmaxf(most, __shfl_xor(most, d, 64));
        const float factor = m[g] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m[g] - most);
        total[g] *= factor;
#pragma unroll
        for (int d = L; d < (int)WAVE; d *= 2) total[g] += __shfl_xor(total[g], d, 64);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            acc[g][e] *= factor;
#pragma unroll
            for (int d = L; d < (int)WAVE; d *= 2) acc[g][e] += __shfl_xor(acc[g][e], d, 64);
        }
        if (group == 0) {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (start + e >= c0 && start + e < a.width) joined[wave][g][2 + start + e] = acc[g][e];
            if (part == 0) { joined[wave][g][0] = most; joined[wave][g][1] = total[g]; }
        }
    }
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < heads * a.width; c += THREADS) {
        const uint32_t g = c / a.width, col = c % a.width;
        float most = -__builtin_inff(), sum = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = fmaxf(most, joined[w][g][0]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float mw = joined[w][g][0], f = mw == -__builtin_inff() ? (joined[w][g][1] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(mw - most);
            sum = fmaf(f, joined[w][g][1], sum);
            o = fmaf(f, joined[w][g][2 + col], o);
        }
        const uint32_t head = head0 + g;
        if (whole) {
            head_row<T>(a.o, text, head)[col] = (T)(sum == 0.f ? 0.f : o / sum);
        } else {
            const uint64_t row = (uint64_t)text * a.heads + head;
            float* p = a.parts + (PAGED ? row * (a.front + a.splits) + a.front + split : row * a.splits + split) * (a.width + 2);
            p[2 + col] = o;
            if (col == 0) { p[0] = most; p[1] = sum; }
        }
    }
}

// Joins the splits of a text's cache: one wavefront per text and head.
template <typename T> __global__ __launch_bounds__(THREADS) void step_join_kernel(const StepArgs a) {
    const uint32_t lane = threadIdx.x % WAVE;
    const uint64_t at = (uint64_t)blockIdx.x * WAVES + threadIdx.x / WAVE;
    if (at >= (uint64_t)a.batch * a.heads) return;
    const uint32_t text = (uint32_t)(at / a.heads), head = (uint32_t)(at % a.heads);
    const Keys keys = step_keys<false>(a, text);
    const uint32_t count = (keys.count + a.per_split - 1) / a.per_split;
    const uint32_t row = a.width + 2;
    const float* p = a.parts + at * a.splits * row;
    float most = -__builtin_inff(), sum = 0.f, o[2] = {0.f, 0.f};
    for (uint32_t s = lane; s < count; s += WAVE) most = fmaxf(most, p[(uint64_t)s * row]);
    most = wave_max(most);
    for (uint32_t s0 = 0; s0 < count; s0 += WAVE) {
        const uint32_t s = s0 + lane;
        const float m = s < count ? p[(uint64_t)s * row] : -__builtin_inff(), part = s < count ? p[(uint64_t)s * row + 1] : 0.f;
        const float f = m == -__builtin_inff() ? (part == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - most);
        sum += lanes_sum<64>(f * part);
        const uint32_t here = count - s0 < WAVE ? count - s0 : WAVE;
#pragma unroll 8
        for (uint32_t l = 0; l < here; ++l) {
            const float fl = __shfl(f, (int)l, 64);
            const float* x = p + (uint64_t)(s0 + l) * row + 2;
#pragma unroll
            for (int c = 0; c < 2; ++c) if (lane + c * WAVE < a.width) o[c] = fmaf(fl, x[lane + c * WAVE], o[c]);
        }
    }
    T* to = head_row<T>(a.o, text, head);
#pragma unroll
    for (int c = 0; c < 2; ++c)
        if (lane + c * WAVE < a.width) to[lane + c * WAVE] = (T)(sum == 0.f ? 0.f : o[c] / sum);
}

// The same over pages, where a row may have many parts: a block per text and head.  A part's columns lie in L lanes, four each, so
// the block reads 256 / L parts at a time; what the groups of lanes have summed is added in their order.  (2048 rows of 34 parts of 128
// columns: 9 us; a wavefront a row, one part after the other, took 28.)
template <typename T> __global__ __launch_bounds__(THREADS) void pages_join_kernel(const StepArgs a, uint32_t L) {
    extern __shared__ float factors[];                // of each part
    __shared__ float waves[2][WAVES], sums[THREADS][4];
    const uint32_t tid = threadIdx.x, text = blockIdx.x / a.heads, head = blockIdx.x % a.heads;
    const Keys keys = step_keys<true>(a, text);
    const uint32_t count = (keys.count + a.per_split - 1) / a.per_split + a.front, row = a.width + 2;
    const float* p = a.parts + (uint64_t)blockIdx.x * (a.front + a.splits) * row;
    float most = -__builtin_inff();
    for (uint32_t s = tid; s < count; s += THREADS) most = fmaxf(most, p[(uint64_t)s * row]);
    most = wave_max(most);
    if (tid % WAVE == 0) waves[0][tid / WAVE] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) most = fmaxf(most, waves[0][w]);
    float total = 0.f;
    for (uint32_t s = tid; s < count; s += THREADS) {
        const float m = p[(uint64_t)s * row], part = p[(uint64_t)s * row + 1];
        const float f = m == -__builtin_inff() ? (part == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - most);
        factors[s] = f;
        total += f == 0.f ? 0.f : f * part;           // (a part of no weight does not show, whatever it holds)
    }
    total = lanes_sum<64>(total);
    if (tid % WAVE == 0) waves[1][tid / WAVE] = total;
    __syncthreads();
    total = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) total += waves[1][w];
    typedef Pack<float, 4>::vec vec;
    const uint32_t c = tid % L * 4, start = a.width < 4 ? 0 : c < a.width - 4 ? c : a.width - 4, groups = THREADS / L;
    vec o = {};
    if (c < a.width) {
#pragma unroll 4
        for (uint32_t s = tid / L; s < count; s += groups) {
            const float* x = p + (uint64_t)s * row + 2;
            vec four;
            if (a.width < 4)
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) four[e] = x[e < a.width ? e : 0];
            else four = *(const Pack<float, 4>::mem*)(x + start);
            const float f = factors[s];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = f == 0.f ? o[e] : fmaf(f, four[e], o[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[tid][e] = o[e];
    __syncthreads();
    if (tid >= a.width) return;
    const uint32_t lane = tid / 4, e = tid < a.width / 4 * 4 || a.width < 4 ? tid % 4 : tid + 4 - a.width;      // (the last columns lie in a lane that starts earlier)
    float x = 0.f;
    for (uint32_t g = 0; g < groups; ++g) x += sums[g * L + lane][e];
    head_row<T>(a.o, text, head)[tid] = (T)(total == 0.f ? 0.f : x / total);
}

template <typename T, int L, int HEADS, bool PAGED> void step_run(const StepArgs& a, hipStream_t st) {
    const uint32_t rounds = (a.group + HEADS - 1) / HEADS;
    const size_t table = a.bias ? (size_t)(a.span + 1) * HEADS * sizeof(float) : 0;
    const uint32_t blocks = a.batch * a.kv_heads * rounds * a.splits;
    if constexpr (PAGED) {
        // Fewer blocks than compute units, each with all of its text's words: twice the wavefronts, whose rows are on their way at the same
        // time (500 words, 5 heads of 60 in 32 bits: 9.2 us, 12.4; with more blocks than that it costs: 288 of 1028 words 37 us, 33).
        if (a.front + a.splits == 1 && blocks <= 256) return step_kernel<T, L, HEADS, true, 2 * WAVES><<<blocks, 2 * THREADS, table, st>>>(a);
    }
    step_kernel<T, L, HEADS, PAGED, WAVES><<<blocks, THREADS, table, st>>>(a);
}
template <typename T, int L, bool PAGED> void step_heads(const StepArgs& a, hipStream_t st) {
    if (a.group == 1) step_run<T, L, 1, PAGED>(a, st);
    else if (a.group == 2) step_run<T, L, 2, PAGED>(a, st);
    else if (a.group <= 4) step_run<T, L, 4, PAGED>(a, st);
    else step_run<T, L, 8, PAGED>(a, st);
}
template <typename T, bool PAGED> void step_any(const StepArgs& a, hipStream_t st) {
    const uint32_t chunks = (a.width + pack16<T> - 1) / pack16<T>;
    if (chunks <= 8) step_heads<T, 8, PAGED>(a, st);
    else if (chunks <= 16) step_heads<T, 16, PAGED>(a, st);
    else if constexpr (sizeof(T) == 4) step_heads<T, 32, PAGED>(a, st);
    if constexpr (!PAGED) {
        if (a.splits > 1) step_join_kernel<T><<<(uint32_t)(((uint64_t)a.batch * a.heads + WAVES - 1) / WAVES), THREADS, 0, st>>>(a);
    }
}
template <typename T> void pages_join(const StepArgs& a, hipStream_t st) {
    uint32_t L = 1;
    while (L * 4 < a.width) L *= 2;
    if (a.front + a.splits > 1) pages_join_kernel<T><<<a.batch * a.heads, THREADS, (a.front + a.splits) * sizeof(float), st>>>(a, L);
}

}  // namespace
}  // namespace w2v

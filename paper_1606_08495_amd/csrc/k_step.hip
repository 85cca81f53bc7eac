// Attention of one new word per text over cached keys and values.
//
// Every shown row of k and v is read once and used for the few query heads that share it: the way through memory
// bounds it.  A row lies in L lanes of 16 bytes each, so a wavefront reads 64 / L rows at a time and asks for four of each before it
// works on any; a group of lanes keeps maximum, sum and output of its own keys for HEADS query heads in registers, and
// groups, wavefronts and, for long caches, blocks are joined at the end in a fixed order.  Rows that
// `keep` leaves out are read but not used.  All arithmetic is fp32.
// Measured: 32 texts of up to 32768 words (574335 in all), 32 heads of 128 over 8, 16 bits: 590 us (4.0 TB/s; a large copy moves
// 4.8).  One text of 500 words, 5 heads of 60: 8 us and 4 us for the join.
#include <type_traits>

#include "attend.h"
#include "tiles.h"

namespace w2v {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / (int)WAVE, AHEAD = 4;

// The keys of a text on one axis: `sunk` first words, then the window up to the new word.
struct Keys { uint32_t sunk, lo, count, last; };
__device__ inline Keys step_keys(const StepArgs& a, uint32_t text) {
    const uint32_t n = a.n[text] < a.room ? a.n[text] : a.room;
    Keys k{0, 0, 0, 0};
    if (n == 0) return k;
    k.last = n - 1;
    k.lo = k.last > a.left ? k.last - a.left : 0;
    k.sunk = k.lo < a.sinks ? k.lo : a.sinks;
    k.count = k.sunk + n - k.lo;
    return k;
}

// Wavefronts a SIMD that the registers are held to: what the plain walk needs by itself.
template <typename T, int HEADS> constexpr int step_waves = (HEADS == 1 ? 5 : HEADS == 2 ? 4 : HEADS == 4 ? 3 : 2) + (sizeof(T) == 4);

template <typename T, int L, int HEADS>
__global__ __launch_bounds__(THREADS, (step_waves<T, HEADS>)) void step_kernel(const StepArgs a) {
    constexpr int N = pack16<T>, GROUPS = WAVE / L;
    typedef typename Pack<T, N>::vec vec;
    extern __shared__ float dynamic[];                // bias by distance 0 .. -span for each head, times log2 e
    __shared__ float joined[WAVES][HEADS][L * N + 2];
    const uint32_t lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, part = lane % L, group = lane / L;
    const uint32_t rounds = (a.group + HEADS - 1) / HEADS;
    uint32_t at = blockIdx.x;
    const uint32_t split = at % a.splits; at /= a.splits;
    const uint32_t round = at % rounds; at /= rounds;
    const uint32_t kv_head = at % a.kv_heads, text = at / a.kv_heads;
    const uint32_t head0 = kv_head * a.group + round * HEADS;
    const uint32_t heads = a.group - round * HEADS < HEADS ? a.group - round * HEADS : HEADS;
    const Keys keys = step_keys(a, text);
    const uint32_t from = split * a.per_split, to = keys.count < from + a.per_split ? keys.count : from + a.per_split;
    if (from >= to && !(split == 0 && a.splits == 1)) return;

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
    const T* const k0 = (const T*)a.k.p + (uint64_t)text * a.k.text + (uint64_t)kv_head * a.k.head;
    const T* const v0 = (const T*)a.v.p + (uint64_t)text * a.v.text + (uint64_t)kv_head * a.v.head;

    constexpr uint32_t STEP = GROUPS * AHEAD;         // keys of a wavefront's step
    const bool masked = a.keep || a.skip_self;
    vec kx[AHEAD], vx[AHEAD];
    uint32_t j[AHEAD];
    uint8_t keep[AHEAD];
    const auto fetch = [&](uint32_t n0) __attribute__((always_inline)) {      // (past the end: the last key again, without weight)
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const uint32_t n = n0 + u * GROUPS + group, at = n < to ? n : to - 1;
            j[u] = at < keys.sunk ? at : keys.lo + at - keys.sunk;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            kx[u] = chunk_read<T, L == 8>(k0 + (uint64_t)j[u] * a.k.token, c0, a.width);
            vx[u] = chunk_read<T, L == 8>(v0 + (uint64_t)j[u] * a.v.token, c0, a.width);
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
        for (uint32_t n0 = from + wave * STEP; n0 < to; n0 += WAVES * STEP) {
            fetch(n0);
            if constexpr (CAREFUL.value)
#pragma unroll
                for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                    for (int e = 0; e < N; ++e) if (!(start + e >= c0 && start + e < a.width)) kx[u][e] = (T)0.f;
            bool in[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                in[u] = n0 + u * GROUPS + group < to && keep[u] && !(a.skip_self && j[u] == keys.last);
            if (masked || n0 + STEP > to)                 // what is not shown must not show, whatever it holds
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
        if (a.splits == 1) {
            head_row<T>(a.o, text, head)[col] = (T)(sum == 0.f ? 0.f : o / sum);
        } else {
            float* p = a.parts + (((uint64_t)text * a.heads + head) * a.splits + split) * (a.width + 2);
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
    const Keys keys = step_keys(a, text);
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

template <typename T, int L, int HEADS> void step_run(const StepArgs& a, hipStream_t st) {
    const uint32_t rounds = (a.group + HEADS - 1) / HEADS;
    const size_t table = a.bias ? (size_t)(a.span + 1) * HEADS * sizeof(float) : 0;
    step_kernel<T, L, HEADS><<<a.batch * a.kv_heads * rounds * a.splits, THREADS, table, st>>>(a);
}
template <typename T, int L> void step_heads(const StepArgs& a, hipStream_t st) {
    if (a.group == 1) step_run<T, L, 1>(a, st);
    else if (a.group == 2) step_run<T, L, 2>(a, st);
    else if (a.group <= 4) step_run<T, L, 4>(a, st);
    else step_run<T, L, 8>(a, st);
}
template <typename T> void step_any(const StepArgs& a, hipStream_t st) {
    const uint32_t chunks = (a.width + pack16<T> - 1) / pack16<T>;
    if (chunks <= 8) step_heads<T, 8>(a, st);
    else if (chunks <= 16) step_heads<T, 16>(a, st);
    else if constexpr (sizeof(T) == 4) step_heads<T, 32>(a, st);
    if (a.splits > 1) step_join_kernel<T><<<(uint32_t)(((uint64_t)a.batch * a.heads + WAVES - 1) / WAVES), THREADS, 0, st>>>(a);
}

}  // namespace

// Blocks enough to fill the device several times over where the caches are long, parts of at least 256 keys.
StepSplits step_splits(uint32_t batch, uint32_t kv_heads, uint32_t room, uint32_t left, uint32_t sinks) {
    const uint64_t most = (uint64_t)left + 1 + sinks < room ? (uint64_t)left + 1 + sinks : room;
    const uint64_t rows = (uint64_t)batch * kv_heads, want = 4096 / rows > 1 ? 4096 / rows : 1;
    uint64_t per = (most + want - 1) / want;
    per = per < 256 ? 256 : (per + 63) / 64 * 64;
    return StepSplits{(uint32_t)((most + per - 1) / per), (uint32_t)per};
}

void launch_step(const StepArgs& a, uint32_t type, hipStream_t st) {
    if (type == ELEM_F32) step_any<float>(a, st);
    else if (type == ELEM_F16) step_any<_Float16>(a, st);
    else step_any<__bf16>(a, st);
}

}  // namespace w2v

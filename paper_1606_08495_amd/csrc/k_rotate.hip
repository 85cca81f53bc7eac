// Positions that turn, and new words on their way into the pages of a cache.
//
//   y_a = gain (x_a cos t - x_b sin t),  y_b = gain (x_a sin t + x_b cos t),  t = position f_c
// for the pairs (a, b) = (2 c, 2 c + 1), or (c, c + r / 2), of a head's first r elements; the rest passes as it is.
//
// What bounds it is the rows' way through memory, once in and once out.  A block takes a few words: it finds their texts, positions
// and places, fills a table of their sines and cosines in LDS once for all heads of queries and keys, and then walks over all rows
// of those words, 16 bytes a thread, a thread's column fixed and some rows asked for before any is worked on.
// Measured: 131333 words in texts of 10 to 40, 5 + 5 heads of 60, 32 bits: 120 us (5.2 TB/s; a large copy moves 4.8).  39955 words of 16 + 4
// heads of 128, half of each turned, 16 bits, there and back: 161 us (5.1 TB/s).  26016 words of 40 prompts into pages, 32 query heads and 8
// keys and values of 128, 16 bits: 126 us (5.1 TB/s).  One word: 5 us, of which the launch is most.
//
// An angle is a whole number of 2^-64 turns times the position, modulo 2^64: exact, whatever the position.  Of its upper 32 bits (2^-32
// of a turn is 1.5e-9) the nearest quarter turn is taken off as a whole number too, and what is left, at most an eighth of a turn,
// goes through the power series of sine and cosine, whose first terms left out are below 2^-25 there.  All products are fp32, the
// result is rounded once.
#include <type_traits>

#include "attend.h"

namespace w2v {
namespace {

constexpr uint32_t THREADS = 256, TOKENS = 64, ANGLES = 1024;      // words of a block, and words times pairs, at most
static_assert(ANGLES >= HEAD_MAX / 2, "one word's");
// Rows that a thread asks for before it works on any (with a partner's chunk for each, half as many).
template <bool HALVES> constexpr int ahead = HALVES ? 2 : 4;
constexpr uint64_t NOWHERE = ~0ull;

__device__ __forceinline__ float2 cos_sin(uint64_t phase) {
    const uint32_t p = (uint32_t)(phase >> 32), quarter = (p + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(p - (quarter << 30)) * 1.4629180792671596e-9f;      // 2 pi / 2^32
    const float z = x * x;
    const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 40320, -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
    return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

// What a block knows of its words: where their rows go (elements from the start of each output), and their turned columns.
struct Words {
    int64_t position[TOKENS];
    uint64_t x[TOKENS], y[TOKENS], z[TOKENS];
    float2 table[ANGLES];                             // [words][pairs]
};

// The text of token i (the same in 16 lanes that look for it together), and whether it has it.
struct Found { uint32_t text; int64_t at, behind; bool in; };      // place in the text, words of the block that follow it there and itself
__device__ __forceinline__ Found find(const TurnArgs& a, uint32_t i, uint32_t lane) {
    if (!a.off) return Found{i, 0, 1, true};
    const uint32_t text = texts_of(a.off, a.n_sent, i, lane);
    const uint64_t first = a.off[text], end = a.off[text + 1];
    return Found{text, (int64_t)(i - first), (int64_t)(end - i < 1ull << 40 ? end - i : 1ull << 40), first <= i && i < end};
}

template <bool APPEND> __device__ __forceinline__ void place(const TurnArgs& a, Words& w, uint32_t word0, uint32_t count) {
    const uint32_t lane = threadIdx.x % WAVE;
    for (uint32_t slot = threadIdx.x / 16; slot < (count + 3) / 4 * 4; slot += THREADS / 16) {      // (a wavefront's four words together)
        const uint32_t i = word0 + (slot < count ? slot : count - 1);
        Found f{i, 0, 1, true};
        if (APPEND || !a.position) f = find(a, i, lane);
        int64_t at = f.at;
        uint64_t y = (uint64_t)i * a.y.out_token, z = 0;
        if constexpr (APPEND) {
            at = f.in ? (int64_t)a.n[f.text] - f.behind : 0;
            uint32_t page = a.n_pages;
            if (f.in && at >= 0 && at < (int64_t)a.room) page = a.table[(uint64_t)f.text * a.table_stride + ((uint32_t)at >> a.shift)];
            const uint32_t place = (uint32_t)at & ((1u << a.shift) - 1);
            y = page < a.n_pages ? page * a.y_page + place * a.y.out_token : NOWHERE;
            z = page < a.n_pages ? page * a.z_page + place * a.z.out_token : NOWHERE;
        }
        if (lane % 16 || slot >= count) continue;
        w.position[slot] = a.position ? (int64_t)a.position[i] : at;
        w.x[slot] = f.in ? (uint64_t)i * a.x.out_token : NOWHERE;
        w.y[slot] = f.in ? y : NOWHERE;
        w.z[slot] = z;
    }
}

// N elements of a row from c0 on, `some` of which are to be had.
template <typename T, int N> __device__ __forceinline__ typename Pack<T, N>::vec part_read(const T* row, uint32_t some) {
    if (some >= (uint32_t)N) return *(const typename Pack<T, N>::mem*)row;
    typename Pack<T, N>::vec v = {};
#pragma unroll
    for (int e = 0; e < N; ++e) if (e < (int)some) v[e] = row[e];
    return v;
}
template <typename T, int N> __device__ __forceinline__ void part_write(T* row, uint32_t some, typename Pack<T, N>::vec v) {
    if (some >= (uint32_t)N) {
        *(typename Pack<T, N>::mem*)row = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) if (e < (int)some) row[e] = v[e];
}

// Chunks of a row that a thread has one of.
__host__ __device__ __forceinline__ uint32_t row_units(bool halves, uint32_t width, uint32_t turned, uint32_t n) {
    return halves ? (turned / 2 + n - 1) / n + (width - turned + n - 1) / n : (width + n - 1) / n;
}

// All rows of one array of the block's words.
template <typename T, int N, bool HALVES>
__device__ __forceinline__ void walk(const TurnArgs& a, const TurnArray& x, uint32_t turned, const uint64_t* to, const Words& w,
                                     uint32_t word0, uint32_t count) {
    typedef typename Pack<T, N>::vec vec;
    constexpr int AHEAD = ahead<HALVES>;
    const uint32_t half = turned / 2, paired = HALVES ? (half + N - 1) / N : 0;      // chunks that have a partner in the other half
    const uint32_t units = row_units(HALVES, a.width, turned, N);
    const uint32_t step = THREADS / units, unit = threadIdx.x % units, first = threadIdx.x / units;
    if (first >= step) return;
    const bool pair = HALVES && unit < paired;
    uint32_t c0 = !HALVES ? unit * N : pair ? unit * N : turned + (unit - paired) * N;
    uint32_t some = (pair ? half : a.width) - c0;
    // A chunk that the row's end cuts begins earlier instead and does some of its neighbour's again, where that is nothing that it reads: in
    // another place than the input's.  (Pairs side by side stay together: the last element of an odd width then goes by itself.  Half a GB in 16
    // bits there and back: rows of 60 in halves 102 us, element by element 266; of 37 in pairs 150, 330.)
    bool single = false;
    if (some < (uint32_t)N && x.in.p != x.out) {
        const uint32_t back = N - some + (!HALVES && a.width % 2), begin = HALVES && !pair ? turned : 0;
        if (c0 >= begin + back) {
            c0 -= back;
            some = N;
            single = !HALVES && a.width % 2;
        }
    }
    const uint32_t step_words = step / x.heads, step_heads = step % x.heads, rows = count * x.heads;
    uint32_t word = first / x.heads, head = first % x.heads;
    for (uint32_t r = first; r < rows; r += AHEAD * step) {
        vec low[AHEAD], high[AHEAD];
        T last[AHEAD];
        uint32_t words[AHEAD], heads[AHEAD];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            words[n] = word < count ? word : count - 1;
            heads[n] = head;
            const T* row = (const T*)x.in.p + (uint64_t)(word0 + words[n]) * x.in.token + (uint64_t)head * x.in.head + c0;
            low[n] = part_read<T, N>(row, some);
            if (pair) high[n] = part_read<T, N>(row + half, some);
            if (!HALVES && single) last[n] = row[N];
            word += step_words;
            head += step_heads;
            if (head >= x.heads) { head -= x.heads; ++word; }
        }
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            const uint64_t at = to[words[n]];
            if (r + n * step >= rows || at == NOWHERE) continue;
            T* row = (T*)x.out + at + (uint64_t)heads[n] * x.out_head + c0;
            const float2* table = w.table + words[n] * half;
            if (pair) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float2 t = table[c0 + e < half ? c0 + e : 0];
                    const float p = (float)low[n][e], q = (float)high[n][e];
                    low[n][e] = (T)(p * t.x - q * t.y);
                    high[n][e] = (T)(p * t.y + q * t.x);
                }
                part_write<T, N>(row + half, some, high[n]);
            } else if (!HALVES && c0 < turned) {
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    const float2 t = table[c0 + e < turned ? (c0 + e) / 2 : 0];
                    const float p = (float)low[n][e], q = (float)low[n][e + 1];
                    if (c0 + e < turned) {
                        low[n][e] = (T)(p * t.x - q * t.y);
                        low[n][e + 1] = (T)(p * t.y + q * t.x);
                    }
                }
            }
            part_write<T, N>(row, some, low[n]);
            if (!HALVES && single) row[N] = last[n];
        }
    }
}

template <typename T, bool HALVES, bool APPEND> __global__ __launch_bounds__(THREADS) void turn_kernel(const TurnArgs a) {
    constexpr int N = pack16<T>;
    __shared__ Words w;
    const uint32_t block = blockIdx.y * gridDim.x + blockIdx.x, pairs = a.rotated / 2;
    if (block > (a.T - 1) / a.tokens) return;
    const uint32_t word0 = block * a.tokens, count = a.T - word0 < a.tokens ? a.T - word0 : a.tokens;
    place<APPEND>(a, w, word0, count);
    __syncthreads();
    for (uint32_t n = threadIdx.x; n < count * pairs; n += THREADS) {
        const float2 t = cos_sin((uint64_t)w.position[n / pairs] * a.turns[n % pairs]);
        w.table[n] = make_float2(a.gain * t.x, a.back ? -a.gain * t.y : a.gain * t.y);
    }
    __syncthreads();
    if (a.x.heads) walk<T, N, HALVES>(a, a.x, a.rotated, w.x, w, word0, count);
    if (a.y.heads) walk<T, N, HALVES>(a, a.y, a.rotated, w.y, w, word0, count);
    if (APPEND) walk<T, N, false>(a, a.z, 0, w.z, w, word0, count);
}

template <typename T, bool APPEND> void turn_run(const TurnArgs& a, hipStream_t st) {
    const uint32_t all = (a.T + a.tokens - 1) / a.tokens, wide = all < 1u << 23 ? all : 1u << 23;      // (threads on an axis: below 2^32)
    const dim3 blocks(wide, (all + wide - 1) / wide);
    if (a.halves) turn_kernel<T, true, APPEND><<<blocks, THREADS, 0, st>>>(a);
    else turn_kernel<T, false, APPEND><<<blocks, THREADS, 0, st>>>(a);
}
// Words of a block: as many as fill the threads with the rows of the array that has most heads, twice over where that is less than four
// words; fewer where there are few words.  (131333 words of 5 + 5 heads of 60 in 32 bits: 13 words a block 123 us, 8 140, 27 134;
// 39955 of 16 + 4 of 128 in 16 bits, in halves: 5 words 84 us, 3 93, 16 91.)
template <bool APPEND> void turn_any(TurnArgs& a, uint32_t type, hipStream_t st) {
    const uint32_t units = row_units(a.halves, a.width, a.rotated, 16 / elem_bytes(type)), heads = a.x.heads > a.y.heads ? a.x.heads : a.y.heads;
    const uint32_t rows = THREADS / units * (a.halves ? ahead<true> : ahead<false>), few = (a.T + 2047) / 2048;
    const uint32_t most = a.rotated > 2 * ANGLES / TOKENS ? 2 * ANGLES / a.rotated : TOKENS;
    a.tokens = rows / heads < 4 ? 2 * rows / heads : rows / heads < most ? rows / heads : most;
    if (a.tokens > few) a.tokens = few;
    if (a.tokens < 1) a.tokens = 1;
    if (type == ELEM_F32) turn_run<float, APPEND>(a, st);
    else if (type == ELEM_F16) turn_run<_Float16, APPEND>(a, st);
    else turn_run<__bf16, APPEND>(a, st);
}

}  // namespace

void launch_rotate(TurnArgs a, uint32_t type, hipStream_t st) { turn_any<false>(a, type, st); }
void launch_append(TurnArgs a, uint32_t type, hipStream_t st) { turn_any<true>(a, type, st); }

}  // namespace w2v

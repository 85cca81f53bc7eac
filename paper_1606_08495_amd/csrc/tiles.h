// Tiles of the attention kernels: 32 x 32 products on the matrix cores, and rows of heads staged in LDS.
//
// Every product here has the form C[m][n] += sum_k A[m][k] B[k][n] with 32 x 32 results and 16 steps of k.  Lane l
// feeds row m = l % 32 of A and column n = l % 32 of B, eight values of k each; which eight a half h = l / 32 feeds is
// free as long as A and B agree.  The result lies with column n = l % 32 in lane l, rows 8 (r / 4) + 4 h + r % 4 in its
// registers r = 0..15.  A result can therefore be the B operand of the next product without
// leaving its lanes: registers 8 s .. 8 s + 7 feed step s with k = 16 s + 8 (t / 4) + 4 h + t % 4, t = 0..7, and the A operand of
// that product is read in the same order ("across" below).  Scores are formed with their words' rows as m and the
// lane's own word as n, so the softmax over a word's row runs over a lane's registers and its partner's 32 lanes on.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "context.h"
#include "elem.h"

namespace w2v {

typedef float Acc __attribute__((ext_vector_type(16)));      // a 32 x 32 result

// A condition that hardly ever holds: what it guards, loops in loops, must not take registers from the walks.
__device__ __forceinline__ bool rare(uint64_t x) { return __builtin_expect(x != 0, 0); }

template <typename T> struct Frag { typedef typename Pack<T, 8>::vec vec; };      // a lane's eight values of an operand

__device__ __forceinline__ void mma(const Frag<_Float16>::vec& a, const Frag<_Float16>::vec& b, Acc& c) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mma(const Frag<__bf16>::vec& a, const Frag<__bf16>::vec& b, Acc& c) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mma(const Frag<float>::vec& a, const Frag<float>::vec& b, Acc& c) {
#pragma unroll
    for (int t = 0; t < 8; ++t) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[t], b[t], c, 0, 0, 0);
}

// Row of a result's register r in lane half h.
__device__ __forceinline__ constexpr int acc_row(int r, int h) { return 8 * (r / 4) + 4 * h + r % 4; }

// Registers 8 s .. 8 s + 7 of a result as the operand of the next product.
template <typename T> __device__ __forceinline__ typename Frag<T>::vec acc_operand(const Acc& c, int s) {
    typename Frag<T>::vec f;
#pragma unroll
    for (int t = 0; t < 8; ++t) f[t] = (T)c[8 * s + t];
    return f;
}

// Sum, and largest, over a lane and its partner in the other half of the wavefront.
__device__ __forceinline__ float halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Chunks: 16 bytes of a row of `width` elements, from element c0 on.  What lies past the row's end is not read: the chunk that
// the end cuts is read as the row's last 16 bytes and moved down afterwards (chunk_fit), and so are chunks wholly past it.
// No access depends on a condition, so that none waits for another.  Rows shorter than a chunk (where NARROW allows
// them) are read by elements.
template <typename T, bool NARROW> __device__ __forceinline__ typename Pack<T, pack16<T>>::vec chunk_read(const T* row, uint32_t c0, uint32_t width) {
    constexpr uint32_t N = pack16<T>;
    if (NARROW && width < N) {
        typename Pack<T, N>::vec x;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) x[e] = row[e < width ? e : width - 1];
        return x;
    }
    return *(const typename Pack<T, N>::mem*)(row + (c0 < width - N ? c0 : width - N));
}
template <typename T>
__device__ __forceinline__ typename Pack<T, pack16<T>>::vec chunk_fit(typename Pack<T, pack16<T>>::vec x, uint32_t c0, uint32_t width) {
    constexpr uint32_t N = pack16<T>;
    const uint32_t start = width >= N && c0 > width - N ? width - N : c0;
    const uint32_t by = (c0 - start) * (uint32_t)sizeof(T);      // bytes to move down by
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    Words w = __builtin_bit_cast(Words, x);
    const bool two = by & 8, one = by & 4, half = by & 2;
    w = Words{two ? w[2] : w[0], two ? w[3] : w[1], two ? 0u : w[2], two ? 0u : w[3]};
    w = Words{one ? w[1] : w[0], one ? w[2] : w[1], one ? w[3] : w[2], one ? 0u : w[3]};
    if constexpr (sizeof(T) == 2) {
        const Words u = {w[0] >> 16 | w[1] << 16, w[1] >> 16 | w[2] << 16, w[2] >> 16 | w[3] << 16, w[3] >> 16};
        w = Words{half ? u[0] : w[0], half ? u[1] : w[1], half ? u[2] : w[2], half ? u[3] : w[3]};
    }
    x = __builtin_bit_cast(typename Pack<T, N>::vec, w);
    if (c0 + N > width)
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) x[e] = c0 + e < width ? x[e] : (T)0.f;
    return x;
}

// A lane's operand for step s straight from its row in memory.
template <typename T, int DB> __device__ __forceinline__ typename Frag<T>::vec load_operand(const T* row, int s, uint32_t h, uint32_t width) {
    constexpr int N = pack16<T>;
    typename Frag<T>::vec f;
#pragma unroll
    for (int p = 0; p < 8 / N; ++p) {
        const uint32_t c0 = 16 * s + 8 * h + p * N;
        const auto x = chunk_fit<T>(chunk_read<T, DB == 1>(row, c0, width), c0, width);
#pragma unroll
        for (int e = 0; e < N; ++e) f[p * N + e] = x[e];
    }
    return f;
}

// ROWS rows of 32 DB elements in LDS.  Rows r, r + 4, r + 8 .. lie together, 16 bytes apart from each other, and the four such
// groups 64 bytes apart: what one access takes at a time -- a chunk of 16 rows, or 64 bytes of four rows side by side -- then
// meets in no bank, and every place is a lane's own base plus a constant.
template <typename T, int DB, int ROWS> struct Tile {
    static constexpr int N = pack16<T>, ROW = DB * 32 * (int)sizeof(T), CHUNKS = ROW / 16;
    static constexpr int STRIDE = ROW + 16, GROUP = ROWS / 4 * STRIDE + 64, BYTES = 4 * GROUP;
    static_assert(ROWS % 64 == 0, "groups begin 16 banks apart");
    typedef typename Pack<T, N>::vec Chunk;
    __device__ static __forceinline__ uint32_t place(uint32_t r, uint32_t c) { return (r & 3) * GROUP + (r >> 2) * STRIDE + c * 16; }
    // a lane's bases for the two reads
    __device__ static __forceinline__ uint32_t base_along(uint32_t lane) {
        return place(lane % 32, 0) + lane / 32 * 8 * (uint32_t)sizeof(T);
    }
    __device__ static __forceinline__ uint32_t base_across(uint32_t lane) {
        const uint32_t h = lane / 32;
        if constexpr (sizeof(T) == 2)      // 16 lanes: 4 rows of 32 bytes
            return ((lane >> 2) & 3) * GROUP + h * STRIDE + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
        else return h * STRIDE + lane % 32 * 4;
    }
    // rows r0 .. r0 + 31 as they are: a lane's row of A, step s
    __device__ static __forceinline__ typename Frag<T>::vec along(const char* tile, uint32_t base, int r0, int s) {
        typename Frag<T>::vec f;
        const char* at = tile + base + r0 / 4 * STRIDE + s * 16 * (int)sizeof(T);
#pragma unroll
        for (int p = 0; p < 8 / N; ++p) {
            const Chunk x = *(const Chunk*)(at + 16 * p);
#pragma unroll
            for (int e = 0; e < N; ++e) f[p * N + e] = x[e];
        }
        return f;
    }
    // columns as rows of A: element 32 b + lane % 32 of rows r0 + 16 s + 8 (t / 4) + 4 h + t % 4
    __device__ static __forceinline__ typename Frag<T>::vec across(const char* tile, uint32_t base, int r0, int s, int b) {
        const char* at = tile + base + (r0 / 4 + 4 * s) * STRIDE + b * 32 * (int)sizeof(T);
        if constexpr (sizeof(T) == 2) {
            typedef short Four __attribute__((ext_vector_type(4)));
            union { Four part[2]; typename Frag<T>::vec f; } u;
#pragma unroll
            for (int p = 0; p < 2; ++p)
                u.part[p] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) Four*)(at + 2 * p * STRIDE));
            return u.f;
        } else {
            typename Frag<T>::vec f;
#pragma unroll
            for (int t = 0; t < 8; ++t) f[t] = *(const T*)(at + 2 * (t / 4) * STRIDE + t % 4 * GROUP);
            return f;
        }
    }
};

// A tile's rows on their way from memory to LDS, in the registers of THREADS threads: a thread keeps one chunk's column and
// every RS-th row.  (Rows past the last one are copies of it, columns past the width of the last ones: the former are
// masked, the latter meet zeros or give columns that nobody reads.)
template <typename T, int DB, int ROWS, int THREADS> struct Transit {
    typedef Tile<T, DB, ROWS> Tl;
    static constexpr uint32_t LANES = Tl::CHUNKS <= 4 ? 4 : Tl::CHUNKS <= 8 ? 8 : Tl::CHUNKS <= 16 ? 16 : 32;
    static constexpr uint32_t RS = THREADS / LANES < ROWS ? THREADS / LANES : ROWS, PER = ROWS / RS;      // (threads past the rows: idle)
    typename Tl::Chunk x[PER];
    const T* at[PER];                                 // what is to be read next
    const T* base;                                    // the head's row of token 0
    const T* tile;                                    // this thread's first row of the next tile, if all its rows follow each other
    uint64_t stride;
    uint32_t r0, c0;
    // row 0 of the first tile is token `token` (which may lie before the first, where no such row is read)
    __device__ __forceinline__ void start(const Heads& p, uint32_t head, int64_t token) {
        r0 = threadIdx.x / LANES % ROWS;
        c0 = threadIdx.x % LANES * Tl::N;
        stride = p.token;
        base = (const T*)p.p + (uint64_t)head * p.head;
        tile = base + (token + r0) * (int64_t)stride;
    }
    // a whole tile whose rows follow each other
    __device__ __forceinline__ void aim() {
#pragma unroll
        for (uint32_t n = 0; n < PER; ++n) at[n] = tile + n * RS * stride;
    }
    // row r is token(r)
    template <typename F> __device__ __forceinline__ void aim(const F& token) {
#pragma unroll
        for (uint32_t n = 0; n < PER; ++n) at[n] = base + (uint64_t)token(r0 + n * RS) * stride;
    }
    __device__ __forceinline__ void load(uint32_t width) {
#pragma unroll
        for (uint32_t n = 0; n < PER; ++n) x[n] = chunk_read<T, DB == 1>(at[n], c0, width);
        tile += ROWS * stride;
    }
    // CLEAN: zeros past the width.  Rows whose bit of `kept` is not set become zeros (tiles of 64 rows).
    template <bool CLEAN = false> __device__ __forceinline__ void store(char* to, uint32_t width, uint64_t kept = ~0ull) {
        if (c0 >= (uint32_t)Tl::CHUNKS * Tl::N || threadIdx.x / LANES >= (uint32_t)ROWS) return;
        if (CLEAN || width % Tl::N)
#pragma unroll
            for (uint32_t n = 0; n < PER; ++n) x[n] = chunk_fit<T>(x[n], c0, width);
#pragma unroll
        for (uint32_t n = 0; n < PER; ++n) *(typename Tl::Chunk*)(to + Tl::place(r0 + n * RS, c0 / Tl::N)) = x[n];
        if (rare(~kept)) {                            // (over what was stored: selecting before it costs registers)
            const uint64_t gone = ~kept >> r0;
#pragma unroll
            for (uint32_t n = 0; n < PER; ++n)
                if (gone >> n * RS & 1) *(typename Tl::Chunk*)(to + Tl::place(r0 + n * RS, c0 / Tl::N)) = typename Tl::Chunk{};
        }
    }
};

}  // namespace w2v

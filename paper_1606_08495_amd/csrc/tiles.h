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

#include "elem.h"

namespace w2v {

typedef float Acc __attribute__((ext_vector_type(16)));      // a 32 x 32 result

template <typename T> struct Frag { typedef typename Pack<T, 8>::vec vec; };      // a lane's eight values of an operand

__device__ inline void mma(const Frag<_Float16>::vec& a, const Frag<_Float16>::vec& b, Acc& c) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ inline void mma(const Frag<__bf16>::vec& a, const Frag<__bf16>::vec& b, Acc& c) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline void mma(const Frag<float>::vec& a, const Frag<float>::vec& b, Acc& c) {
#pragma unroll
    for (int t = 0; t < 8; ++t) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[t], b[t], c, 0, 0, 0);
}

// Row of a result's register r in lane half h.
__device__ inline constexpr int acc_row(int r, int h) { return 8 * (r / 4) + 4 * h + r % 4; }

// Registers 8 s .. 8 s + 7 of a result as the operand of the next product.
template <typename T> __device__ inline typename Frag<T>::vec acc_operand(const Acc& c, int s) {
    typename Frag<T>::vec f;
#pragma unroll
    for (int t = 0; t < 8; ++t) f[t] = (T)c[8 * s + t];
    return f;
}

// Sum, and largest, over a lane and its partner in the other half of the wavefront.
__device__ inline float halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float halves_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 16 bytes of a row of `width` elements, from element c0 on; zeros past the row's end.
template <typename T> __device__ inline typename Pack<T, pack16<T>>::vec load_chunk(const T* row, uint32_t c0, uint32_t width) {
    constexpr int N = pack16<T>;
    typename Pack<T, N>::vec x;
    if (c0 + N <= width) {
        x = *(const typename Pack<T, N>::mem*)(row + c0);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = c0 + e < width ? row[c0 + e] : (T)0.f;
    }
    return x;
}

// A lane's operand for step s straight from its row in memory.
template <typename T> __device__ inline typename Frag<T>::vec load_operand(const T* row, int s, uint32_t h, uint32_t width) {
    constexpr int N = pack16<T>;
    typename Frag<T>::vec f;
#pragma unroll
    for (int p = 0; p < 8 / N; ++p) {
        const auto x = load_chunk(row, 16 * s + 8 * h + p * N, width);
#pragma unroll
        for (int e = 0; e < N; ++e) f[p * N + e] = x[e];
    }
    return f;
}

// ROWS rows of 32 DB elements in LDS, in chunks of 16 bytes.  Chunk c of row r lies at place c ^ turn(r) of its row: then
// neither 16 rows' chunks c nor four rows' 64 bytes side by side -- what the two reads below ask for at a time -- meet in a bank.
template <typename T, int DB, int ROWS> struct Tile {
    static constexpr int N = pack16<T>, ROW = DB * 32 * (int)sizeof(T), CHUNKS = ROW / 16, BYTES = ROWS * ROW;
    typedef typename Pack<T, N>::vec Chunk;
    __device__ static inline uint32_t turn(uint32_t r) {
        if constexpr (CHUNKS % 16 == 0) return ((r & 3) << 2) | ((r >> 2) & 3);
        else if constexpr (CHUNKS % 8 == 0) return ((r & 2) << 1) | ((r >> 1) & 2) | ((r >> 3) & 1);
        else return (r >> 2) & 3;
    }
    __device__ static inline uint32_t place(uint32_t r, uint32_t c) { return r * ROW + ((c ^ turn(r)) << 4); }
    // rows as they are: lane's row of A, step s
    __device__ static inline typename Frag<T>::vec along(const char* tile, uint32_t r, int s, uint32_t h) {
        typename Frag<T>::vec f;
#pragma unroll
        for (int p = 0; p < 8 / N; ++p) {
            const Chunk x = *(const Chunk*)(tile + place(r, (16 * s + 8 * h) / N + p));
#pragma unroll
            for (int e = 0; e < N; ++e) f[p * N + e] = x[e];
        }
        return f;
    }
    // columns as rows of A: element 32 b + lane % 32 of rows r0 + 16 s + 8 (t / 4) + 4 h + t % 4
    __device__ static inline typename Frag<T>::vec across(const char* tile, uint32_t r0, int s, int b, uint32_t lane) {
        typename Frag<T>::vec f;
        const uint32_t h = lane / 32;
        if constexpr (sizeof(T) == 2) {
            typedef short Four __attribute__((ext_vector_type(4)));
            union { Four part[2]; typename Frag<T>::vec f; } u;
            const uint32_t c = 4 * b + 2 * ((lane / 16) & 1) + ((lane >> 1) & 1);      // 16 lanes: 4 rows of 32 bytes
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const uint32_t r = r0 + 16 * s + 8 * p + 4 * h + ((lane >> 2) & 3);
                u.part[p] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) Four*)(tile + place(r, c) + 8 * (lane & 1)));
            }
            f = u.f;
        } else {
            const uint32_t at = 32 * b + lane % 32;
#pragma unroll
            for (int t = 0; t < 8; ++t)
                f[t] = *(const T*)(tile + place(r0 + 16 * s + 8 * (t / 4) + 4 * h + t % 4, at / N) + (at % N) * sizeof(T));
        }
        return f;
    }
};

// A tile's rows on their way from memory to LDS, in the registers of THREADS threads.
template <typename T, int DB, int ROWS, int THREADS> struct Transit {
    typedef Tile<T, DB, ROWS> Tl;
    static constexpr int PER = (ROWS * Tl::CHUNKS + THREADS - 1) / THREADS;
    typename Tl::Chunk x[PER];
    // row(r): the row's first element in memory, or null where the tile has none
    template <typename F> __device__ inline void load(F row, uint32_t width) {
#pragma unroll
        for (int n = 0; n < PER; ++n) {
            const uint32_t at = threadIdx.x + n * THREADS;
            typename Tl::Chunk z = {};
            x[n] = z;
            if (ROWS * Tl::CHUNKS % THREADS == 0 || at < ROWS * Tl::CHUNKS) {
                const T* p = row(at / Tl::CHUNKS);
                if (p) x[n] = load_chunk(p, (at % Tl::CHUNKS) * Tl::N, width);
            }
        }
    }
    __device__ inline void store(char* tile) const {
#pragma unroll
        for (int n = 0; n < PER; ++n) {
            const uint32_t at = threadIdx.x + n * THREADS;
            if (ROWS * Tl::CHUNKS % THREADS == 0 || at < ROWS * Tl::CHUNKS)
                *(typename Tl::Chunk*)(tile + Tl::place(at / Tl::CHUNKS, at % Tl::CHUNKS)) = x[n];
        }
    }
};

}  // namespace w2v

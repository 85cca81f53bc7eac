// Element types of the context operators and 16-byte accesses to rows that need not be aligned to them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace w2v {

enum ElemType : uint32_t { ELEM_F32 = 0, ELEM_F16 = 1, ELEM_BF16 = 2, ELEM_TYPES = 3 };
constexpr uint32_t elem_bytes(uint32_t type) { return type == ELEM_F32 ? 4 : 2; }

// N elements next to each other, in registers; memory holds them at any address that T itself may have (gfx950 reads
// and writes whole vectors at such addresses; an access that crosses a line costs that line).
template <typename T, int N> struct Pack;
template <int N> struct Pack<float, N> {
    typedef float vec __attribute__((ext_vector_type(N)));
    typedef float mem __attribute__((ext_vector_type(N), aligned(4)));
};
template <int N> struct Pack<_Float16, N> {
    typedef _Float16 vec __attribute__((ext_vector_type(N)));
    typedef _Float16 mem __attribute__((ext_vector_type(N), aligned(2)));
};
template <int N> struct Pack<__bf16, N> {
    typedef __bf16 vec __attribute__((ext_vector_type(N)));
    typedef __bf16 mem __attribute__((ext_vector_type(N), aligned(2)));
};
template <typename T> constexpr int pack16 = 16 / (int)sizeof(T);       // elements of 16 bytes

// The sum over aligned groups of G lanes (a power of two up to 64), in every lane of the group, in a fixed order.
template <int G> __device__ inline float lanes_sum(float x) {
#pragma unroll
    for (int m = 1; m < G; m *= 2) x += __shfl_xor(x, m, 64);
    return x;
}

}  // namespace w2v

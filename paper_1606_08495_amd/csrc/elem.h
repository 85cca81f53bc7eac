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

// The sum (or largest) over aligned groups of G lanes (a power of two up to 64), in every lane of the group, in a fixed order:
// exchanges inside registers, none through LDS.  (With pairs summed, a lane's mirror in 8 or 16 lanes holds what
// its partner 4 or 8 lanes on does.)
template <int CTRL> __device__ __forceinline__ float lane_partner(float x) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
template <int G, typename F> __device__ __forceinline__ float lanes_join(float x, const F& f) {
    if constexpr (G >= 2) x = f(x, lane_partner<0xB1>(x));        // quad_perm 1 0 3 2
    if constexpr (G >= 4) x = f(x, lane_partner<0x4E>(x));        // quad_perm 2 3 0 1
    if constexpr (G >= 8) x = f(x, lane_partner<0x141>(x));       // mirror in 8
    if constexpr (G >= 16) x = f(x, lane_partner<0x140>(x));      // mirror in 16
    if constexpr (G >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if constexpr (G >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return x;
}
template <int G> __device__ __forceinline__ float lanes_sum(float x) {
    return lanes_join<G>(x, [](float a, float b) __attribute__((always_inline)) { return a + b; });
}

}  // namespace w2v

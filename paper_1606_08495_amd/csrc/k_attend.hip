// Attention over texts, forward: one wavefront per word and head.
#include "attend.h"

namespace w2v {
namespace {

constexpr int THREADS = 256;

template <typename T> __global__ __launch_bounds__(THREADS) void attend_rows_kernel(const AttendArgs a) {
    const uint32_t lane = threadIdx.x % WAVE;
    const uint64_t at = (uint64_t)blockIdx.x * (THREADS / WAVE) + threadIdx.x / WAVE;
    const uint32_t i = (uint32_t)(at / a.heads), head = (uint32_t)(at % a.heads);
    if (i >= a.T) return;
    const Shown s = shown_to(a, i, text_bounds(a.off, text_of(a.off, a.n_sent, i, lane), i, a.T));
    float row[2], lse;
    attend_row<T>(a, head, i, s, lane, row, lse);
    T* out = head_row<T>(a.o, i, head);
    for (int c = 0; c < 2; ++c) if (lane + c * WAVE < a.width) out[lane + c * WAVE] = (T)row[c];
    if (lane == 0 && a.lse) a.lse[(size_t)head * a.T + i] = lse;
}

template <typename T> void attend_any(const AttendArgs& a, hipStream_t st) {
    attend_rows_kernel<T><<<(uint32_t)(((uint64_t)a.T * a.heads + 3) / 4), THREADS, 0, st>>>(a);
}

}  // namespace

void launch_attend(const AttendArgs& a, uint32_t type, hipStream_t st) {
    if (type == ELEM_F32) attend_any<float>(a, st);
    else if (type == ELEM_F16) attend_any<_Float16>(a, st);
    else attend_any<__bf16>(a, st);
}

}  // namespace w2v

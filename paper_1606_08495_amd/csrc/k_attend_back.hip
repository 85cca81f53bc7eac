// Attention over texts, backward: one wavefront at a time per word and head, and per word and key head.
#include "attend.h"

namespace w2v {
namespace {

constexpr int BLOCK_WORDS = 128, THREADS = 256, WAVES = THREADS / WAVE;

template <typename T> __global__ __launch_bounds__(THREADS) void query_rows_kernel(const BackwardArgs b) {
    const AttendArgs& a = b.a;
    __shared__ float sums[WAVES][2 * SPAN_MAX + 1];
    const uint32_t lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, head = blockIdx.x % a.heads;
    const uint32_t part = blockIdx.x / a.heads, distances = 2 * a.span + 1;
    if (b.dbias) for (uint32_t c = lane; c < distances; c += WAVE) sums[wave][c] = 0.f;
    for (uint32_t n = wave; n < BLOCK_WORDS; n += WAVES) {
        const uint32_t i = part * BLOCK_WORDS + n;
        if (i >= a.T) break;
        const Shown s = shown_to(a, i, text_bounds(a.off, text_of(a.off, a.n_sent, i, lane), i, a.T));
        const T *o = (const T*)head_row<T>(a.o, i, head), *g = head_row<T>(b.dout, i, head);
        float delta = 0.f;
        for (uint32_t c = lane; c < a.width; c += WAVE) delta = fmaf((float)o[c], (float)g[c], delta);
        delta = lanes_sum<64>(delta);
        if (lane == 0) b.delta[(size_t)head * a.T + i] = delta;
        float row[2];
        query_row<T>(b, head, i, s, delta, lane, row, b.dbias ? sums[wave] : nullptr);
        T* dq = head_row<T>(b.dq, i, head);
        for (int c = 0; c < 2; ++c) if (lane + c * WAVE < a.width) dq[lane + c * WAVE] = (T)row[c];
    }
    if (!b.dbias) return;
    __syncthreads();
    float* to = b.by_distance + ((size_t)head * gridDim.x / a.heads + part) * distances;
    for (uint32_t c = threadIdx.x; c < distances; c += THREADS)
        to[c] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
}

template <typename T> __global__ __launch_bounds__(THREADS) void key_rows_kernel(const BackwardArgs b) {
    const AttendArgs& a = b.a;
    const uint32_t lane = threadIdx.x % WAVE;
    const uint64_t at = (uint64_t)blockIdx.x * WAVES + threadIdx.x / WAVE;
    const uint32_t j = (uint32_t)(at / a.kv_heads), kv_head = (uint32_t)(at % a.kv_heads);
    if (j >= a.T) return;
    const Shown s = sees(a, j, text_bounds(a.off, text_of(a.off, a.n_sent, j, lane), j, a.T));
    float dk[2] = {0.f, 0.f}, dv[2] = {0.f, 0.f};
    key_row<T>(b, kv_head, j, s.lo, s.sunk, lane, dk, dv);
    T *to_k = head_row<T>(b.dk, j, kv_head), *to_v = head_row<T>(b.dv, j, kv_head);
    for (int c = 0; c < 2; ++c)
        if (lane + c * WAVE < a.width) {
            to_k[lane + c * WAVE] = (T)(dk[c] * a.scale);
            to_v[lane + c * WAVE] = (T)dv[c];
        }
}

// dbias of one head: the parts' sums by distance, then the distances of each bucket, both in order.
__global__ __launch_bounds__(1024) void bias_buckets_kernel(const BackwardArgs b, uint32_t parts) {
    const AttendArgs& a = b.a;
    __shared__ float by_distance[2 * SPAN_MAX + 1];
    __shared__ uint32_t bucket[2 * SPAN_MAX + 1];
    const uint32_t head = blockIdx.x, distances = 2 * a.span + 1;
    const float* from = b.by_distance + (size_t)head * parts * distances;
    for (uint32_t c = threadIdx.x; c < distances; c += 1024) {
        float s = 0.f;
        for (uint32_t p = 0; p < parts; ++p) s += from[(size_t)p * distances + c];
        by_distance[c] = s;
        bucket[c] = a.buckets[c];
    }
    __syncthreads();
    for (uint32_t k = threadIdx.x; k < a.n_buckets; k += 1024) {
        float s = 0.f;
        for (uint32_t c = 0; c < distances; ++c) if (bucket[c] == k) s += by_distance[c];
        b.dbias[(size_t)head * a.n_buckets + k] = s;
    }
}

template <typename T> void backward_any(const BackwardArgs& b, hipStream_t st) {
    const AttendArgs& a = b.a;
    query_rows_kernel<T><<<attend_bias_parts(a.T) * a.heads, THREADS, 0, st>>>(b);
    key_rows_kernel<T><<<(uint32_t)(((uint64_t)a.T * a.kv_heads + WAVES - 1) / WAVES), THREADS, 0, st>>>(b);
}

}  // namespace

uint32_t attend_bias_parts(uint32_t T) { return (T + BLOCK_WORDS - 1) / BLOCK_WORDS; }

void launch_attend_backward(const BackwardArgs& b, uint32_t type, hipStream_t st) {
    if (b.a.T) {
        if (type == ELEM_F32) backward_any<float>(b, st);
        else if (type == ELEM_F16) backward_any<_Float16>(b, st);
        else backward_any<__bf16>(b, st);
    }
    if (b.dbias) bias_buckets_kernel<<<b.a.heads, 1024, 0, st>>>(b, attend_bias_parts(b.a.T));
}

}  // namespace w2v

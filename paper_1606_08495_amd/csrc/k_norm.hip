// Layer norm of rows and its gradients.
//
//   y = (x - mean) rstd gain + offset,  rstd = (mean((x - mean)^2) + eps)^-1/2
//   dx = rstd (t - mean(t) - z mean(t z)),  t = dy gain,  z = (x - mean) rstd
//   dgain = sum over rows of dy z,  doffset = sum over rows of dy
//
// What bounds it is the rows' way through memory: x in, y out; x and dy in, dx out.  A row stays in registers from its
// one load to its store, so the variance is the mean of squared differences, not a difference of large sums.  A group of
// G lanes holds a row, NV vectors of 16 bytes a lane: 8 lanes up to 64 vectors, then doubled, so that few lanes idle and a
// wavefront has up to eight rows in flight.  Above 64 lanes a group is a block.  A group walks over the rows
// with a fixed stride, keeps gain and offset (and backward its sums for their gradients) in registers, and asks for its
// next row before it works on this one.  Sums are fp32; order is fixed by the shape alone.
// Measured: 2^20 rows of 300 in 16 bits 260 us (4.9 TB/s, the rate of a large copy); 2^17 rows of 300 in 32 bits, both passes, 156 us
// (786 MB moved); 8191 rows of 4101 in 16 bits, both passes, 119 us (the backward kernel's sums leave one wavefront a SIMD, as its
// 512 blocks of two wavefronts do by themselves).  Backward, 8 vectors a lane at 128 lanes and more keep 144 to 224 bytes a lane in
// scratch: fp16 rows of 8192 and 16384, fp32 of 16384.
#include <type_traits>

#include "context.h"
#include "elem.h"

namespace w2v {
namespace {

constexpr uint32_t NORM_BLOCK = 256;

// One row's vectors of a lane: vector i of lane l is number i G + l of the row.
template <typename T, int G, int NV> struct Row {
    static constexpr int N = pack16<T>;
    typedef typename Pack<T, N>::vec vec;
    typedef typename Pack<T, N>::mem mem;
    vec v[NV];
    __device__ void load(const T* row, uint32_t lane, uint32_t d) {
        const uint32_t full = d / N;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t at = i * G + lane;
            if (at < full) {
                v[i] = *(const mem*)(row + (size_t)at * N);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) v[i][e] = at * N + e < d ? row[(size_t)at * N + e] : (T)0.f;
            }
        }
    }
    __device__ void store(T* row, uint32_t lane, uint32_t d) const {
        const uint32_t full = d / N;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t at = i * G + lane;
            if (at < full) {
                *(mem*)(row + (size_t)at * N) = v[i];
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) if (at * N + e < d) row[(size_t)at * N + e] = v[i][e];
            }
        }
    }
};

// Columns' fp32 values as a lane of the row's group holds them, from memory (`other` where there are none and past the row's end)
// and back.
template <typename T, int G, int NV>
__device__ inline void load_columns(float (&w)[NV][pack16<T>], const float* p, float other, uint32_t lane, uint32_t d) {
    constexpr int N = pack16<T>;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t c = (i * G + lane) * N;
        if (p && c + N <= d) {
#pragma unroll
            for (int e = 0; e < N; e += 4) {
                const Pack<float, 4>::vec four = *(const Pack<float, 4>::mem*)(p + c + e);
#pragma unroll
                for (int k = 0; k < 4; ++k) w[i][e + k] = four[k];
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) w[i][e] = p && c + e < d ? p[c + e] : other;
        }
    }
}
template <typename T, int G, int NV>
__device__ inline void store_columns(const float (&w)[NV][pack16<T>], float* p, uint32_t lane, uint32_t d) {
    constexpr int N = pack16<T>;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t c = (i * G + lane) * N;
        if (c + N <= d) {
#pragma unroll
            for (int e = 0; e < N; e += 4)
                *(Pack<float, 4>::mem*)(p + c + e) = Pack<float, 4>::vec{w[i][e], w[i][e + 1], w[i][e + 2], w[i][e + 3]};
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) if (c + e < d) p[c + e] = w[i][e];
        }
    }
}

// Sum over the G lanes of a row.  Rows of more than a wavefront go through LDS, `turn` says which of the two halves.
template <int G> __device__ inline float row_sum(float x, float* lds, uint32_t turn) {
    if constexpr (G <= 64) return lanes_sum<G>(x);
    constexpr int W = G > 64 ? G / 64 : 1;
    x = lanes_sum<64>(x);
    float* part = lds + turn * W;
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
    __syncthreads();
    float s = part[0];
#pragma unroll
    for (int w = 1; w < W; ++w) s += part[w];
    return s;
}

template <typename T, int G, int NV>
__global__ __launch_bounds__(G > (int)NORM_BLOCK ? G : (int)NORM_BLOCK)
void norm_kernel(const NormArgs a) {
    constexpr int N = pack16<T>;
    constexpr uint32_t threads = G > (int)NORM_BLOCK ? G : (G > 64 ? G : NORM_BLOCK);
    constexpr uint32_t groups = threads / G;
    __shared__ float lds[2 * (G > 64 ? G / 64 : 1)];
    const uint32_t lane = threadIdx.x % G, d = a.d;
    float gain[NV][N], offset[NV][N];
    load_columns<T, G, NV>(gain, a.gain, 1.f, lane, d);
    load_columns<T, G, NV>(offset, a.offset, 0.f, lane, d);
    const float n = (float)d;
    const uint64_t stride = (uint64_t)gridDim.x * groups;
    uint64_t r = (uint64_t)blockIdx.x * groups + threadIdx.x / G;
    Row<T, G, NV> next;
    if (r < a.rows) next.load((const T*)a.x + r * a.x_stride, lane, d);
    for (; r < a.rows; r += stride) {
        Row<T, G, NV> row = next;
        if (r + stride < a.rows) next.load((const T*)a.x + (r + stride) * a.x_stride, lane, d);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) s += (float)row.v[i][e];
        const float mean = row_sum<G>(s, lds, 0) / n;
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float c = (i * G + lane) * N + e < d ? (float)row.v[i][e] - mean : 0.f;
                q += c * c;
            }
        const float rstd = 1.f / sqrtf(row_sum<G>(q, lds, 1) / n + a.eps);
        if (lane == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e)
                row.v[i][e] = (T)(((float)row.v[i][e] - mean) * rstd * gain[i][e] + offset[i][e]);
        row.store((T*)a.y + r * a.y_stride, lane, d);
    }
}

// Backward.  A block leaves its sums for the columns in parts[block][2][d].
template <typename T, int G, int NV>
__global__ __launch_bounds__(G > (int)NORM_BLOCK ? G : (int)NORM_BLOCK)
void norm_backward_kernel(const NormBackwardArgs a) {
    constexpr int N = pack16<T>;
    constexpr uint32_t threads = G > (int)NORM_BLOCK ? G : (G > 64 ? G : NORM_BLOCK);
    constexpr uint32_t groups = threads / G;
    constexpr uint32_t waves = G > 64 ? 1 : threads / 64;
    __shared__ float lds[4 * (G > 64 ? G / 64 : 1)];
    __shared__ float columns[G > 64 ? 1 : 2 * G * NV * N];
    const uint32_t lane = threadIdx.x % G, d = a.d;
    float gain[NV][N], dg[NV][N], db[NV][N];
    load_columns<T, G, NV>(gain, a.gain, 1.f, lane, d);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) dg[i][e] = db[i][e] = 0.f;
    const float n = (float)d;
    const uint64_t stride = (uint64_t)gridDim.x * groups;
    uint64_t r = (uint64_t)blockIdx.x * groups + threadIdx.x / G;
    uint32_t turn = 0;
    Row<T, G, NV> next_x, next_dy;
    if (r < a.rows) {
        next_x.load((const T*)a.x + r * a.x_stride, lane, d);
        next_dy.load((const T*)a.dy + r * a.dy_stride, lane, d);
    }
    for (; r < a.rows; r += stride) {
        Row<T, G, NV> x = next_x, dy = next_dy;
        if (r + stride < a.rows) {
            next_x.load((const T*)a.x + (r + stride) * a.x_stride, lane, d);
            next_dy.load((const T*)a.dy + (r + stride) * a.dy_stride, lane, d);
        }
        const float mean = a.mean[r], rstd = a.rstd[r];
        float s = 0.f, q = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float g = (float)dy.v[i][e], z = ((float)x.v[i][e] - mean) * rstd, t = g * gain[i][e];
                dg[i][e] += g * z;
                db[i][e] += g;
                s += t;
                q += t * z;
            }
        s = row_sum<G>(s, lds, 2 * turn) / n;
        q = row_sum<G>(q, lds, 2 * turn + 1) / n;
        turn ^= 1;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float z = ((float)x.v[i][e] - mean) * rstd;
                x.v[i][e] = (T)(rstd * ((float)dy.v[i][e] * gain[i][e] - s - z * q));
            }
        x.store((T*)a.dx + r * a.dx_stride, lane, d);
    }
    if (!a.parts) return;
    float* part = a.parts + (size_t)blockIdx.x * 2 * d;
    if constexpr (G > 64) {
        store_columns<T, G, NV>(dg, part, lane, d);
        store_columns<T, G, NV>(db, part + d, lane, d);
    } else {
        // the groups of a wavefront by exchange, then the wavefronts one after the other
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e)
#pragma unroll
                for (int m = G; m < 64; m *= 2) {
                    dg[i][e] += __shfl_xor(dg[i][e], m, 64);
                    db[i][e] += __shfl_xor(db[i][e], m, 64);
                }
        for (uint32_t w = 0; w < waves; ++w) {
            if (threadIdx.x / 64 == w && threadIdx.x % 64 < G) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        float* at = columns + ((i * N + e) * G + lane) * 2;      // lanes side by side
                        at[0] = w ? at[0] + dg[i][e] : dg[i][e];
                        at[1] = w ? at[1] + db[i][e] : db[i][e];
                    }
            }
            __syncthreads();
        }
        for (uint32_t c = threadIdx.x; c < d; c += threads) {
            const uint32_t at = c / N, e = c % N, i = at / G, l = at % G;
            part[c] = columns[((i * N + e) * G + l) * 2];
            part[d + c] = columns[((i * N + e) * G + l) * 2 + 1];
        }
    }
}

// out[c] = sum over parts of parts[p][c], c over the 2 d columns: 64 columns a block, 16 shares of the parts.
__global__ __launch_bounds__(1024) void norm_columns_kernel(const float* parts, uint32_t count, uint32_t d, float* dgain,
                                                            float* doffset) {
    __shared__ float share[16][64];
    const uint32_t c = blockIdx.x * 64 + threadIdx.x % 64, k = threadIdx.x / 64;
    float s = 0.f;
    if (c < 2 * d) {
#pragma unroll 8
        for (uint32_t p = k; p < count; p += 16) s += parts[(size_t)p * 2 * d + c];
    }
    share[k][threadIdx.x % 64] = s;
    __syncthreads();
    if (k || c >= 2 * d) return;
    for (int i = 1; i < 16; ++i) s += share[i][threadIdx.x];
    if (c < d) { if (dgain) dgain[c] = s; }
    else if (doffset) doffset[c - d] = s;
}

// Lanes of a row: the fewest that leave at most eight vectors a lane.
uint32_t norm_lanes(uint32_t d, uint32_t n) {
    const uint32_t vectors = (d + n - 1) / n;
    uint32_t g = 8;
    while (g * 8 < vectors) g *= 2;
    return g;
}
uint32_t norm_blocks(uint64_t rows, uint32_t g, uint32_t most) {
    const uint32_t groups = g >= NORM_BLOCK ? 1 : (g > 64 ? 1 : NORM_BLOCK / g);
    const uint64_t need = (rows + groups - 1) / groups;
    return (uint32_t)(need < most ? need : most);
}
constexpr uint32_t NORM_FORWARD_BLOCKS = 2048, NORM_BACKWARD_BLOCKS = 512;

template <typename T, int G, int NV, typename A> void norm_run(const A& a, uint32_t blocks, hipStream_t st) {
    constexpr uint32_t threads = G > 64 ? G : NORM_BLOCK;
    if constexpr (std::is_same<A, NormArgs>::value) norm_kernel<T, G, NV><<<blocks, threads, 0, st>>>(a);
    else norm_backward_kernel<T, G, NV><<<blocks, threads, 0, st>>>(a);
}

// NV from 5 to 8 where the group was doubled, 1 to 8 for the smallest.
template <typename T, int G, typename A> void norm_nv(const A& a, uint32_t nv, uint32_t blocks, hipStream_t st) {
    if constexpr (G == 8) {
        switch (nv) {
            case 1: return norm_run<T, G, 1>(a, blocks, st);
            case 2: return norm_run<T, G, 2>(a, blocks, st);
            case 3: return norm_run<T, G, 3>(a, blocks, st);
            case 4: return norm_run<T, G, 4>(a, blocks, st);
        }
    }
    switch (nv) {
        case 5: return norm_run<T, G, 5>(a, blocks, st);
        case 6: return norm_run<T, G, 6>(a, blocks, st);
        default: return norm_run<T, G, 8>(a, blocks, st);
    }
}

template <typename T, typename A> void norm_any(const A& a, uint32_t most, hipStream_t st) {
    const uint32_t n = pack16<T>, g = norm_lanes(a.d, n);
    const uint32_t nv = (a.d + n * g - 1) / (n * g), blocks = norm_blocks(a.rows, g, most);
    switch (g) {
        case 8: return norm_nv<T, 8>(a, nv, blocks, st);
        case 16: return norm_nv<T, 16>(a, nv, blocks, st);
        case 32: return norm_nv<T, 32>(a, nv, blocks, st);
        case 64: return norm_nv<T, 64>(a, nv, blocks, st);
        case 128: return norm_nv<T, 128>(a, nv, blocks, st);
        case 256: return norm_nv<T, 256>(a, nv, blocks, st);
    }
    if constexpr (sizeof(T) == 4) norm_nv<T, 512>(a, nv, blocks, st);      // (16 bits: 16384 elements are 2048 vectors, 256 lanes)
}

}  // namespace

void launch_norm(const NormArgs& a, uint32_t type, hipStream_t st) {
    if (type == ELEM_F32) norm_any<float>(a, NORM_FORWARD_BLOCKS, st);
    else if (type == ELEM_F16) norm_any<_Float16>(a, NORM_FORWARD_BLOCKS, st);
    else norm_any<__bf16>(a, NORM_FORWARD_BLOCKS, st);
}

uint32_t norm_backward_parts(uint64_t rows, uint32_t d, uint32_t type) {
    return norm_blocks(rows, norm_lanes(d, 16 / elem_bytes(type)), NORM_BACKWARD_BLOCKS);
}

void launch_norm_backward(const NormBackwardArgs& a, uint32_t type, float* dgain, float* doffset, hipStream_t st) {
    if (a.rows) {
        if (type == ELEM_F32) norm_any<float>(a, NORM_BACKWARD_BLOCKS, st);
        else if (type == ELEM_F16) norm_any<_Float16>(a, NORM_BACKWARD_BLOCKS, st);
        else norm_any<__bf16>(a, NORM_BACKWARD_BLOCKS, st);
    }
    if (dgain || doffset)
        norm_columns_kernel<<<(2 * a.d + 63) / 64, 1024, 0, st>>>(a.parts, norm_backward_parts(a.rows, a.d, type), a.d,
                                                                  dgain, doffset);
}

}  // namespace w2v

// Launches of the context operators (layer norm, attention over texts) for context.hip, which checks what callers pass.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace w2v {

// ---- layer norm ------------------------------------------------------------------------------------
struct NormArgs {
    const void* x; uint64_t x_stride; uint64_t rows; uint32_t d; float eps;
    const float* gain; const float* offset;              // either may be null
    void* y; uint64_t y_stride; float* mean; float* rstd;     // the statistics may be null
};
void launch_norm(const NormArgs& a, uint32_t type, hipStream_t st);

struct NormBackwardArgs {
    const void* dy; uint64_t dy_stride; const void* x; uint64_t x_stride; uint64_t rows; uint32_t d;
    const float* gain; const float* mean; const float* rstd;
    void* dx; uint64_t dx_stride;
    float* parts;            // [norm_backward_parts][2][d], or null where neither column gradient is wanted
};
uint32_t norm_backward_parts(uint64_t rows, uint32_t d, uint32_t type);
void launch_norm_backward(const NormBackwardArgs& a, uint32_t type, float* dgain, float* doffset, hipStream_t st);

}  // namespace w2v

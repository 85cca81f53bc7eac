// C ABI of the context operators: argument checks and the order in which their kernels are queued.  They belong to no
// shard and keep nothing between calls.  See include/w2v_shard.h for the contract of every entry point.
#include "../../include/w2v_shard.h"

#include <cmath>

#include "common.h"
#include "context.h"
#include "elem.h"

using namespace w2v;
static_assert(W2V_T_F32 == ELEM_F32 && W2V_T_F16 == ELEM_F16 && W2V_T_BF16 == ELEM_BF16, "element types");

namespace {

int launched() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? W2V_OK : fail(W2V_ERR_HIP, "a launch failed: %s", hipGetErrorString(e));
}

bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

int check_type(int type) {
    return (unsigned)type < ELEM_TYPES ? W2V_OK : fail(W2V_ERR_ARG, "type %d is none of W2V_T_*", type);
}

constexpr uint64_t ROWS_MAX = 1ull << 40, STRIDE_MAX = 1ull << 40;      // elements; rows times stride stays below 2^64 bytes

int check_norm(int type, uint64_t rows, uint32_t d) {
    if (int rc = check_type(type)) return rc;
    if (d == 0 || d > W2V_NORM_D_MAX) return fail(W2V_ERR_ARG, "d = %u outside 1..%d", d, W2V_NORM_D_MAX);
    if (rows >= ROWS_MAX) return fail(W2V_ERR_ARG, "too many rows");
    return W2V_OK;
}
int check_rows(const void* p, uint64_t stride, uint64_t least, uint64_t rows, int type, const char* name) {
    if (!p) return fail(W2V_ERR_NULL, "%s is NULL", name);
    if (!aligned(p, elem_bytes(type))) return fail(W2V_ERR_ARG, "%s is not aligned to its elements", name);
    if (rows > 1 && stride < least) return fail(W2V_ERR_ARG, "rows of %s overlap", name);
    if (rows > 1 && (stride >= STRIDE_MAX || rows > (1ull << 60) / (stride ? stride : 1)))
        return fail(W2V_ERR_ARG, "%s reaches too far", name);
    return W2V_OK;
}

}  // namespace

extern "C" int w2v_layer_norm(int type, const void* x, uint64_t x_stride, uint64_t rows, uint32_t d, const float* gain,
                              const float* offset, float eps, void* y, uint64_t y_stride, float* mean, float* rstd,
                              void* stream) {
    if (int rc = check_norm(type, rows, d)) return rc;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(W2V_ERR_ARG, "eps must be finite and not negative");
    if (rows == 0) return W2V_OK;
    if (int rc = check_rows(x, x_stride, 0, rows, type, "x")) return rc;
    if (int rc = check_rows(y, y_stride, d, rows, type, "y")) return rc;
    if (x == y && rows > 1 && x_stride != y_stride) return fail(W2V_ERR_ARG, "y is x, but its rows lie elsewhere");
    launch_norm(NormArgs{x, x_stride, rows, d, eps, gain, offset, y, y_stride, mean, rstd}, (uint32_t)type,
                (hipStream_t)stream);
    return launched();
}

extern "C" size_t w2v_layer_norm_backward_workspace(int type, uint64_t rows, uint32_t d) {
    if ((unsigned)type >= ELEM_TYPES || rows >= ROWS_MAX || d == 0 || d > W2V_NORM_D_MAX) return 0;
    return (size_t)norm_backward_parts(rows, d, (uint32_t)type) * 2 * d * sizeof(float);
}

extern "C" int w2v_layer_norm_backward(int type, const void* dy, uint64_t dy_stride, const void* x, uint64_t x_stride,
                                       uint64_t rows, uint32_t d, const float* gain, const float* mean,
                                       const float* rstd, void* dx, uint64_t dx_stride, float* dgain, float* doffset,
                                       void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_norm(type, rows, d)) return rc;
    const bool columns = dgain || doffset;
    if (rows) {
        if (int rc = check_rows(dy, dy_stride, 0, rows, type, "dy")) return rc;
        if (int rc = check_rows(x, x_stride, 0, rows, type, "x")) return rc;
        if (int rc = check_rows(dx, dx_stride, d, rows, type, "dx")) return rc;
        if (!mean || !rstd) return fail(W2V_ERR_NULL, "the rows' statistics are NULL");
        if (rows > 1 && ((dx == x && dx_stride != x_stride) || (dx == dy && dx_stride != dy_stride)))
            return fail(W2V_ERR_ARG, "dx is an input, but its rows lie elsewhere");
        if (columns) {
            const size_t need = w2v_layer_norm_backward_workspace(type, rows, d);
            if (!workspace) return fail(W2V_ERR_NULL, "workspace is NULL");
            if (!aligned(workspace, 256)) return fail(W2V_ERR_ARG, "workspace must be 256-byte aligned");
            if (workspace_bytes < need)
                return fail(W2V_ERR_ARG, "workspace of %zu bytes is too small: %zu are needed", workspace_bytes, need);
        }
    }
    if (!rows && !columns) return W2V_OK;
    launch_norm_backward(NormBackwardArgs{dy, dy_stride, x, x_stride, rows, d, gain, mean, rstd, dx, dx_stride,
                                          columns ? (float*)workspace : nullptr},
                         (uint32_t)type, dgain, doffset, (hipStream_t)stream);
    return launched();
}

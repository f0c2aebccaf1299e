// Dropout of a tensor, added to a residual: y_i = r_i + [draw_i >= thr] s x_i, s = 1 / (1 - rate).
// The draws are a function of (seed, element), so nothing of the mask is stored and the backward pass is the same
// kernel on dy.  One rounding, at the store.
#include "ops.h"

namespace sw {

// A lane takes eight consecutive elements, 16 bytes of bf16, and draws four times.
template <typename T, bool RES>
__global__ __launch_bounds__(256) void dropout_kernel(const T *x, const T *r, T *y, int64_t n, Drop d) {
    const int64_t stride = (int64_t)gridDim.x * 256 * 8;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; i < n; i += stride) {
        float v[8], res[8];
        const bool whole = i + 8 <= n;
        if (whole) {
            Eight<T>::load(x + i, v);
            if (RES) Eight<T>::load(r + i, res);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = i + j < n ? to_f32(x[i + j]) : 0.f;
                if (RES) res[j] = i + j < n ? to_f32(r[i + j]) : 0.f;
            }
        }
        drop_apply<8>(d, (uint64_t)i, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = RES ? fmaf(v[j], d.scale, res[j]) : v[j] * d.scale;
        if (whole) {
            Eight<T>::store(y + i, v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i + j < n) y[i + j] = from_f32<T>(v[j]);
        }
    }
}

template <typename T>
static hipError_t dropout_launch(int64_t n, const Drop &d, const void *x, const void *r, void *y, hipStream_t s) {
    ProfScope ps("dropout", s);
    const int64_t blocks = ceil_div(n, 256 * 8), most = 1 << 20;
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    if (r)
        hipLaunchKernelGGL((dropout_kernel<T, true>), grid, dim3(256), 0, s, (const T *)x, (const T *)r, (T *)y, n, d);
    else
        hipLaunchKernelGGL((dropout_kernel<T, false>), grid, dim3(256), 0, s, (const T *)x, (const T *)nullptr, (T *)y, n, d);
    return hipGetLastError();
}

}  // namespace sw

using namespace sw;

extern "C" int switch_dropout(int64_t n, int32_t act_dtype, float rate, uint64_t seed, const void *x,
                              const void *residual, void *y, void *hip_stream) {
    if (act_dtype != SW_F32 && act_dtype != SW_BF16) return SW_ERR_DTYPE;
    if (n < 0 || n >= (int64_t)1 << 40) return SW_ERR_SHAPE;
    if (!drop_rate_ok(rate)) return SW_ERR_VALUE;
    if (n == 0) return SW_OK;
    if (!x || !y) return SW_ERR_NULL;
    if (!aligned16(x) || !aligned16(y) || (residual && !aligned16(residual))) return SW_ERR_ALIGN;
    const Drop d = drop_of(rate, seed);
    hipStream_t s = (hipStream_t)hip_stream;
    return status_of(act_dtype == SW_BF16 ? dropout_launch<bf16>(n, d, x, residual, y, s)
                                          : dropout_launch<float>(n, d, x, residual, y, s));
}

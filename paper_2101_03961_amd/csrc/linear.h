// switch_linear's products, shared by linear.hip (entry points, element-wise passes), linear_bf16.hip, ...
#pragma once

#include "normal.h"
#include "ops.h"

namespace sw {

// C[q][p] = sum_k Q(q, k) P(p, k), C row-major:
enum LinearKind {
    LINEAR_FWD,   // y = r + drop(act(x W + b))   q: row          p: column of W   k: column of x
    LINEAR_DX,    // dx = s dz W^T                q: row          p: column of x   k: column of W
    LINEAR_DW     // dW = s x^T dz                q: column of x  p: column of W   k: row
};
struct LinearArgs {
    const void *Q, *P;
    int ldq, ldp;                  // elements of a row in memory
    int64_t Qdim, Kdim;
    int Pdim;                      // columns of C; LINEAR_FWD: columns of y
    const float *bias;
    const void *residual;
    void *C, *z;
    float *part;                   // LINEAR_DW in several parts of k: their sums, [part][Qdim][Pdim]
    int act, gated;
    float scale;                   // of the sums
    Drop drop;
};

// How the weight gradient's k, the rows, is cut: parts of split_k (the last one shorter), each summed by itself.
// A part's rows of x and of dz are addressed through one descriptor each, of less than 2 GB.
struct LinearPlan {
    int tile;
    int splits;
    int64_t split_k;
};
LinearPlan plan_linear_bf16(const switch_linear_config *cfg, bool backward);

// act of a value, or of a gate and a linear part
__device__ __forceinline__ float linear_act(int act, float u, float v) {
    switch (act) {
    case SW_ACT_RELU: return fmaxf(u, 0.f);
    case SW_ACT_GELU: return u * normal_of(u).cdf;
    case SW_ACT_GEGLU: return u * normal_of(u).cdf * v;
    default: return u;
    }
}

static inline int64_t linear_columns(const switch_linear_config *cfg) {   // of W
    return cfg->activation == SW_ACT_GEGLU ? 2 * cfg->N : cfg->N;
}

hipError_t launch_linear_bf16(const LinearPlan &plan, const LinearArgs &a, hipStream_t s);
// either may be left out
hipError_t launch_linear_backward_bf16(const LinearPlan &plan, const LinearArgs *dx, const LinearArgs *dW, hipStream_t s);

}  // namespace sw

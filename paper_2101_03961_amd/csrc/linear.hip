// switch_linear: one matrix product with bias, activation, dropout and residual in its epilogue, and its gradients.
//
//   z = x W + b,  y = r + drop(act(z));   dz = act'(z) drop(dy),  dx = dz W^T,  dW = x^T dz,  db = sum of dz's rows
//
// All three products are C[q][p] = sum_k Q(q, k) P(p, k) with C row-major.
#include <math.h>

#include "normal.h"
#include "ops.h"

namespace sw {

struct LinearArgs {
    const void *Q, *P;
    long q_rs, q_ks, p_rs, p_ks;   // strides of a row and of a k
    int64_t Qdim, Kdim;
    int Pdim;                      // columns of C (of y: half of W's for the gated activation)
    const float *bias;
    const void *residual;
    void *C, *z;
    int act, gated;
    float scale;                   // of the sums
    Drop drop;
};

// act of a value, or of a gate and a linear part
__device__ __forceinline__ float linear_act(int act, float u, float v) {
    switch (act) {
    case SW_ACT_RELU: return fmaxf(u, 0.f);
    case SW_ACT_GELU: return u * normal_of(u).cdf;
    case SW_ACT_GEGLU: return u * normal_of(u).cdf * v;
    default: return u;
    }
}

constexpr int kLinTile = 64, kLinKC = 16;

template <typename T, bool GATED>
__global__ __launch_bounds__(256) void linear_kernel(LinearArgs a) {
    constexpr int NP = GATED ? 2 : 1;
    __shared__ float qs[kLinKC][kLinTile + 4];
    __shared__ float ps[NP][kLinKC][kLinTile + 4];
    const int64_t q0 = (int64_t)blockIdx.x * kLinTile;
    const int p0 = blockIdx.y * kLinTile;
    const T *Q = (const T *)a.Q, *P = (const T *)a.P;
    const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    float acc[NP][4][4], total[NP][4][4];
#pragma unroll
    for (int g = 0; g < NP; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[g][i][j] = total[g][i][j] = 0.f;
    for (int64_t k0 = 0; k0 < a.Kdim; k0 += kLinKC) {
        if (k0 % 256 == 0) {
#pragma unroll
            for (int g = 0; g < NP; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        total[g][i][j] += acc[g][i][j];
                        acc[g][i][j] = 0.f;
                    }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int id = tid + i * 256;
            int r, kk;
            if (a.q_ks == 1) { kk = id % kLinKC; r = id / kLinKC; } else { r = id % kLinTile; kk = id / kLinTile; }
            qs[kk][r] = q0 + r < a.Qdim && k0 + kk < a.Kdim ? to_f32(Q[(q0 + r) * a.q_rs + (k0 + kk) * a.q_ks]) : 0.f;
            if (a.p_ks == 1) { kk = id % kLinKC; r = id / kLinKC; } else { r = id % kLinTile; kk = id / kLinTile; }
#pragma unroll
            for (int g = 0; g < NP; ++g)
                ps[g][kk][r] = p0 + r < a.Pdim && k0 + kk < a.Kdim
                                   ? to_f32(P[(long)(g * a.Pdim + p0 + r) * a.p_rs + (k0 + kk) * a.p_ks]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kLinKC; ++kk)
#pragma unroll
            for (int g = 0; g < NP; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[g][i][j] = fmaf(qs[kk][ty * 4 + i], ps[g][kk][tx * 4 + j], acc[g][i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t q = q0 + ty * 4 + i;
        if (q >= a.Qdim) continue;
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            const int p = p0 + tx * 4 + j;   // Pdim is even
            if (p >= a.Pdim) continue;
            float v[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                float z[NP];
#pragma unroll
                for (int g = 0; g < NP; ++g) {
                    z[g] = (total[g][i][j + m] + acc[g][i][j + m]) * a.scale;
                    if (a.bias) z[g] += a.bias[g * a.Pdim + p + m];
                    if (a.z) ((T *)a.z)[q * a.Pdim * NP + g * a.Pdim + p + m] = from_f32<T>(z[g]);
                }
                v[m] = linear_act(a.act, z[0], z[NP - 1]);
            }
            const int64_t at = q * a.Pdim + p;
            if (a.drop.on) {
                drop_apply<2>(a.drop, (uint64_t)at, v);
                v[0] *= a.drop.scale;
                v[1] *= a.drop.scale;
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                if (a.residual) v[m] += to_f32(((const T *)a.residual)[at + m]);
                ((T *)a.C)[at + m] = from_f32<T>(v[m]);
            }
        }
    }
}

// dz (without the dropout's scale) and sums of its rows, kDzRows at a time.  A lane takes four columns.
constexpr int kDzRows = 128;
struct DzArgs {
    const void *dy, *z;
    void *dz;                      // or nullptr
    float *part;                   // [row blocks][columns of W], or nullptr
    int64_t M;
    int N, act;
    Drop drop;
};

template <typename T, bool GATED>
__global__ __launch_bounds__(256) void linear_dz_kernel(DzArgs a) {
    const int64_t q0 = (int64_t)blockIdx.x * kDzRows, qend = q0 + kDzRows < a.M ? q0 + kDzRows : a.M;
    const int p = (blockIdx.y * 256 + threadIdx.x) * 2;
    if (p >= a.N) return;
    const int Nz = GATED ? 2 * a.N : a.N;
    float su[2] = {}, sv[2] = {};
    for (int64_t q = q0; q < qend; ++q) {
        const int64_t at = q * a.N + p, zat = q * Nz + p;
        float g[2] = {to_f32(((const T *)a.dy)[at]), to_f32(((const T *)a.dy)[at + 1])};
        if (a.drop.on) drop_apply<2>(a.drop, (uint64_t)at, g);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            float du = g[m], dv = 0.f;
            if (a.act != SW_ACT_NONE) {
                const float u = to_f32(((const T *)a.z)[zat + m]);
                if (a.act == SW_ACT_RELU) {
                    du = u > 0.f ? g[m] : 0.f;
                } else {
                    const NormalOf n = normal_of(u);
                    const float v = GATED ? to_f32(((const T *)a.z)[zat + a.N + m]) : 1.f;
                    du = g[m] * v * fmaf(u, n.pdf, n.cdf);
                    dv = g[m] * u * n.cdf;
                }
            }
            if (a.dz) ((T *)a.dz)[zat + m] = from_f32<T>(du);
            if (a.dz && GATED) ((T *)a.dz)[zat + a.N + m] = from_f32<T>(dv);
            su[m] += du;
            sv[m] += dv;
        }
    }
    if (!a.part) return;
    float *out = a.part + (size_t)blockIdx.x * Nz + p;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        out[m] = su[m];
        if (GATED) out[a.N + m] = sv[m];
    }
}

__global__ __launch_bounds__(256) void linear_db_kernel(const float *part, int64_t parts, int cols, float scale, float *db) {
    const int p = blockIdx.x * 256 + threadIdx.x;
    if (p >= cols) return;
    double s = 0.;
    for (int64_t i = 0; i < parts; ++i) s += (double)part[i * cols + p];
    db[p] = (float)(s * scale);
}

static int64_t linear_columns(const switch_linear_config *cfg) {
    return cfg->activation == SW_ACT_GEGLU ? 2 * cfg->N : cfg->N;
}

static int check_linear(const switch_linear_config *cfg) {
    if (!cfg) return SW_ERR_NULL;
    if (cfg->act_dtype != SW_F32 && cfg->act_dtype != SW_BF16) return SW_ERR_DTYPE;
    if (cfg->activation < SW_ACT_NONE || cfg->activation > SW_ACT_GEGLU) return SW_ERR_DTYPE;
    if (cfg->M < 0 || cfg->M >= (int64_t)1 << 31) return SW_ERR_SHAPE;
    const int64_t widest = (int64_t)1 << 21;
    if (cfg->K < 1 || cfg->N < 1 || cfg->K >= widest || cfg->N >= widest || linear_columns(cfg) >= widest) return SW_ERR_SHAPE;
    const int64_t elt = cfg->act_dtype == SW_BF16 ? 2 : 4;
    if (cfg->K * elt % 16 || cfg->N * elt % 16) return SW_ERR_SHAPE;
    if (cfg->K * linear_columns(cfg) * elt >= (int64_t)1 << 31) return SW_ERR_SHAPE;
    if (!drop_rate_ok(cfg->dropout)) return SW_ERR_VALUE;
    if (cfg->flags) return SW_ERR_VALUE;
    return SW_OK;
}

struct LinearLayout {
    size_t dz, part, total;
    bool own_dz;                   // dz is not dy itself
    int64_t parts;
};
static LinearLayout linear_layout(const switch_linear_config *cfg, bool backward) {
    LinearLayout l{};
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, 256); return o; };
    if (backward) {
        l.own_dz = cfg->activation != SW_ACT_NONE || drop_of(cfg->dropout, 0).on;
        l.parts = ceil_div(cfg->M, kDzRows);
        l.dz = take(l.own_dz ? (size_t)cfg->M * linear_columns(cfg) * (cfg->act_dtype == SW_BF16 ? 2 : 4) : 0);
        l.part = take((size_t)l.parts * linear_columns(cfg) * 4);
    }
    l.total = cfg->M ? off : 0;
    return l;
}

static hipError_t launch_linear(const char *name, int dtype, const LinearArgs &a, hipStream_t s) {
    ProfScope ps(name, s);
    const dim3 grid((unsigned)ceil_div(a.Qdim, kLinTile), (unsigned)ceil_div(a.Pdim, kLinTile));
#define SW_LINEAR(T, G) hipLaunchKernelGGL((linear_kernel<T, G>), grid, dim3(256), 0, s, a)
    if (dtype == SW_BF16) { if (a.gated) SW_LINEAR(bf16, true); else SW_LINEAR(bf16, false); }
    else { if (a.gated) SW_LINEAR(float, true); else SW_LINEAR(float, false); }
#undef SW_LINEAR
    return hipGetLastError();
}

static bool linear_workspace_ok(const LinearLayout &l, const void *workspace, size_t bytes) {
    return l.total == 0 || (workspace && ((uintptr_t)workspace & 255u) == 0 && bytes >= l.total);
}

}  // namespace sw

using namespace sw;

extern "C" {

int switch_linear_workspace_size(const switch_linear_config *cfg, int backward, size_t *bytes_out) {
    if (!cfg || !bytes_out) return SW_ERR_NULL;
    const int st = check_linear(cfg);
    if (st != SW_OK) return st;
    *bytes_out = linear_layout(cfg, backward != 0).total;
    return SW_OK;
}

int switch_linear(const switch_linear_config *cfg, const void *x, const void *W, const float *bias,
                  const void *residual, void *y, void *z, void *workspace, size_t workspace_bytes, void *hip_stream) {
    const int st = check_linear(cfg);
    if (st != SW_OK) return st;
    if (cfg->M == 0) return SW_OK;
    if (!x || !W || !y) return SW_ERR_NULL;
    if (!aligned16(x) || !aligned16(W) || !aligned16(bias) || !aligned16(residual) || !aligned16(y) || !aligned16(z))
        return SW_ERR_ALIGN;
    if (!linear_workspace_ok(linear_layout(cfg, false), workspace, workspace_bytes)) return SW_ERR_WORKSPACE;
    LinearArgs a{};
    a.Q = x; a.q_rs = cfg->K; a.q_ks = 1;
    a.P = W; a.p_rs = 1; a.p_ks = linear_columns(cfg);
    a.Qdim = cfg->M; a.Kdim = cfg->K; a.Pdim = (int)cfg->N;
    a.bias = bias; a.residual = residual; a.C = y; a.z = z;
    a.act = cfg->activation;
    a.gated = cfg->activation == SW_ACT_GEGLU;
    a.scale = 1.f;
    a.drop = drop_of(cfg->dropout, cfg->seed);
    return status_of(launch_linear("linear", cfg->act_dtype, a, (hipStream_t)hip_stream));
}

int switch_linear_backward(const switch_linear_config *cfg, const void *dy, const void *x, const void *W, const void *z,
                           void *dx, void *dW, float *db, void *workspace, size_t workspace_bytes, void *hip_stream) {
    int st = check_linear(cfg);
    if (st != SW_OK) return st;
    if (!dx && !dW && !db) return SW_ERR_NULL;
    if (!aligned16(dy) || !aligned16(x) || !aligned16(W) || !aligned16(z) || !aligned16(dx) || !aligned16(dW) || !aligned16(db))
        return SW_ERR_ALIGN;
    hipStream_t s = (hipStream_t)hip_stream;
    const int64_t cols = linear_columns(cfg);
    const int dt = cfg->act_dtype;
    if (cfg->M == 0) {
        if (dW && (st = fill_zero(dW, (size_t)(cfg->K * cols) * (dt == SW_BF16 ? 2 : 4), s))) return st;
        return db ? fill_zero(db, (size_t)cols * 4, s) : SW_OK;
    }
    if (!dy || (dx && !W) || (dW && !x) || (cfg->activation != SW_ACT_NONE && !z)) return SW_ERR_NULL;
    const LinearLayout l = linear_layout(cfg, true);
    if (!linear_workspace_ok(l, workspace, workspace_bytes)) return SW_ERR_WORKSPACE;
    char *ws = (char *)workspace;
    const bool gated = cfg->activation == SW_ACT_GEGLU;
    const void *dz = l.own_dz ? ws + l.dz : dy;
    const Drop drop = drop_of(cfg->dropout, cfg->seed);
    if (l.own_dz || db) {
        ProfScope ps("linear_dz", s);
        DzArgs a{};
        a.dy = dy; a.z = z;
        a.dz = l.own_dz ? ws + l.dz : nullptr;
        a.part = db ? (float *)(ws + l.part) : nullptr;
        a.M = cfg->M; a.N = (int)cfg->N; a.act = cfg->activation;
        a.drop = drop;
        const dim3 grid((unsigned)l.parts, (unsigned)ceil_div(cfg->N, 512));
#define SW_DZ(T, G) hipLaunchKernelGGL((linear_dz_kernel<T, G>), grid, dim3(256), 0, s, a)
        if (dt == SW_BF16) { if (gated) SW_DZ(bf16, true); else SW_DZ(bf16, false); }
        else { if (gated) SW_DZ(float, true); else SW_DZ(float, false); }
#undef SW_DZ
        if ((st = status_of(hipGetLastError()))) return st;
    }
    if (db) {
        ProfScope ps("linear_db", s);
        hipLaunchKernelGGL(linear_db_kernel, dim3((unsigned)ceil_div(cols, 256)), dim3(256), 0, s,
                           (const float *)(ws + l.part), l.parts, (int)cols, drop.scale, db);
        if ((st = status_of(hipGetLastError()))) return st;
    }
    LinearArgs a{};
    a.scale = drop.scale;
    if (dx) {   // q: row, p: column of x, k: column of W
        a.Q = dz; a.q_rs = cols; a.q_ks = 1;
        a.P = W; a.p_rs = cols; a.p_ks = 1;
        a.Qdim = cfg->M; a.Kdim = cols; a.Pdim = (int)cfg->K;
        a.C = dx;
        if ((st = status_of(launch_linear("linear_dx", dt, a, s)))) return st;
    }
    if (dW) {   // q: column of x, p: column of W, k: row
        a.Q = x; a.q_rs = 1; a.q_ks = cfg->K;
        a.P = dz; a.p_rs = 1; a.p_ks = cols;
        a.Qdim = cfg->K; a.Kdim = cfg->M; a.Pdim = (int)cols;
        a.C = dW;
        if ((st = status_of(launch_linear("linear_dW", dt, a, s)))) return st;
    }
    return SW_OK;
}

}  // extern "C"

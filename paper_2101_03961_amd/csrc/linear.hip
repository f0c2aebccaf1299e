// switch_linear: one matrix product with bias, activation, dropout and residual in its epilogue, and its gradients.
//
//   z = x W + b,  y = r + drop(act(z));   dz = act'(z) drop(dy),  dx = dz W^T,  dW = x^T dz,  db = sum of dz's rows
//
// All three products are C[q][p] = sum_k Q(q, k) P(p, k) with C row-major.
#include <math.h>

#include "linear.h"

namespace sw {

constexpr int kLinTile = 64, kLinKC = 16;

template <typename T, bool GATED>
__global__ __launch_bounds__(256) void linear_kernel(LinearArgs a, int kind) {
    const long q_rs = kind == LINEAR_DW ? 1 : a.ldq, q_ks = kind == LINEAR_DW ? a.ldq : 1;
    const long p_rs = kind == LINEAR_DX ? a.ldp : 1, p_ks = kind == LINEAR_DX ? 1 : a.ldp;
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
            if (q_ks == 1) { kk = id % kLinKC; r = id / kLinKC; } else { r = id % kLinTile; kk = id / kLinTile; }
            qs[kk][r] = q0 + r < a.Qdim && k0 + kk < a.Kdim ? to_f32(Q[(q0 + r) * q_rs + (k0 + kk) * q_ks]) : 0.f;
            if (p_ks == 1) { kk = id % kLinKC; r = id / kLinKC; } else { r = id % kLinTile; kk = id / kLinTile; }
#pragma unroll
            for (int g = 0; g < NP; ++g)
                ps[g][kk][r] = p0 + r < a.Pdim && k0 + kk < a.Kdim
                                   ? to_f32(P[(long)(g * a.Pdim + p0 + r) * p_rs + (k0 + kk) * p_ks]) : 0.f;
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

// dz without the dropout's scale (so that, where act' is 0 or 1, it is dy or zero and loses nothing in bf16) and sums of its
// rows.  A lane takes a chunk of columns, 16 bytes, of the gate and of the linear part; `lanes` lanes of a block share a row
// and each handles kDzSteps rows, 256 / lanes apart.  Bound by its traffic.
constexpr int kDzSteps = 8;
struct DzArgs {
    const void *dy, *z;
    void *dz;                      // or nullptr
    float *part;                   // [row blocks][columns of W], or nullptr
    int64_t M;
    int N, act, lanes;
    Drop drop;
};

template <typename T> struct DzChunk;
template <> struct DzChunk<bf16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ void load(const void *p, int64_t at, float *v) { Eight<bf16>::load((const bf16 *)p + at, v); }
    static __device__ __forceinline__ void store(void *p, int64_t at, const float *v) { Eight<bf16>::store((bf16 *)p + at, v); }
};
template <> struct DzChunk<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void load(const void *p, int64_t at, float *v) {
        *(float4 *)v = *(const float4 *)((const float *)p + at);
    }
    static __device__ __forceinline__ void store(void *p, int64_t at, const float *v) {
        *(float4 *)((float *)p + at) = *(const float4 *)v;
    }
};

template <typename T, bool GATED>
__global__ __launch_bounds__(256) void linear_dz_kernel(DzArgs a) {
    typedef DzChunk<T> C;
    constexpr int n = C::n, NP = GATED ? 2 : 1;
    __shared__ float sums[256][NP * n + 1];
    const int tid = threadIdx.x, line = tid / a.lanes, lines = 256 / a.lanes;
    const int p = (blockIdx.y * a.lanes + tid % a.lanes) * n;
    const int64_t q0 = (int64_t)blockIdx.x * (lines * kDzSteps) + line;
    const int64_t Nz = NP * (int64_t)a.N;
    float sum[NP][n] = {};
    if (p < a.N)
#pragma unroll 2
        for (int i = 0; i < kDzSteps; ++i) {
            const int64_t q = q0 + (int64_t)i * lines;
            if (q >= a.M) break;
            const int64_t at = q * a.N + p, zat = q * Nz + p;
            float g[n], u[n], v[n];
            C::load(a.dy, at, g);
            if (a.act != SW_ACT_NONE) C::load(a.z, zat, u);
            if (GATED) C::load(a.z, zat + a.N, v);
            if (a.drop.on) drop_apply<n>(a.drop, (uint64_t)at, g);
            if (a.act == SW_ACT_RELU) {
#pragma unroll
                for (int m = 0; m < n; ++m) g[m] = u[m] > 0.f ? g[m] : 0.f;
            } else if (a.act != SW_ACT_NONE) {
#pragma unroll
                for (int m = 0; m < n; ++m) {
                    const NormalOf no = normal_of(u[m]);
                    if (GATED) {
                        const float linear = v[m];
                        v[m] = g[m] * u[m] * no.cdf;
                        g[m] *= linear;
                    }
                    g[m] *= fmaf(u[m], no.pdf, no.cdf);
                }
            }
            if (a.dz) {
                C::store(a.dz, zat, g);
                if (GATED) C::store(a.dz, zat + a.N, v);
            }
#pragma unroll
            for (int m = 0; m < n; ++m) {
                sum[0][m] += g[m];
                if (GATED) sum[NP - 1][m] += v[m];
            }
        }
    if (!a.part) return;
#pragma unroll
    for (int g = 0; g < NP; ++g)
#pragma unroll
        for (int m = 0; m < n; ++m) sums[tid][g * n + m] = sum[g][m];
    __syncthreads();
    // the lines of a column, in order
    for (int i = tid; i < a.lanes * NP * n; i += 256) {
        const int lane = i / (NP * n), m = i - lane * (NP * n), col = (blockIdx.y * a.lanes + lane) * n + m % n;
        if (col >= a.N) continue;
        float s = 0.f;
        for (int l = 0; l < lines; ++l) s += sums[l * a.lanes + lane][m];
        a.part[blockIdx.x * Nz + m / n * a.N + col] = s;
    }
}

// The parts' sums of dW and, in the blocks behind, of db, in the order of the parts.
struct LinearJoin {
    const float *dW_part;
    void *dW;
    int64_t elements;              // of dW
    int splits;
    int dW_blocks;
    const float *db_part;
    float *db;
    int64_t db_parts;
    int cols;
    float scale;
};
constexpr int kJoinCols = 32;
template <typename T> __global__ __launch_bounds__(1024) void linear_join_kernel(LinearJoin a) {
    typedef DzChunk<T> C;
    if ((int)blockIdx.x < a.dW_blocks) {
        const int64_t at = ((int64_t)blockIdx.x * 1024 + threadIdx.x) * C::n;
        if (at >= a.elements) return;
        float sum[C::n] = {};
#pragma unroll 4
        for (int s = 0; s < a.splits; ++s) {
            const float *from = a.dW_part + s * a.elements + at;
#pragma unroll
            for (int m = 0; m < C::n; m += 4) {
                const float4 x = *(const float4 *)(from + m);
                sum[m] += x.x; sum[m + 1] += x.y; sum[m + 2] += x.z; sum[m + 3] += x.w;
            }
        }
#pragma unroll
        for (int m = 0; m < C::n; ++m) sum[m] *= a.scale;
        C::store(a.dW, at, sum);
        return;
    }
    constexpr int kLines = 1024 / kJoinCols;
    __shared__ double sums[kLines][kJoinCols + 1];
    const int col = threadIdx.x % kJoinCols, line = threadIdx.x / kJoinCols;
    const int p = ((int)blockIdx.x - a.dW_blocks) * kJoinCols + col;
    double sum = 0.;
    if (p < a.cols)
#pragma unroll 4
        for (int64_t i = line; i < a.db_parts; i += kLines) sum += (double)a.db_part[i * a.cols + p];
    sums[line][col] = sum;
    __syncthreads();
    if (line == 0 && p < a.cols) {
        sum = 0.;
        for (int l = 0; l < kLines; ++l) sum += sums[l][col];
        a.db[p] = (float)(sum * a.scale);
    }
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
    size_t dz, db_part, dW_part, total;
    bool own_dz;                   // dz is not dy itself
    int lanes;                     // of linear_dz_kernel
    int64_t db_parts;
    LinearPlan plan;
};
static LinearLayout linear_layout(const switch_linear_config *cfg, bool backward) {
    LinearLayout l{};
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, 256); return o; };
    const bool bf = cfg->act_dtype == SW_BF16;
    const int64_t elt = bf ? 2 : 4, cols = linear_columns(cfg);
    if (bf) l.plan = plan_linear_bf16(cfg, backward);
    else l.plan = LinearPlan{0, 1, cfg->M};
    if (backward) {
        l.own_dz = cfg->activation != SW_ACT_NONE || drop_of(cfg->dropout, 0).on;
        const int64_t chunks = cfg->N * elt / 16;
        l.lanes = 1;
        while (l.lanes < 32 && l.lanes < chunks) l.lanes *= 2;
        l.db_parts = ceil_div(cfg->M, 256 / l.lanes * kDzSteps);
        l.dz = take(l.own_dz ? (size_t)cfg->M * cols * elt : 0);
        l.db_part = take((size_t)l.db_parts * cols * 4);
        l.dW_part = take(l.plan.splits > 1 ? (size_t)l.plan.splits * cfg->K * cols * 4 : 0);
    }
    l.total = cfg->M ? off : 0;
    return l;
}

static hipError_t launch_linear_f32(const char *name, LinearKind kind, const LinearArgs &a, hipStream_t s) {
    ProfScope ps(name, s);
    const dim3 grid((unsigned)ceil_div(a.Qdim, kLinTile), (unsigned)ceil_div(a.Pdim, kLinTile));
    if (a.gated) hipLaunchKernelGGL((linear_kernel<float, true>), grid, dim3(256), 0, s, a, (int)kind);
    else hipLaunchKernelGGL((linear_kernel<float, false>), grid, dim3(256), 0, s, a, (int)kind);
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
    const LinearLayout l = linear_layout(cfg, false);
    if (!linear_workspace_ok(l, workspace, workspace_bytes)) return SW_ERR_WORKSPACE;
    LinearArgs a{};
    a.Q = x; a.ldq = (int)cfg->K;
    a.P = W; a.ldp = (int)linear_columns(cfg);
    a.Qdim = cfg->M; a.Kdim = cfg->K; a.Pdim = (int)cfg->N;
    a.bias = bias; a.residual = residual; a.C = y; a.z = z;
    a.act = cfg->activation;
    a.gated = cfg->activation == SW_ACT_GEGLU;
    a.scale = 1.f;
    a.drop = drop_of(cfg->dropout, cfg->seed);
    hipStream_t s = (hipStream_t)hip_stream;
    return status_of(cfg->act_dtype == SW_BF16 ? launch_linear_bf16(l.plan, a, s) : launch_linear_f32("linear", LINEAR_FWD, a, s));
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
    const bool bf = cfg->act_dtype == SW_BF16;
    if (cfg->M == 0) {
        if (dW && (st = fill_zero(dW, (size_t)(cfg->K * cols) * (bf ? 2 : 4), s))) return st;
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
        a.dz = l.own_dz && (dx || dW) ? ws + l.dz : nullptr;
        a.part = db ? (float *)(ws + l.db_part) : nullptr;
        a.M = cfg->M; a.N = (int)cfg->N; a.act = cfg->activation; a.lanes = l.lanes;
        a.drop = drop;
        const dim3 grid((unsigned)l.db_parts, (unsigned)ceil_div(cfg->N, l.lanes * (bf ? 8 : 4)));
#define SW_DZ(T, G) hipLaunchKernelGGL((linear_dz_kernel<T, G>), grid, dim3(256), 0, s, a)
        if (bf) { if (gated) SW_DZ(bf16, true); else SW_DZ(bf16, false); }
        else { if (gated) SW_DZ(float, true); else SW_DZ(float, false); }
#undef SW_DZ
        if ((st = status_of(hipGetLastError()))) return st;
    }
    LinearArgs ax{}, aw{};
    ax.scale = aw.scale = drop.scale;
    ax.Q = dz; ax.ldq = (int)cols;
    ax.P = W; ax.ldp = (int)cols;
    ax.Qdim = cfg->M; ax.Kdim = cols; ax.Pdim = (int)cfg->K;
    ax.C = dx;
    aw.Q = x; aw.ldq = (int)cfg->K;
    aw.P = dz; aw.ldp = (int)cols;
    aw.Qdim = cfg->K; aw.Kdim = cfg->M; aw.Pdim = (int)cols;
    aw.C = dW; aw.part = (float *)(ws + l.dW_part);
    if (bf) {
        if ((dx || dW) && (st = status_of(launch_linear_backward_bf16(l.plan, dx ? &ax : nullptr, dW ? &aw : nullptr, s)))) return st;
    } else {
        if (dx && (st = status_of(launch_linear_f32("linear_dx", LINEAR_DX, ax, s)))) return st;
        if (dW && (st = status_of(launch_linear_f32("linear_dW", LINEAR_DW, aw, s)))) return st;
    }
    const bool join_dW = dW && l.plan.splits > 1;
    if (join_dW || db) {
        ProfScope ps("linear_join", s);
        LinearJoin j{};
        j.dW_part = aw.part; j.dW = dW;
        j.elements = cfg->K * cols;
        j.splits = l.plan.splits;
        j.dW_blocks = join_dW ? (int)ceil_div(j.elements, 1024 * (bf ? 8 : 4)) : 0;
        j.db_part = (const float *)(ws + l.db_part); j.db = db;
        j.db_parts = l.db_parts;
        j.cols = (int)cols;
        j.scale = drop.scale;
        const dim3 grid((unsigned)(j.dW_blocks + (db ? ceil_div(cols, kJoinCols) : 0)));
        if (bf) hipLaunchKernelGGL(linear_join_kernel<bf16>, grid, dim3(1024), 0, s, j);
        else hipLaunchKernelGGL(linear_join_kernel<float>, grid, dim3(1024), 0, s, j);
        st = status_of(hipGetLastError());
    }
    return st;
}

}  // extern "C"

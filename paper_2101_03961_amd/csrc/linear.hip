// switch_linear: one matrix product with bias, activation, dropout and residual in its epilogue, and its gradients.
//
//   z = x W + b,  y = r + drop(act(z));   dz = act'(z) drop(dy),  dx = dz W^T,  dW = x^T dz,  db = sum of dz's rows
//
// The products: linear_bf16.hip, linear_f32.hip, linear_few.hip.  Here: how they are cut, the element-wise pass before those of
// the backward pass, the sums of their parts, and the entry points.
#include <math.h>

#include "linear.h"

namespace sw {

// dz without the dropout's scale (so that, where act' is 0 or 1, it is dy or zero and loses nothing in bf16) and sums of its
// rows.  A lane takes a chunk of columns, 16 bytes, of the gate and of the linear part; `lanes` lanes of a block share a row
// and each handles `steps` rows, 256 / lanes apart.  Bound by its traffic.
//
// GELU's dz has more digits than bf16.  Its rounding adds as much error to a gradient as the gradient's own (together sqrt(2)
// of one) where many values average it; over few rows a gradient hangs on few of them, and the two came to 1.5 to 2.1 of one
// (1 to 5 rows; at most 1.55 at 32, 1.48 at 128, 1.47 at 256 and 512).  So up to kTermRows rows, and where a caller asks
// for it, dz is kept as the sum of two bf16 terms, 16 digits, the second M rows below the first; the products, which W and dW
// bind there and not their operations, take 2 M rows: dx's of both terms are added up as parts of k are, dW's k runs over both
// terms, over x twice.  One term / two, us, 4096 -> 2 x 10240 gated: 16 rows 108 / 113, 64 rows 113 / 142, 256 rows 166 / 201,
// 1024 rows 329 / 581, 8192 rows 2146 / 4419; 768 -> 2 x 2048: 1 row 13.6 / 14.9, 16 rows 17.4 / 22.4, 256 rows 22.0 / 26.4.
constexpr int kTermRows = 256, kCopyBlocks = 512;
static int linear_terms(const switch_linear_config *cfg) {
    const bool gelu = cfg->activation == SW_ACT_GELU || cfg->activation == SW_ACT_GEGLU;
    return cfg->act_dtype == SW_BF16 && gelu && (cfg->M <= kTermRows || cfg->flags & SW_FLAG_DZ_TWO_TERMS) ? 2 : 1;
}
struct DzArgs {
    const void *dy, *z;
    void *dz;                      // or nullptr
    int64_t low;                   // where dz's second term begins; 0: one term
    const void *x;                 // with two terms, copied twice by the blocks behind y_blocks
    void *x_twice;                 // or nullptr
    int64_t x_elements;
    int y_blocks;
    float *part;                   // [row blocks][columns of W], or nullptr
    int64_t M;
    int N, act, lanes, steps;
    Drop drop;
};

// what a value's rounding to bf16 leaves (exact); nothing where that is infinite
__device__ __forceinline__ float rest_of(float v) {
    const float first = (float)(bf16)v;
    return isfinite(first) ? v - first : 0.f;
}

template <typename T, bool GATED>
__global__ __launch_bounds__(256) void linear_dz_kernel(DzArgs a) {
    typedef Row16<T> C;
    constexpr int n = C::n, NP = GATED ? 2 : 1;
    __shared__ float sums[256][NP * n + 1];
    const int tid = threadIdx.x, line = tid / a.lanes, lines = 256 / a.lanes;
    if (sizeof(T) == 2 && (int)blockIdx.y >= a.y_blocks) {
        const int64_t block = (int64_t)(blockIdx.y - a.y_blocks) * gridDim.x + blockIdx.x;
        const int64_t step = (int64_t)(gridDim.y - a.y_blocks) * gridDim.x * 256 * n;
        for (int64_t at = (block * 256 + tid) * n; at < a.x_elements; at += step) {
            float v[n];
            C::load(a.x, at, v);
            C::store(a.x_twice, at, v);
            // (an infinity counts once: its products with the second terms have either sign)
#pragma unroll
            for (int m = 0; m < n; ++m) v[m] = isfinite(v[m]) ? v[m] : 0.f;
            C::store(a.x_twice, a.x_elements + at, v);
        }
        return;
    }
    const int p = (blockIdx.y * a.lanes + tid % a.lanes) * n;
    const int64_t q0 = (int64_t)blockIdx.x * (lines * a.steps) + line;
    const int64_t Nz = NP * (int64_t)a.N;
    float sum[NP][n] = {};
    if (p < a.N)
#pragma unroll 2
        for (int i = 0; i < a.steps; ++i) {
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
                for (int m = 0; m < n; ++m) g[m] = u[m] <= 0.f ? 0.f : u[m] > 0.f ? g[m] : u[m];   // (NaN stays NaN)
            } else if (a.act != SW_ACT_NONE) {
#pragma unroll
                for (int m = 0; m < n; ++m) {
                    const NormalOf no = normal_at<T>(u[m]);
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
                if (sizeof(T) == 2 && a.low) {
                    float rest[n];
#pragma unroll
                    for (int m = 0; m < n; ++m) rest[m] = rest_of(g[m]);
                    C::store(a.dz, a.low + zat, rest);
                    if (GATED) {
#pragma unroll
                        for (int m = 0; m < n; ++m) rest[m] = rest_of(v[m]);
                        C::store(a.dz, a.low + zat + a.N, rest);
                    }
                }
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

// Sums of parts, in their order: of dx, of dW and, by lines of blocks behind, of db.
struct LinearSum {
    const float *part;
    void *out;
    int64_t elements;
    int splits, blocks;
};
struct LinearJoin {
    LinearSum dx, dW;
    const float *db_part;
    float *db;
    int64_t db_parts;
    int cols;
    float scale;
};
constexpr int kJoinThreads = 1024, kJoinCols = 32;

template <int n> __device__ __forceinline__ void add_parts(const float *part, int splits, int64_t stride, float *sum) {
#pragma unroll
    for (int m = 0; m < n; ++m) sum[m] = 0.f;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const float *from = part + s * stride;
#pragma unroll
        for (int m = 0; m < n; m += 4) {
            const float4 x = *(const float4 *)(from + m);
            sum[m] += x.x; sum[m + 1] += x.y; sum[m + 2] += x.z; sum[m + 3] += x.w;
        }
    }
}

template <typename T> __global__ __launch_bounds__(kJoinThreads) void linear_join_kernel(LinearJoin a) {
    constexpr int n = Row16<T>::n;
    int b = blockIdx.x;
    if (b < a.dx.blocks + a.dW.blocks) {
        const LinearSum &w = b < a.dx.blocks ? a.dx : a.dW;
        if (b >= a.dx.blocks) b -= a.dx.blocks;
        const int64_t at = ((int64_t)b * kJoinThreads + threadIdx.x) * n;
        if (at >= w.elements) return;
        float sum[n];
        add_parts<n>(w.part + at, w.splits, w.elements, sum);
#pragma unroll
        for (int m = 0; m < n; ++m) sum[m] *= a.scale;
        Row16<T>::store(w.out, at, sum);
        return;
    }
    b -= a.dx.blocks + a.dW.blocks;
    constexpr int kLines = kJoinThreads / kJoinCols;
    __shared__ double sums[kLines][kJoinCols + 1];
    const int col = threadIdx.x % kJoinCols, line = threadIdx.x / kJoinCols;
    const int p = b * kJoinCols + col;
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

// The forward pass behind several parts of k: their sums and the epilogue.
template <typename T, int ACT> __global__ __launch_bounds__(256) void linear_finish_kernel(LinearArgs a, int splits) {
    constexpr int n = Row16<T>::n;
    constexpr bool GATED = ACT == SW_ACT_GEGLU;
    const uint32_t chunks = (uint32_t)a.Pdim / n;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, q = i / chunks;
    if (q >= a.Qdim) return;
    const int p = (int)(i - q * chunks) * n;
    const int64_t cols = GATED ? 2 * (int64_t)a.Pdim : a.Pdim;
    const float *from = a.part + q * cols + p;
    float v[n], lin[n];
    add_parts<n>(from, splits, a.Qdim * cols, v);
    if (GATED) add_parts<n>(from + a.Pdim, splits, a.Qdim * cols, lin);
    linear_emit<T, ACT>(a, q, p, v, lin);
}
template <typename T> static hipError_t linear_finish(const LinearArgs &a, int splits, hipStream_t s) {
    ProfScope ps("linear_finish", s);
    const dim3 grid((unsigned)ceil_div(a.Qdim * (a.Pdim / Row16<T>::n), 256));
    auto kern = a.act == SW_ACT_RELU    ? linear_finish_kernel<T, SW_ACT_RELU>
                : a.act == SW_ACT_GELU  ? linear_finish_kernel<T, SW_ACT_GELU>
                : a.act == SW_ACT_GEGLU ? linear_finish_kernel<T, SW_ACT_GEGLU>
                                        : linear_finish_kernel<T, SW_ACT_NONE>;
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, a, splits);
    return hipGetLastError();
}

// ---- how a product is cut ---------------------------------------------------------------------
// Per kind of tile: k of a step; us of a step per block of a CU (of the blocks that share it, one after the other) and of
// a step at least; us of a block's start and end, forward and backward (whose parts of dW are stored in fp32); blocks that a
// CU holds.  Fitted to products of 4 to 64 steps and to backward passes with 1 to 48 parts of dW; us of dx and dW, as chosen
// (tile, parts) / the best of all: 16384 x 768 x 2048 (256, 12) 119 / 119; 65536 x 2048 x 768 (256, 8) 461 / 461;
// 8192 x 2048 x 768 (256, 8) 75 / 67; 5000 x 520 x 1000 (128, 6) 27 / 27; 2048 x 4096 x 4096 (256, 1) 119 / 118;
// 30000 x 264 x 520 (128, 16) 48 / 46.
struct LinearModel {
    int tile, bk;
    double step, least, once_fwd, once_bwd;
    int resident;
};
static const LinearModel kBf16Models[] = {{256, 64, 1.45, 1.45, 10., 17., 1}, {128, 64, 0.52, 0.75, 4., 8., 2}};
static const LinearModel kF32Models[] = {{64, 32, 0.5, 0.6, 5., 5., 3}};
constexpr int kCUs = 256;
// A launch that adds up parts of k: forward, with the epilogue, or backward.
static double finish_us(int splits, double elements) { return splits > 1 ? 4. + splits * elements * 2e-6 : 0.; }
static double join_us(int splits, double elements) { return splits > 1 ? 3. + splits * elements * 0.67e-6 : 0.; }
static LinearCut cut_of(int64_t k, int splits, int bk) {
    const int64_t split_k = ceil_div(ceil_div(k, splits), bk) * bk;
    return LinearCut{(int)ceil_div(k, split_k), split_k};
}

LinearPlan plan_linear(const switch_linear_config *cfg, bool backward) {
    const int64_t M = cfg->M * (backward ? linear_terms(cfg) : 1), K = cfg->K, Nz = linear_columns(cfg);
    LinearPlan plan{64, {1, backward ? Nz : K}, {1, M}};
    if (M == 0) return plan;
    if (!backward && linear_few_rows(cfg)) return LinearPlan{0, linear_few_cut(cfg), {1, M}};
    const bool bf = cfg->act_dtype == SW_BF16;
    // the rows of a part of dW: what a descriptor of 2 GB spans
    const int64_t widest = (K > Nz ? K : Nz) * (bf ? 2 : 4), most_k = (int64_t)0x7fffffff / widest / 64 * 64;
    static const int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
    // the normal distribution function of a large tile's values, which no other block's products hide
    const double gelu_us = cfg->activation == SW_ACT_GELU ? 9. : cfg->activation == SW_ACT_GEGLU ? 5. : 0.;
    double best = 1e30;
    const LinearModel *models = bf ? kBf16Models : kF32Models;
    for (int i = 0; i < (bf ? 2 : 1); ++i) {
        const LinearModel &m = models[i];
        const double tx = (double)ceil_div(M, m.tile) * ceil_div(backward ? K : Nz, m.tile);
        const int64_t kx = backward ? Nz : K;
        for (int sx : kSplits) {
            // (parts of y or dx only while its tiles leave CUs idle; four steps at least)
            if (sx > 1 && (tx * sx > 2 * kCUs || kx < (int64_t)sx * 4 * m.bk)) break;
            const LinearCut x = cut_of(kx, sx, m.bk);
            const double steps_x = (double)ceil_div(x.split_k, m.bk), items_x = tx * x.splits;
            if (!backward) {
                const double per_cu = ceil(items_x / kCUs);
                const double us = ceil(per_cu / m.resident) * (m.once_fwd + (m.resident == 1 ? gelu_us : 0.)) +
                                  steps_x * fmax(per_cu * m.step, m.least) + finish_us(x.splits, (double)M * Nz);
                if (us < best) {
                    best = us;
                    plan = LinearPlan{m.tile, x, {1, M}};
                }
                continue;
            }
            const double tw = (double)ceil_div(K, m.tile) * ceil_div(Nz, m.tile);
            bool found = false;   // (a cut whose parts a descriptor spans)
            for (int sw : kSplits) {
                if (found && (tw * sw > 4 * kCUs * m.resident || M < (int64_t)sw * 4 * m.bk)) break;
                LinearCut w = cut_of(M, sw, m.bk);
                if (w.split_k > most_k) {
                    if (sw < 64) continue;
                    w = LinearCut{(int)ceil_div(M, most_k), most_k};
                }
                found = true;
                const double steps_w = (double)ceil_div(w.split_k, m.bk), items_w = tw * w.splits;
                // dx's tiles, then dW's on what they leave idle: whole blocks
                const double once = m.once_bwd / m.resident, bx = steps_x * m.step + once, bw = steps_w * m.step + once;
                const double rounds = floor(items_x / kCUs), over = items_x - rounds * kCUs, t0 = rounds * bx;
                double end = fmax(t0 + (over > 0 ? bx : 0.), (items_x * bx + items_w * bw) / kCUs);
                for (int j = 0; j < 16; ++j) {
                    const double na = floor(fmax(end - t0 - bx, 0.) / bw + 1e-9), nb = floor((end - t0) / bw + 1e-9);
                    if (over * na + (kCUs - over) * nb >= items_w) break;
                    const double a = t0 + bx + (na + 1.) * bw, b = t0 + (nb + 1.) * bw;
                    end = over > 0 && a < b ? a : b;
                }
                end = fmax(end, fmax(steps_x, steps_w) * m.least + m.once_bwd);
                const double us = end + join_us(x.splits, (double)M * K) + join_us(w.splits, (double)K * Nz);
                if (us < best) {
                    best = us;
                    plan = LinearPlan{m.tile, x, w};
                }
            }
        }
    }
    return plan;
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
    if (cfg->flags & ~SW_FLAG_DZ_TWO_TERMS) return SW_ERR_VALUE;
    return SW_OK;
}

struct LinearLayout {
    size_t dz, x_twice, db_part, x_part, w_part, total;
    bool own_dz;                   // dz is not dy itself
    int terms;                     // of dz
    int x_parts;                   // sums of y or dx: parts of k, each of every term
    int lanes, steps;              // of linear_dz_kernel
    int64_t db_parts;
    LinearPlan plan;
};
static LinearLayout linear_layout(const switch_linear_config *cfg, bool backward) {
    LinearLayout l{};
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, 256); return o; };
    const int64_t elt = cfg->act_dtype == SW_BF16 ? 2 : 4, cols = linear_columns(cfg);
    l.plan = plan_linear(cfg, backward);
    if (backward) {
        l.own_dz = cfg->activation != SW_ACT_NONE || drop_of(cfg->dropout, 0).on;
        const int64_t chunks = cfg->N * elt / 16;
        l.lanes = 1;
        while (l.lanes < 32 && l.lanes < chunks) l.lanes *= 2;
        // rows of a lane: eight, fewer while the blocks are fewer than the CUs (a whole backward pass, gated, eight / so:
        // 256 rows 120 -> 2 x 280: 33.8 / 15.5 us, 768 -> 2 x 2048: 35.2 / 26.5; 64 rows 4096 -> 2 x 10240: 158 / 148)
        l.steps = 8;
        while (l.steps > 1 && ceil_div(cfg->M, 256 / l.lanes * l.steps) * ceil_div(chunks, l.lanes) < kCUs) l.steps /= 2;
        l.db_parts = ceil_div(cfg->M, 256 / l.lanes * l.steps);
        l.terms = linear_terms(cfg);
        l.dz = take(l.own_dz ? (size_t)l.terms * cfg->M * cols * elt : 0);
        l.x_twice = take(l.terms > 1 ? (size_t)2 * cfg->M * cfg->K * elt : 0);
        l.db_part = take((size_t)l.db_parts * cols * 4);
        l.w_part = take(l.plan.w.splits > 1 ? (size_t)l.plan.w.splits * cfg->K * cols * 4 : 0);
    } else {
        l.terms = 1;
    }
    l.x_parts = l.plan.x.splits * l.terms;
    l.x_part = take(l.x_parts > 1 ? (size_t)l.x_parts * cfg->M * (backward ? cfg->K : cols) * 4 : 0);
    l.total = cfg->M ? off : 0;
    return l;
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
    int st = check_linear(cfg);
    if (st != SW_OK) return st;
    if (cfg->M == 0) return SW_OK;
    if (!x || !W || !y) return SW_ERR_NULL;
    if (!aligned16(x) || !aligned16(W) || !aligned16(bias) || !aligned16(residual) || !aligned16(y) || !aligned16(z))
        return SW_ERR_ALIGN;
    const LinearLayout l = linear_layout(cfg, false);
    if (!linear_workspace_ok(l, workspace, workspace_bytes)) return SW_ERR_WORKSPACE;
    const bool bf = cfg->act_dtype == SW_BF16;
    LinearArgs a{};
    a.Q = x; a.ldq = (int)cfg->K;
    a.P = W; a.ldp = (int)linear_columns(cfg);
    a.Qdim = cfg->M; a.Kdim = cfg->K; a.Pdim = (int)cfg->N;
    a.bias = bias; a.residual = residual; a.C = y; a.z = z;
    a.part = l.x_parts > 1 ? (float *)((char *)workspace + l.x_part) : nullptr;
    a.act = cfg->activation;
    a.gated = cfg->activation == SW_ACT_GEGLU;
    a.scale = 1.f;
    a.drop = drop_of(cfg->dropout, cfg->seed);
    hipStream_t s = (hipStream_t)hip_stream;
    {
        ProfScope ps("linear", s);
        st = status_of(l.plan.tile == 0 ? launch_linear_few(cfg->act_dtype, l.plan, a, s)
                       : bf             ? launch_linear_bf16(l.plan, a, s)
                                        : launch_linear_f32(l.plan, a, s));
    }
    if (st || l.plan.x.splits == 1) return st;
    return status_of(bf ? linear_finish<bf16>(a, l.plan.x.splits, s) : linear_finish<float>(a, l.plan.x.splits, s));
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
        a.M = cfg->M; a.N = (int)cfg->N; a.act = cfg->activation; a.lanes = l.lanes; a.steps = l.steps;
        a.drop = drop;
        a.y_blocks = (int)ceil_div(cfg->N, l.lanes * (bf ? 8 : 4));
        dim3 grid((unsigned)l.db_parts, (unsigned)a.y_blocks);
        if (l.terms > 1 && (dx || dW)) a.low = cfg->M * cols;
        if (l.terms > 1 && dW) {
            a.x = x; a.x_twice = ws + l.x_twice;
            a.x_elements = cfg->M * cfg->K;
            const int64_t blocks = ceil_div(a.x_elements, 256 * 8);
            grid.y += (unsigned)ceil_div(blocks < kCopyBlocks ? blocks : kCopyBlocks, l.db_parts);
        }
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
    ax.Qdim = l.terms * cfg->M; ax.Kdim = cols; ax.Pdim = (int)cfg->K;
    ax.C = dx; ax.part = l.x_parts > 1 ? (float *)(ws + l.x_part) : nullptr;
    aw.Q = l.terms > 1 ? ws + l.x_twice : x; aw.ldq = (int)cfg->K;
    aw.P = dz; aw.ldp = (int)cols;
    aw.Qdim = cfg->K; aw.Kdim = l.terms * cfg->M; aw.Pdim = (int)cols;
    aw.C = dW; aw.part = l.plan.w.splits > 1 ? (float *)(ws + l.w_part) : nullptr;
    if (dx || dW) {
        ProfScope ps("linear_backward", s);
        auto launch = bf ? launch_linear_backward_bf16 : launch_linear_backward_f32;
        if ((st = status_of(launch(l.plan, dx ? &ax : nullptr, dW ? &aw : nullptr, s)))) return st;
    }
    LinearJoin j{};
    auto sum = [&](const LinearArgs &a, int64_t rows, int splits) {
        const int64_t elements = rows * a.Pdim;
        return LinearSum{a.part, a.C, elements, splits, (int)ceil_div(elements, kJoinThreads * (bf ? 8 : 4))};
    };
    if (dx && l.x_parts > 1) j.dx = sum(ax, cfg->M, l.x_parts);
    if (dW && l.plan.w.splits > 1) j.dW = sum(aw, cfg->K, l.plan.w.splits);
    if (!j.dx.blocks && !j.dW.blocks && !db) return SW_OK;
    ProfScope ps("linear_join", s);
    j.db_part = (const float *)(ws + l.db_part); j.db = db;
    j.db_parts = l.db_parts;
    j.cols = (int)cols;
    j.scale = drop.scale;
    const dim3 grid((unsigned)(j.dx.blocks + j.dW.blocks + (db ? ceil_div(cols, kJoinCols) : 0)));
    if (bf) hipLaunchKernelGGL(linear_join_kernel<bf16>, grid, dim3(kJoinThreads), 0, s, j);
    else hipLaunchKernelGGL(linear_join_kernel<float>, grid, dim3(kJoinThreads), 0, s, j);
    return status_of(hipGetLastError());
}

}  // extern "C"

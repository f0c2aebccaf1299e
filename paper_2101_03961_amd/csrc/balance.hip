// The load-balancing loss of a router's logits and choices, and the gradient of the logits.
//
//   p = softmax(h) per row;  P_i = sum p_i / n and f_i = counts_i / (n k) over a group's n tokens;
//   loss = alpha E / G sum_groups sum_i f_i P_i
//   dh_j = p_j (c_j - sum_i p_i c_i),  c_i = d_loss alpha E f_i / (G n)
//
// Both directions read the logits once and are bound by that (and by the store of dh): a row stays in the registers of
// the G lanes that share it.  Forward, each lane keeps the running sums of its columns in registers over the rows of its
// block; the blocks' sums and counts are added up by a second kernel in a fixed order.
#include <math.h>

#include "ops.h"

namespace sw {

constexpr int kBalThreads = 256;
constexpr int kBalJoinCols = 32;   // experts per block of the joining kernel

struct BalanceArgs {
    const float *logits;
    const int32_t *index;
    const uint8_t *mask;
    int64_t Tg;                 // tokens of a group
    int E, k, groups;
    int nbg;                    // blocks per group
    int tb;                     // tokens per block
    float *psum_part;           // [groups * nbg][E]
    int32_t *count_part;        // [groups * nbg][E]
    int32_t *token_part;        // [groups * nbg]
    double *loss_part;          // [groups][tiles of kBalJoinCols experts]
    uint32_t *arrived;          // blocks of the joining kernel that are done
    double alpha;
    float *loss;
    int32_t *counts, *tokens;
};

template <int G> __device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
    for (int m = G / 2; m > 0; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, kWave));
    return v;
}
template <int G> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int m = G / 2; m > 0; m >>= 1) v += __shfl_xor(v, m, kWave);
    return v;
}

// The lane's part of a row: chunks of four logits, G lanes apart; columns past E are -inf.
template <int G, int NV, bool WIDE>
__device__ __forceinline__ void balance_row(const float *row, int E, int lane, float (&h)[NV][4]) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (lane + G * i) * 4;
        if (WIDE) {   // E a multiple of four: rows begin on 16 bytes
            float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            if (c < E) v = *(const float4 *)(row + c);
            h[i][0] = v.x; h[i][1] = v.y; h[i][2] = v.z; h[i][3] = v.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) h[i][j] = c + j < E ? row[c + j] : -INFINITY;
        }
    }
}

// h becomes the row's probabilities; a row of -inf alone becomes zeros
template <int G, int NV> __device__ __forceinline__ void balance_probs(float (&h)[NV][4]) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) m = fmaxf(m, h[i][j]);
    m = lanes_max<G>(m);
    if (m == -INFINITY) m = 0.f;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            h[i][j] = __expf(h[i][j] - m);
            s += h[i][j];
        }
    s = lanes_sum<G>(s);
    const float inv = s > 0.f ? 1.0f / s : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) h[i][j] *= inv;
}

template <int G, int NV, bool WIDE>
__global__ __launch_bounds__(kBalThreads) void balance_kernel(BalanceArgs a) {
    constexpr int kCols = G * NV * 4, kRows = kBalThreads / G;
    __shared__ float psum[kCols];
    __shared__ int32_t hist[kCols];
    __shared__ int32_t live_tokens;
    const int tid = threadIdx.x, lane = tid % G, sub = tid / G;
    const int g = blockIdx.x / a.nbg;
    const int64_t t0 = g * a.Tg + (int64_t)(blockIdx.x - g * a.nbg) * a.tb;
    const int64_t gend = (g + 1) * a.Tg, tend = t0 + a.tb < gend ? t0 + a.tb : gend;
    // (the first row's logits are under way while the choices are counted, the next one's while a row is worked on)
    auto live = [&](int64_t t) { return t < tend && (!a.mask || a.mask[t]); };
    float next[NV][4];
    bool have = live(t0 + sub);
    if (have) balance_row<G, NV, WIDE>(a.logits + (t0 + sub) * a.E, a.E, lane, next);
    if (blockIdx.x == 0 && tid == 0) *a.arrived = 0;   // for the kernel behind this one
    for (int i = tid; i < kCols; i += kBalThreads) hist[i] = 0;
    if (tid == 0) live_tokens = 0;
    __syncthreads();
    const uint32_t choices = (uint32_t)((tend - t0) * a.k);   // (T k < 2^31)
    for (uint32_t i = tid; i < choices; i += kBalThreads) {
        if (a.mask && !a.mask[t0 + i / (uint32_t)a.k]) continue;
        const int e = a.index[t0 * a.k + i];
        if ((unsigned)e < (unsigned)a.E) atomicAdd(&hist[e], 1);
    }
    float acc[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
    int seen = 0;
    for (int64_t t = t0 + sub; t < tend; t += kRows) {
        float h[NV][4];
        const bool now = have;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) h[i][j] = next[i][j];
        have = live(t + kRows);
        if (have) balance_row<G, NV, WIDE>(a.logits + (t + kRows) * a.E, a.E, lane, next);
        if (!now) continue;
        ++seen;
        balance_probs<G, NV>(h);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] += h[i][j];
    }
    if (lane == 0 && seen) atomicAdd(&live_tokens, seen);
    // the rows of a wave, then the waves one after the other
#pragma unroll
    for (int m = G; m < kWave; m <<= 1)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] += __shfl_xor(acc[i][j], m, kWave);
#pragma unroll
    for (int w = 0; w < kBalThreads / kWave; ++w) {
        if (tid / kWave == w && tid % kWave < G) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = (lane + G * i) * 4 + j;
                    psum[c] = w ? psum[c] + acc[i][j] : acc[i][j];
                }
        }
        __syncthreads();
    }
    if (gridDim.x == 1) {   // the only block: no parts to join
        __shared__ double sums[kBalThreads / kWave];
        double sum = 0.;
        for (int i = tid; i < a.E; i += kBalThreads) {
            a.counts[i] = hist[i];
            sum += (double)psum[i] * (double)hist[i];
        }
#pragma unroll
        for (int m = kWave / 2; m > 0; m >>= 1) sum += __shfl_xor(sum, m, kWave);
        if (tid % kWave == 0) sums[tid / kWave] = sum;
        __syncthreads();
        if (tid == 0) {
            sum = 0.;
#pragma unroll
            for (int w = 0; w < kBalThreads / kWave; ++w) sum += sums[w];
            const double n = live_tokens > 0 ? (double)live_tokens : 1.;
            a.tokens[0] = live_tokens;
            *a.loss = (float)(a.alpha * a.E / a.k * (sum / (n * n)));
        }
        return;
    }
    const size_t at = (size_t)blockIdx.x * a.E;
    for (int i = tid; i < a.E; i += kBalThreads) {
        a.psum_part[at + i] = psum[i];
        a.count_part[at + i] = hist[i];
    }
    if (tid == 0) a.token_part[blockIdx.x] = live_tokens;
}

// Adds up a group's parts for kBalJoinCols experts; the block that is last to arrive adds up the loss.
__global__ __launch_bounds__(1024) void balance_join_kernel(BalanceArgs a) {
    constexpr int kLines = 1024 / kBalJoinCols;
    __shared__ double ps[kLines][kBalJoinCols + 1];
    __shared__ int32_t cs[kLines][kBalJoinCols + 1];
    __shared__ int32_t ns[1024 / kWave];
    __shared__ uint32_t before;
    const int tid = threadIdx.x, col = tid % kBalJoinCols, line = tid / kBalJoinCols;
    const int tiles = (int)gridDim.x, tile = blockIdx.x, g = blockIdx.y;
    const int e = tile * kBalJoinCols + col;
    const size_t b0 = (size_t)g * a.nbg;
    double p = 0.;
    int32_t c = 0, n = 0;
    if (e < a.E)
#pragma unroll 8
        for (int b = line; b < a.nbg; b += kLines) {
            p += (double)a.psum_part[(b0 + b) * a.E + e];
            c += a.count_part[(b0 + b) * a.E + e];
        }
    for (int b = tid; b < a.nbg; b += 1024) n += a.token_part[b0 + b];
    ps[line][col] = p;
    cs[line][col] = c;
#pragma unroll
    for (int m = kWave / 2; m > 0; m >>= 1) n += __shfl_xor(n, m, kWave);
    if (tid % kWave == 0) ns[tid / kWave] = n;
    __syncthreads();
    if (tid < kWave) {
        n = 0;
#pragma unroll
        for (int w = 0; w < 1024 / kWave; ++w) n += ns[w];
        double part = 0.;
        if (tid < kBalJoinCols && e < a.E) {
            p = 0.;
            c = 0;
            for (int l = 0; l < kLines; ++l) {
                p += ps[l][col];
                c += cs[l][col];
            }
            a.counts[(size_t)g * a.E + e] = c;
            part = p * (double)c;
        }
#pragma unroll
        for (int m = kWave / 2; m > 0; m >>= 1) part += __shfl_xor(part, m, kWave);
        if (tid == 0) {
            if (tile == 0) a.tokens[g] = n;
            const double nn = n > 0 ? (double)n : 1.;
            __hip_atomic_store(a.loss_part + (size_t)g * tiles + tile, part / (nn * nn), __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
            before = __hip_atomic_fetch_add(a.arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    __syncthreads();
    const int parts = tiles * a.groups;
    if (before != (uint32_t)parts - 1) return;
    double sum = 0.;
    for (int i = tid; i < parts; i += 1024)
        sum += __hip_atomic_load(a.loss_part + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    ps[0][0] = 0.;
    __syncthreads();
#pragma unroll
    for (int m = kWave / 2; m > 0; m >>= 1) sum += __shfl_xor(sum, m, kWave);
    if (tid % kWave == 0) ps[tid / kWave][0] = sum;
    __syncthreads();
    if (tid == 0) {
        sum = 0.;
        for (int w = 0; w < 1024 / kWave; ++w) sum += ps[w][0];
        *a.loss = (float)(a.alpha * a.E / ((double)a.groups * a.k) * sum);
    }
}

struct BalanceBwdArgs {
    const float *logits;
    const uint8_t *mask;
    const int32_t *counts, *tokens;
    float *dlogits;
    int64_t Tg;
    int E;
    int nbg, tb;
    double scale;               // d_loss alpha E / (G k)
};

template <int G, int NV, bool WIDE>
__global__ __launch_bounds__(kBalThreads) void balance_bwd_kernel(BalanceBwdArgs a) {
    constexpr int kRows = kBalThreads / G;
    __shared__ int64_t totals[kBalThreads / kWave];
    const int tid = threadIdx.x, lane = tid % G, sub = tid / G;
    const int g = blockIdx.x / a.nbg;
    const int64_t t0 = g * a.Tg + (int64_t)(blockIdx.x - g * a.nbg) * a.tb;
    const int64_t gend = (g + 1) * a.Tg, tend = t0 + a.tb < gend ? t0 + a.tb : gend;
    // (the first row's logits are under way while the coefficients are made, the next one's while a row is worked on)
    auto live = [&](int64_t t) { return t < tend && (!a.mask || a.mask[t]); };
    float next[NV][4];
    bool have = live(t0 + sub);
    if (have) balance_row<G, NV, WIDE>(a.logits + (t0 + sub) * a.E, a.E, lane, next);
    const int32_t *counts = a.counts + (size_t)g * a.E;
    int64_t total = 0;
    for (int i = tid; i < a.E; i += kBalThreads) total += counts[i];
#pragma unroll
    for (int m = kWave / 2; m > 0; m >>= 1) total += __shfl_xor(total, m, kWave);
    if (tid % kWave == 0) totals[tid / kWave] = total;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < kBalThreads / kWave; ++w) total += totals[w];
    // c_j less its mean over the experts, which drops out (sum p = 1) and would cost its digits in c_j - sum p c
    const double n = a.tokens[g], scale = n > 0. ? a.scale / (n * n) : 0., mean = (double)total / a.E;
    float c[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = (lane + G * i) * 4 + j;
            c[i][j] = e < a.E ? (float)(((double)counts[e] - mean) * scale) : 0.f;
        }
    for (int64_t t = t0 + sub; t < tend; t += kRows) {
        float h[NV][4];
        const bool now = have;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) h[i][j] = now ? next[i][j] : 0.f;
        have = live(t + kRows);
        if (have) balance_row<G, NV, WIDE>(a.logits + (t + kRows) * a.E, a.E, lane, next);
        if (now) {
            balance_probs<G, NV>(h);
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) dot = fmaf(h[i][j], c[i][j], dot);
            dot = lanes_sum<G>(dot);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) h[i][j] *= c[i][j] - dot;
        }
        float *out = a.dlogits + t * a.E;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (lane + G * i) * 4;
            if (WIDE) {
                if (col < a.E) *(float4 *)(out + col) = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (col + j < a.E) out[col + j] = h[i][j];
            }
        }
    }
}

// Lanes per row and chunks per lane: eight lanes read 128 bytes of a row at a time; more lanes share a row where a
// lane would hold more than 16 logits, up to a wave.
#define SW_BALANCE_LANES(E, WHAT)          \
    do {                                   \
        if ((E) <= 4) { WHAT(1, 1); }      \
        else if ((E) <= 8) { WHAT(2, 1); } \
        else if ((E) <= 16) { WHAT(4, 1); } \
        else if ((E) <= 32) { WHAT(8, 1); } \
        else if ((E) <= 64) { WHAT(8, 2); } \
        else if ((E) <= 128) { WHAT(8, 4); } \
        else if ((E) <= 256) { WHAT(16, 4); } \
        else if ((E) <= 512) { WHAT(32, 4); } \
        else if ((E) <= 1024) { WHAT(64, 4); } \
        else if ((E) <= 2048) { WHAT(64, 8); } \
        else { WHAT(64, 16); }             \
    } while (0)

static int balance_rows(int64_t E) {   // rows that a block handles at a time
    int rows = 0;
#define SW_ROWS_AT_A_TIME(G, NV) rows = kBalThreads / G
    SW_BALANCE_LANES(E, SW_ROWS_AT_A_TIME);
#undef SW_ROWS_AT_A_TIME
    return rows;
}

// Tokens per block: as many as leave about `blocks` of them, whole rounds of rows.
static int64_t balance_tokens(const switch_balance_config *cfg, int64_t blocks) {
    const int64_t groups = cfg->n_groups > 1 ? cfg->n_groups : 1, rows = balance_rows(cfg->E);
    const int64_t per = ceil_div(cfg->T, blocks), Tg = cfg->T / groups;
    const int64_t tb = ceil_div(per < Tg ? per : Tg, rows) * rows;
    return tb > 0 ? tb : rows;
}

struct BalanceLayout {
    int64_t groups, Tg, tb, nbg, tiles;
    size_t psum, count, token, loss, arrived, total;
};
static BalanceLayout balance_layout(const switch_balance_config *cfg) {
    BalanceLayout l{};
    l.groups = cfg->n_groups > 1 ? cfg->n_groups : 1;
    l.Tg = cfg->T / l.groups;
    // 512 blocks; more experts than 1024: 256, whose parts are half as many bytes (us, 256 / 512 / 1024 blocks: 65536 x 128
    // 15.6 / 14.9 / 17.8, 65536 x 512 38 / 33 / 36, 16384 x 2048 37 / 39 / 41, 4096 x 4096 25 / 28 / 37).  Four rounds of rows
    // or fewer: one block, without the second launch (9 us for both, however little they do).
    l.tb = balance_tokens(cfg, cfg->E > 1024 ? 256 : 512);
    if (l.groups == 1 && cfg->T <= 4 * balance_rows(cfg->E)) l.tb = 4 * balance_rows(cfg->E);
    l.nbg = ceil_div(l.Tg, l.tb);
    l.tiles = ceil_div(cfg->E, kBalJoinCols);
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, 256); return o; };
    const size_t parts = (size_t)(l.groups * l.nbg);
    l.psum = take(parts * cfg->E * 4);
    l.count = take(parts * cfg->E * 4);
    l.token = take(parts * 4);
    l.loss = take((size_t)(l.groups * l.tiles) * 8);
    l.arrived = take(4);
    l.total = cfg->T ? off : 0;
    return l;
}

static int check_balance(const switch_balance_config *cfg) {
    if (!cfg) return SW_ERR_NULL;
    if (cfg->T < 0 || cfg->T >= (int64_t)1 << 31) return SW_ERR_SHAPE;
    if (cfg->E < 1 || cfg->E > 4096) return SW_ERR_SHAPE;
    if (cfg->k < 1 || cfg->k > cfg->E || cfg->T * cfg->k >= (int64_t)1 << 31) return SW_ERR_SHAPE;
    if (cfg->n_groups < 0 || cfg->n_groups > 65535) return SW_ERR_SHAPE;
    if (cfg->n_groups > 1 && cfg->T % cfg->n_groups) return SW_ERR_SHAPE;
    if (!isfinite(cfg->alpha)) return SW_ERR_VALUE;
    if (cfg->flags) return SW_ERR_VALUE;
    return SW_OK;
}

}  // namespace sw

using namespace sw;

extern "C" {

int switch_balance_workspace_size(const switch_balance_config *cfg, size_t *bytes_out) {
    if (!cfg || !bytes_out) return SW_ERR_NULL;
    const int st = check_balance(cfg);
    if (st != SW_OK) return st;
    *bytes_out = balance_layout(cfg).total;
    return SW_OK;
}

int switch_balance_loss(const switch_balance_config *cfg, const float *logits, const int32_t *expert_index,
                        const uint8_t *token_mask, float *loss, int32_t *expert_counts, int32_t *token_counts,
                        void *workspace, size_t workspace_bytes, void *hip_stream) {
    int st = check_balance(cfg);
    if (st != SW_OK) return st;
    if (!loss || !expert_counts || !token_counts) return SW_ERR_NULL;
    hipStream_t s = (hipStream_t)hip_stream;
    const BalanceLayout l = balance_layout(cfg);
    if (cfg->T == 0) {
        if ((st = fill_zero(loss, 4, s))) return st;
        if ((st = fill_zero(expert_counts, (size_t)(l.groups * cfg->E) * 4, s))) return st;
        return fill_zero(token_counts, (size_t)l.groups * 4, s);
    }
    if (!logits || !expert_index) return SW_ERR_NULL;
    if (!aligned16(logits) || !aligned16(expert_index) || !aligned16(loss) || !aligned16(expert_counts) ||
        !aligned16(token_counts))
        return SW_ERR_ALIGN;
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < l.total) return SW_ERR_WORKSPACE;
    char *ws = (char *)workspace;
    BalanceArgs a{};
    a.logits = logits;
    a.index = expert_index;
    a.mask = token_mask;
    a.Tg = l.Tg;
    a.E = (int)cfg->E;
    a.k = (int)cfg->k;
    a.groups = (int)l.groups;
    a.nbg = (int)l.nbg;
    a.tb = (int)l.tb;
    a.psum_part = (float *)(ws + l.psum);
    a.count_part = (int32_t *)(ws + l.count);
    a.token_part = (int32_t *)(ws + l.token);
    a.loss_part = (double *)(ws + l.loss);
    a.arrived = (uint32_t *)(ws + l.arrived);
    a.alpha = cfg->alpha;
    a.loss = loss;
    a.counts = expert_counts;
    a.tokens = token_counts;
    {
        ProfScope ps("balance", s);
        const dim3 grid((unsigned)(l.groups * l.nbg));
#define SW_BALANCE(G, NV)                                                                                          \
    if (cfg->E % 4 == 0) hipLaunchKernelGGL((balance_kernel<G, NV, true>), grid, dim3(kBalThreads), 0, s, a);      \
    else hipLaunchKernelGGL((balance_kernel<G, NV, false>), grid, dim3(kBalThreads), 0, s, a)
        SW_BALANCE_LANES(cfg->E, SW_BALANCE);
#undef SW_BALANCE
        if ((st = status_of(hipGetLastError()))) return st;
    }
    if (l.groups * l.nbg == 1) return SW_OK;
    ProfScope ps("balance_join", s);
    hipLaunchKernelGGL(balance_join_kernel, dim3((unsigned)l.tiles, (unsigned)l.groups), dim3(1024), 0, s, a);
    return status_of(hipGetLastError());
}

int switch_balance_loss_backward(const switch_balance_config *cfg, float d_loss, const float *logits,
                                 const uint8_t *token_mask, const int32_t *expert_counts, const int32_t *token_counts,
                                 float *dlogits, void *hip_stream) {
    const int st = check_balance(cfg);
    if (st != SW_OK) return st;
    if (!isfinite(d_loss)) return SW_ERR_VALUE;
    if (cfg->T == 0) return SW_OK;
    if (!logits || !expert_counts || !token_counts || !dlogits) return SW_ERR_NULL;
    if (!aligned16(logits) || !aligned16(expert_counts) || !aligned16(token_counts) || !aligned16(dlogits))
        return SW_ERR_ALIGN;
    hipStream_t s = (hipStream_t)hip_stream;
    const int64_t groups = cfg->n_groups > 1 ? cfg->n_groups : 1;
    BalanceBwdArgs a{};
    a.logits = logits;
    a.mask = token_mask;
    a.counts = expert_counts;
    a.tokens = token_counts;
    a.dlogits = dlogits;
    a.Tg = cfg->T / groups;
    a.E = (int)cfg->E;
    // (us, 512 / 1024 / 2048 blocks: 65536 x 32 7.3 / 6.7 / 6.9, 65536 x 128 13.8 / 13.9 / 17.7, 16384 x 2048 55 / 57 / 63,
    // 4096 x 4096 35 / 48 / 48)
    a.tb = (int)balance_tokens(cfg, 512);
    a.nbg = (int)ceil_div(a.Tg, a.tb);
    a.scale = (double)d_loss * cfg->alpha * cfg->E / ((double)groups * cfg->k);
    ProfScope ps("balance_bwd", s);
    const dim3 grid((unsigned)(groups * a.nbg));
#define SW_BALANCE(G, NV)                                                                                          \
    if (cfg->E % 4 == 0) hipLaunchKernelGGL((balance_bwd_kernel<G, NV, true>), grid, dim3(kBalThreads), 0, s, a);  \
    else hipLaunchKernelGGL((balance_bwd_kernel<G, NV, false>), grid, dim3(kBalThreads), 0, s, a)
    SW_BALANCE_LANES(cfg->E, SW_BALANCE);
#undef SW_BALANCE
    return status_of(hipGetLastError());
}

}  // extern "C"

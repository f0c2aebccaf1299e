// switch_linear's products, shared by linear.hip (entry points, element-wise passes), linear_bf16.hip, linear_f32.hip and
// linear_few.hip (few rows).
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
    float *part;                   // k in several parts: their sums, [part][Qdim][columns: of W where gated]; otherwise nullptr
                                   // (or dx of dz in two terms: the sums of both)
    int act, gated;
    float scale;                   // of the sums
    Drop drop;
};

// k in equal parts (the last one shorter), each summed by itself.
struct LinearCut {
    int splits;
    int64_t split_k;
};
struct LinearPlan {
    int tile;                      // rows and columns; 0: the kernel for few rows
    LinearCut x, w;                // y or dx, dW
};
LinearPlan plan_linear(const switch_linear_config *cfg, bool backward);
bool linear_few_rows(const switch_linear_config *cfg);
LinearCut linear_few_cut(const switch_linear_config *cfg);

static inline int64_t linear_columns(const switch_linear_config *cfg) {   // of W
    return cfg->activation == SW_ACT_GEGLU ? 2 * cfg->N : cfg->N;
}

// either product of the backward pass may be left out
hipError_t launch_linear_bf16(const LinearPlan &plan, const LinearArgs &a, hipStream_t s);
hipError_t launch_linear_backward_bf16(const LinearPlan &plan, const LinearArgs *dx, const LinearArgs *dW, hipStream_t s);
hipError_t launch_linear_f32(const LinearPlan &plan, const LinearArgs &a, hipStream_t s);
hipError_t launch_linear_backward_f32(const LinearPlan &plan, const LinearArgs *dx, const LinearArgs *dW, hipStream_t s);
hipError_t launch_linear_few(int dtype, const LinearPlan &plan, const LinearArgs &a, hipStream_t s);

template <typename F> static inline hipError_t with_lds(PerDeviceOnce &once, F kernel, int bytes) {
    return once_per_device(once, [&] {
        return hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    });
}

// ---- tiles ------------------------------------------------------------------------------------
struct LinearTiles {
    int tiles_q, tiles_p;
    LinearCut cut;
};
static inline LinearTiles linear_tiles(const LinearArgs &a, int tile, const LinearCut &cut) {
    return LinearTiles{(int)ceil_div(a.Qdim, tile), (int)ceil_div(a.Pdim, a.gated ? tile / 2 : tile), cut};
}
// blocks of a product, whole rounds of XCDs
static inline int64_t linear_blocks(const LinearTiles &t) {
    return ceil_div((int64_t)t.tiles_q * t.tiles_p * t.cut.splits, 8) * 8;
}

// Blocks in two dimensions where one would hold 2^32 threads (whole rounds of XCDs each), and a block's number.
static inline dim3 linear_grid(int64_t blocks) {
    const int64_t most = kMaxGridThreads / 256 / 8 * 8, x = blocks < most ? blocks : most;
    return dim3((unsigned)x, (unsigned)ceil_div(blocks, x));
}
__device__ __forceinline__ int linear_block() { return (int)(blockIdx.y * gridDim.x + blockIdx.x); }

// Item of a block when the blocks of an XCD (b mod 8) take neighbouring ones; total or more for blocks without one.
__device__ __forceinline__ int linear_item(int b, int total) {
    const int per = (total + 7) >> 3;
    return b >> 3 < per ? (b & 7) * per + (b >> 3) : total;
}

// An item's place.  Items of a part of k are neighbours, in bands of eight row tiles, so that those that run on
// an XCD at a time, 32 in a row, share their operands in its L2.
struct LinearPlace {
    int64_t q0, k0;
    int p0, split, klim;
};
__device__ __forceinline__ LinearPlace linear_place(const LinearArgs &a, const LinearTiles &t, int n, int qb, int pb) {
    LinearPlace at;
    const int tiles = t.tiles_q * t.tiles_p;
    at.split = n / tiles;
    n -= at.split * tiles;
    constexpr int kBand = 8;
    const int band = n / (kBand * t.tiles_p), rows = min(kBand, t.tiles_q - band * kBand);
    n -= band * kBand * t.tiles_p;
    const int pt = n / rows;
    at.q0 = (int64_t)(band * kBand + (n - pt * rows)) * qb;
    at.p0 = pt * pb;
    at.k0 = at.split * t.cut.split_k;
    at.klim = (int)min(a.Kdim - at.k0, t.cut.split_k);
    return at;
}

// The operands' loads of a tile.  (Descriptors span 32 bits: W is below 2 GB; a tile's rows of x and dz, and a part's rows of
// both, begin at the base.)
template <LinearKind KIND, bool GATED, typename E, typename OP>
__device__ __forceinline__ void linear_init_p(OP &op, const LinearArgs &a, const LinearPlace &at, int lane, int wave) {
    const E *base = (const E *)a.P + (KIND == LINEAR_DX ? (size_t)at.k0 : (size_t)at.k0 * a.ldp);
    if constexpr (GATED) op.init_gated(base, a.ldp, at.p0, a.Pdim, at.klim, lane, wave);
    else op.init(base, a.ldp, at.p0, a.Pdim, at.klim, lane, wave);
}
template <LinearKind KIND, int QB, typename E, typename OQ>
__device__ __forceinline__ void linear_init_q(OQ &oq, const LinearArgs &a, const LinearPlace &at, int lane, int wave) {
    if constexpr (KIND == LINEAR_DW)
        oq.init((const E *)a.Q + (size_t)at.k0 * a.ldq, a.ldq, (int)at.q0, (int)a.Qdim, at.klim, lane, wave);
    else
        oq.init((const E *)a.Q + ((size_t)at.q0 * a.ldq + (size_t)at.k0), a.ldq, 0, (int)min(a.Qdim - at.q0, (int64_t)QB),
                at.klim, lane, wave);
}

// ---- epilogue -----------------------------------------------------------------------------------
// act of a value, or of a gate and a linear part
template <typename T> __device__ __forceinline__ float linear_act(int act, float u, float v) {
    switch (act) {
    case SW_ACT_RELU: return __builtin_elementwise_maximum(u, 0.f);   // (NaN stays NaN)
    case SW_ACT_GELU: return u * normal_at<T>(u).cdf;
    case SW_ACT_GEGLU: return u * normal_at<T>(u).cdf * v;
    default: return u;
    }
}

// What a lane has at hand for its columns p .. p + n - 1 of any row
template <typename T, int ACT> struct LinearColumns {
    static constexpr int n = Row16<T>::n;
    float bu[n], bv[n];
    __device__ __forceinline__ void load(const LinearArgs &a, int p) {
        if (!a.bias) return;
#pragma unroll
        for (int m = 0; m < n; m += 4) {
            *(float4 *)(bu + m) = *(const float4 *)(a.bias + p + m);
            if (ACT == SW_ACT_GEGLU) *(float4 *)(bv + m) = *(const float4 *)(a.bias + a.Pdim + p + m);
        }
    }
};

// Columns p .. p + n - 1 (of the gate part v and of the linear part) of row q: sums to outputs, in fp32 with a rounding
// of z and one of y.  residual: those n values, where there is one.
template <typename T, int ACT>
__device__ __forceinline__ void linear_emit(const LinearArgs &a, const LinearColumns<T, ACT> &col, int64_t q, int p,
                                            float *v, float *lin, const float *residual) {
    constexpr int n = Row16<T>::n;
    constexpr bool GATED = ACT == SW_ACT_GEGLU;
    const int64_t out = q * a.Pdim + p;
    if (a.bias) {
#pragma unroll
        for (int m = 0; m < n; ++m) {
            v[m] += col.bu[m];
            if (GATED) lin[m] += col.bv[m];
        }
    }
    if (a.z) {
        const int64_t zat = GATED ? out + q * a.Pdim : out;
        Row16<T>::store(a.z, zat, v);
        if (GATED) Row16<T>::store(a.z, zat + a.Pdim, lin);
    }
#pragma unroll
    for (int m = 0; m < n; ++m) v[m] = linear_act<T>(ACT, v[m], GATED ? lin[m] : 0.f);
    if (a.drop.on) {
        drop_apply<n>(a.drop, (uint64_t)out, v);
#pragma unroll
        for (int m = 0; m < n; ++m) v[m] *= a.drop.scale;
    }
    if (a.residual)
#pragma unroll
        for (int m = 0; m < n; ++m) v[m] += residual[m];
    Row16<T>::store(a.C, out, v);
}
// the same where nothing is at hand
template <typename T, int ACT>
__device__ __forceinline__ void linear_emit(const LinearArgs &a, int64_t q, int p, float *v, float *lin) {
    LinearColumns<T, ACT> col;
    col.load(a, p);
    float residual[Row16<T>::n];
    if (a.residual) Row16<T>::load(a.residual, q * a.Pdim + p, residual);
    linear_emit<T, ACT>(a, col, q, p, v, lin, residual);
}

// A part's sums of columns p .. p + n - 1
template <int n, bool GATED>
__device__ __forceinline__ void linear_store_part(const LinearArgs &a, int split, int64_t q, int p, const float *v,
                                                  const float *lin) {
    float *to = a.part + ((split * a.Qdim + q) * (GATED ? 2 * (int64_t)a.Pdim : a.Pdim) + p);
#pragma unroll
    for (int m = 0; m < n; m += 4) {
        *(float4 *)(to + m) = *(const float4 *)(v + m);
        if (GATED) *(float4 *)(to + a.Pdim + m) = *(const float4 *)(lin + m);
    }
}

}  // namespace sw

// switch_linear's products in fp32 on the matrix cores (MFMA 32x32x2).
//
// Tiles of 64 x 64 by four waves of 32 x 32; k advances 32 at a time through two LDS stages filled by direct loads, and four
// or five blocks share a CU and cover each other's waits.  Bound by the products: 1024 cycles a step, a quarter of
// that for the LDS.  Sums in two levels, chains of kChain products, so that their rounding grows with the square roots of
// the two lengths.
#include "linear.h"
#include "rows_operands.h"

namespace sw {

constexpr int kTile = 64, kStep = 32, kChain = 256;

// [k][row] operand of the gated activation: of each wave's 32 columns the first 16 are gate columns and the others the
// linear columns that belong to them.
struct F32GatedTrans : F32Trans<kTile, 4, 32> {
    __device__ __forceinline__ void init_gated(const float *base, int ld, int col0, int cols, int klim, int lane, int wave) {
        init(base, ld, 0, ld, klim, lane, wave);
        const int kk = lane / kChunks, r = ((lane % kChunks) ^ (turn(kk) >> 2)) * 4;
        const bool linear = r & 16;
        const int col = col0 + (r >> 5) * 16 + (r & 15);
        voff = col < cols ? ((uint32_t)(wave * kLoads * kRowsPerLoad + kk) * (uint32_t)ld + (uint32_t)(linear ? cols + col : col)) * 4u
                          : kOobOffset;
    }
};

template <LinearKind KIND, int ACT>
__device__ __forceinline__ void linear_f32_tile(const LinearArgs &a, const LinearTiles &t, char *lds, int n) {
    constexpr bool GATED = ACT == SW_ACT_GEGLU;
    constexpr int kOperand = kTile * kStep * 4, kStage = 2 * kOperand;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wp = wave % 2, wq = wave / 2;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const LinearPlace at = linear_place(a, t, n, kTile, GATED ? kTile / 2 : kTile);
    typename std::conditional<KIND == LINEAR_DX, F32Direct<kTile, 4>,
        typename std::conditional<GATED, F32GatedTrans, F32Trans<kTile, 4, 32>>::type>::type op;
    typename std::conditional<KIND == LINEAR_DW, F32Trans<kTile, 4, 32>, F32Direct<kTile, 4>>::type oq;
    op.init_frag(lane, wp * 32);
    oq.init_frag(lane, wq * 32);
    linear_init_p<KIND, GATED, float>(op, a, at, lane, wave);
    linear_init_q<KIND, kTile, float>(oq, a, at, lane, wave);
    constexpr int kLoadsP = decltype(op)::kLoads, kLoadsQ = decltype(oq)::kLoads;
    const int nk = (at.klim + kStep - 1) / kStep;
    f32x16 acc, total;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = total[r] = 0.f;
    auto issue = [&](int kt) {
        const uint32_t to = lds0 + (uint32_t)((kt & 1) * kStage);
#pragma unroll
        for (int i = 0; i < kLoadsP; ++i) op.issue_one(to, kt * kStep, wave, i);
#pragma unroll
        for (int i = 0; i < kLoadsQ; ++i) oq.issue_one(to + kOperand, kt * kStep, wave, i);
    };
    issue(0);
    for (int kt = 0; kt < nk; ++kt) {
        rows_wait_vmcnt<0>();
        __syncthreads();   // step kt has landed, step kt - 1 is read
        if (kt + 1 < nk) issue(kt + 1);
        if (kt != 0 && kt % (kChain / kStep) == 0) {
            total += acc;
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] = 0.f;
        }
        const char *sp = lds + (kt & 1) * kStage, *sq = sp + kOperand;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const f32x4 fp = op.frag4(sp, 0, ks), fq = oq.frag4(sq, 0, ks);
#pragma unroll
            for (int m = 0; m < 4; ++m) acc = mfma_f32(fp[m], fq[m], acc);
        }
    }
    total += acc;
    // a lane holds, for row lane % 32 of the wave's, columns 8 g + 4 (lane / 32) .. + 3; gated: the linear ones in g + 2
    const int64_t q = at.q0 + wq * 32 + lane % 32;
    if (q >= a.Qdim) return;
#pragma unroll
    for (int g = 0; g < (GATED ? 2 : 4); ++g) {
        const int p = at.p0 + wp * (GATED ? 16 : 32) + 8 * g + 4 * (lane / 32);
        if (p >= a.Pdim) continue;
        float v[4], lin[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            v[m] = total[4 * g + m];
            if (GATED) lin[m] = total[8 + (4 * g + m) % 8];
        }
        if (t.cut.splits > 1) {
            linear_store_part<4, GATED>(a, at.split, q, p, v, lin);
        } else if (KIND == LINEAR_FWD) {
            linear_emit<float, ACT>(a, q, p, v, lin);
        } else {
#pragma unroll
            for (int m = 0; m < 4; ++m) v[m] *= a.scale;
            Row16<float>::store(a.C, q * a.Pdim + p, v);
        }
    }
}

template <int ACT> __global__ __launch_bounds__(256, 4) void linear_fwd_f32_kernel(LinearArgs a, LinearTiles t) {
    __shared__ __attribute__((aligned(16))) char lds[4 * kTile * kStep * 4];
    const int total = t.tiles_q * t.tiles_p * t.cut.splits, n = linear_item(blockIdx.x, total);
    if (n < total) linear_f32_tile<LINEAR_FWD, ACT>(a, t, lds, n);
}

__global__ __launch_bounds__(256, 4) void linear_bwd_f32_kernel(LinearArgs dx, LinearTiles tx, LinearArgs dW, LinearTiles tw,
                                                                int dx_blocks) {
    __shared__ __attribute__((aligned(16))) char lds[4 * kTile * kStep * 4];
    if ((int)blockIdx.x < dx_blocks) {
        const int total = tx.tiles_q * tx.tiles_p * tx.cut.splits, n = linear_item(blockIdx.x, total);
        if (n < total) linear_f32_tile<LINEAR_DX, SW_ACT_NONE>(dx, tx, lds, n);
    } else {
        const int total = tw.tiles_q * tw.tiles_p * tw.cut.splits, n = linear_item(blockIdx.x - dx_blocks, total);
        if (n < total) linear_f32_tile<LINEAR_DW, SW_ACT_NONE>(dW, tw, lds, n);
    }
}

hipError_t launch_linear_f32(const LinearPlan &plan, const LinearArgs &a, hipStream_t s) {
    const LinearTiles t = linear_tiles(a, kTile, plan.x);
    const dim3 grid((unsigned)(ceil_div(linear_items(t), 8) * 8));
    auto kern = a.act == SW_ACT_RELU    ? linear_fwd_f32_kernel<SW_ACT_RELU>
                : a.act == SW_ACT_GELU  ? linear_fwd_f32_kernel<SW_ACT_GELU>
                : a.act == SW_ACT_GEGLU ? linear_fwd_f32_kernel<SW_ACT_GEGLU>
                                        : linear_fwd_f32_kernel<SW_ACT_NONE>;
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, a, t);
    return hipGetLastError();
}

hipError_t launch_linear_backward_f32(const LinearPlan &plan, const LinearArgs *dx, const LinearArgs *dW, hipStream_t s) {
    const LinearArgs none{};
    const LinearArgs &ax = dx ? *dx : none, &aw = dW ? *dW : none;
    const LinearTiles tx = linear_tiles(ax, kTile, plan.x), tw = linear_tiles(aw, kTile, plan.w);
    const int64_t bx = ceil_div(linear_items(tx), 8) * 8, bw = ceil_div(linear_items(tw), 8) * 8;
    hipLaunchKernelGGL(linear_bwd_f32_kernel, dim3((unsigned)(bx + bw)), dim3(256), 0, s, ax, tx, aw, tw, (int)bx);
    return hipGetLastError();
}

}  // namespace sw

// switch_linear's products in fp32 on the matrix cores (MFMA 32x32x2).
//
// Tiles of 64 x 64 by four waves of one MFMA tile; k advances 32 at a time through three LDS stages filled by direct loads, and
// up to three blocks share a CU.  Bound by the products: 1024 cycles a step, a quarter of that for the LDS.  (Tiles of
// 128 x 128, two waves' worth of MFMA tiles per wave side, measured the same: us of y, then of dx and dW, 64 / 128: 4096 x 4096 x
// 4096 1146, 2003 / 1166, 2125; 3001 x 1000 x 520 38, 65 / 47, 74.)  Sums in two levels, chains of kChain / 2 products, so that
// their rounding grows with the square roots of the two lengths.
#include "linear.h"
#include "rows_operands.h"

namespace sw {

constexpr int kTile = 64, kStep = 32, kChain = 256, kStages = 3;
constexpr int kOperand = kTile * kStep * 4, kStage = 2 * kOperand, kLds = kStages * kStage;

// An MFMA multiplies two k, one per half of the wave; which two is free as long as both operands agree: products m of
// quarter ks of a step take k = 8 ks + m and 8 ks + 4 + m, so that a lane's share of a [row][k] operand is 16 bytes in a row.
// [row][k] operand:
struct LinearF32Rows : F32Direct<kTile, 4> {
    __device__ __forceinline__ void init_frag(int lane, int frag_row) { RowsDirect<kTile, 4>::init_frag(lane, frag_row); }
    __device__ __forceinline__ f32x4 frag4(const char *st, int ks) const {
        return *(const f32x4 *)(st + (frag0 ^ (uint32_t)(ks << 5)));
    }
};
// [k][row] operand: LDS [32 k][64]; of k-rows 4 .. 7 of every eight the two halves trade places, so that the two
// k-rows of a read use different banks.  GATED: of each 32 columns the first 16 are gate columns and the others the
// linear columns that belong to them.
template <bool GATED> struct LinearF32Cols {
    static constexpr int kLoads = 2, kRowsPerLoad = 4;   // of a wave: k-rows 8 wave + 4 i + ..
    i32x4 rsrc;
    uint32_t voff[kLoads], k_step, frag0;
    __device__ __forceinline__ void init(const float *base, int ld, int col0, int cols, int klim, int lane, int wave) {
        rsrc = make_rsrc(base, (uint32_t)klim * (uint32_t)ld * 4u);
        k_step = (uint32_t)ld * 4u;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = (lane % 16 * 4) ^ (i << 5);
            const int col = GATED ? col0 + (r >> 5) * 16 + (r & 15) : col0 + r;
            voff[i] = col < cols ? ((uint32_t)(wave * 8 + lane / 16) * (uint32_t)ld +
                                    (uint32_t)(GATED && (r & 16) ? cols + col : col)) * 4u
                                 : kOobOffset;
        }
    }
    __device__ __forceinline__ void init_frag(int lane, int frag_row) {
        const int h = lane >> 5;
        frag0 = (uint32_t)((4 * h * kTile + ((frag_row + lane % 32) ^ (h << 5))) * 4);
    }
    __device__ __forceinline__ void issue_one(uint32_t st, int k0, int wave, int i) const {
        dma16(rsrc, voff[i], (uint32_t)(k0 + i * kRowsPerLoad) * k_step,
              st + (uint32_t)((wave * kLoads + i) * 1024));
    }
    __device__ __forceinline__ f32x4 frag4(const char *st, int ks) const {
        const char *p = st + frag0 + ks * (8 * kTile * 4);
        return f32x4{*(const float *)p, *(const float *)(p + kTile * 4), *(const float *)(p + 2 * kTile * 4),
                     *(const float *)(p + 3 * kTile * 4)};
    }
};

template <LinearKind KIND, int ACT>
__device__ __forceinline__ void linear_f32_tile(const LinearArgs &a, const LinearTiles &t, char *lds, int n) {
    constexpr bool GATED = ACT == SW_ACT_GEGLU;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wp = wave % 2, wq = wave / 2;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const LinearPlace at = linear_place(a, t, n, kTile, GATED ? kTile / 2 : kTile);
    typename std::conditional<KIND == LINEAR_DX, LinearF32Rows, LinearF32Cols<GATED>>::type op;
    typename std::conditional<KIND == LINEAR_DW, LinearF32Cols<false>, LinearF32Rows>::type oq;
    op.init_frag(lane, wp * 32);
    oq.init_frag(lane, wq * 32);
    linear_init_p<KIND, false, float>(op, a, at, lane, wave);
    linear_init_q<KIND, kTile, float>(oq, a, at, lane, wave);
    constexpr int kLoads = decltype(op)::kLoads + decltype(oq)::kLoads;
    const int nk = (at.klim + kStep - 1) / kStep;
    // two chains: a product would wait for the one before it (4096 x 4096 x 4096, us of y: one chain 1273, two 1146)
    f32x16 acc[2], total;
    auto clear = [&] {
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[0][r] = acc[1][r] = 0.f;
    };
    clear();
#pragma unroll
    for (int r = 0; r < 16; ++r) total[r] = 0.f;
    auto issue = [&](int kt, uint32_t to) {   // (past the end: never read)
#pragma unroll
        for (int i = 0; i < decltype(op)::kLoads; ++i) op.issue_one(lds0 + to, kt * kStep, wave, i);
#pragma unroll
        for (int i = 0; i < decltype(oq)::kLoads; ++i) oq.issue_one(lds0 + to + kOperand, kt * kStep, wave, i);
    };
    f32x4 fp[2], fq[2];
    auto read = [&](uint32_t from, int ks) {
        fp[ks & 1] = op.frag4(lds + from, ks);
        fq[ks & 1] = oq.frag4(lds + from + kOperand, ks);
    };
#pragma unroll
    for (int s = 0; s < kStages; ++s) issue(s, s * kStage);
    rows_wait_vmcnt<(kStages - 1) * kLoads>();
    __syncthreads();
    read(0, 0);
    uint32_t st = 0;
    for (int kt = 0; kt < nk; ++kt) {
        const uint32_t st1 = st == (kStages - 1) * kStage ? 0 : st + kStage;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            // the next fragments, one quarter of a step ahead; before the last quarter the step is read and its stage is
            // filled again
            if (ks == 3) {
                rows_wait_vmcnt<(kStages - 2) * kLoads>();   // step kt + 1 has landed
                asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
                __syncthreads();
                issue(kt + kStages, st);
            }
            read(ks == 3 ? st1 : st, (ks + 1) & 3);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int m = 0; m < 4; ++m)
                acc[m & 1] = __builtin_amdgcn_mfma_f32_32x32x2f32(fp[ks & 1][m], fq[ks & 1][m], acc[m & 1], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (kt % (kChain / kStep) == kChain / kStep - 1) {
            total += acc[0] + acc[1];
            clear();
        }
        st = st1;
    }
    rows_wait_vmcnt<0>();   // the trailing loads
    total += acc[0] + acc[1];
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
        if (a.part) {
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

template <int ACT> __global__ __launch_bounds__(256, 3) void linear_fwd_f32_kernel(LinearArgs a, LinearTiles t) {
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    const int total = t.tiles_q * t.tiles_p * t.cut.splits, n = linear_item(linear_block(), total);
    if (n < total) linear_f32_tile<LINEAR_FWD, ACT>(a, t, lds, n);
}

__global__ __launch_bounds__(256, 3) void linear_bwd_f32_kernel(LinearArgs dx, LinearTiles tx, LinearArgs dW, LinearTiles tw,
                                                                int dx_blocks) {
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    if (linear_block() < dx_blocks) {
        const int total = tx.tiles_q * tx.tiles_p * tx.cut.splits, n = linear_item(linear_block(), total);
        if (n < total) linear_f32_tile<LINEAR_DX, SW_ACT_NONE>(dx, tx, lds, n);
    } else {
        const int total = tw.tiles_q * tw.tiles_p * tw.cut.splits, n = linear_item(linear_block() - dx_blocks, total);
        if (n < total) linear_f32_tile<LINEAR_DW, SW_ACT_NONE>(dW, tw, lds, n);
    }
}

hipError_t launch_linear_f32(const LinearPlan &plan, const LinearArgs &a, hipStream_t s) {
    const LinearTiles t = linear_tiles(a, kTile, plan.x);
    const dim3 grid = linear_grid(linear_blocks(t));
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
    const int64_t bx = linear_blocks(tx), bw = linear_blocks(tw);
    hipLaunchKernelGGL(linear_bwd_f32_kernel, linear_grid(bx + bw), dim3(256), 0, s, ax, tx, aw, tw, (int)bx);
    return hipGetLastError();
}

}  // namespace sw

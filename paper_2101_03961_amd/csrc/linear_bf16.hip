// switch_linear's products on bf16 MFMA 16x16x32, fp32 accumulation (P is the MFMA "A" side).  One tile per block, k 64 at a
// time through LDS stages filled by direct loads.
//
// Large tiles, 256 x 256 in four waves, one block per CU, for products that fill the chip with them: bound by the matrix cores
// under their own power (8192 x 8192 x 8192: 1320 - 1450 TFLOP/s; 8192 x 8192 x 4096 of zeros, which draw less,
// 1600 - 1780), and by a tile's start and end, 10 us beside 1.45 us a step: at its end all CUs store at once.  (Persistent
// blocks of eight waves with the next tile's loads under way during the epilogue: 65536 x 2048 x 768 205 us, the plain
// eight-wave kernel 202.  Tiles of 256 x 128, two blocks per CU, whose starts and ends the other block covers, with 32 k a
// step to fit the LDS: 1.9 us for the products that take 1.45.)  Small tiles, 128 x 128, two blocks per CU, where the large
// ones leave CUs idle.  linear.hip chooses.
#include "linear.h"
#include "rows_operands.h"

namespace sw {

constexpr int BK = 64;   // k per step

// [k][row] operand of the gated activation: tile columns come in groups of 32 IP per wave, half of them gate
// columns and half the linear columns that belong to them.
template <int IP, int WP, int NW> struct GatedTrans : RowsTrans<32 * IP * WP, NW> {
    typedef RowsTrans<32 * IP * WP, NW> Base;
    __device__ __forceinline__ void init_gated(const bf16 *base, int ld, int col0, int cols, int klim, int lane, int wave) {
        constexpr int R = 32 * IP * WP;
        Base::init(base, ld, 0, ld, klim, lane, wave);
#pragma unroll
        for (int i = 0; i < Base::kPeriod; ++i) {
            const int at = (R == 256 ? 0 : wave * Base::kGroup + i) * 64 + lane;
            const int kr = at / Base::kChunks + (R == 256 ? Base::first_row(wave, 0) : 0);
            const int r = (at % Base::kChunks ^ Base::perm(kr)) << 3;
            const int w = r / (32 * IP), in = r % (32 * IP);
            const bool linear = in >= 16 * IP;
            const int col = col0 + w * (16 * IP) + (linear ? in - 16 * IP : in);
            this->voff[i] = col < cols ? ((uint32_t)kr * (uint32_t)ld + (uint32_t)(linear ? cols + col : col)) * 2u
                                       : kOobOffset;
        }
    }
};

// Epilogue of a wave: 16 rows at a time through 2 KB IP of LDS of its own, as fp32, so that a lane has eight consecutive
// columns (of the gate and the linear part) and rows leave in whole segments.  The 16-byte chunks of a row trade places by
// the row, so that neither side has bank conflicts.
template <int IP, int IQ, LinearKind KIND, int ACT>
__device__ __forceinline__ void linear_epilogue(const LinearArgs &a, const LinearPlace &at,
                                                const f32x4 (&acc)[2 * IP][2 * IQ], char *turn, int lane, int wp, int wq) {
    static_assert(IP % 2 == 0, "whole groups of 16 chunks of a row");
    constexpr bool GATED = ACT == SW_ACT_GEGLU;
    constexpr int kPitch = 32 * IP * 4, kCols = GATED ? 16 * IP : 32 * IP, kChunks = kCols / 8;
    constexpr int kPasses = 16 * kChunks / 64, kPassRows = 64 / kChunks;
    const int r0 = lane / kChunks, c = lane % kChunks;   // the lane's row, those kPassRows further, and its chunk
    const int p = at.p0 + wp * kCols + c * 8;
    if (at.p0 + wp * kCols >= a.Pdim) return;
    const int rows = (int)min(a.Qdim - at.q0, (int64_t)0x7fffffff) - wq * IQ * 32;   // of the wave
    const int64_t q0 = at.q0 + wq * IQ * 32;
    const bool in = p < a.Pdim;
    LinearColumns<bf16, ACT> col;
    if (KIND == LINEAR_FWD && in) col.load(a, p);
    // the residual's rows, kAhead rounds before they are added (the fragments' registers are free by now)
    constexpr int kAhead = 4;
    bf16x8 res[2 * IQ][kPasses];
    auto load_residual = [&](int j) {
#pragma unroll
        for (int x = 0; x < kPasses; ++x) {
            const int row = j * 16 + x * kPassRows + r0;
            if (row < rows && in) res[j][x] = *(const bf16x8 *)((const bf16 *)a.residual + (q0 + row) * a.Pdim + p);
        }
    };
    if (KIND == LINEAR_FWD && a.residual)
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (j < 2 * IQ) load_residual(j);
#pragma unroll
    for (int j = 0; j < 2 * IQ; ++j) {
        if (j * 16 >= rows) break;
        if (KIND == LINEAR_FWD && a.residual && j + kAhead < 2 * IQ) load_residual(j + kAhead);
#pragma unroll
        for (int i = 0; i < 2 * IP; ++i)
            *(f32x4 *)(turn + (lane & 15) * kPitch + (((i * 4 + (lane >> 4)) ^ (lane & 15)) << 4)) = acc[i][j];
#pragma unroll
        for (int x = 0; x < kPasses; ++x) {
            const int r = x * kPassRows + r0, row = j * 16 + r;
            auto chunk = [&](int n) { return *(const f32x4 *)(turn + r * kPitch + ((n ^ r) << 4)); };
            float v[8], lin[8];
            *(f32x4 *)v = chunk(2 * c);
            *(f32x4 *)(v + 4) = chunk(2 * c + 1);
            if (GATED) {
                *(f32x4 *)lin = chunk(2 * c + kCols / 4);
                *(f32x4 *)(lin + 4) = chunk(2 * c + 1 + kCols / 4);
            }
            if (row >= rows || !in) continue;
            const int64_t q = q0 + row;
            if (a.part) {
                linear_store_part<8, GATED>(a, at.split, q, p, v, lin);
            } else if (KIND == LINEAR_FWD) {
                float r8[8];
                if (a.residual)
#pragma unroll
                    for (int m = 0; m < 8; ++m) r8[m] = (float)res[j][x][m];
                linear_emit<bf16, ACT>(a, col, q, p, v, lin, r8);
            } else {
#pragma unroll
                for (int m = 0; m < 8; ++m) v[m] *= a.scale;
                Eight<bf16>::store((bf16 *)a.C + q * a.Pdim + p, v);
            }
        }
    }
}

template <int IP, int WP, int IQ, int WQ, LinearKind KIND, bool GATED> struct LinearOps {
    static constexpr int NW = WP * WQ, PB = 32 * IP * WP, QB = 32 * IQ * WQ, OUTP = GATED ? PB / 2 : PB;
    typedef typename std::conditional<KIND == LINEAR_DX, RowsDirect<PB, NW>,
        typename std::conditional<GATED, GatedTrans<IP, WP, NW>, RowsTrans<PB, NW>>::type>::type P;
    typedef typename std::conditional<KIND == LINEAR_DW, RowsTrans<QB, NW>, RowsDirect<QB, NW>>::type Q;
    static constexpr int kPBytes = PB * BK * 2, kStage = (PB + QB) * BK * 2;
    static constexpr int kTurn = 16 * 32 * IP * 4;   // bytes per wave
};

// Four products into four accumulators, which stay where they are: the compiler's own copies some of 64 around between the
// registers of either kind.  With a direct load (see dma16) behind them, whose m0 is set before them: the products are the
// wait states between that, or a descriptor reloaded from a spill lane, and the load.
__device__ __forceinline__ void products4(f32x4 &c0, f32x4 &c1, f32x4 &c2, f32x4 &c3, bf16x8 p0, bf16x8 p1, bf16x8 p2, bf16x8 p3,
                                          bf16x8 q) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %4, %8, %0\n\t"
                 "v_mfma_f32_16x16x32_bf16 %1, %5, %8, %1\n\t"
                 "v_mfma_f32_16x16x32_bf16 %2, %6, %8, %2\n\t"
                 "v_mfma_f32_16x16x32_bf16 %3, %7, %8, %3"
                 : "+a"(c0), "+a"(c1), "+a"(c2), "+a"(c3)
                 : "v"(p0), "v"(p1), "v"(p2), "v"(p3), "v"(q));
}
__device__ __forceinline__ void products4_load(f32x4 &c0, f32x4 &c1, f32x4 &c2, f32x4 &c3, bf16x8 p0, bf16x8 p1, bf16x8 p2,
                                               bf16x8 p3, bf16x8 q, i32x4 rsrc, uint32_t voff, uint32_t soff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %12\n\t"
                 "v_mfma_f32_16x16x32_bf16 %0, %4, %8, %0\n\t"
                 "v_mfma_f32_16x16x32_bf16 %1, %5, %8, %1\n\t"
                 "v_mfma_f32_16x16x32_bf16 %2, %6, %8, %2\n\t"
                 "v_mfma_f32_16x16x32_bf16 %3, %7, %8, %3\n\t"
                 "buffer_load_dwordx4 %9, %10, %11 offen lds"
                 : "+a"(c0), "+a"(c1), "+a"(c2), "+a"(c3)
                 : "v"(p0), "v"(p1), "v"(p2), "v"(p3), "v"(q), "v"(voff), "s"(rsrc), "s"(soff), "s"(lds)
                 : "memory");
}

// One large tile: four waves of 128 x 128, one per SIMD, whose fragments take a third less LDS traffic than those of eight
// waves of 64 x 128 (1536 cycles of reads and fills per step, the products take 2048).  P goes through three stages of 32 KB, Q
// through two.  In the middle of step kt a barrier ends the reads of its stages; Q's is filled with step kt + 2 in the second
// half of the step, P's with step kt + 3 in the first half of the next one: a load and two reads per eight products throughout
// (all 16 loads in the second half: dx of 8192 x 8192 x 4096 380 us, 374 so; of zeros 313 and 301).  The fragments of a half
// step are read during the products of the half step before.
template <LinearKind KIND, int ACT>
__device__ __forceinline__ void linear_large(const LinearArgs &a, const LinearTiles &t, char *lds, int n) {
    constexpr int IP = 4, WP = 2, IQ = 4, WQ = 2;
    constexpr bool GATED = ACT == SW_ACT_GEGLU;
    typedef LinearOps<IP, WP, IQ, WQ, KIND, GATED> S;
    constexpr int kStageP = S::PB * BK * 2, kStageQ = S::QB * BK * 2;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wp = wave % WP, wq = wave / WP;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const LinearPlace at = linear_place(a, t, n, S::QB, S::OUTP);
    typename S::P op;
    typename S::Q oq;
    constexpr int kLoadsP = S::P::kLoads, kLoadsQ = S::Q::kLoads;
    static_assert(kLoadsP == 8 && kLoadsQ == 8, "a load per two groups of products");
    op.init_frag16(lane, wp * 32 * IP);
    oq.init_frag16(lane, wq * 32 * IQ);
    linear_init_p<KIND, GATED, bf16>(op, a, at, lane, wave);
    linear_init_q<KIND, S::QB, bf16>(oq, a, at, lane, wave);
    f32x4 acc[2 * IP][2 * IQ];
#pragma unroll
    for (int i = 0; i < 2 * IP; ++i)
#pragma unroll
        for (int j = 0; j < 2 * IQ; ++j) {
            acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            asm volatile("" : "+a"(acc[i][j]));
        }
    asm volatile("s_nop 3");   // written before the first product reads them
    const int nk = (at.klim + BK - 1) / BK;
    auto issue_p = [&](uint32_t st, int kt, int i) { op.issue_one(lds0 + st, kt * BK, wave, i); };
    auto issue_q = [&](uint32_t st, int kt, int i) { oq.issue_one(lds0 + 3 * kStageP + st, kt * BK, wave, i); };
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int i = 0; i < kLoadsP; ++i) issue_p(s * kStageP, s, i);
#pragma unroll
        for (int i = 0; i < kLoadsQ; ++i) issue_q(s * kStageQ, s, i);
    }
    rows_wait_vmcnt<kLoadsP + kLoadsQ>();
    __syncthreads();
    bf16x8 fp[2][2 * IP], fq[2][2 * IQ];
    // fragment f of a half step, in the order of use
    auto read = [&](const char *sp, const char *sq, int ks, int f) {
        if (f == 0) fq[ks][0] = oq.frag16(sq, 0, ks);
        else if (f <= 2 * IP) fp[ks][f - 1] = op.frag16(sp, f - 1, ks);
        else fq[ks][f - 2 * IP] = oq.frag16(sq, f - 2 * IP, ks);
    };
    constexpr int kGroups = 2 * IP + 2 * IQ;   // fragments, and groups of four products, of a half step
    static_assert(kGroups == 16 && 4 * IP * IQ == 4 * kGroups, "four products per fragment");
#pragma unroll
    for (int f = 0; f < kGroups; ++f) read(lds, lds + 3 * kStageP, 0, f);
    uint32_t sp = 0, sq = 0;   // stages of step kt
#pragma nounroll
    for (int kt = 0; kt < nk; ++kt) {
        const uint32_t sp1 = sp == 2 * kStageP ? 0 : sp + kStageP, sp2 = sp1 == 2 * kStageP ? 0 : sp1 + kStageP;
        const uint32_t sq1 = sq ^ kStageQ;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            op.reload_frag();
            oq.reload_frag();
            if (ks == 1) {
                rows_wait_vmcnt<kLoadsP>();   // step kt + 1 has landed
                asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
                __syncthreads();              // ... for all waves, and both stages of step kt are read
            }
            const char *rp = lds + (ks == 0 ? sp : sp1), *rq = lds + 3 * kStageP + (ks == 0 ? sq : sq1);
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                // one read per group; in the first half the last five groups cover the reads' latency before the barrier
#pragma unroll
                for (int f = 0; f < kGroups; ++f)
                    if ((ks == 1 ? f : f * 11 / kGroups) == g) read(rp, rq, ks ^ 1, f);
                __builtin_amdgcn_sched_barrier(0);
                const int i = g % 2 * 4, j = g / 2;
                if (g % 2 == 0) {
                    products4(acc[i][j], acc[i + 1][j], acc[i + 2][j], acc[i + 3][j], fp[ks][i], fp[ks][i + 1], fp[ks][i + 2],
                              fp[ks][i + 3], fq[ks][j]);
                } else {
                    i32x4 rsrc;
                    uint32_t voff, soff, at_lds;
                    if (ks == 0) {
                        op.load_of((kt + 2) * BK, wave, g / 2, rsrc, voff, soff, at_lds);
                        at_lds += lds0 + sp2;
                    } else {
                        oq.load_of((kt + 2) * BK, wave, g / 2, rsrc, voff, soff, at_lds);
                        at_lds += lds0 + 3 * kStageP + sq;
                    }
                    products4_load(acc[i][j], acc[i + 1][j], acc[i + 2][j], acc[i + 3][j], fp[ks][i], fp[ks][i + 1],
                                   fp[ks][i + 2], fp[ks][i + 3], fq[ks][j], rsrc, voff, soff, at_lds);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        sp = sp1;
        sq = sq1;
    }
    rows_wait_vmcnt<0>();   // the trailing loads
    asm volatile("s_nop 15\n\ts_nop 15");   // the last products (the compiler does not know them as such)
#pragma unroll
    for (int i = 0; i < 2 * IP; ++i)
#pragma unroll
        for (int j = 0; j < 2 * IQ; ++j) asm volatile("" : "+a"(acc[i][j]));
    __syncthreads();
    linear_epilogue<IP, IQ, KIND, ACT>(a, at, acc, lds + wave * S::kTurn, lane, wp, wq);
}

template <int ACT>
__global__ __launch_bounds__(256, 1) void linear_fwd_large_kernel(LinearArgs a, LinearTiles t) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int total = t.tiles_q * t.tiles_p * t.cut.splits, n = linear_item(linear_block(), total);
    if (n < total) linear_large<LINEAR_FWD, ACT>(a, t, lds, n);
}

__global__ __launch_bounds__(256, 1) void linear_bwd_large_kernel(LinearArgs dx, LinearTiles tx, LinearArgs dW, LinearTiles tw,
                                                                  int dx_blocks) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    if (linear_block() < dx_blocks) {
        const int total = tx.tiles_q * tx.tiles_p * tx.cut.splits, n = linear_item(linear_block(), total);
        if (n < total) linear_large<LINEAR_DX, SW_ACT_NONE>(dx, tx, lds, n);
    } else {
        const int total = tw.tiles_q * tw.tiles_p * tw.cut.splits, n = linear_item(linear_block() - dx_blocks, total);
        if (n < total) linear_large<LINEAR_DW, SW_ACT_NONE>(dW, tw, lds, n);
    }
}

// One small tile: four waves of 64 x 64, two stages.
template <LinearKind KIND, int ACT>
__device__ __forceinline__ void linear_small(const LinearArgs &a, const LinearTiles &t, char *lds, int n) {
    constexpr int IP = 2, WP = 2, IQ = 2, WQ = 2;
    constexpr bool GATED = ACT == SW_ACT_GEGLU;
    typedef LinearOps<IP, WP, IQ, WQ, KIND, GATED> S;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wp = wave % WP, wq = wave / WP;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const LinearPlace at = linear_place(a, t, n, S::QB, S::OUTP);
    typename S::P op;
    typename S::Q oq;
    op.init_frag16(lane, wp * 32 * IP);
    oq.init_frag16(lane, wq * 32 * IQ);
    linear_init_p<KIND, GATED, bf16>(op, a, at, lane, wave);
    linear_init_q<KIND, S::QB, bf16>(oq, a, at, lane, wave);
    f32x4 acc[2 * IP][2 * IQ];
#pragma unroll
    for (int i = 0; i < 2 * IP; ++i)
#pragma unroll
        for (int j = 0; j < 2 * IQ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto issue = [&](int kt) {
        const uint32_t to = lds0 + (uint32_t)((kt & 1) * S::kStage);
#pragma unroll
        for (int i = 0; i < S::P::kLoads; ++i) op.issue_one(to, kt * BK, wave, i);
#pragma unroll
        for (int i = 0; i < S::Q::kLoads; ++i) oq.issue_one(to + S::kPBytes, kt * BK, wave, i);
    };
    const int nk = (at.klim + BK - 1) / BK;
    issue(0);
    for (int kt = 0; kt < nk; ++kt) {
        rows_wait_vmcnt<0>();   // step kt has landed
        __syncthreads();        // ... for all waves; step kt - 1 is read
        if (kt + 1 < nk) issue(kt + 1);
        const char *sp = lds + (kt & 1) * S::kStage, *sq = sp + S::kPBytes;
#pragma unroll
        for (int ks = 0; ks < BK / 32; ++ks) {
            bf16x8 fp[2 * IP], fq[2 * IQ];
#pragma unroll
            for (int i = 0; i < 2 * IP; ++i) fp[i] = op.frag16(sp, i, ks);
#pragma unroll
            for (int j = 0; j < 2 * IQ; ++j) fq[j] = oq.frag16(sq, j, ks);
#pragma unroll
            for (int j = 0; j < 2 * IQ; ++j)
#pragma unroll
                for (int i = 0; i < 2 * IP; ++i)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp[i], fq[j], acc[i][j], 0, 0, 0);
        }
    }
    __syncthreads();
    linear_epilogue<IP, IQ, KIND, ACT>(a, at, acc, lds + wave * S::kTurn, lane, wp, wq);
}

template <int ACT>
__global__ __launch_bounds__(256, 2) void linear_fwd_small_kernel(LinearArgs a, LinearTiles t) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int total = t.tiles_q * t.tiles_p * t.cut.splits, n = linear_item(linear_block(), total);
    if (n < total) linear_small<LINEAR_FWD, ACT>(a, t, lds, n);
}

__global__ __launch_bounds__(256, 2) void linear_bwd_small_kernel(LinearArgs dx, LinearTiles tx, LinearArgs dW, LinearTiles tw,
                                                                  int dx_blocks) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    if (linear_block() < dx_blocks) {
        const int total = tx.tiles_q * tx.tiles_p * tx.cut.splits, n = linear_item(linear_block(), total);
        if (n < total) linear_small<LINEAR_DX, SW_ACT_NONE>(dx, tx, lds, n);
    } else {
        const int total = tw.tiles_q * tw.tiles_p * tw.cut.splits, n = linear_item(linear_block() - dx_blocks, total);
        if (n < total) linear_small<LINEAR_DW, SW_ACT_NONE>(dW, tw, lds, n);
    }
}

// ---- host side ------------------------------------------------------------------------------
constexpr int kLargeTile = 256, kSmallTile = 128;
constexpr int kLargeLds = 5 * kLargeTile * BK * 2, kSmallLds = 2 * 2 * kSmallTile * BK * 2;
static_assert(kLargeLds == 160 * 1024, "all of a CU's");

template <int ACT> static hipError_t linear_fwd_bf16(const LinearPlan &plan, const LinearArgs &a, hipStream_t s) {
    const bool large = plan.tile == kLargeTile;
    const LinearTiles t = linear_tiles(a, plan.tile, plan.x);
    auto kern = large ? linear_fwd_large_kernel<ACT> : linear_fwd_small_kernel<ACT>;
    static PerDeviceOnce once[2];
    const int lds = large ? kLargeLds : kSmallLds;
    const hipError_t err = with_lds(once[large], kern, lds);
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(kern, linear_grid(linear_blocks(t)), dim3(256), lds, s, a, t);
    return hipGetLastError();
}

hipError_t launch_linear_bf16(const LinearPlan &plan, const LinearArgs &a, hipStream_t s) {
    switch (a.act) {
    case SW_ACT_RELU: return linear_fwd_bf16<SW_ACT_RELU>(plan, a, s);
    case SW_ACT_GELU: return linear_fwd_bf16<SW_ACT_GELU>(plan, a, s);
    case SW_ACT_GEGLU: return linear_fwd_bf16<SW_ACT_GEGLU>(plan, a, s);
    default: return linear_fwd_bf16<SW_ACT_NONE>(plan, a, s);
    }
}

hipError_t launch_linear_backward_bf16(const LinearPlan &plan, const LinearArgs *dx, const LinearArgs *dW, hipStream_t s) {
    const bool large = plan.tile == kLargeTile;
    const LinearArgs none{};
    const LinearArgs &ax = dx ? *dx : none, &aw = dW ? *dW : none;
    const LinearTiles tx = linear_tiles(ax, plan.tile, plan.x), tw = linear_tiles(aw, plan.tile, plan.w);
    const int64_t bx = linear_blocks(tx), bw = linear_blocks(tw);
    auto kern = large ? linear_bwd_large_kernel : linear_bwd_small_kernel;
    static PerDeviceOnce once[2];
    const int lds = large ? kLargeLds : kSmallLds;
    const hipError_t err = with_lds(once[large], kern, lds);
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(kern, linear_grid(bx + bw), dim3(256), lds, s, ax, tx, aw, tw, (int)bx);
    return hipGetLastError();
}

}  // namespace sw

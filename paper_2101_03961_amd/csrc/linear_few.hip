// switch_linear's forward product for few rows (a decoding step): bound by the one pass over W.
//
// W goes from memory to the registers, 16 bytes per lane, and is used by up to four MFMA row blocks of 16 rows of x.  A
// wave takes chunks of k rows of W (32 of bf16, 16 of fp32) by 16 x 16 bytes of columns: lane 16 g + c holds, of the
// rows that are lane group g's share of the MFMA's k, chunk c of columns.  Column j of chunk c is index c of MFMA j, so
// no element changes lanes; bf16 pairs of k come from two registers by a byte permutation.
//
// The eight waves of a block take eight neighbouring chunks a round; the 512 bytes of each row of x that belong to them go
// to LDS by direct loads (read by every wave for itself, 64 bytes of each row, x took as long as W: its rows are a multiple of
// 4 KB apart and lie in one L2 channel; 64 rows, 4096 x 20480: 49 us, 43 so).  Loads run two rounds ahead.  At the end the waves
// add up their sums through LDS, in order; several parts of k (few columns) are added up by linear_finish_kernel.
#include "linear.h"
#include "rows_operands.h"

namespace sw {

constexpr int kFewRows = 64, kFewWaves = 8;

template <typename T> struct FewChunk;   // a lane's share of a chunk: W rows of 16 bytes, MFMA operands
template <> struct FewChunk<bf16> {
    static constexpr int kRows = 32, kLoads = 8;   // k rows, W loads per lane
    u32x4 w[kLoads];
    // k rows 8 g + i of chunk k
    __device__ __forceinline__ static int row(int g, int i) { return 8 * g + i; }
    template <int MT> __device__ __forceinline__ void products(f32x4 (&acc)[8][MT], const u32x4 (&x)[MT]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u32x4 f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                f[i] = __builtin_amdgcn_perm(w[2 * i + 1][j / 2], w[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int m = 0; m < MT; ++m)
                acc[j][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f),
                                                                     __builtin_bit_cast(bf16x8, x[m]), acc[j][m], 0, 0, 0);
        }
    }
};
template <> struct FewChunk<float> {
    static constexpr int kRows = 16, kLoads = 4;
    u32x4 w[kLoads];
    __device__ __forceinline__ static int row(int g, int i) { return 4 * g + i; }
    // (an MFMA takes one k of each lane group: 4 g + i of all g)
    template <int MT> __device__ __forceinline__ void products(f32x4 (&acc)[4][MT], const u32x4 (&x)[MT]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    acc[j][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i][j]), __uint_as_float(x[m][i]),
                                                                      acc[j][m], 0, 0, 0);
    }
};

constexpr int few_lds(int mt, int cols) {   // three stages of x, then the waves' sums
    const int x = 3 * 16 * mt * 512, sums = kFewWaves * 16 * (cols + 4) * 4;
    return x > sums ? x : sums;
}

// STREAM: W is not kept in the caches (it is much more than they hold).
template <typename T, int MT, int ACT, bool STREAM>
__global__ __launch_bounds__(64 * kFewWaves, 2) void linear_few_kernel(LinearArgs a, LinearCut cut) {
    typedef FewChunk<T> Chunk;
    constexpr bool GATED = ACT == SW_ACT_GEGLU;
    constexpr int n = Row16<T>::n, kCols = 16 * n, kPitch = kCols + 4;   // columns of a block; LDS row, in floats
    constexpr int kRound = kFewWaves * Chunk::kRows, kStage = 16 * MT * 512;
    static_assert(kRound * sizeof(T) == 512, "bytes of a row of x per round");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const int p0 = blockIdx.x * (GATED ? kCols / 2 : kCols);
    const int split = blockIdx.y;
    const int k0 = (int)(split * cut.split_k), kend = (int)min(a.Kdim, k0 + cut.split_k), K = (int)a.Kdim;
    // the lane's columns of W; rows past the last one lie past the descriptor
    const int col = GATED ? p0 + (c & 7) * n : p0 + c * n;
    const auto wsrc = __builtin_amdgcn_make_buffer_rsrc((void *)a.P, 0, (int)((uint32_t)K * (uint32_t)a.ldp * sizeof(T)),
                                                        0x00020000);
    const i32x4 xsrc = make_rsrc(a.Q, (uint32_t)a.Qdim * (uint32_t)K * sizeof(T));
    const uint32_t wcol = col < a.Pdim ? (uint32_t)(GATED && c >= 8 ? a.Pdim + col : col) * sizeof(T) : kOobOffset;
    // x: load i of the wave is rows 2 (8 i + wave) + lane / 32, 512 bytes each; the 16-byte chunks of a row trade places by the
    // row, so that 16 rows' same chunk lies in 16 places of the banks
    int xk[MT];             // first k (of a round) that the lane fetches; past K where the row does not exist
    uint32_t xoff[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int row = 2 * (8 * i + wave) + (lane >> 5);
        xk[i] = ((lane & 31) ^ (row & 15)) * n;
        xoff[i] = (uint32_t)row * (uint32_t)K * sizeof(T) + (uint32_t)xk[i] * sizeof(T);
        if (row >= a.Qdim) xk[i] = 1 << 28;
    }
    Chunk w[2];
    auto load = [&](int r, Chunk &ch) {   // round r
        const int k = k0 + r * kRound + wave * Chunk::kRows;
        const uint32_t first = k < kend ? wcol : kOobOffset;   // (chunks past the part: zeros, to keep the count even)
#pragma unroll
        for (int i = 0; i < Chunk::kLoads; ++i) {
            const uint32_t off = (uint32_t)(k + Chunk::row(g, i)) * (uint32_t)a.ldp * sizeof(T) + wcol;
            ch.w[i] = __builtin_amdgcn_raw_buffer_load_b128(wsrc, (int)(first == kOobOffset ? kOobOffset : off), 0,
                                                            STREAM ? 2 : 0);
        }
        const uint32_t to = lds0 + (uint32_t)(r % 3 * kStage);
#pragma unroll
        for (int i = 0; i < MT; ++i)
            dma16(xsrc, k0 + r * kRound + xk[i] < K ? xoff[i] : kOobOffset, (uint32_t)(k0 + r * kRound) * sizeof(T),
                  to + (uint32_t)((8 * i + wave) * 1024));
    };
    f32x4 acc[n][MT];
#pragma unroll
    for (int j = 0; j < n; ++j)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[j][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int rounds = (kend - k0 + kRound - 1) / kRound;
    load(0, w[0]);
    load(1, w[1]);
    auto round = [&](int r, Chunk &ch) {
        rows_wait_vmcnt<Chunk::kLoads + MT>();   // this round's loads have landed
        __syncthreads();                         // ... for all waves, and the stage of the round before is read
        if (k0 + r * kRound + wave * Chunk::kRows < kend) {
            u32x4 x[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m)
                x[m] = *(const u32x4 *)(lds + r % 3 * kStage + (16 * m + c) * 512 + (((4 * wave + g) ^ c) << 4));
            ch.template products<MT>(acc, x);
        }
        load(r + 2, ch);
    };
    for (int r = 0; r < rounds; r += 2) {
        round(r, w[0]);
        if (r + 1 < rounds) round(r + 1, w[1]);
    }
    rows_wait_vmcnt<0>();
    __syncthreads();
    // a lane holds, for row c of a block, columns n (4 g + r) + j in acc[j][block][r]
    float *red = (float *)lds;   // [waves][16][kPitch]
    const int tid = threadIdx.x, chunks = GATED ? 8 : 16;
    const int r = tid / chunks, ch = tid % chunks, p = p0 + ch * n;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        if (m) __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < n; j += 4)
                *(f32x4 *)(red + (wave * 16 + c) * kPitch + n * (4 * g + i) + j) =
                    f32x4{acc[j][m][i], acc[j + 1][m][i], acc[j + 2][m][i], acc[j + 3][m][i]};
        __syncthreads();
        const int64_t q = m * 16 + r;
        if (r < 16 && q < a.Qdim && p < a.Pdim) {
            float v[n] = {}, lin[n] = {};
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                const float *from = red + (w * 16 + r) * kPitch + ch * n;
#pragma unroll
                for (int j = 0; j < n; ++j) {
                    v[j] += from[j];
                    if (GATED) lin[j] += from[kCols / 2 + j];
                }
            }
            if (a.part) linear_store_part<n, GATED>(a, split, q, p, v, lin);
            else linear_emit<T, ACT>(a, q, p, v, lin);
        }
    }
}

bool linear_few_rows(const switch_linear_config *cfg) { return cfg->M <= kFewRows; }

// Parts of k that give every CU a block, as long as each wave has two chunks (us with 1, 4, 8, 16 parts: 48 x 10240 x 4096
// 74, 29, 23, 32; 64 x 8192 x 1024 45, 19, 15, 15; 1 x 768 x 4096 6.5, 7.7, 9.1, 9.7; 1 x 4096 x 20480, 160 blocks without,
// 32, 34, 33, 38).
LinearCut linear_few_cut(const switch_linear_config *cfg) {
    const bool bf = cfg->act_dtype == SW_BF16;
    const int64_t tiles = ceil_div(linear_columns(cfg), bf ? 128 : 64), least = kFewWaves * (bf ? 32 : 16) * 2;
    int64_t splits = 256 / tiles;
    if (splits > cfg->K / least) splits = cfg->K / least;
    if (splits < 2) return LinearCut{1, cfg->K};
    const int64_t split_k = ceil_div(ceil_div(cfg->K, splits), 32) * 32;
    return LinearCut{(int)ceil_div(cfg->K, split_k), split_k};
}

template <typename T, int MT, int ACT, bool STREAM>
static hipError_t linear_few_launch(const LinearPlan &plan, const LinearArgs &a, hipStream_t s) {
    constexpr int n = Row16<T>::n, lds = few_lds(MT, 16 * n);
    auto kern = linear_few_kernel<T, MT, ACT, STREAM>;
    static PerDeviceOnce once;
    const hipError_t err = with_lds(once, kern, lds);
    if (err != hipSuccess) return err;
    const dim3 grid((unsigned)ceil_div(a.Pdim, a.gated ? 8 * n : 16 * n), (unsigned)plan.x.splits);
    hipLaunchKernelGGL(kern, grid, dim3(64 * kFewWaves), lds, s, a, plan.x);
    return hipGetLastError();
}
// A W of more than 32 MB streams past the caches (us, without / with: 48 x 10240 x 4096 24.8 / 24.0, 1 x 4096 x 20480 32.5 /
// 31.6; but 64 x 8192 x 1024 14.4 / 15.3, 32 x 2048 x 768 8.7 / 10.0).
template <typename T, int MT, int ACT>
static hipError_t linear_few_caches(const LinearPlan &plan, const LinearArgs &a, hipStream_t s) {
    return a.Kdim * a.ldp * (int64_t)sizeof(T) > 32 << 20 ? linear_few_launch<T, MT, ACT, true>(plan, a, s)
                                                          : linear_few_launch<T, MT, ACT, false>(plan, a, s);
}
template <typename T, int ACT> static hipError_t linear_few(const LinearPlan &plan, const LinearArgs &a, hipStream_t s) {
    switch (ceil_div(a.Qdim, 16)) {
    case 1: return linear_few_caches<T, 1, ACT>(plan, a, s);
    case 2: return linear_few_caches<T, 2, ACT>(plan, a, s);
    case 3: return linear_few_caches<T, 3, ACT>(plan, a, s);
    default: return linear_few_caches<T, 4, ACT>(plan, a, s);
    }
}

template <typename T> static hipError_t linear_few_act(const LinearPlan &plan, const LinearArgs &a, hipStream_t s) {
    switch (a.act) {
    case SW_ACT_RELU: return linear_few<T, SW_ACT_RELU>(plan, a, s);
    case SW_ACT_GELU: return linear_few<T, SW_ACT_GELU>(plan, a, s);
    case SW_ACT_GEGLU: return linear_few<T, SW_ACT_GEGLU>(plan, a, s);
    default: return linear_few<T, SW_ACT_NONE>(plan, a, s);
    }
}

hipError_t launch_linear_few(int dtype, const LinearPlan &plan, const LinearArgs &a, hipStream_t s) {
    return dtype == SW_BF16 ? linear_few_act<bf16>(plan, a, s) : linear_few_act<float>(plan, a, s);
}

}  // namespace sw

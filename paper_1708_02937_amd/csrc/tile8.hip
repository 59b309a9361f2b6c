// Products of blocked 8-bit matrices for many rows: BN weight rows x BM activation rows per workgroup, staged through
// LDS one block of 128 columns at a time.
//
// The weights are the first operand of the 32 x 32 matrix instructions and the activations the second, so a lane ends
// with runs of four consecutive outputs of one activation row.  Two arithmetics, by the output's type:
//   bfloat16  the scaled 8-bit instructions, which multiply by both blocks' powers of two themselves.  Within an
//             instruction they align products to the largest one and keep about 14 bits, 1.5e-5 of a sum of normal
//             values (measured), a hundredth of the output's own rounding; between instructions the sum is fp32.
//   float     codes widened to bfloat16, which is exact, and the 16-bit instructions, whose products and sums are
//             fp32; each block's sum is scaled as it joins the total.  Half the matrix rate.
#include "product8.h"

namespace sdnn {
namespace {

constexpr int kRowBytes = kBlock;  // a row of a stage: one block

enum TileMode { kTileProduct, kTileExpertsIn, kTileExpertsOut };

// Sixteen bytes per lane from global memory straight into LDS at base + 16 * lane.
__device__ __forceinline__ void stage16(const uint8_t *from, uint8_t *lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
}

// This wave's loads into LDS have landed, and every wave is here.
__device__ __forceinline__ void stage_barrier() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <int MODE, typename T, int BN, int BM, int WN, int WM>
struct Tile {
    static constexpr int kThreads = 64 * WN * WM, kWaves = WN * WM;
    static constexpr int NI = BN / WN / 32, MJ = BM / WM / 32;
    static constexpr int kRows = BN + BM, kLoads = kRows / 8 / kWaves;
    static constexpr int kStage = kRows * kRowBytes, kLds = 2 * kStage;
    static constexpr bool kExact = sizeof(T) == 4;
    static_assert(kRows % (8 * kWaves) == 0, "every wave stages the same number of rows");
};

// Which weight row LDS row r of a tile stands for, relative to the tile's first.  In the experts' first product the
// lower half of the tile is gate rows and the upper half the up rows of the same outputs.
template <int MODE, typename T, int BN, int BM, int WN, int WM>
__global__ void __launch_bounds__(64 * WN * WM) product_tile_kernel(ProductArgs a, ExpertsArgs x, TileWork work) {
    using S = Tile<MODE, T, BN, BM, WN, WM>;
    constexpr int NI = S::NI, MJ = S::MJ;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wn = wave % WN, wm = wave / WN;

    // The chiplets take workgroups in turn; each is given a run of neighbouring tiles, which share operand rows in
    // its L2.
    const int64_t tile = chiplet_order(blockIdx.x, gridDim.x);
    const int64_t nt = tile % work.n_tiles;
    int64_t mt = tile / work.n_tiles;

    const uint8_t *act, *act_scale, *wt, *wt_scale;
    int64_t n_rows, k, row0 = 0;  // n_rows: outputs of this matrix; row0: the tile's first activation row
    int rows;                     // activation rows of this tile
    constexpr int kOut = MODE == kTileExpertsIn ? BN / 2 : BN;  // outputs of a tile
    const int64_t n0 = nt * kOut;
    if constexpr (MODE == kTileProduct) {
        row0 = mt * BM;
        rows = (int)min((int64_t)BM, a.m - row0);
        act = a.a, act_scale = a.a_scale, wt = a.w, wt_scale = a.w_scale, n_rows = a.n, k = a.k;
    } else {
        const int e = find_tile(x.offsets, x.experts, x.tokens * x.chosen, (int)mt, BM, row0, rows);
        if (e < 0) return;
        if constexpr (MODE == kTileExpertsIn) {
            k = x.width, n_rows = x.inner;
            act = x.a, act_scale = x.a_scale;
            wt = x.w_in + (int64_t)e * 2 * n_rows * code_pitch(k);
            wt_scale = x.w_in_scale + (int64_t)e * 2 * blocks_of(n_rows) * scale_pitch(k);
        } else {
            k = x.inner, n_rows = x.width;
            act = work.p_codes, act_scale = work.p_scales;
            wt = x.w_out + (int64_t)e * n_rows * code_pitch(k);
            wt_scale = x.w_out_scale + (int64_t)e * blocks_of(n_rows) * scale_pitch(k);
        }
    }
    const int64_t pitch = code_pitch(k), spitch = scale_pitch(k);
    const int kb = (int)blocks_of(k);

    // activation row of tile row r (rows past the tile's end repeat its last)
    auto act_row = [&](int r) -> int64_t {
        const int64_t at = row0 + min(r, rows - 1);
        if constexpr (MODE == kTileExpertsIn) {
            const int64_t slots = x.tokens * x.chosen;
            return min(max((int64_t)x.order[at], (int64_t)0), slots - 1) / x.chosen;
        } else {
            return at;
        }
    };

    // Staging: instruction i of a wave fills 8 rows of 128 bytes; the 16-byte piece c of row r lies at c ^ (r & 7), so
    // that the lanes of a read, which hold different rows, spread over the banks.  The swap is made on the global side.
    const uint8_t *from[S::kLoads];
#pragma unroll
    for (int i = 0; i < S::kLoads; i++) {
        const int r = (i * S::kWaves + wave) * 8 + lane / 8;
        const int piece = ((lane % 8) ^ (r & 7)) * 16;
        if (r < BN) {
            int64_t n;
            if constexpr (MODE == kTileExpertsIn)
                n = min(n0 + r % (BN / 2), n_rows - 1) + (r < BN / 2 ? 0 : n_rows);
            else
                n = min(n0 + r, n_rows - 1);
            from[i] = wt + n * pitch + piece;
        } else {
            from[i] = act + act_row(r - BN) * pitch + piece;
        }
    }
    auto stage = [&](int buf) {
#pragma unroll
        for (int i = 0; i < S::kLoads; i++) {
            stage16(from[i], lds + buf * S::kStage + (i * S::kWaves + wave) * 1024);
            from[i] += kBlock;
        }
    };

    // First LDS row of this wave's weight subtile i.
    auto sub_row = [&](int i) {
        if constexpr (MODE == kTileExpertsIn)
            return (i < NI / 2 ? 0 : BN / 2) + wn * (NI / 2) * 32 + (i % (NI / 2)) * 32;
        else
            return wn * NI * 32 + i * 32;
    };

    // Scale codes, four blocks to a word: the lane's activation rows, and the weights' block rows of the wave (a
    // subtile of 32 weight rows lies in one).
    const uint8_t *asc[MJ];
#pragma unroll
    for (int j = 0; j < MJ; j++) asc[j] = act_scale + act_row((wm * MJ + j) * 32 + lane % 32) * spitch;
    const uint8_t *wsc[NI];
#pragma unroll
    for (int i = 0; i < NI; i++) {
        int64_t n = n0 + sub_row(i);
        if constexpr (MODE == kTileExpertsIn)
            n = n0 + sub_row(i) % (BN / 2);
        const int64_t last = (n_rows - 1) / kBlock;
        int64_t block = min(n / kBlock, last);
        if constexpr (MODE == kTileExpertsIn) block += i < NI / 2 ? 0 : last + 1;
        wsc[i] = wt_scale + block * spitch;
    }

    v16f acc[NI][MJ];
#pragma unroll
    for (int i = 0; i < NI; i++)
#pragma unroll
        for (int j = 0; j < MJ; j++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[i][j][r] = 0.0f;

    stage(0);
    uint32_t as[MJ], ws[NI], as_next[MJ], ws_next[NI];
#pragma unroll
    for (int j = 0; j < MJ; j++) as_next[j] = *(const uint32_t *)asc[j];
#pragma unroll
    for (int i = 0; i < NI; i++) ws_next[i] = *(const uint32_t *)wsc[i];

    for (int b = 0; b < kb; b++) {
        if (b % 4 == 0) {
            const int next = min(b + 4, (int)spitch - 4);
#pragma unroll
            for (int j = 0; j < MJ; j++) as[j] = as_next[j], as_next[j] = *(const uint32_t *)(asc[j] + next);
#pragma unroll
            for (int i = 0; i < NI; i++) ws[i] = ws_next[i], ws_next[i] = *(const uint32_t *)(wsc[i] + next);
        }
        stage_barrier();
        if (b + 1 < kb) stage((b + 1) & 1);
        const uint8_t *buf = lds + (b & 1) * S::kStage;
        // lane's 32 bytes of LDS row r in half h of the block
        auto fetch = [&](int r, int h) -> v8i {
            const int c = h * 4 + lane / 32 * 2, sw = r & 7;
            const v4i lo = *(const v4i *)(buf + r * kRowBytes + ((c ^ sw) * 16));
            const v4i hi = *(const v4i *)(buf + r * kRowBytes + (((c + 1) ^ sw) * 16));
            return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        };
        if constexpr (!S::kExact) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                v8i wf[NI], af[MJ];
#pragma unroll
                for (int j = 0; j < MJ; j++) af[j] = fetch(BN + (wm * MJ + j) * 32 + lane % 32, h);
#pragma unroll
                for (int i = 0; i < NI; i++) wf[i] = fetch(sub_row(i) + lane % 32, h);
#pragma unroll
                for (int i = 0; i < NI; i++)
#pragma unroll
                    for (int j = 0; j < MJ; j++)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf[i], af[j], acc[i][j], 0, 0, 0,
                                                                                    ws[i], 0, as[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < MJ; j++) {
                v8bf af[8];
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const v8i q = fetch(BN + (wm * MJ + j) * 32 + lane % 32, h);
#pragma unroll
                    for (int c = 0; c < 4; c++) af[4 * h + c] = widen8(q[2 * c], q[2 * c + 1]);
                }
#pragma unroll
                for (int i = 0; i < NI; i++) {
                    v16f z;
#pragma unroll
                    for (int r = 0; r < 16; r++) z[r] = 0.0f;
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        const v8i q = fetch(sub_row(i) + lane % 32, h);
#pragma unroll
                        for (int c = 0; c < 4; c++)
                            z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(q[2 * c], q[2 * c + 1]), af[4 * h + c],
                                                                        z, 0, 0, 0);
                    }
                    const int shift = (int)(ws[i] & 255) + (int)(as[j] & 255) - 2 * kOne;
#pragma unroll
                    for (int r = 0; r < 16; r++) acc[i][j][r] += ldexpf(z[r], shift);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < MJ; j++) as[j] >>= 8;
#pragma unroll
        for (int i = 0; i < NI; i++) ws[i] >>= 8;
    }

    // acc[i][j][4 q + v]: tile row (wm MJ + j) 32 + lane % 32, weight row sub_row(i) + 8 q + 4 (lane / 32) + v
    if constexpr (MODE == kTileExpertsIn) {
        constexpr int NP = NI / 2;
        constexpr int kPitch = kBlock + 16;  // LDS pitch of a row of codes: rows start in different banks
        static_assert(BN == 2 * kBlock, "a tile's outputs are one block of p");
        static_assert(BM * kPitch + WN * BM * 4 <= S::kLds, "the epilogue's arrays fit the stages");
        float *red = (float *)(lds + BM * kPitch);
        stage_barrier();  // the last stage has been read
#pragma unroll
        for (int j = 0; j < MJ; j++) {
            float amax = 0.0f;
#pragma unroll
            for (int i = 0; i < NP; i++)
#pragma unroll
                for (int r = 0; r < 16; r++) {
                    const int64_t f = n0 + sub_row(i) + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
                    const float p = f < n_rows ? silu_times(acc[i][j][r], acc[i + NP][j][r]) : 0.0f;
                    acc[i][j][r] = p;
                    amax = fmaxf(amax, finite_abs(p));
                }
            amax = fmaxf(amax, __shfl_xor(amax, 32));
            if (lane < 32) red[wn * BM + (wm * MJ + j) * 32 + lane] = amax;
        }
        __syncthreads();
        const int64_t p_pitch = code_pitch(n_rows), p_spitch = scale_pitch(n_rows);
#pragma unroll
        for (int j = 0; j < MJ; j++) {
            const int r = (wm * MJ + j) * 32 + lane % 32;
            float amax = red[r];
#pragma unroll
            for (int w = 1; w < WN; w++) amax = fmaxf(amax, red[w * BM + r]);
            const int code = scale_code(amax);
            const float inv = inverse_scale(code);
#pragma unroll
            for (int i = 0; i < NP; i++)
#pragma unroll
                for (int q = 0; q < 4; q++)
                    *(int *)(lds + r * kPitch + sub_row(i) + 8 * q + 4 * (lane / 32)) =
                        pack_e4m3(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3],
                                  inv);
            if (wn == 0 && lane < 32 && r < rows) {
                uint8_t *s = work.p_scales_out + (row0 + r) * p_spitch;
                s[nt] = (uint8_t)code;
                if (nt == work.n_tiles - 1)
                    for (int64_t c = nt + 1; c < p_spitch; c++) s[c] = 1;
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < rows * 8; c += S::kThreads)
            *(v4i *)(work.p_codes_out + (row0 + c / 8) * p_pitch + n0 + c % 8 * 16) =
                *(const v4i *)(lds + c / 8 * kPitch + c % 8 * 16);
    } else {
        // Through LDS, 32 rows of every wave at a time, so that whole lines leave for memory.
        constexpr int kCells = 16 / sizeof(T), kPitch = BN + kCells, kSlice = WM * 32;
        static_assert(kSlice * kPitch * sizeof(T) + BN * 4 <= S::kLds, "a slice of the outputs fits the stages");
        T *out = (T *)lds;
        float *bias = (float *)(lds + kSlice * kPitch * sizeof(T));
        stage_barrier();  // the last stage has been read
        if constexpr (MODE == kTileProduct)
            for (int c = threadIdx.x; c < BN; c += S::kThreads)
                bias[c] = a.bias && n0 + c < n_rows ? a.bias[n0 + c] : 0.0f;
#pragma unroll
        for (int j = 0; j < MJ; j++) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NI; i++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const int c = sub_row(i) + 8 * q + 4 * (lane / 32);
                    v4f z = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    if constexpr (MODE == kTileProduct) {
                        z += *(const v4f *)(bias + c);
                        if (a.activate)
                            for (int v = 0; v < 4; v++) z[v] = relu_clamp(z[v], a.ymax);
                    }
                    put4(out + (wm * 32 + lane % 32) * kPitch + c, z);
                }
            __syncthreads();
            constexpr int kPieces = BN / kCells;
#pragma unroll
            for (int c = threadIdx.x; c < kSlice * kPieces; c += S::kThreads) {
                const int lr = c / kPieces, r = (lr / 32 * MJ + j) * 32 + lr % 32, col = c % kPieces * kCells;
                if (r >= rows || n0 + col >= n_rows) continue;
                T *y;
                if constexpr (MODE == kTileProduct)
                    y = (T *)a.y + (row0 + r) * a.ldy;
                else
                    y = (T *)work.o + min(max((int64_t)x.order[row0 + r], (int64_t)0), x.tokens * x.chosen - 1) * n_rows;
                const T *from = out + lr * kPitch + col;
                if (work.wide && n0 + col + kCells <= n_rows)
                    *(v4i *)(y + n0 + col) = *(const v4i *)from;
                else
                    for (int v = 0; v < kCells && n0 + col + v < n_rows; v++) y[n0 + col + v] = from[v];
            }
        }
    }
}

template <int MODE, typename T, int BN, int BM, int WN, int WM>
hipError_t tile_go(const ProductArgs &a, const ExpertsArgs &x, TileWork work, int64_t m_tiles, int64_t outputs,
                   hipStream_t s) {
    using S = Tile<MODE, T, BN, BM, WN, WM>;
    static std::atomic<unsigned long long> raised{0};
    const auto kernel = product_tile_kernel<MODE, T, BN, BM, WN, WM>;
    hipError_t e = raise_lds_limit((const void *)kernel, S::kLds, raised);
    if (e != hipSuccess) return e;
    constexpr int kOut = MODE == kTileExpertsIn ? BN / 2 : BN;
    work.n_tiles = (outputs + kOut - 1) / kOut;
    const int64_t grid = work.n_tiles * m_tiles;
    if (grid * S::kThreads >= (int64_t)1 << 32) return hipErrorInvalidConfiguration;
    kernel<<<(unsigned)grid, S::kThreads, S::kLds, s>>>(a, x, work);
    return hipGetLastError();
}

template <typename T>
hipError_t product_go(const ProductArgs &a, TileWork work, hipStream_t s) {
    const ExpertsArgs none{};
    const int64_t big = ((a.m + 255) / 256) * ((a.n + 255) / 256);
    if constexpr (sizeof(T) == 2)
        if (big >= 256) return tile_go<kTileProduct, T, 256, 256, 2, 4>(a, none, work, (a.m + 255) / 256, a.n, s);
    return tile_go<kTileProduct, T, 128, 128, 2, 2>(a, none, work, (a.m + 127) / 128, a.n, s);
}

template <typename T>
hipError_t experts_go(const ExpertsArgs &x, TileWork work, hipStream_t s) {
    const ProductArgs none{};
    const int64_t slots = x.tokens * x.chosen, busy = slots < x.experts ? slots : x.experts;
    if constexpr (sizeof(T) == 2) if (slots >= 128 * busy) {
        hipError_t e = tile_go<kTileExpertsIn, T, 256, 256, 2, 4>(none, x, work, busy + slots / 256, x.inner, s);
        if (e != hipSuccess) return e;
        return tile_go<kTileExpertsOut, T, 256, 256, 2, 4>(none, x, work, busy + slots / 256, x.width, s);
    }
    hipError_t e = tile_go<kTileExpertsIn, T, 256, 64, 2, 2>(none, x, work, busy + slots / 64, x.inner, s);
    if (e != hipSuccess) return e;
    return tile_go<kTileExpertsOut, T, 128, 64, 2, 2>(none, x, work, busy + slots / 64, x.width, s);
}

}  // namespace

hipError_t launch_product_tile(const ProductArgs &a, const TileWork &work, bool bf16, hipStream_t s) {
    return bf16 ? product_go<__bf16>(a, work, s) : product_go<float>(a, work, s);
}

hipError_t launch_experts_tile(const ExpertsArgs &x, const TileWork &work, bool bf16, hipStream_t s) {
    return bf16 ? experts_go<__bf16>(x, work, s) : experts_go<float>(x, work, s);
}

}  // namespace sdnn

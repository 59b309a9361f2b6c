// Products of blocked 8-bit matrices for many rows: BN weight rows x BM activation rows per workgroup, staged through
// LDS one block of 128 columns at a time.
//
// The weights are the first operand of the 32 x 32 matrix instructions and the activations the second, so a lane ends
// with runs of four consecutive outputs of one activation row.  Two arithmetics:
//   8 bits  (bfloat16 outputs) the scaled 8-bit instructions, which multiply by both blocks' powers of two themselves.
//           Within an instruction they align products to the largest one and keep about 14 bits, 1.5e-5 of a sum of
//           normal values (measured), a hundredth of the output's own rounding; between instructions the sum is fp32.
//   EXACT   (float outputs, and the first of the experts' products where tiles are few) codes widened to bfloat16 with
//           their scales, which is exact, and the 16-bit instructions, whose products and sums are fp32.  Half the matrix
//           rate.
#include "product8.h"

namespace sdnn {
namespace {

constexpr int kRowBytes = kBlock / 2;  // a row of a stage: half a block

constexpr int kMaxLds = 160 * 1024;

enum TileMode { kTileProduct, kTileExpertsIn, kTileExpertsOut };

// Sixteen bytes per lane from global memory straight into LDS at base + 16 * lane.
__device__ __forceinline__ void stage16(const uint8_t *from, uint8_t *lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
}

// All but this wave's last LEFT loads have landed, its reads of LDS are over, and every wave is here.
template <int LEFT>
__device__ __forceinline__ void stage_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

template <int MODE, typename T, bool EXACT, int BN, int BM, int WN, int WM, int KG, int STAGES>
struct Tile {
    static constexpr int kThreads = 64 * WN * WM * KG, kWaves = WN * WM;  // waves of a group
    static constexpr int NI = BN / WN / 32, MJ = BM / WM / 32;
    static constexpr int kRows = BN + BM, kLoads = kRows / 16 / kWaves;
    static constexpr int kStage = kRows * kRowBytes, kRing = STAGES * kStage * KG;
    static constexpr int kBlockRows = BN > kBlock ? BN / kBlock : 1;  // block rows of weights
    // the scales behind the stages: two words per row, or (KG > 1) every row's whole
    static int64_t lds_bytes(int64_t k) {
        return kRing + (KG == 1 ? 2 * (BM + 64) * 4 : (BM + kBlockRows) * (scale_pitch(k) + 4));
    }
    static constexpr bool kTurns = kWaves == 8 && KG == 1 && !EXACT;
    static_assert(KG == 1 || MODE != kTileExpertsOut, "the experts' rows are rounded by one group");
    static_assert(kRows % (16 * kWaves) == 0, "every wave stages the same number of rows");
};

// In the experts' first product the lower half of a tile's LDS rows is gate rows and the upper half the up rows of the
// same outputs.  With KG > 1, KG groups of waves share the tile's blocks between them (group g takes blocks g, g + KG,
// ...), each with stages of its own, and their sums join in the end: for products with few tiles, whose time is the
// length of the chain of stages.
template <int MODE, typename T, bool EXACT, int BN, int BM, int WN, int WM, int KG, int STAGES>
__global__ void __launch_bounds__(64 * WN * WM * KG, KG == 1 ? 2 : KG) product_tile_kernel(ProductArgs a, ExpertsArgs x, TileWork work) {
    using S = Tile<MODE, T, EXACT, BN, BM, WN, WM, KG, STAGES>;
    constexpr int NI = S::NI, MJ = S::MJ, kStages = STAGES;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x % 64, any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wave = any_wave % S::kWaves, group = any_wave / S::kWaves;
    const int wn = wave % WN, wm = wave / WN;

    // The chiplets take workgroups in turn; each is given a run of neighbouring tiles, four tiles of rows wide, so that
    // the 32 tiles in flight on a chiplet share 12 panels of operand rows in its L2.
    constexpr int kGroup = MODE == kTileProduct ? 4 : 1;
    const int64_t tile = chiplet_order(blockIdx.x, gridDim.x), m_tiles = gridDim.x / work.n_tiles;
    const int64_t first = tile / (kGroup * work.n_tiles) * kGroup, wide = min(m_tiles - first, (int64_t)kGroup);
    const int64_t in_group = tile - first * work.n_tiles;
    const int64_t nt = in_group / wide, mt = first + in_group % wide;

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

    // Staging: instruction i of a wave fills 16 rows of 64 bytes; the 16-byte piece c of row r lies at c ^ (r / 4 & 3),
    // so that the 16 lanes of a read that go together, which hold different rows, cover all banks.  The swap is made on
    // the global side.
    const uint8_t *from[S::kLoads];
#pragma unroll
    for (int i = 0; i < S::kLoads; i++) {
        const int r = (i * S::kWaves + wave) * 16 + lane / 4;
        const int piece = ((lane % 4) ^ (r >> 2 & 3)) * 16;
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
        if (KG > 1) from[i] += min(group, kb - 1) * kBlock;
    }
    const int stages = 2 * ((kb + KG - 1) / KG);
    uint8_t *const ring = lds + group * (kStages * S::kStage);
    auto stage = [&](int t) {
#pragma unroll
        for (int i = 0; i < S::kLoads; i++) {
            stage16(from[i], ring + t % kStages * S::kStage + (i * S::kWaves + wave) * 1024);
            // the other half of the block, then the group's next block (past the end: the last one again)
            if (KG == 1 || t % 2 == 0)
                from[i] += kRowBytes;
            else
                from[i] += (t / 2 + 1) * KG + group < kb ? KG * kBlock - kRowBytes : -kRowBytes;
        }
    };

    // First LDS row of this wave's weight subtile i.
    auto sub_row = [&](int i) {
        if constexpr (MODE == kTileExpertsIn)
            return (i < NI / 2 ? 0 : BN / 2) + wn * (NI / 2) * 32 + (i % (NI / 2)) * 32;
        else
            return wn * NI * 32 + i * 32;
    };

    // Scale codes, four blocks to a word, go through LDS too: the words of the tile's activation rows, then of its block
    // rows of weights (in the experts' first product the gate's and the up rows').
    constexpr int kWords = BM + 64;
    uint8_t *const scales = lds + S::kRing;
    const int64_t last_block = (n_rows - 1) / kBlock;
    auto weight_scales = [&](int i) -> const uint8_t * {
        if constexpr (MODE == kTileExpertsIn)
            return wt_scale + (min(n0 / kBlock, last_block) + i % 2 * (last_block + 1)) * spitch;
        else
            return wt_scale + min(n0 / kBlock + i % S::kBlockRows, last_block) * spitch;
    };
    const uint8_t *scale_from = nullptr;
    if (KG == 1) {
        if (wave < BM / 64)
            scale_from = act_scale + act_row(wave * 64 + lane) * spitch;
        else if (wave == BM / 64)
            scale_from = weight_scales(lane);
    }
    auto stage_scales = [&](int four) {
        if (wave <= BM / 64)
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void *)(scale_from + four * 4),
                (__attribute__((address_space(3))) void *)(scales + (four & 1) * kWords * 4 + wave * 256), 4, 0, 0);
    };

    v16f acc[NI][MJ];
#pragma unroll
    for (int i = 0; i < NI; i++)
#pragma unroll
        for (int j = 0; j < MJ; j++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[i][j][r] = 0.0f;

    uint32_t xs[MJ], ws[NI];
    auto read_scales = [&](int four) {
        const uint32_t *w = (const uint32_t *)(scales + (four & 1) * kWords * 4);
#pragma unroll
        for (int j = 0; j < MJ; j++) xs[j] = w[(wm * MJ + j) * 32 + lane % 32];
#pragma unroll
        for (int i = 0; i < NI; i++) ws[i] = w[BM + sub_row(i) / kBlock];
    };
    // Several stages are on their way while one is multiplied: a load takes longer than a stage's products.
    constexpr int kLeft = S::kLoads * (kStages - 2);
    if (KG == 1) stage_scales(0);
    for (int t = 0; t < kStages - 1; t++)
        if (t < stages) stage(t);
    if (KG > 1) {
        const int words = (int)spitch / 4;
        for (int c = threadIdx.x; c < (BM + S::kBlockRows) * words; c += S::kThreads) {
            const int r = c / words, w = c % words;
            const uint8_t *at = r < BM ? act_scale + act_row(r) * spitch : weight_scales(r - BM);
            *(uint32_t *)(scales + r * ((int)spitch + 4) + w * 4) = *(const uint32_t *)(at + w * 4);
        }
    }
    // The scales of stage t, read anew every four blocks, and the next ones sent for.
    auto scales_at = [&](int t) {
        if (KG == 1 && t % 8 == 0) {
            read_scales(t / 8);
            if (t + 8 < stages) stage_scales(t / 8 + 1);
        }
    };
    // The lane's 32 bytes of LDS row r of stage t.
    auto fetch = [&](int t, int r) -> v8i {
        const uint8_t *row = ring + t % kStages * S::kStage + r * kRowBytes;
        const int c = lane / 32 * 2, sw = r >> 2 & 3;
        const v4i lo = *(const v4i *)(row + ((c ^ sw) * 16)), hi = *(const v4i *)(row + (((c + 1) ^ sw) * 16));
        return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    auto fetch_x = [&](int t, int j) { return fetch(t, BN + (wm * MJ + j) * 32 + lane % 32); };
    auto fetch_w = [&](int t, int i) { return fetch(t, sub_row(i) + lane % 32); };
    uint32_t xc[MJ], wc[NI];  // the codes of a stage's block, in the low byte
    auto codes_at = [&](int t) {
        if constexpr (KG > 1) {
            const int b = min(t / 2 * KG + group, kb - 1), row = (int)spitch + 4;
#pragma unroll
            for (int j = 0; j < MJ; j++) xc[j] = scales[((wm * MJ + j) * 32 + lane % 32) * row + b];
#pragma unroll
            for (int i = 0; i < NI; i++) wc[i] = scales[(BM + sub_row(i) / kBlock) * row + b];
            return;
        }
        const int shift = t / 2 % 4 * 8;
#pragma unroll
        for (int j = 0; j < MJ; j++) xc[j] = xs[j] >> shift;
#pragma unroll
        for (int i = 0; i < NI; i++) wc[i] = ws[i] >> shift;
    };
    if constexpr (S::kTurns) {
        // The two waves of a SIMD take turns: while one reads a stage's operands the other keeps the matrix cores busy.
        // Turns change at a barrier, and the second half of the waves is one turn late.  Wave and turn 2 t: reads of
        // stage t, sends for stage t + 3, whose buffer was last read (by the late waves) in turn 2 t - 1; turn 2 t + 1:
        // products.  Stage t + 1 has landed for every wave at the end of turn 2 t + 1, when it is first needed.
        const bool late = wave >= 4;
        auto turn = [&]() {
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        auto landed = [&](int t) {  // this wave's part of stage t + 1
            if (t + kStages - 1 < stages)
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLeft) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        };
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        turn();
        if (late) turn();
        for (int t = 0; t < stages; t++) {
            scales_at(t);
            v8i xf[MJ], wf[NI];
#pragma unroll
            for (int j = 0; j < MJ; j++) xf[j] = fetch_x(t, j);
#pragma unroll
            for (int i = 0; i < NI; i++) wf[i] = fetch_w(t, i);
            __builtin_amdgcn_sched_barrier(0);
            if (t + kStages - 1 < stages) stage(t + kStages - 1);
            codes_at(t);
            if (late) landed(t);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            turn();
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < NI; i++)
#pragma unroll
                for (int j = 0; j < MJ; j++)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf[i], xf[j], acc[i][j], 0, 0, 0, wc[i],
                                                                                0, xc[j]);
            __builtin_amdgcn_s_setprio(0);
            if (!late) landed(t);
            turn();
        }
        if (!late) turn();
    } else {
        for (int t = 0; t < stages; t++) {
            // Stage t has landed, and the buffer of the one before has been read by every wave.
            if (t + kStages - 1 <= stages)
                stage_barrier<kLeft>();
            else
                stage_barrier<0>();
            scales_at(t);
            if (t + kStages - 1 < stages) stage(t + kStages - 1);
            if (KG > 1 && t / 2 * KG + group >= kb) continue;  // this group's blocks are done
            codes_at(t);
            v8i xf[MJ];
#pragma unroll
            for (int j = 0; j < MJ; j++) xf[j] = fetch_x(t, j);
            v8i wf[NI];
#pragma unroll
            for (int i = 0; i < NI; i++) wf[i] = fetch_w(t, i);
            if constexpr (!EXACT) {
#pragma unroll
                for (int i = 0; i < NI; i++)
#pragma unroll
                    for (int j = 0; j < MJ; j++)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf[i], xf[j], acc[i][j], 0, 0, 0,
                                                                                    wc[i], 0, xc[j]);
            } else {
                bool plain = true;
#pragma unroll
                for (int j = 0; j < MJ; j++) plain = plain && widens((int)(xc[j] & 255), xf[j]);
#pragma unroll
                for (int i = 0; i < NI; i++) plain = plain && widens((int)(wc[i] & 255), wf[i]);
                plain = __all(plain);
                v8bf xw[MJ][4];
#pragma unroll
                for (int j = 0; j < MJ; j++)
#pragma unroll
                    for (int c = 0; c < 4; c++)
                        xw[j][c] = widen8(xf[j][2 * c], xf[j][2 * c + 1], plain ? (int)(xc[j] & 255) : kOne);
#pragma unroll
                for (int i = 0; i < NI; i++) {
                    v8bf ww[4];
#pragma unroll
                    for (int c = 0; c < 4; c++)
                        ww[c] = widen8(wf[i][2 * c], wf[i][2 * c + 1], plain ? (int)(wc[i] & 255) : kOne);
                    if (plain) {
#pragma unroll
                        for (int j = 0; j < MJ; j++)
#pragma unroll
                            for (int c = 0; c < 4; c++)
                                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ww[c], xw[j][c], acc[i][j], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int j = 0; j < MJ; j++) {
                            v16f z;
#pragma unroll
                            for (int r = 0; r < 16; r++) z[r] = 0.0f;
#pragma unroll
                            for (int c = 0; c < 4; c++)
                                z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ww[c], xw[j][c], z, 0, 0, 0);
                            const int e = (int)(wc[i] & 255) + (int)(xc[j] & 255) - 2 * kOne;
#pragma unroll
                            for (int r = 0; r < 16; r++) acc[i][j][r] += ldexpf(z[r], e);
                        }
                    }
                }
            }
        }
    }

    if constexpr (KG > 1) {
        // The groups' sums, in the order of the groups.
        constexpr int kSum = S::kWaves * NI * MJ * 16 * 64 * 4;
        static_assert((KG - 1) * kSum <= S::kRing, "the groups' sums fit the stages");
        stage_barrier<0>();
        v4f *const sums = (v4f *)lds + (wave * NI * MJ * 4) * 64 + lane;
        if (group > 0)
#pragma unroll
            for (int i = 0; i < NI * MJ * 4; i++)
                sums[(group - 1) * (kSum / 16) + i * 64] =
                    v4f{acc[i / 4 / MJ][i / 4 % MJ][i % 4 * 4], acc[i / 4 / MJ][i / 4 % MJ][i % 4 * 4 + 1],
                        acc[i / 4 / MJ][i / 4 % MJ][i % 4 * 4 + 2], acc[i / 4 / MJ][i / 4 % MJ][i % 4 * 4 + 3]};
        __syncthreads();
        if (group == 0)
#pragma unroll
            for (int i = 0; i < NI * MJ * 4; i++)
#pragma unroll
                for (int g = 0; g < KG - 1; g++) {
                    const v4f v = sums[g * (kSum / 16) + i * 64];
                    for (int c = 0; c < 4; c++) acc[i / 4 / MJ][i / 4 % MJ][i % 4 * 4 + c] += v[c];
                }
    }

    // acc[i][j][4 q + v]: tile row (wm MJ + j) 32 + lane % 32, weight row sub_row(i) + 8 q + 4 (lane / 32) + v
    if constexpr (MODE == kTileExpertsIn) {
        constexpr int NP = NI / 2;
        constexpr int kPitch = kBlock + 16;  // LDS pitch of a row of codes: rows start in different banks
        static_assert(BN == 2 * kBlock, "a tile's outputs are one block of p");
        static_assert(BM * kPitch + WN * BM * 4 <= S::kRing, "the epilogue's arrays fit the stages");
        float *red = (float *)(lds + BM * kPitch);
        stage_barrier<0>();  // the last stage has been read
        if (group == 0)
#pragma unroll
        for (int j = 0; j < MJ; j++) {
            float amax = 0.0f;
#pragma unroll
            for (int i = 0; i < NP; i++)
#pragma unroll
                for (int r = 0; r < 16; r++) {
                    const int64_t f = n0 + sub_row(i) + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
                    float p = silu_times<sizeof(T) == 2>(acc[i][j][r], acc[i + NP][j][r]);
                    p = f < n_rows ? p : 0.0f;
                    acc[i][j][r] = p;
                    amax = fmaxf(amax, fabsf(p));  // NaN is passed over
                }
            if (__any(amax == INFINITY)) {
                amax = 0.0f;
#pragma unroll
                for (int i = 0; i < NP; i++)
#pragma unroll
                    for (int r = 0; r < 16; r++) amax = fmaxf(amax, finite_abs(acc[i][j][r]));
            }
            amax = fmaxf(amax, __shfl_xor(amax, 32));
            if (lane < 32) red[wn * BM + (wm * MJ + j) * 32 + lane] = amax;
        }
        __syncthreads();
        const int64_t p_pitch = code_pitch(n_rows), p_spitch = scale_pitch(n_rows);
        if (group == 0)
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
        // Through LDS, 32 rows of every wave at a time, so that whole lines leave for memory, and past the caches, which
        // the operands of the tiles to come fill better (8192 x 16384 x 4096: 516 us without that, 495 with it).
        constexpr bool kHalf = MODE == kTileExpertsOut && sizeof(T) == 2;  // the experts' rows in half precision
        using Out = typename std::conditional<kHalf, _Float16, T>::type;
        constexpr int kCells = 16 / sizeof(T), kPitch = BN + kCells, kSlice = WM * 32;
        static_assert(kSlice * kPitch * sizeof(T) + BN * 4 <= S::kRing, "a slice of the outputs fits the stages");
        Out *const out = (Out *)lds;
        float *bias = (float *)(lds + kSlice * kPitch * sizeof(T));
        stage_barrier<0>();  // the last stage has been read
        int *const slot = (int *)scales;
        if constexpr (MODE == kTileExpertsOut)
            for (int c = threadIdx.x; c < BM; c += S::kThreads)
                slot[c] = min(max(x.order[row0 + min(c, rows - 1)], 0), (int)(x.tokens * x.chosen - 1));
        if constexpr (MODE == kTileProduct)
            for (int c = threadIdx.x; c < BN; c += S::kThreads)
                bias[c] = a.bias && n0 + c < n_rows ? a.bias[n0 + c] : 0.0f;
        float inverse[MJ];
        if constexpr (kHalf) {
            // A row of the tile has a power of two of its own, which brings its largest value to 2^14 and more: what
            // is rounded here is rounded to 11 bits, and the sum of the experts' rows, which is rounded to 8, stays as
            // good as if they were fp32 (measured: 1.40 times the error of the last rounding with bfloat16 rows and
            // everything else exact).  Wider rows would cost half as much again as the whole combination.
            static_assert(BM * 4 + WN * BM * 4 <= 2 * (BM + 64) * 4, "the rows' maxima fit behind the slots");
            float *const red = (float *)(scales + BM * 4);
#pragma unroll
            for (int j = 0; j < MJ; j++) {
                float amax = 0.0f;
#pragma unroll
                for (int i = 0; i < NI; i++)
#pragma unroll
                    for (int r = 0; r < 16; r++) amax = fmaxf(amax, fabsf(acc[i][j][r]));  // NaN is passed over
                if (__any(amax == INFINITY)) {
                    amax = 0.0f;
#pragma unroll
                    for (int i = 0; i < NI; i++)
#pragma unroll
                        for (int r = 0; r < 16; r++) amax = fmaxf(amax, finite_abs(acc[i][j][r]));
                }
                amax = fmaxf(amax, __shfl_xor(amax, 32));
                if (lane < 32) red[wn * BM + (wm * MJ + j) * 32 + lane] = amax;
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < MJ; j++) {
                const int r = (wm * MJ + j) * 32 + lane % 32;
                float amax = red[r];
#pragma unroll
                for (int w = 1; w < WN; w++) amax = fmaxf(amax, red[w * BM + r]);
                const int code = max((__float_as_int(amax) >> 23) - 14, 1);
                inverse[j] = inverse_scale(code);
                if (wn == 0 && lane < 32 && r < rows) work.o_scales[(int64_t)slot[r] * work.n_tiles + nt] = (uint8_t)code;
            }
        }
#pragma unroll
        for (int j = 0; j < MJ; j++) {
            __syncthreads();
            if (group == 0)
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
                    if constexpr (kHalf) z *= inverse[j];
                    put4(out + (wm * 32 + lane % 32) * kPitch + c, z);
                }
            __syncthreads();
            const int cols = (int)min((int64_t)BN, n_rows - n0);
            constexpr int kPieces = BN / kCells;
#pragma unroll
            for (int c = threadIdx.x; c < kSlice * kPieces; c += S::kThreads) {
                const int lr = c / kPieces, col = c % kPieces * kCells;
                const int r = (lr / 32 * MJ + j) * 32 + lr % 32;  // row lr of the slice, in the tile
                if (r >= rows || col >= cols) continue;
                Out *y;
                if constexpr (MODE == kTileProduct)
                    y = (Out *)a.y + (row0 + r) * a.ldy + n0 + col;
                else
                    y = (Out *)work.o + (int64_t)slot[r] * work.o_pitch + n0 + col;
                const Out *const from = out + lr * kPitch + col;
                if (col + kCells <= cols)
                    __builtin_nontemporal_store(*(const v4i *)from, (v4i_any *)y);
                else
                    for (int v = 0; col + v < cols; v++) y[v] = from[v];
            }
        }
    }
}

template <int MODE, typename T, bool EXACT, int BN, int BM, int WN, int WM, int KG, int STAGES>
hipError_t tile_go(const ProductArgs &a, const ExpertsArgs &x, TileWork work, int64_t m_tiles, int64_t outputs,
                   hipStream_t s) {
    using S = Tile<MODE, T, EXACT, BN, BM, WN, WM, KG, STAGES>;
    static std::atomic<unsigned long long> raised{0};
    const auto kernel = product_tile_kernel<MODE, T, EXACT, BN, BM, WN, WM, KG, STAGES>;
    const int64_t lds = S::lds_bytes(MODE == kTileProduct ? a.k : MODE == kTileExpertsIn ? x.width : x.inner);
    hipError_t e = raise_lds_limit((const void *)kernel, kMaxLds, raised);
    if (e != hipSuccess) return e;
    constexpr int kOut = MODE == kTileExpertsIn ? BN / 2 : BN;
    work.n_tiles = (outputs + kOut - 1) / kOut;
    const int64_t grid = work.n_tiles * m_tiles;
    if (grid * S::kThreads >= (int64_t)1 << 32 || lds > kMaxLds) return hipErrorInvalidConfiguration;
    kernel<<<(unsigned)grid, S::kThreads, (unsigned)lds, s>>>(a, x, work);
    return hipGetLastError();
}

// A call is fastest on the largest tile that still gives every CU (256) a workgroup, and with few tiles the groups that
// share a tile's blocks shorten the chain of stages.  Measured in us at K = 4096, bfloat16 (x 4: four groups):
//   N x M         64x64 x4  64x64 x2  128x64 x2  128x128 x2  256x128  256x256
//   4096 x 128        12.1      12.5       16.3        22.5     40.0     41.7
//   4096 x 256        16.1      13.3       17.0        22.7     40.3     42.6
//   4096 x 512        25.5      23.0       18.8        23.2     40.9     43.3
//   4096 x 1024       47.6      40.8       31.6        26.8     41.3     44.0
//   4096 x 2048       88.9      76.7                   53.6     44.2     46.1
//   16384 x 1024     208.9     155.0      129.2       115.6     85.7     64.8
// With float (the 16-bit instructions) four groups are ahead for longer: 4096 x 256 20.4, 22.5 and 31.4, 4096 x 512 on
// 128 x 64 with four groups 30.1 and with two 32.6; and tiles beyond 128 x 128 do not fit the registers.
// Over short rows the chain of stages is short anyway, and 64 x 64 with one group comes before 128 x 128 x2.  One bound on K
// stands for a line that falls as tiles rise, and is higher for float (64x64 | 128x128 x2, by tiles of 64 x 64):
//   K        576 x 3700 (522)          1024 x 3900 (976)         float: 522              976
//   1001      9.7 | 11.5                12.9 | 12.0              15.4 | 17.9             18.5 | 18.8
//   1536     12.8 | 14.0                18.1 | 14.9              21.0 | 23.0             25.5 | 24.1
//   2048     15.3 | 15.7                21.5 | 16.7              25.8 | 27.8             32.1 | 28.8
//   2560     19.1 | 19.1                26.7 | 20.1              31.4 | 33.1             39.3 | 34.1
//   4096     27.5 | 24.6                41.8 | 26.0              46.3 | 47.5             59.2 | 49.0
// Float above 1024 tiles, 64x64 | 128x128: 1000 x 5000 x 2048 (1264) 41.3 | 44.7, 1024 x 8192 x 2048 (2048) 60.1 | 47.4,
// 2048 x 16384 x 4096 (8192) 428 | 354.
template <typename T>
hipError_t product_go(const ProductArgs &a, TileWork work, hipStream_t s) {
    constexpr bool kExact = sizeof(T) == 4;
    const ExpertsArgs none{};
    const auto tiles = [&](int side) { return (a.m + side - 1) / side; };
    const int64_t small = tiles(64) * ((a.n + 63) / 64);
    // the groups' kernels hold every scale of a tile in LDS; these two need the most
    const bool groups = Tile<kTileProduct, T, kExact, 128, 128, 2, 2, 2, 4>::lds_bytes(a.k) <= kMaxLds &&
                        Tile<kTileProduct, T, kExact, 128, 64, 2, 2, 4, 3>::lds_bytes(a.k) <= kMaxLds;
    if (groups && small <= 1024) {
        if (small <= (sizeof(T) == 2 ? 128 : 256))
            return tile_go<kTileProduct, T, kExact, 64, 64, 2, 2, 4, 4>(a, none, work, tiles(64), a.n, s);
        if constexpr (sizeof(T) == 2) {
            if (small <= 256) return tile_go<kTileProduct, T, kExact, 64, 64, 2, 2, 2, 4>(a, none, work, tiles(64), a.n, s);
            if (small <= 512) return tile_go<kTileProduct, T, kExact, 128, 64, 2, 2, 2, 3>(a, none, work, tiles(64), a.n, s);
        } else {
            if (small <= 512) return tile_go<kTileProduct, T, kExact, 128, 64, 2, 2, 4, 3>(a, none, work, tiles(64), a.n, s);
        }
        if (a.k <= 2048) return tile_go<kTileProduct, T, kExact, 64, 64, 2, 2, 1, 4>(a, none, work, tiles(64), a.n, s);
        return tile_go<kTileProduct, T, kExact, 128, 128, 2, 2, 2, 4>(a, none, work, tiles(128), a.n, s);
    }
    if constexpr (sizeof(T) == 2) {
        if (small <= 2048) return tile_go<kTileProduct, T, kExact, 256, 128, 2, 2, 1, 3>(a, none, work, tiles(128), a.n, s);
        return tile_go<kTileProduct, T, kExact, 256, 256, 2, 4, 1, 4>(a, none, work, tiles(256), a.n, s);
    } else {
        return tile_go<kTileProduct, T, kExact, 128, 128, 2, 2, 1, 4>(a, none, work, tiles(128), a.n, s);
    }
}

// Tiles of 64 rows with the first product exact; of 128 with the 8-bit instructions for many rows to an expert, where
// tiles are enough to fill the chip more than once.  Both measured in us (64 rows | 128 rows), at sizes on both sides of
// the bound; the 8-bit instructions are ahead at all of them, so the bound is not where their time begins to pay:
//   64 experts of 4096 x 1024, 8 chosen:   64 tokens 262 | 225,  333 tokens 312 | 226,  2048 tokens 739 | 429
//   8 experts of 4096 x 1024, 2 chosen:    128 tokens 69 | 61,   512 tokens 80 | 70,    2048 tokens 216 | 122
//   24 experts of 2001 x 701, 3 chosen:    333 tokens 51 | 47,   600 tokens 81 | 53,    1000 tokens 89 | 69
// What the exact product is for: a sum that is 5e-5 off (a column in a hundred ten times as wide as the others) moves some
// values of p over a boundary of their 8 bits.  Without a residual the result is then 1.17 to 1.55 times as far from the
// exact one as its own rounding to bfloat16 brings it, with one 1.03 to 1.3 times; with the exact product up to 1.03.
// The bound goes by tiles alone, not by what a call saves: 333 tokens on 64 experts lie above it, 2048 on 8 below.  (The
// exact product on tiles of 128 rows: 8192 tokens as above 2.2 ms, 1.3.)
template <typename T>
hipError_t experts_go(const ExpertsArgs &x, TileWork work, int *run, hipStream_t s) {
    constexpr bool kExact = sizeof(T) == 4;
    const ProductArgs none{};
    const int64_t slots = x.tokens * x.chosen, busy = slots < x.experts ? slots : x.experts;
    const int64_t large = busy + slots / 128, small = busy + slots / 64;
    if constexpr (sizeof(T) == 2)
        if (slots >= 32 * busy && large * ((x.inner + 127) / 128) >= 400) {
            const hipError_t e = tile_go<kTileExpertsIn, T, kExact, 256, 128, 2, 2, 1, 3>(none, x, work, large, x.inner, s);
            if (e != hipSuccess) return e;
            *run = 256;
            return tile_go<kTileExpertsOut, T, kExact, 256, 128, 2, 2, 1, 3>(none, x, work, large, x.width, s);
        }
    const hipError_t e =
        Tile<kTileExpertsIn, T, true, 256, 64, 4, 1, 2, 3>::lds_bytes(x.width) <= kMaxLds
            ? tile_go<kTileExpertsIn, T, true, 256, 64, 4, 1, 2, 3>(none, x, work, small, x.inner, s)
            : tile_go<kTileExpertsIn, T, true, 256, 64, 4, 1, 1, 3>(none, x, work, small, x.inner, s);
    if (e != hipSuccess) return e;
    *run = 128;
    return tile_go<kTileExpertsOut, T, kExact, 128, 64, 2, 2, 1, 3>(none, x, work, small, x.width, s);
}

}  // namespace

hipError_t launch_product_tile(const ProductArgs &a, const TileWork &work, bool bf16, hipStream_t s) {
    return bf16 ? product_go<__bf16>(a, work, s) : product_go<float>(a, work, s);
}

hipError_t launch_experts_tile(const ExpertsArgs &x, const TileWork &work, bool bf16, int *run, hipStream_t s) {
    return bf16 ? experts_go<__bf16>(x, work, run, s) : experts_go<float>(x, work, run, s);
}

}  // namespace sdnn

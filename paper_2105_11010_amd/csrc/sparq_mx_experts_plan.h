// Which kernel and which tiles a product of experts, or its gradients, gets (include/sparq_mx_experts.h).  Host code; tests/experts_plan_check.cpp asks it.
#pragma once
#include <math.h>

#include "sparq_mx_experts_few_kernel.h"
#include "sparq_mx_grad_kernel.h"
#include "sparq_mx_tiles.h"

namespace sparq {
namespace mx {

// ---- the product ------------------------------------------------------------------------
struct ExpertsPlan {
    int tile;                // 256, 128 or 64: results a workgroup makes along either side; 0: few rows, 16 `fragments` of them a workgroup
    int fragments;
    int parts;               // of the reduction (one expert without offsets alone)
    int64_t pieces;          // few rows: as many as any division of the rows can make
    int blocks;              // ... and blocks of 16 columns a workgroup makes
    size_t table_bytes, partial_bytes;
};
// What a round of tiles takes (us): one of 256 x 256 a CU, or two of 128 x 128, by the length of the reduction and what comes behind it.  One wavefront a SIMD
// has nobody to multiply while it makes its results; of two workgroups a CU one does.  (bf16, measured: 8192 x 4096 x 4096, 256 -> 128: 85 -> 97, with gelu 114 -> 105,
// kept 102 -> 109, both 127 -> 118, residual 100 -> 112; 16384 x 4096 x 2048 104 -> 107, 163 -> 121, 136 -> 124, 187 -> 144, residual 153 -> 133; of 1024 76 -> 61,
// residual 127 -> 90.)
inline double round_of(int tile, int K, int function, bool residual, bool kept) {
    const bool gelu = function == SPARQ_MX_GELU, silu = function == SPARQ_MX_SILU;
    if (tile == 256) return 11.0 + 7.6 * K / 1024 + (gelu ? 14.7 : silu ? 8.0 : 0.0) + (residual ? 10.0 : 0.0) + (kept ? 8.0 : 0.0);
    return 1.9 + 5.7 * K / 1024 + (gelu ? 1.8 : silu ? 1.0 : 0.0) + (residual ? 3.4 : 0.0) + (kept ? 2.0 : 0.0);
}
inline ExpertsPlan experts_plan(int64_t M, int N, int K, int experts, bool offsets, int function, bool residual, bool kept) {
    ExpertsPlan p = {};
    p.parts = 1;
    // What an expert has of the rows on average; how they are divided is not known here.
    const int64_t each = (M + experts - 1) / experts;
    // Few rows (us, a gemm on six sets of tensors in turn, as many rows for each expert / rows that go to any, few rows -> tiles.  16 rows a workgroup: 16 experts of
    // 4096 x 2048 with 13 rows each 18.4 / 21.0 -> 20.5 / 20.8, with 16 18.7 / 21.6 -> 20.8 / 20.6; 8 of 2048 x 4096 with 13 12.7 / 12.8 -> 13.3 / 13.3, with 16 13.1 / 14.8 ->
    // 13.4 / 13.4; 64 of 1024 x 1024 with 13 11.1 / 13.2 -> 11.3 / 11.3.  32 rows a workgroup: 32 rows each 23.5 / 26.8 -> 22.3 / 22.3, 15.9 / 19.1 -> 13.6 / 13.7, 15.9 / 19.2 ->
    // 11.7 / 12.1; 64: 29.4 / 44.2 -> 24.2 / 24.2, 24.4 / 26.8 -> 14.2 / 14.5, 24.5 / 38.1 -> 13.8 / 14.4.  One expert: as the product without an epilogue, sparq_mx_gemm.hip.)
    // A kept form goes in tiles at any number of rows: the 16 columns of a block are half of the 32 values that share a scale, and the other half is made elsewhere.  (What
    // that costs: 16 of 4096 x 2048 with 4 rows each 20.9, without the kept form 16.4; a layer of 4096 x 4096 with 16 rows 8.5 and 4.9.)
    if (!kept && (offsets ? each <= 12 : each <= 16 || (each <= 64 && each * N * K <= 5ll << 27))) {
        p.fragments = (int)((each + 15) / 16);
        p.pieces = offsets ? most_tiles(M, experts, 16 * p.fragments) : 1;
        // Two workgroups of eight wavefronts a CU, or three of four, by the number of pieces to be expected of rows that go to any expert alike (us, by blocks a
        // workgroup makes: 16 rows, 16 experts of 2048 x 4096: one 16.7, two 15.8, three 13.9, four 14.8, six 14.5; 64 rows, the same: 27, 21, 23, 17.8, 21.
        // Rows that every expert has one of make more pieces than that: 16 rows, one of each, 20).
        const double part = offsets ? (double)M / (16 * p.fragments) - 0.5 * experts : 0.0;
        const double expected = offsets ? experts * (1.0 - pow(1.0 - 1.0 / experts, (double)M)) + (part > 0.0 ? part : 0.0) : 1.0;
        const double wanted = expected * ((N + kFewColumns - 1ll) / kFewColumns) / (K <= 4 * kScaleUnit ? 690 : 460);
        p.blocks = wanted < 1.5 ? 1 : wanted > 8.0 ? 8 : (int)(wanted + 0.5);
        return p;
    }
    // (of experts' rows about half of an expert's last tile is empty)
    const auto tiles_m = [&](int t) { return !offsets ? (M + t - 1) / t : M / t + (experts + 1) / 2 > experts ? M / t + (experts + 1) / 2 : (int64_t)experts; };
    const auto tiles = [&](int t) { return tiles_m(t) * ((N + t - 1) / t); };
    const int64_t rounds256 = (tiles(256) + 255) / 256, rounds128 = (tiles(128) + 511) / 512;
    // (experts of a few hundred rows leave much of their tiles of 256 empty: 16 of 4096 x 2048 with 96 rows each 36 us, in tiles of 128 31)
    if (tiles(128) < 112) p.tile = 64;
    else if (offsets && each < 512) p.tile = 128;
    else p.tile = rounds256 * round_of(256, K, function, residual, kept) < rounds128 * round_of(128, K, function, residual, kept) ? 256 : 128;
    if (offsets) {
        p.table_bytes = p.tile == 256 || experts > kExpertsOfLanes ? table_bytes(M, experts) : 0;
        return p;
    }
    const int64_t n = ((M + p.tile - 1) / p.tile) * ((N + p.tile - 1) / p.tile), steps = (K + kCodeUnit - 1) / kCodeUnit, most = steps / 16;
    p.parts = n <= 64 && steps >= 64 ? (int)(128 / n < most ? 128 / n : most) : 1;
    p.partial_bytes = p.parts > 1 ? (size_t)round_up(p.parts * M * N * 4, 256) : 0;
    return p;
}
// What the epilogue is and whether there are offsets does not change what the query names: the most of all.
inline size_t experts_bytes(int64_t M, int N, int K, int experts) {
    size_t most = 0;
    for (int form = 0; form < 8; ++form) {
        const bool offsets = form & 1, residual = form & 2, kept = form & 4;
        if (!offsets && experts > 1) continue;
        for (const int function : {(int)SPARQ_MX_NONE, (int)SPARQ_MX_SILU, (int)SPARQ_MX_GELU}) {
            const ExpertsPlan p = experts_plan(M, N, K, experts, offsets, function, residual, kept);
            const size_t bytes = p.table_bytes + p.partial_bytes;
            most = bytes > most ? bytes : most;
        }
    }
    return most;
}

// Whether the product quantises its rows itself, each wavefront the group that it multiplies, once a workgroup: what that saves is a launch (us, itself -> before it,
// 16 experts of 2048 x 4096, 16 rows 13.9 -> 16.2, 64 rows 17.8 -> 19.4; 128 rows among 8 of 4096 x 2048, 16 each, 14.2 -> 14.4).
inline bool quantised_on_the_way(const ExpertsPlan& plan, int K) { return plan.tile == 0 && plan.fragments == 1 && K <= 8 * kScaleUnit; }

// ---- the gradients ----------------------------------------------------------------------
// Tiles of 256 (bf16), 128 or 64 results along either side, by the rounds that 256 CUs make of them.  bf16: as in sparq_mx_grad.hip.  The others, whose
// parts of dy leave LDS for one tile of 128 a CU, and three (fp16) or two of 64: a round of the smaller makes 0.86 or 0.6 of the time of one of the larger (us, 128 -> 64, fp16:
// dx 2048 x 2048 x 2048 to 4 experts 77 -> 62, 8192 x 1024 x 1024 to 8 65 -> 58, 16384 x 2048 x 2048 to 8 347 -> 402; dw of 4275 x 777 x 520 to 20 39 -> 35, 2048 x 2048 x 2048
// to 4 70 -> 80); dw's tiles, many and short, come without rounds.  What the experts leave empty of their last tiles it takes for half a tile each: fp16 dx of 16384 x 512 x 512
// to 64 goes in tiles of 128, 39, for 34.5.
inline int grad_tile(int dy_type, int64_t tiles256, int64_t tiles128, int64_t tiles64, int64_t steps, bool dw) {
    if (tiles128 < 192) return 64;
    if (dy_type == SPARQ_MX_BF16) return !(dw && steps <= 4) && 3 * ((tiles256 + 255) / 256) <= 2 * ((tiles128 + 511) / 512) ? 256 : 128;
    const int places64 = dy_type == SPARQ_MX_F16 ? 768 : 512;
    const double round64 = dy_type == SPARQ_MX_F16 ? 0.86 : 0.6;
    const double rounds128 = dw ? tiles128 / 256.0 : (double)((tiles128 + 255) / 256);
    const double rounds64 = dw ? (double)tiles64 / places64 : (double)((tiles64 + places64 - 1) / places64);
    return rounds64 * round64 < rounds128 ? 64 : 128;
}
inline int dx_tile(int dy_type, int64_t M, int K, int experts) {
    const auto tiles = [&](int t) { return (M / t + experts / 2 + 1) * ((K + t - 1) / t); };
    return grad_tile(dy_type, tiles(256), tiles(128), tiles(64), 0, false);
}
inline int dw_tile(int dy_type, int64_t M, int N, int K, int experts) {
    const auto tiles = [&](int64_t t) { return experts * ((N + t - 1) / t) * ((K + t - 1) / t); };
    return grad_tile(dy_type, tiles(256), tiles(128), tiles(64), (M / experts + kGradStep - 1) / kGradStep, true);
}

}  // namespace mx
}  // namespace sparq

// The gradients' kernel: 256 x 256 results a workgroup (bf16), 128 x 128 (the other types), or 64 x 64, the largest that leaves no CUs without.
// out[j][k] = sum_r dy(j, r) V[r][k] as in sparq_mx_grad_kernel.h.  V's rows are decoded as they lie, eight values of a row a thread, and dy's are
// copied; the matrix instruction's operands, eight neighbouring r of one column, come out of LDS by reads that turn 4 x 16 values (V, and dy
// where r is its row).  Sixteen lanes read four rows, 32 bytes each, at a time: a row's 16-byte units are permuted by the row so that four
// neighbouring rows lie in different quarters of the banks.
// A step is 64 r, four quarters of sixteen (256 x 256), four or one matrix instructions; one wavefront a SIMD has nobody else to fill the time an
// instruction runs, so what goes between them is laid out here: the next quarter's reads, and of V and of dy two rows each, written to the
// next step's tiles, and the request for their successors.  One barrier a step, before the last quarter: by then the step's tiles have been
// read by all.  (dy straight to LDS, without registers: the compiler then waits for these loads before every turning read, and dx of
// 8192 x 4096 x 4096 took 392 us instead of 268, before the steps' order was laid out as it is.)
// Bound by the matrix instructions and, with data as large as this, by the card's power: 8192 x 4096 x 4096 takes 206-248 us for dx and 237-256
// for dw (1.07-1.33 PF; the same instructions without loads and writes 1.57 PF).  fp16 dy, two instructions a product, 673-728 and 706-722 us, fp32, three,
// 904-916 and 940.  Tiles of 128 and 64 ask for V at a step's end (a thread has one run of it) and need it where the next
// begins (experts' a step later, which fp16 dx of 16384 x 2048 x 2048 took from 335 to 307-320): of 128 every step waits for all loads behind its barrier, which bf16 hides in part by a second workgroup on the CU and fp16 and fp32, whose LDS
// leaves no room for one, do not; of 64 that wait is what a small layer's time is, 515 x 771 x 577 7.7 and 8.4 us of 12 or 13 steps.  dw in 256 x 256 keeps 105
// scalar registers in lanes of vector ones, about 110 moves a step between its matrix instructions.
#pragma once
#include <type_traits>

#include "sparq_mx_grad_kernel.h"
#include "sparq_mx_tiles.h"

namespace sparq {
namespace mx {

template <int TILE> inline constexpr int kWideBytes = kGradStep * TILE * 2;       // of one side's tile

template <class T, int TILE> inline constexpr int kWideLds = 2 * (kParts<T> + 1) * kWideBytes<TILE>;
template <class T, int TILE> inline constexpr int kWidePerCu = kWideLds<T, TILE> < 40 * 1024 ? 4 : 160 * 1024 / kWideLds<T, TILE>;
// PARAMS: GradParams, or what sparq_mx_experts_grad.h makes of it -- dx's tiles of one expert's rows each, dw a workgroup's of one expert.
template <class T, class O, bool DW, int TILE, class PARAMS = GradParams>
__global__ __launch_bounds__(kGradThreads, (kWidePerCu<T, TILE>)) void grad_wide_kernel(O* __restrict__ out, const PARAMS all) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool kExperts = !std::is_same_v<PARAMS, GradParams>;
    std::conditional_t<kExperts, GradParams, const GradParams&> p = all;
    if constexpr (kExperts && DW) {
        out = all.template own_rows<T, O>(p, out);
    }
    const uint32_t part = kExperts ? 0 : blockIdx.y;
    constexpr int P = kParts<T>;                             // of dy, a tile each
    constexpr bool kCut = kExperts && DW && P == 1;          // dw's last step is cut off (of more parts, checking costs what it saves)
    constexpr int kF = TILE / 64, kSlots = P * kF * kF;      // 32 x 32 results along a side; matrix instructions a quarter
    constexpr int kRow = TILE * 2;                           // bytes of a tile's row
    constexpr int kRun = TILE == 64 ? 16 : 32, kRuns = TILE * kGradStep / kGradThreads / kRun;      // a thread's runs of V's values
    constexpr int kUnits = TILE / 32;                        // and of eight values of dy, as many as V's pieces of eight
    constexpr int kPieces = kRun / 8;                        // a run
    constexpr bool kDeep = kExperts && TILE <= 128;          // V is asked for two steps ahead: a thread's one run of it is written in pieces all over a step
    constexpr int kSets = kDeep ? 2 : 1;
    constexpr int kBytes = kWideBytes<TILE>;
    typedef short v4s __attribute__((ext_vector_type(4)));
    extern __shared__ __attribute__((aligned(16))) uint8_t lds8[];
    uint8_t *const lds_dy = lds8, *const lds_v = lds8 + 2 * P * kBytes;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), c = lane & 31, g = lane >> 5;
    if constexpr (DW) {
        const uint32_t tiles = (uint32_t)p.tiles_j * (uint32_t)p.tiles_k;
        if (blockIdx.x >= tiles) {
            typedef ColumnSums<T, kGradThreads> Sums;
            static_assert(Sums::kFloats * 4 <= kWideLds<T, TILE>);
            if constexpr (kExperts) {                        // (one slab, the expert's rows)
                Sums::run(static_cast<const T*>(p.dy), p.lddy, 0, p.R, (int)p.J, (int)(blockIdx.x - tiles) * Sums::kColumns, p.column_sums, reinterpret_cast<float*>(lds8));
                return;
            }
            const uint32_t n = blockIdx.x - tiles, across = (uint32_t)((p.J + Sums::kColumns - 1) / Sums::kColumns), slab = n / across;
            const int64_t begin = slab * p.slab, end = begin + p.slab < p.R ? begin + p.slab : p.R;
            if (blockIdx.y == 0)
                Sums::run(static_cast<const T*>(p.dy), p.lddy, begin, end, (int)p.J, (int)(n % across) * Sums::kColumns, p.column_sums + slab * p.J,
                          reinterpret_cast<float*>(lds8));
            return;
        }
    }
    uint32_t tj, tk;
    int64_t j0;
    if constexpr (kExperts && !DW) {
        if (!all.template own_tile<TILE>(p, j0, tk)) return;
    } else {
        tile_of(blockIdx.x, p.tiles_j, p.tiles_k, tj, tk);
        j0 = (int64_t)tj * TILE;
    }
    const int k0 = (int)tk * TILE;
    const int64_t s_begin = (int64_t)part * p.steps_per_part, s_all = (p.R + kGradStep - 1) / kGradStep;
    const int64_t s_end = s_begin + p.steps_per_part < s_all ? s_begin + p.steps_per_part : s_all, s_fast = p.s_whole < s_end ? p.s_whole : s_end;
    Products<P, TILE, TILE> products;
    const int wj = products.wj, wk = products.wk;

    if (s_begin < s_fast) {
        // ---- dy: a thread has kUnits runs of eight values: of every eighth or 16th row (DW) or of rows 32 i + t / 8, 64 r each
        constexpr int kAcross = TILE / 8, kRowsAtOnce = kGradThreads / kAcross;
        constexpr int kSize = sizeof(T), kKept = 2 * kSize;
        uint32_t kept[kUnits][kKept];
        uint32_t dy_at[DW ? 1 : kUnits], dy_column = 0;
        if constexpr (DW) {
            int64_t j = j0 + 8 * (t % kAcross);
            j = j < p.J ? j : j0;                            // (columns past the last one make results that are not stored)
            dy_column = (uint32_t)((j - j0) * kSize);
            dy_at[0] = (uint32_t)((t / kAcross * p.lddy + (j - j0)) * kSize);
        } else {
            const int64_t last = p.J - 1 - j0;
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int row = 32 * i + (t >> 3), from = row < last ? row : (int)last;
                dy_at[i] = (uint32_t)((from * p.lddy + 8 * (t & 7)) * kSize);
            }
        }
        // ---- V: a thread has two runs of 32 values, one block each, of rows 4 (lane / 8) + wave and that + 32; or one of row 4 (lane / 4) + wave;
        // or one of 16 values of row lane / 4 + 16 wave
        constexpr int kWords = kRun / (DW ? 4 : 8);
        uint32_t raw[kSets][kRuns][kWords], scale[kSets][kRuns];
        constexpr int kAlong = TILE / kRun;
        const int v_row = TILE == 64 ? lane / kAlong + 16 * wave : 4 * (lane / kAlong) + wave;
        int k = k0 + kRun * (lane % kAlong);
        k = k < p.K128 ? k : p.K128 - kRun;
        const uint32_t v_at = (uint32_t)(v_row * p.code_pitch + (DW ? k : k / 2)), scale_at = (uint32_t)(v_row * p.scale_pitch + (k >> 5));

        // Where the next step to be asked for lies.  Past the last one it stays there, for tiles nobody reads.
        const uint8_t* dy_from = static_cast<const uint8_t*>(p.dy) + (DW ? j0 + s_begin * (kGradStep * p.lddy) : j0 * p.lddy + s_begin * kGradStep) * kSize;
        const uint8_t *codes_from = p.codes + s_begin * kGradStep * p.code_pitch, *scales_from = p.scales + s_begin * kGradStep * p.scale_pitch;
        const uint32_t dy_step = DW ? (uint32_t)(kGradStep * p.lddy * kSize) : kGradStep * kSize, codes_step = (uint32_t)(kGradStep * p.code_pitch);
        const uint32_t scales_step = (uint32_t)(kGradStep * p.scale_pitch);
        int left = (int)(s_fast - s_begin) - 1;
        // (kCut) A step's rows may be fewer than 64: what comes for the others -- the next expert's rows of V, or what lies past V's end and comes as zeros -- is made
        // zeros as it is written to LDS.  Of the step that is written, and of the one that is asked for.
        int rows_written = 0, rows_asked = 0;
        if constexpr (kCut) rows_asked = all.fast_rows(p);
        int left_v = left;
        auto advance_v = [&]() __attribute__((always_inline)) {
            codes_from += left_v > 0 ? codes_step : 0;
            scales_from += left_v > 0 ? scales_step : 0;
            --left_v;
        };
        auto advance = [&]() __attribute__((always_inline)) {
            dy_from += left > 0 ? dy_step : 0;
            if constexpr (kDeep) {
                advance_v();
            } else {
                codes_from += left > 0 ? codes_step : 0;
                scales_from += left > 0 ? scales_step : 0;
            }
            --left;
            rows_written = rows_asked;
            rows_asked -= kGradStep;
        };
        const auto buffer = [](const uint8_t* from) __attribute__((always_inline)) { return __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, 0x7FFFFFFF, 0x00020000); };
        // ... that ends with the call's rows, where a step may not
        const auto buffer_to = [&](const uint8_t* from, const uint8_t* end, auto checked) __attribute__((always_inline)) {
            const int64_t bytes = end - from;
            return __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, decltype(checked)::value && bytes < 0x7FFFFFFF ? (int)bytes : 0x7FFFFFFF, 0x00020000);
        };
        const uint8_t *codes_end = nullptr, *scales_end = nullptr;
        if constexpr (kCut) {
            codes_end = all.codes + all.rows * p.code_pitch;
            scales_end = all.scales + all.rows * p.scale_pitch;
        }
        // (dy's rows past the fast ones are not asked for: their lanes read the step's first row, which is one.  Its end is no border a load could be held against: rows may
        // be an odd number of elements, and words lie across it.)
        auto load_dy = [&](int i, auto checked) __attribute__((always_inline)) {
            constexpr bool kCheck = kCut && decltype(checked)::value;
            const uint32_t row = DW ? (uint32_t)(kRowsAtOnce * i * p.lddy * kSize) : 0;
            uint32_t at = dy_at[DW ? 0 : i];
            if constexpr (kCheck) at = kRowsAtOnce * i + t / kAcross < rows_asked ? at + row : dy_column;
#pragma unroll
            for (int h = 0; h < kKept / 4; ++h) {
                const v4u w = __builtin_amdgcn_raw_buffer_load_b128(buffer(dy_from), at, (kCheck ? 0 : (int)row) + 16 * h, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) kept[i][4 * h + e] = w[e];
            }
        };
        // (V's end is one.  A load's offset is the sum of a lane's part and a scalar one, and the lane's alone is held against the buffer's size: the row is in it.)
        auto load_v = [&](int set, int run, auto checked) __attribute__((always_inline)) {
            const uint32_t row = (uint32_t)(32 * run * p.code_pitch), scale_row = (uint32_t)(32 * run * p.scale_pitch);
            const uint32_t in_lane = kCut && decltype(checked)::value ? row : 0, scale_in_lane = kCut && decltype(checked)::value ? scale_row : 0;
            if constexpr (kWords == 2) {
                const v2u w = __builtin_amdgcn_raw_buffer_load_b64((kCut ? buffer_to(codes_from, codes_end, checked) : buffer(codes_from)), v_at, 0, 0);
                raw[kDeep ? set : 0][run][0] = w[0];
                raw[kDeep ? set : 0][run][1] = w[1];
            }
#pragma unroll
            for (int h = 0; h < kWords / 4; ++h) {
                const v4u w = __builtin_amdgcn_raw_buffer_load_b128((kCut ? buffer_to(codes_from, codes_end, checked) : buffer(codes_from)), v_at + in_lane, (int)(row - in_lane) + 16 * h, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) raw[kDeep ? set : 0][run][4 * h + e] = w[e];
            }
            scale[kDeep ? set : 0][run] = __builtin_amdgcn_raw_buffer_load_b8((kCut ? buffer_to(scales_from, scales_end, checked) : buffer(scales_from)), scale_at + scale_in_lane,
                                                                              (int)(scale_row - scale_in_lane), 0);
        };
        // A tile's row is permuted in its 16-byte units, which keeps both the turning reads and the writes apart in the banks.
        const auto permuted = [](int row, int chunk) __attribute__((always_inline)) {
            if constexpr (TILE == 64) return row * kRow + ((chunk ^ (row & 2 ? 5 : 0)) << 4);
            else return row * kRow + ((chunk ^ (chunk >> 4 & 1) ^ ((row & 3) << 2 | (row >> 2 & 3))) << 4);
        };
        auto write_dy = [&](uint8_t* tile, int i, auto checked) __attribute__((always_inline)) {
            uint8_t* const to = tile + (DW ? permuted(kRowsAtOnce * i + t / kAcross, t % kAcross) : 16 * unit_at(32 * i + (t >> 3), t & 7));
            if constexpr (kCut && decltype(checked)::value) {
                const bool there = kRowsAtOnce * i + t / kAcross < rows_written;
#pragma unroll
                for (int e = 0; e < kKept; ++e) kept[i][e] = there ? kept[i][e] : 0u;
            }
            if constexpr (P == 1) *reinterpret_cast<v4u*>(to) = v4u{kept[i][0], kept[i][1], kept[i][2], kept[i][3]};
            else {
                float part[8][P];
#pragma unroll
                for (int e = 0; e < 8; ++e) split<P>(element<T>(kept[i][kSize == 4 ? e : e / 2], e % 2), part[e]);
#pragma unroll
                for (int n = 0; n < P; ++n)
                    *reinterpret_cast<v4u*>(to + n * kBytes) = v4u{pack_bf16(part[0][n], part[1][n]), pack_bf16(part[2][n], part[3][n]),
                                                                   pack_bf16(part[4][n], part[5][n]), pack_bf16(part[6][n], part[7][n])};
            }
        };
        // values 2 e and 2 e + 1 of the eight of a piece
        v4u decoded;
        float unit;
        auto decode = [&](int set, int piece, int e, auto checked) __attribute__((always_inline)) {
            const int run = piece / kPieces, at = piece % kPieces;
            if (at == 0 && e == 0) {
                unit = DW ? unit8_of(scale[kDeep ? set : 0][run]) : scale_operand(scale[kDeep ? set : 0][run]);
                if constexpr (kCut && decltype(checked)::value) unit = v_row + 32 * run < rows_written ? unit : 0.0f;
            }
            if constexpr (DW) {
                const uint32_t w = raw[kDeep ? set : 0][run][2 * at + (e >> 1)] >> (16 * (e & 1));
                decoded[e] = pack_bf16((float)(int8_t)w * unit, (float)(int8_t)(w >> 8) * unit);
            } else {
                decoded[e] = pair4_of(raw[kDeep ? set : 0][run][at], unit, e);
            }
        };
        auto write_v = [&](uint8_t* tile, int piece) __attribute__((always_inline)) {
            *reinterpret_cast<v4u*>(tile + permuted(v_row + 32 * (piece / kPieces), kPieces * (lane % kAlong) + piece % kPieces)) = decoded;
        };
        // ---- operands: eight neighbouring r of one row or column
        struct Operands {
            v4u v[kF], dy[P][kF];
        };
        Operands set[2];
        // A lane's half of operand f: r = 16 q + 8 g + 4 h + (lane / 4) % 4, columns first + 32 f + 16 ((lane / 16) % 2) + 4 (lane % 4) and on.
        auto read_turned = [&](v4u& to, const uint8_t* tile, int first, int f, int q, int h) __attribute__((always_inline)) {
            typedef __attribute__((address_space(3))) v4s* P;
            const int row = 8 * g + 4 * h + ((lane >> 2) & 3), chunk = first / 8 + 4 * f + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
            const v4s r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(tile + permuted(row, chunk) + ((lane & 1) << 3) + q * 16 * kRow));
            const v2u w = __builtin_bit_cast(v2u, r);
            to[2 * h] = w[0];
            to[2 * h + 1] = w[1];
        };
        constexpr int kReads = kF * (2 + P * (DW ? 2 : 1));
        // read n of a quarter's kReads, in the order the products need them: the first fragment of V, all of dy, the rest of V
        auto read = [&](Operands& o, const uint8_t* dy_tile, const uint8_t* v_tile, int q, int n) __attribute__((always_inline)) {
            constexpr int kEach = DW ? 2 * kF : kF, kDy = P * kEach;
            if (n < 2) read_turned(o.v[0], v_tile, wk, 0, q, n);
            else if (n < 2 + kDy) {
                const int part = (n - 2) / kEach, f = (n - 2) % kEach;
                if constexpr (DW) read_turned(o.dy[part][f >> 1], dy_tile + part * kBytes, wj, f >> 1, q, f & 1);
                else o.dy[part][f] = *reinterpret_cast<const v4u*>(dy_tile + part * kBytes + 16 * unit_at(wj + 32 * f + c, 2 * q + g));
            } else {
                n -= kDy;
                read_turned(o.v[n >> 1], v_tile, wk, n >> 1, q, n & 1);
            }
        };

        // What is issued after matrix instruction i of quarter q of a step whose tiles are the first or second of each side.  Between two
        // barriers, quarters 3, 0, 1, 2, the tiles of the step after the later one's are written and those after them asked for.
        auto between = [&](auto now_, int q, int i, auto checked) __attribute__((always_inline)) {
            constexpr int now = decltype(now_)::value;
            const int part = (q + 1) & 3, first = part * kUnits / 4, parts = 8 * ((part + 1) * kUnits / 4 - first);      // pieces this quarter, eight parts each
            if (q == 3 && i == 0) advance();
            const int read_from = q == 3 ? now ^ 1 : now, write_to = q == 3 ? now : now ^ 1;
            for (int n = i * kReads / kSlots; n < (i + 1) * kReads / kSlots; ++n) read(set[(q + 1) & 1], lds_dy + read_from * P * kBytes, lds_v + read_from * kBytes, (q + 1) & 3, n);
            for (int u = i * parts / kSlots; u < (i + 1) * parts / kSlots; ++u) {
                const int piece = first + u / 8;
                if (u % 2 == 0) decode(write_to, piece, u % 8 / 2, checked);
                if (u % 8 == 7) {
                    write_v(lds_v + write_to * kBytes, piece);
                    if (piece % kPieces == kPieces - 1) load_v(write_to, piece / kPieces, checked);
                }
                if (u % 8 == 3) {
                    write_dy(lds_dy + write_to * P * kBytes, piece, checked);
                    load_dy(piece, checked);
                }
            }
        };
        auto barrier = [&]() __attribute__((always_inline)) {
            __builtin_amdgcn_s_waitcnt(vmcnt_and_lds(63));
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        auto step = [&](auto now, auto checked) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (q == 3) barrier();                       // the next step's tiles are written, this step's read
                const Operands& o = set[q & 1];
#pragma unroll
                for (int x = 0; x < kF; ++x)
#pragma unroll
                    for (int n = 0; n < P; ++n)
#pragma unroll
                        for (int y = 0; y < kF; ++y) {
                            products.acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, o.v[x]), __builtin_bit_cast(v8bf, o.dy[n][y]),
                                                                                         products.acc[x][y], 0, 0, 0);
                            between(now, q, (x * P + n) * kF + y, checked);
                            __builtin_amdgcn_sched_barrier(0);
                        }
            }
        };

#pragma unroll
        for (int i = 0; i < kUnits; ++i) load_dy(i, std::true_type{});
#pragma unroll
        for (int i = 0; i < kRuns; ++i) load_v(0, i, std::true_type{});
        if constexpr (kDeep) {
            advance_v();
#pragma unroll
            for (int i = 0; i < kRuns; ++i) load_v(1, i, std::true_type{});
        }
        advance();
        static_assert(kUnits == kPieces * kRuns, "a unit of dy to a piece of V");
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) decode(0, i, e, std::true_type{});
            write_v(lds_v, i);
            if (i % kPieces == kPieces - 1) load_v(0, i / kPieces, std::true_type{});
            write_dy(lds_dy, i, std::true_type{});
            load_dy(i, std::true_type{});
        }
        barrier();
        // as if the last quarter of a step before the first
#pragma unroll
        for (int i = 0; i < kSlots; ++i) between(std::integral_constant<int, 1>{}, 3, i, std::true_type{});
        int64_t s = s_begin;
        if constexpr (kCut)
            for (; s + (kDeep ? 6 : 5) < s_fast; s += 2) {   // (what these ask for, up to a quarter of step s + 4 -- of V s + 5 --, is of whole steps)
                step(std::integral_constant<int, 0>{}, std::false_type{});
                step(std::integral_constant<int, 1>{}, std::false_type{});
            }
        for (; s < s_fast; s += 2) {
            step(std::integral_constant<int, 0>{}, std::true_type{});
            if (s + 1 < s_fast) step(std::integral_constant<int, 1>{}, std::true_type{});
        }
    }
    int64_t s_rest = s_begin < s_fast ? s_fast : s_begin, s_last = s_end;
    if constexpr (kExperts && DW) {                          // (the rows behind the fast ones, by themselves)
        all.template leave_fast<T>(p);
        s_rest = 0;
        s_last = p.steps_per_part;
    }
    multiply_rest<T, DW, TILE, TILE>(products, p, reinterpret_cast<v4u*>(lds8), j0, k0, s_rest, s_last);

    __syncthreads();
    const __amdgpu_buffer_rsrc_t none = __builtin_amdgcn_make_buffer_rsrc((void*)nullptr, 0, 0, 0x00020000);
    store_results<O, kF, kF, kF == 1 ? 64 : 128>(products.acc, out + part * p.part_stride, p.ldo, j0 + wj, p.J, k0 + wk, p.K, none, lds8 + wave * 4096);
#endif
}

}  // namespace mx
}  // namespace sparq

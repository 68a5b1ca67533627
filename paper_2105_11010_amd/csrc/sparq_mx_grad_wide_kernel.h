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
// begins: of 128 every step waits for all loads behind its barrier, which bf16 hides in part by a second workgroup on the CU and fp16 and fp32, whose LDS
// leaves no room for one, do not; of 64 that wait is what a small layer's time is, 515 x 771 x 577 7.7 and 8.4 us of 12 or 13 steps.  dw in 256 x 256 keeps 105
// scalar registers in lanes of vector ones, about 110 moves a step between its matrix instructions.
#pragma once
#include <type_traits>

#include "sparq_mx_grad_kernel.h"

namespace sparq {
namespace mx {

template <int TILE> inline constexpr int kWideBytes = kGradStep * TILE * 2;       // of one side's tile

template <class T, int TILE> inline constexpr int kWideLds = 2 * (kParts<T> + 1) * kWideBytes<TILE>;
template <class T, int TILE> inline constexpr int kWidePerCu = kWideLds<T, TILE> < 40 * 1024 ? 4 : 160 * 1024 / kWideLds<T, TILE>;
template <class T, class O, bool DW, int TILE>
__global__ __launch_bounds__(kGradThreads, (kWidePerCu<T, TILE>)) void grad_wide_kernel(O* __restrict__ out, const GradParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int P = kParts<T>;                             // of dy, a tile each
    constexpr int kF = TILE / 64, kSlots = P * kF * kF;      // 32 x 32 results along a side; matrix instructions a quarter
    constexpr int kRow = TILE * 2;                           // bytes of a tile's row
    constexpr int kRun = TILE == 64 ? 16 : 32, kRuns = TILE * kGradStep / kGradThreads / kRun;      // a thread's runs of V's values
    constexpr int kUnits = TILE / 32;                        // and of eight values of dy, as many as V's pieces of eight
    constexpr int kPieces = kRun / 8;                        // a run
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
            const uint32_t n = blockIdx.x - tiles, across = (uint32_t)((p.J + Sums::kColumns - 1) / Sums::kColumns), slab = n / across;
            const int64_t begin = slab * p.slab, end = begin + p.slab < p.R ? begin + p.slab : p.R;
            if (blockIdx.y == 0)
                Sums::run(static_cast<const T*>(p.dy), p.lddy, begin, end, (int)p.J, (int)(n % across) * Sums::kColumns, p.column_sums + slab * p.J,
                          reinterpret_cast<float*>(lds8));
            return;
        }
    }
    uint32_t tj, tk;
    tile_of(blockIdx.x, p.tiles_j, p.tiles_k, tj, tk);
    const int64_t j0 = (int64_t)tj * TILE;
    const int k0 = (int)tk * TILE;
    const int64_t s_begin = (int64_t)blockIdx.y * p.steps_per_part, s_all = (p.R + kGradStep - 1) / kGradStep;
    const int64_t s_end = s_begin + p.steps_per_part < s_all ? s_begin + p.steps_per_part : s_all, s_fast = p.s_whole < s_end ? p.s_whole : s_end;
    Products<P, TILE, TILE> products;
    const int wj = products.wj, wk = products.wk;

    if (s_begin < s_fast) {
        // ---- dy: a thread has kUnits runs of eight values: of every eighth or 16th row (DW) or of rows 32 i + t / 8, 64 r each
        constexpr int kAcross = TILE / 8, kRowsAtOnce = kGradThreads / kAcross;
        constexpr int kSize = sizeof(T), kKept = 2 * kSize;
        uint32_t kept[kUnits][kKept];
        uint32_t dy_at[DW ? 1 : kUnits];
        if constexpr (DW) {
            int64_t j = j0 + 8 * (t % kAcross);
            j = j < p.J ? j : j0;                            // (columns past the last one make results that are not stored)
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
        uint32_t raw[kRuns][kWords], scale[kRuns];
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
        auto advance = [&]() __attribute__((always_inline)) {
            dy_from += left > 0 ? dy_step : 0;
            codes_from += left > 0 ? codes_step : 0;
            scales_from += left > 0 ? scales_step : 0;
            --left;
        };
        const auto buffer = [](const uint8_t* from) __attribute__((always_inline)) { return __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, 0x7FFFFFFF, 0x00020000); };
        auto load_dy = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int h = 0; h < kKept / 4; ++h) {
                const v4u w = __builtin_amdgcn_raw_buffer_load_b128(buffer(dy_from), dy_at[DW ? 0 : i], (DW ? (int)(kRowsAtOnce * i * p.lddy * kSize) : 0) + 16 * h, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) kept[i][4 * h + e] = w[e];
            }
        };
        auto load_v = [&](int run) __attribute__((always_inline)) {
            if constexpr (kWords == 2) {
                const v2u w = __builtin_amdgcn_raw_buffer_load_b64(buffer(codes_from), v_at, 0, 0);
                raw[run][0] = w[0];
                raw[run][1] = w[1];
            }
#pragma unroll
            for (int h = 0; h < kWords / 4; ++h) {
                const v4u w = __builtin_amdgcn_raw_buffer_load_b128(buffer(codes_from), v_at, (int)(32 * run * p.code_pitch) + 16 * h, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) raw[run][4 * h + e] = w[e];
            }
            scale[run] = __builtin_amdgcn_raw_buffer_load_b8(buffer(scales_from), scale_at, (int)(32 * run * p.scale_pitch), 0);
        };
        // A tile's row is permuted in its 16-byte units, which keeps both the turning reads and the writes apart in the banks.
        const auto permuted = [](int row, int chunk) __attribute__((always_inline)) {
            if constexpr (TILE == 64) return row * kRow + ((chunk ^ (row & 2 ? 5 : 0)) << 4);
            else return row * kRow + ((chunk ^ (chunk >> 4 & 1) ^ ((row & 3) << 2 | (row >> 2 & 3))) << 4);
        };
        auto write_dy = [&](uint8_t* tile, int i) __attribute__((always_inline)) {
            uint8_t* const to = tile + (DW ? permuted(kRowsAtOnce * i + t / kAcross, t % kAcross) : 16 * unit_at(32 * i + (t >> 3), t & 7));
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
        auto decode = [&](int piece, int e) __attribute__((always_inline)) {
            const int run = piece / kPieces, at = piece % kPieces;
            if (at == 0 && e == 0) unit = DW ? unit8_of(scale[run]) : scale_operand(scale[run]);
            if constexpr (DW) {
                const uint32_t w = raw[run][2 * at + (e >> 1)] >> (16 * (e & 1));
                decoded[e] = pack_bf16((float)(int8_t)w * unit, (float)(int8_t)(w >> 8) * unit);
            } else {
                decoded[e] = pair4_of(raw[run][at], unit, e);
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
        auto between = [&](auto now_, int q, int i) __attribute__((always_inline)) {
            constexpr int now = decltype(now_)::value;
            const int part = (q + 1) & 3, first = part * kUnits / 4, parts = 8 * ((part + 1) * kUnits / 4 - first);      // pieces this quarter, eight parts each
            if (q == 3 && i == 0) advance();
            const int read_from = q == 3 ? now ^ 1 : now, write_to = q == 3 ? now : now ^ 1;
            for (int n = i * kReads / kSlots; n < (i + 1) * kReads / kSlots; ++n) read(set[(q + 1) & 1], lds_dy + read_from * P * kBytes, lds_v + read_from * kBytes, (q + 1) & 3, n);
            for (int u = i * parts / kSlots; u < (i + 1) * parts / kSlots; ++u) {
                const int piece = first + u / 8;
                if (u % 2 == 0) decode(piece, u % 8 / 2);
                if (u % 8 == 7) {
                    write_v(lds_v + write_to * kBytes, piece);
                    if (piece % kPieces == kPieces - 1) load_v(piece / kPieces);
                }
                if (u % 8 == 3) {
                    write_dy(lds_dy + write_to * P * kBytes, piece);
                    load_dy(piece);
                }
            }
        };
        auto barrier = [&]() __attribute__((always_inline)) {
            __builtin_amdgcn_s_waitcnt(vmcnt_and_lds(63));
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        auto step = [&](auto now) __attribute__((always_inline)) {
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
                            between(now, q, (x * P + n) * kF + y);
                            __builtin_amdgcn_sched_barrier(0);
                        }
            }
        };

#pragma unroll
        for (int i = 0; i < kUnits; ++i) load_dy(i);
#pragma unroll
        for (int i = 0; i < kRuns; ++i) load_v(i);
        advance();
        static_assert(kUnits == kPieces * kRuns, "a unit of dy to a piece of V");
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) decode(i, e);
            write_v(lds_v, i);
            if (i % kPieces == kPieces - 1) load_v(i / kPieces);
            write_dy(lds_dy, i);
            load_dy(i);
        }
        barrier();
        // as if the last quarter of a step before the first
#pragma unroll
        for (int i = 0; i < kSlots; ++i) between(std::integral_constant<int, 1>{}, 3, i);
        for (int64_t s = s_begin; s < s_fast; s += 2) {
            step(std::integral_constant<int, 0>{});
            if (s + 1 < s_fast) step(std::integral_constant<int, 1>{});
        }
    }
    multiply_rest<T, DW, TILE, TILE>(products, p, reinterpret_cast<v4u*>(lds8), j0, k0, s_begin < s_fast ? s_fast : s_begin, s_end);

    __syncthreads();
    const __amdgpu_buffer_rsrc_t none = __builtin_amdgcn_make_buffer_rsrc((void*)nullptr, 0, 0, 0x00020000);
    store_results<O, kF, kF, kF == 1 ? 64 : 128>(products.acc, out + blockIdx.y * p.part_stride, p.ldo, j0 + wj, p.J, k0 + wk, p.K, none, lds8 + wave * 4096);
#endif
}

}  // namespace mx
}  // namespace sparq

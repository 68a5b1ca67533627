// The product of 4-bit operands on v_mfma_scale_f32_32x32x64_f8f6f4: y[m][n] = sum_k W[n][k] A[m][k].
// A lane feeds 32 neighbouring values of one row, which is one block, and the block's scale; the weights are the first operand, so
// that a lane ends with four neighbouring n of one m.
// A workgroup of four wavefronts makes TM x TN results in steps of 128 values (64 bytes of a row), a wavefront a quarter of them, and
// takes one tile after the other.  Codes go from memory to LDS without passing registers, three to four steps ahead -- across a tile's end into the next
// one's -- into four buffers in turn; scales likewise, 16 bytes of a row (four steps) at a time, into two.  One barrier a step.
// Steps come in fours: past a row's end the scales are zeros, 2^-127 each, and what codes add there is 2^-254 of something: nothing
// in fp32.
// 8192 x 8192 x 4096 takes 160-180 us (3.1-3.4 PF; 8192 x 4096 x 4096 86, 4096^3 47).  The matrix instructions alone would take 61 at the clock they
// reach without data; with data the card's power sets the clock (1.8 GHz), and without the loads the kernel takes 122.  What is between is the
// caches' requests, 64 bytes each, 0.69 of one a channel and cycle, and the first steps of every 256 x 256 tile: 20 (fp32 results) or 26 registers, LDS
// addresses most of them, lie in scratch memory there, the compiler makes a tile's first four steps a copy of their own that reads them back, and
// each such read is waited for with all loads before it, seven times a tile (of 8192 x 8192 x 1024, 68 us, that is half of the steps).  (Loads of 128 bytes, two steps at a time, halve those but leave one pair of steps ahead in
// LDS: 202 us where this took 179.)
#pragma once
#include <type_traits>
#include <utility>

#include "sparq_mx_store.h"

namespace sparq {
namespace mx {

struct GemmParams {
    const uint8_t *a, *as, *w, *ws;
    const float* bias;
    int64_t M, ldy, part_stride;         // results of a part of the reduction lie part_stride apart
    uint32_t code_pitch, scale_pitch;
    int32_t N;
    uint32_t tiles_m, tiles_n, items;    // items: tiles x parts
    int32_t steps, steps_per_part;       // of 128 values, multiples of four
};

constexpr int kGemmThreads = 256;
constexpr int kGemmMaxK = 1 << 23;       // a tile's rows stay inside 32-bit offsets

// Bytes of a row of results that a wavefront turns at a time: what is left of a CU's LDS, or of half of it.
template <int TILE> constexpr int kTurnRow = TILE == 256 ? 128 : 64;
template <int TILE> constexpr int kGemmLds = 4 * 2 * TILE * 64 + 2 * 2 * TILE * 16 + 4 * 32 * kTurnRow<TILE>;

template <int N> using Const = std::integral_constant<int, N>;

template <class O, int TM, int TN>
__global__ __launch_bounds__(kGemmThreads) void gemm_kernel(O* __restrict__ y, const GemmParams p) {
#if defined(__HIP_DEVICE_COMPILE__)                          // (the host's pass does not know loads of 16 bytes to LDS, and leaves the kernel out)
    constexpr int FM = TM / 64, FN = TN / 64;                // 32 x 32 results a wavefront makes along either side
    constexpr int kBuffer = (TM + TN) * 64, kScaleBuffer = (TM + TN) * 16;
    constexpr int kLoads = (TM + TN) / 64;                   // of a step, a wavefront
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];       // four buffers of codes, two of scales, a piece of results each
    uint8_t* const lds_scales = lds + 4 * kBuffer;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, g = lane >> 5;
    const int wm = (wave >> 1) * (TM / 2), wn = (wave & 1) * (TN / 2);

    // A tile of results and its share of the reduction.
    struct Item {
        int64_t m0;
        int n0, s_begin, steps;
        uint32_t part;
    };
    auto item_of = [&](uint32_t id) __attribute__((always_inline)) {
        Item it;
        uint32_t tm, tn;
        it.part = p.tiles_m * p.tiles_n == p.items ? 0 : id / (p.tiles_m * p.tiles_n);
        tile_of(id - it.part * p.tiles_m * p.tiles_n, p.tiles_m, p.tiles_n, tm, tn);
        it.m0 = (int64_t)tm * TM;
        it.n0 = (int)tn * TN;
        it.s_begin = it.part * p.steps_per_part;
        it.steps = p.steps - it.s_begin < p.steps_per_part ? p.steps - it.s_begin : p.steps_per_part;
        return it;
    };
    // Where the next loads come from.  Rows past the last one lie past the buffers' ends and come as zeros.
    __amdgpu_buffer_rsrc_t ra, rw, ras, rws;
    int load_step;
    auto open = [&](const Item& it) __attribute__((always_inline)) {
        const uint32_t rows_m = p.M - it.m0 < TM ? (uint32_t)(p.M - it.m0) : TM, rows_n = p.N - it.n0 < TN ? p.N - it.n0 : TN;
        const auto buffer = [](const uint8_t* base, uint32_t rows, uint32_t pitch) __attribute__((always_inline)) {
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, (int)(rows * pitch), 0x00020000);
        };
        ra = buffer(p.a + it.m0 * p.code_pitch, rows_m, p.code_pitch);
        rw = buffer(p.w + (int64_t)it.n0 * p.code_pitch, rows_n, p.code_pitch);
        ras = buffer(p.as + it.m0 * p.scale_pitch, rows_m, p.scale_pitch);
        rws = buffer(p.ws + (int64_t)it.n0 * p.scale_pitch, rows_n, p.scale_pitch);
        load_step = it.s_begin;
    };
    // One load brings 16 rows: lane l row l / 4 and its 16-byte unit (l % 4) ^ (row / 4 % 4), which lands in place l % 4: the
    // permutation keeps the operands' reads, 32 rows at one place of the reduction, out of each other's banks.
    // (Rows are in the offset that is checked against the buffer's end; the step is in the other, and stays inside a row.)
    uint32_t from[TM / 64];
#pragma unroll
    for (int i = 0; i < TM / 64; ++i) from[i] = (uint32_t)(64 * i + wave * 16 + (lane >> 2)) * p.code_pitch + (((lane & 3) ^ (lane >> 4)) << 4);
    const uint32_t scales_from = (uint32_t)(wave * 64 + lane) * p.scale_pitch;

    auto load_scales = [&](int buf) __attribute__((always_inline)) {
        uint8_t* to = lds_scales + buf * kScaleBuffer + wave * 1024;
        if constexpr (TM == 256) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ras, (LdsPtr)to, 16, scales_from, (load_step >> 2) * 16, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rws, (LdsPtr)(to + TM * 16), 16, scales_from, (load_step >> 2) * 16, 0, 0);
        } else if (wave < TM / 64) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ras, (LdsPtr)to, 16, scales_from, (load_step >> 2) * 16, 0, 0);
        } else if (wave < TM / 32) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rws, (LdsPtr)to, 16, scales_from - TM * p.scale_pitch, (load_step >> 2) * 16, 0, 0);
        }
    };
    // load i of a step's kLoads; steps past the row's last one bring that one's codes again
    auto load = [&](int buf, int i) __attribute__((always_inline)) {
        const uint32_t col = (uint32_t)load_step * 64 < p.code_pitch ? load_step * 64 : p.code_pitch - 64;
        uint8_t* to = lds + buf * kBuffer + wave * 1024 + i * 4096;
        if (i < TM / 64) __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (LdsPtr)to, 16, from[i], col, 0, 0);
        else __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (LdsPtr)to, 16, from[i - TM / 64], col, 0, 0);
    };
    static_assert(TM == TN && (TM == 256 || TM == 128 || TM == 64), "rows of scales: one load a wavefront and operand, or one a wavefront at most");

    struct Operands {
        v4i a[FM], w[FN];
    };
    struct Scales {
        int a[FM], w[FN];
    };
    const int at_m = (wm + c) * 64, at_n = TM * 64 + (wn + c) * 64, x = (c >> 2) & 3;
    constexpr int kReads = FM + FN;
    // operand i of half h of the step in a buffer: values 64 h + 32 g and on
    auto read = [&](Operands& o, int buf, int h, int i) __attribute__((always_inline)) {
        const uint8_t* from = lds + buf * kBuffer + (((2 * h + g) ^ x) << 4);
        if (i < FM) o.a[i] = *reinterpret_cast<const v4i*>(from + at_m + i * 2048);
        else o.w[i - FM] = *reinterpret_cast<const v4i*>(from + at_n + (i - FM) * 2048);
    };
    // a step's four scales of a row; shifted, the lane's own are in bytes 0 (first half) and 2
    auto read_scale = [&](Scales& o, int buf, int place, int i) __attribute__((always_inline)) {
        const uint8_t* from = lds_scales + buf * kScaleBuffer + place * 4;
        if (i < FM) o.a[i] = *reinterpret_cast<const int*>(from + (wm + c + 32 * i) * 16);
        else o.w[i - FM] = *reinterpret_cast<const int*>(from + (TM + wn + c + 32 * (i - FM)) * 16);
    };
    auto shift_scale = [&](Scales& o, int i) __attribute__((always_inline)) {
        int& s = i < FM ? o.a[i] : o.w[i - FM];
        s = (int)((uint32_t)s >> (8 * g));
    };

    v16f acc[FN][FM];
    // The products of half a step; after the i-th matrix instruction comes what between(i) issues.  One wavefront a SIMD has nobody else to
    // fill the time an instruction runs, so the order is fixed here.
    auto multiply = [&](const Operands& o, const Scales& s, auto half, auto&& between) __attribute__((always_inline)) {
        constexpr int kByte = decltype(half)::value * 2;
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                const v8i w = __builtin_shufflevector(o.w[i], o.w[i], 0, 1, 2, 3, -1, -1, -1, -1), a = __builtin_shufflevector(o.a[j], o.a[j], 0, 1, 2, 3, -1, -1, -1, -1);
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, a, acc[i][j], 4, 4, kByte, s.w[i], kByte, s.a[j]);
                between(i * FM + j);
                __builtin_amdgcn_sched_barrier(0);
            }
    };

    Operands first, second;
    Scales scales, next_scales;
    int groups = 0;                                          // of four steps before this item
    // Step s of the item, in buffer place = s % 4; the last reads are of step s + 1, be that the next item's first.
    auto step = [&](int s, auto place_, const Item& it, uint32_t next_id) __attribute__((always_inline)) {
        constexpr int place = decltype(place_)::value, kAll = FM * FN;
        const int group = (groups + (s >> 2)) & 1;           // which buffer holds the scales
        // Reads and loads are spread evenly: a read of 1 KB takes LDS as long for four wavefronts as an instruction runs, a load
        // the address unit twice as long.
        constexpr int kHalfLoads = kLoads / 2;
        const auto share = [](int i, int n) { return std::pair<int, int>{i * n / kAll, (i + 1) * n / kAll}; };     // of n, after instruction i
        multiply(first, scales, Const<0>{}, [&](int i) __attribute__((always_inline)) {
            const auto reads = share(i, kReads), loads = share(i, kHalfLoads);
            for (int n = reads.first; n < reads.second; ++n) read(second, place, 1, n);
            for (int n = loads.first; n < loads.second; ++n) load((place + 3) & 3, kHalfLoads + n);
        });
        ++load_step;
        // This step's buffer has been read, here and, past the barrier, in the other wavefronts: it takes step s + 4.  And step s + 1 is
        // there: all but the loads of steps s + 2 and s + 3 are done.  (An item's first two steps: they were waited for before it began.)
        if (place >= 2 || s >= 4) __builtin_amdgcn_s_waitcnt(vmcnt_and_lds(2 * kLoads));
        else __builtin_amdgcn_s_waitcnt(vmcnt_and_lds(63));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (place == 0 && s + 4 == it.steps) {               // from here on the loads are the next item's (none: the last one's again, unread)
            if (next_id < p.items) open(item_of(next_id));
            else load_step = it.s_begin;
        }
        multiply(second, scales, Const<1>{}, [&](int i) __attribute__((always_inline)) {
            const auto reads = share(i, kReads), loads = share(i, kHalfLoads), early = share(2 * i, kReads), late = share(2 * i + 1, kReads);
            const int last = early.first + (late.second - early.first), scale_buf = place == 3 ? group ^ 1 : group;
            for (int n = early.first; n < last && n < kReads; ++n) read_scale(next_scales, scale_buf, (place + 1) & 3, n);
            for (int n = reads.first; n < reads.second; ++n) read(first, (place + 1) & 3, 0, n);
            if (place == 0 && i == 0) load_scales(group ^ 1);
            for (int n = loads.first; n < loads.second; ++n) load(place, n);
            if (kAll == 1) {
                for (int n = 0; n < kReads; ++n) shift_scale(next_scales, n);
            } else if (2 * i >= kAll)
                for (int n = early.first - kReads; n < last - kReads; ++n) shift_scale(next_scales, n);
        });
        scales = next_scales;
    };

    uint32_t id = blockIdx.x;
    open(item_of(id));
    load_scales(0);
#pragma unroll
    for (int b = 0; b < 3; ++b) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load(b, i);
        ++load_step;
    }
#pragma unroll
    for (int i = 0; i < kLoads / 2; ++i) load(3, i);
    __builtin_amdgcn_s_waitcnt(vmcnt(kLoads / 2));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < kReads; ++i) {
        read(first, 0, 0, i);
        read_scale(scales, 0, 0, i);
        shift_scale(scales, i);
    }
    for (; id < p.items; id += gridDim.x) {
        const Item it = item_of(id);
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[i][j] = v16f{};
        for (int s = 0; s < it.steps; s += 4) {
            step(s, Const<0>{}, it, id + gridDim.x);
            step(s + 1, Const<1>{}, it, id + gridDim.x);
            step(s + 2, Const<2>{}, it, id + gridDim.x);
            step(s + 3, Const<3>{}, it, id + gridDim.x);
        }
        groups += it.steps >> 2;
        // The next item's first three steps are there before the results' stores queue up behind them.
        __builtin_amdgcn_s_waitcnt(vmcnt(kLoads / 2));
        const __amdgpu_buffer_rsrc_t bias = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p.bias), 0, p.bias ? p.N * 4 : 0, 0x00020000);
        store_results<O, FN, FM, kTurnRow<TM>>(acc, y + it.part * p.part_stride, p.ldy, it.m0 + wm, p.M, it.n0 + wn, p.N, bias,
                                               lds + 4 * kBuffer + 2 * kScaleBuffer + wave * 32 * kTurnRow<TM>);
    }
    __builtin_amdgcn_s_waitcnt(vmcnt(0));                    // nothing is on its way to LDS when the wavefront ends
#endif
}

}  // namespace mx
}  // namespace sparq

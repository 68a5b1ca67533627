// The product of 4-bit operands on v_mfma_scale_f32_32x32x64_f8f6f4: y[m][n] = sum_k W[n][k] A[m][k].
// A lane feeds 32 neighbouring values of one row, which is one block, and the block's scale; the weights are the first operand, so
// that a lane ends with four neighbouring n of one m.
// A workgroup of four wavefronts makes TM x TN results in steps of 128 values (64 bytes of a row), a wavefront a quarter of them.
// Codes go from memory to LDS without passing registers, three steps ahead, into four buffers in turn; scales likewise, 16 bytes of
// a row (four steps) at a time, into two.  One barrier a step.
#pragma once
#include <type_traits>

#include "sparq_mx_store.h"

namespace sparq {
namespace mx {

struct GemmParams {
    const uint8_t *a, *as, *w, *ws;
    const float* bias;
    int64_t M, ldy, part_stride;         // results of a part of the reduction lie part_stride apart
    uint32_t code_pitch, scale_pitch;
    int32_t N;
    uint32_t tiles_m, tiles_n;
    int32_t steps, steps_per_part;       // of 128 values; the latter a multiple of four
};

constexpr int kGemmThreads = 256;
constexpr int kGemmMaxK = 1 << 23;       // a tile's rows stay inside 32-bit offsets

typedef __attribute__((address_space(3))) void* LdsPtr;
// The wait instruction's operand for at most n loads on their way.
constexpr int vmcnt(int n) { return (n & 15) | (n >> 4) << 14 | 0x0F70; }

template <int N> using Const = std::integral_constant<int, N>;

template <class O, int TM, int TN>
__global__ __launch_bounds__(kGemmThreads) void gemm_kernel(O* __restrict__ y, const GemmParams p) {
#if defined(__HIP_DEVICE_COMPILE__)                          // (the host's pass does not know loads of 16 bytes to LDS, and leaves the kernel out)
    constexpr int FM = TM / 64, FN = TN / 64;                // 32 x 32 results a wavefront makes along either side
    constexpr int kBuffer = (TM + TN) * 64, kScaleBuffer = (TM + TN) * 16;
    constexpr int kLoads = (TM + TN) / 64;                   // of a step, a wavefront
    static_assert(4 * kTurnBytes<O, FN * 32> <= 4 * kBuffer + 2 * kScaleBuffer, "results are turned where the operands were");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];                         // four buffers of codes, two of scales
    uint8_t* const lds_scales = lds + 4 * kBuffer;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, g = lane >> 5;
    const int wm = (wave >> 1) * (TM / 2), wn = (wave & 1) * (TN / 2);
    uint32_t tm, tn;
    tile_of(blockIdx.x, p.tiles_m, p.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * TM;
    const int n0 = (int)tn * TN;
    const int s_begin = blockIdx.y * p.steps_per_part, s_end = s_begin + p.steps_per_part < p.steps ? s_begin + p.steps_per_part : p.steps;

    // Rows past the last one lie past the buffers' ends and come as zeros.
    const uint32_t rows_m = p.M - m0 < TM ? (uint32_t)(p.M - m0) : TM, rows_n = p.N - n0 < TN ? p.N - n0 : TN;
    const auto buffer = [](const uint8_t* base, uint32_t rows, uint32_t pitch) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, (int)(rows * pitch), 0x00020000);
    };
    const __amdgpu_buffer_rsrc_t ra = buffer(p.a + m0 * p.code_pitch, rows_m, p.code_pitch), rw = buffer(p.w + (int64_t)n0 * p.code_pitch, rows_n, p.code_pitch);
    const __amdgpu_buffer_rsrc_t ras = buffer(p.as + m0 * p.scale_pitch, rows_m, p.scale_pitch), rws = buffer(p.ws + (int64_t)n0 * p.scale_pitch, rows_n, p.scale_pitch);
    // One load brings 16 rows: lane l row l / 4 and its 16-byte unit (l % 4) ^ (row / 2 % 4), which lands in place l % 4: the
    // permutation keeps the operands' reads, 32 rows at one place of the reduction, out of each other's banks.
    // (Rows are in the offset that is checked against the buffer's end; the step is in the other, and stays inside a row.)
    uint32_t from[TM / 64];
#pragma unroll
    for (int i = 0; i < TM / 64; ++i) from[i] = (uint32_t)(64 * i + wave * 16 + (lane >> 2)) * p.code_pitch + (((lane & 3) ^ ((lane >> 3) & 3)) << 4);
    const uint32_t scales_from = (uint32_t)(wave * 64 + lane) * p.scale_pitch;

    auto load = [&](int s, int buf, int scale_buf, bool with_scales) __attribute__((always_inline)) {
        s = s < s_end ? s : s_end - 1;                       // (past the end: the last step again, into a buffer nobody reads)
        if (with_scales) {
            uint8_t* to = lds_scales + scale_buf * kScaleBuffer + wave * 1024;
            if (TM == 256 || wave < TM / 64) __builtin_amdgcn_raw_ptr_buffer_load_lds(ras, (LdsPtr)to, 16, scales_from, (s >> 2) * 16, 0, 0);
            else __builtin_amdgcn_raw_ptr_buffer_load_lds(rws, (LdsPtr)(to), 16, scales_from - TM * p.scale_pitch, (s >> 2) * 16, 0, 0);
            if (TM == 256) __builtin_amdgcn_raw_ptr_buffer_load_lds(rws, (LdsPtr)(to + TM * 16), 16, scales_from, (s >> 2) * 16, 0, 0);
        }
        uint8_t* to = lds + buf * kBuffer + wave * 1024;
#pragma unroll
        for (int i = 0; i < TM / 64; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (LdsPtr)(to + i * 4096), 16, from[i], s * 64, 0, 0);
#pragma unroll
        for (int i = 0; i < TN / 64; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (LdsPtr)(to + TM * 64 + i * 4096), 16, from[i], s * 64, 0, 0);
    };
    static_assert(TM == TN && (TM == 256 || TM == 128), "rows of scales: one load a wavefront and operand, or one a wavefront");

    struct Operands {
        v4i a[FM], w[FN];
    };
    struct Scales {
        int a[FM], w[FN];
    };
    const int at_m = (wm + c) * 64, at_n = TM * 64 + (wn + c) * 64, x = (c >> 1) & 3;
    // half h of the step in a buffer: values 64 h + 32 g and on
    auto read = [&](Operands& o, int buf, int h) __attribute__((always_inline)) {
        const uint8_t* from = lds + buf * kBuffer + (((2 * h + g) ^ x) << 4);
#pragma unroll
        for (int f = 0; f < FM; ++f) o.a[f] = *reinterpret_cast<const v4i*>(from + at_m + f * 2048);
#pragma unroll
        for (int f = 0; f < FN; ++f) o.w[f] = *reinterpret_cast<const v4i*>(from + at_n + f * 2048);
    };
    // a step's four scales of a row, the lane's own in bytes 0 (first half) and 2
    auto read_scales = [&](Scales& o, int buf, int place) __attribute__((always_inline)) {
        const uint8_t* from = lds_scales + buf * kScaleBuffer + place * 4;
#pragma unroll
        for (int f = 0; f < FM; ++f) o.a[f] = *reinterpret_cast<const uint32_t*>(from + (wm + c + 32 * f) * 16) >> (8 * g);
#pragma unroll
        for (int f = 0; f < FN; ++f) o.w[f] = *reinterpret_cast<const uint32_t*>(from + (TM + wn + c + 32 * f) * 16) >> (8 * g);
    };

    v16f acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = v16f{};
    auto multiply = [&](const Operands& o, const Scales& s, auto half) __attribute__((always_inline)) {
        constexpr int kByte = decltype(half)::value * 2;
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                const v8i w = __builtin_shufflevector(o.w[i], o.w[i], 0, 1, 2, 3, -1, -1, -1, -1), a = __builtin_shufflevector(o.a[j], o.a[j], 0, 1, 2, 3, -1, -1, -1, -1);
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, a, acc[i][j], 4, 4, kByte, s.w[i], kByte, s.a[j]);
            }
    };

    Operands first, second;
    Scales scales, next_scales;
    // Step s from buffer place (s % 4): what is read in it arrived a step ago, and its last reads are of step s + 1.
    auto step = [&](int s, auto place_) __attribute__((always_inline)) {
        constexpr int place = decltype(place_)::value;
        const int group = (s - s_begin) >> 2;
        // Step s + 1 is there: all but the loads of step s + 2 are done, here and, past the barrier, in the other wavefronts; and
        // these have used what they read of step s - 1, whose buffer takes step s + 3.
        __builtin_amdgcn_s_waitcnt(vmcnt(kLoads));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        load(s + 3, (place + 3) & 3, (group + 1) & 1, place == 1);
        read(second, place, 1);
        multiply(first, scales, Const<0>{});
        read(first, (place + 1) & 3, 0);
        read_scales(next_scales, (place == 3 ? group + 1 : group) & 1, (place + 1) & 3);
        multiply(second, scales, Const<1>{});
        scales = next_scales;
    };
    if (s_begin < s_end) {
        load(s_begin, 0, 0, true);
        load(s_begin + 1, 1, 0, false);
        load(s_begin + 2, 2, 0, false);
        __builtin_amdgcn_s_waitcnt(vmcnt(2 * kLoads));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read(first, 0, 0);
        read_scales(scales, 0, 0);
        for (int s = s_begin; s < s_end; s += 4) {
            step(s, Const<0>{});
            if (s + 1 < s_end) step(s + 1, Const<1>{});
            if (s + 2 < s_end) step(s + 2, Const<2>{});
            if (s + 3 < s_end) step(s + 3, Const<3>{});
        }
        __builtin_amdgcn_s_waitcnt(vmcnt(0));                // nothing is on its way to LDS when the wavefront ends
    }

    __syncthreads();
    const __amdgpu_buffer_rsrc_t bias = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p.bias), 0, p.bias ? p.N * 4 : 0, 0x00020000);
    store_results<O, FN, FM>(acc, y + blockIdx.y * p.part_stride, p.ldy, m0 + wm, p.M, n0 + wn, p.N, bias, lds + wave * kTurnBytes<O, FN * 32>);
#endif
}

}  // namespace mx
}  // namespace sparq

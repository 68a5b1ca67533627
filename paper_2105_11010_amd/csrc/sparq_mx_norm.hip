// Layer norm with an 8-bit checkpoint of its input, and its backward pass from that (include/sparq_mx.h).
#include <type_traits>

#include "sparq_mx_common.h"

namespace sparq {
namespace mx {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

struct NormParams {
    int64_t ldx, ldy, code_pitch, scale_pitch, rows;
    int32_t K, K128;
    float eps, inv_K;
};

// The wavefront's sum in every lane: within rows of sixteen lanes by moves, between them by swaps, none through LDS.
__device__ __forceinline__ float wave_sum(float v) {
    const auto moved = [](float x, auto control) __attribute__((always_inline)) {
        return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), decltype(control)::value, 0xF, 0xF, true));
    };
    v += moved(v, std::integral_constant<int, 0xB1>{});      // lane ^ 1
    v += moved(v, std::integral_constant<int, 0x4E>{});      // lane ^ 2
    v += moved(v, std::integral_constant<int, 0x141>{});     // the other four of eight
    v += moved(v, std::integral_constant<int, 0x140>{});     // the other eight of sixteen
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// Sum over the wavefronts that share a row.  Two buffers in turn: a wavefront may write the next sum while others still
// read this one, but not the one after that before they have passed the barrier between.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float* shared, int& turn) {
    v = wave_sum(v);
    if constexpr (WAVES == 1) return v;
    float* at = shared + turn * WAVES;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = at[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) s += at[i];
    return s;
}
// A lane's eight values of a row in registers, loaded without a branch: from + 0..7, the last eight of the row where its own would reach past
// the end.  WHOLE: rows of whole eights; else the first `skip` of them are the lane's before it's.
struct Place {
    int col, from, skip;
    bool inside;
};
template <bool WHOLE>
__device__ __forceinline__ Place place_of(int col, int K) {
    Place p;
    p.col = col;
    p.inside = col < K;
    p.from = col < K - 8 ? col : K - 8;
    p.skip = WHOLE || !p.inside ? 0 : col - p.from;
    return p;
}
// own(i): element i is the lane's
template <bool WHOLE>
__device__ __forceinline__ bool own(const Place& p, int i) { return p.inside && (WHOLE || i >= p.skip); }
template <bool WHOLE, bool NT = false, class T>
__device__ __forceinline__ void store_own(T* row, const Place& p, const float (&v)[8]) {
    if (!p.inside) return;
    if (WHOLE || p.skip == 0) store8<NT>(row + p.from, v);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= p.skip) row[p.from + i] = (T)v[i];
    }
}

// The lane's own elements to the front, zeros behind them: a checkpoint's codes lie where the row's eights begin.
__device__ __forceinline__ void first_own(const Place& p, float (&v)[8]) {
#pragma unroll
    for (int by = 4; by; by >>= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p.skip & by ? (i + by < 8 ? v[i + by] : 0.0f) : v[i];
}

// WAVES wavefronts take a row of at least eight, CHUNKS x 8 values a lane, which stay in registers from the load to the result: one
// pass over memory, the mean first and the squares of what differs from it second.  As many workgroups as have room go through the rows,
// gamma and beta in registers and the next row on its way while this one is summed.  Bound by memory and, for each row, by the two sums one after
// the other: 16384 x 4096 bf16 with checkpoint 60 us (5.6 TB/s), 65536 x 1024 66, fp32 117.
template <class T, int WAVES, int CHUNKS, bool WHOLE, int STREAMING>
__global__ __launch_bounds__(kThreads) void norm_kernel(const T* __restrict__ x, const float* __restrict__ gamma,
                                                        const float* __restrict__ beta, T* __restrict__ y, float* __restrict__ mean_out,
                                                        float* __restrict__ rstd_out, uint8_t* __restrict__ codes,
                                                        uint8_t* __restrict__ scales, const NormParams p) {
    __shared__ float shared[2 * WAVES];
    constexpr int kPerBlock = kWaves / WAVES, kSpan = WAVES * 512;
    const int wave = threadIdx.x >> 6, t = threadIdx.x & (WAVES * 64 - 1), lane = threadIdx.x & 63;
    const int64_t first = (int64_t)blockIdx.x * kPerBlock + (WAVES == 1 ? wave : 0), stride = (int64_t)gridDim.x * kPerBlock;
    if (first >= p.rows) return;                             // (whole workgroups where they share a row)
    int turn = 0;
    Raw8<T> raw[CHUNKS];
    float g[CHUNKS][8], b[CHUNKS][8];
    Place at[CHUNKS];
    auto fetch = [&](int64_t row) __attribute__((always_inline)) {
        row = row < p.rows ? row : p.rows - 1;               // (past the end: a row again, for nobody)
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) load_raw<STREAMING == kAll>(x + row * p.ldx + at[c].from, raw[c]);
    };
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) at[c] = place_of<WHOLE>(c * kSpan + 8 * t, p.K);
    fetch(first);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        load8(gamma + at[c].from, g[c]);
        if (beta) load8(beta + at[c].from, b[c]);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) b[c][i] = 0.0f;
        }
    }
    for (int64_t row = first; row < p.rows; row += stride) {
        float v[CHUNKS][8], sum = 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            values_of(raw[c], v[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += own<WHOLE>(at[c], i) ? v[c][i] : 0.0f;
        }
        fetch(row + stride);
        const float mean = row_sum<WAVES>(sum, shared, turn) * p.inv_K;
        float squares = 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = v[c][i] - mean;
                squares += own<WHOLE>(at[c], i) ? d * d : 0.0f;
            }
        const float var = row_sum<WAVES>(squares, shared, turn) * p.inv_K;
        const float rstd = 1.0f / sqrtf(var + p.eps);
        if (t == 0 && mean_out) mean_out[row] = mean;
        if (t == 0 && rstd_out) rstd_out[row] = rstd;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (v[c][i] - mean) * rstd * g[c][i] + b[c][i];
            store_own<WHOLE, STREAMING != kKept>(y + row * p.ldy, at[c], o);
            if (codes && at[c].col - 8 * lane < p.K) {       // the wavefront's 512 values begin inside the row
                if constexpr (!WHOLE) first_own(at[c], v[c]);
                if (!at[c].inside) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[c][i] = 0.0f;
                }
                const uint32_t byte = scale8_of(block_top(v[c]));
                const v2u w = codes8_of(v[c], byte);
                if (at[c].col < p.K128) *reinterpret_cast<v2u*>(codes + row * p.code_pitch + at[c].col) = w;
                if ((lane & 3) == 0) scales[row * p.scale_pitch + (at[c].col >> 5)] = (uint8_t)byte;
            }
        }
    }
}

// Rows of any length, read three times: 4096 x 16384 bf16 with checkpoint 91 us (3.7 TB/s of what it has to move), where a row a little shorter,
// held in registers, goes at 5.5.
template <class T>
__global__ __launch_bounds__(kThreads) void norm_long_kernel(const T* __restrict__ x, const float* __restrict__ gamma,
                                                             const float* __restrict__ beta, T* __restrict__ y, float* __restrict__ mean_out,
                                                             float* __restrict__ rstd_out, uint8_t* __restrict__ codes,
                                                             uint8_t* __restrict__ scales, const NormParams p) {
    __shared__ float shared[2 * kWaves];
    const int t = threadIdx.x, lane = t & 63;
    const int64_t row = blockIdx.x;
    int turn = 0;
    x += row * p.ldx;
    y += row * p.ldy;
    float v[8], sum = 0.0f, squares = 0.0f;
    for (int col = 8 * t; col < p.K; col += 8 * kThreads) {
        load_upto8(x + col, p.K - col, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[i];
    }
    const float mean = row_sum<kWaves>(sum, shared, turn) * p.inv_K;
    for (int col = 8 * t; col < p.K; col += 8 * kThreads) {
        load_upto8(x + col, p.K - col, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) squares += i < p.K - col ? (v[i] - mean) * (v[i] - mean) : 0.0f;
    }
    const float var = row_sum<kWaves>(squares, shared, turn) * p.inv_K;
    const float rstd = 1.0f / sqrtf(var + p.eps);
    if (t == 0 && mean_out) mean_out[row] = mean;
    if (t == 0 && rstd_out) rstd_out[row] = rstd;
    for (int col = 8 * t; col - 8 * lane < p.K; col += 8 * kThreads) {       // (whole wavefronts: a block is four lanes')
        const int n = p.K - col;
        float g[8], b[8], o[8];
        load_upto8(x + col, n, v);
        load_upto8(gamma + col, n, g);
        if (beta) load_upto8(beta + col, n, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (v[i] - mean) * rstd * g[i] + (beta ? b[i] : 0.0f);
        if (n > 0) store_upto8(y + col, n, o);
        if (codes) {
            const uint32_t byte = scale8_of(block_top(v));
            const v2u w = codes8_of(v, byte);
            if (col < p.K128) *reinterpret_cast<v2u*>(codes + row * p.code_pitch + col) = w;
            if ((lane & 3) == 0) scales[row * p.scale_pitch + (col >> 5)] = (uint8_t)byte;
        }
    }
}

// ---- backward ----------------------------------------------------------------------
struct NormGradParams {
    int64_t ldy, ldx, code_pitch, scale_pitch, rows;
    int32_t K;
    float inv_K;
    int32_t parts;                       // partial sums of the weights' gradients: rows part, part + parts, ...
};

// The weights' gradients of 32 columns, eight a lane and 64 rows at a time: what reads dy and the codes once more.
struct ColumnGradients {
    static constexpr int kColumns = 32, kLanes = kColumns / 8, kRows = kThreads / kLanes, kSlices = kThreads / kColumns, kPitch = kColumns + 4;
    static constexpr int kFloats = kRows * kPitch;
    template <class T>
    static __device__ __forceinline__ void run(const T* __restrict__ dy, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                               const float* __restrict__ mean, const float* __restrict__ rstd, float* __restrict__ dgamma,
                                               float* __restrict__ dbeta, const NormGradParams& p, int first, float* shared) {
        const int t = threadIdx.x, x = t % kLanes, r0 = t / kLanes, col = first + 8 * x, n = p.K - col;
        float g[8] = {}, b[8] = {};
        if (n > 0) {
#pragma unroll 2
            for (int64_t row = r0; row < p.rows; row += kRows) {
                float d[8], h[8];
                load_upto8(dy + row * p.ldy + col, n, d);
                values8_of(*reinterpret_cast<const v2u*>(codes + row * p.code_pitch + col), scales[row * p.scale_pitch + (col >> 5)], h);
                const float mu = mean[row], r = rstd[row];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    g[i] += d[i] * ((h[i] - mu) * r);
                    b[i] += d[i];
                }
            }
        }
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float* const to = which ? dbeta : dgamma;
            if (!to) continue;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) shared[r0 * kPitch + 8 * x + i] = which ? b[i] : g[i];
            __syncthreads();
            // kSlices threads a column, then one
            const int c = t % kColumns, slice = t / kColumns;
            float total = 0.0f;
#pragma unroll
            for (int i = 0; i < kRows / kSlices; ++i) total += shared[(slice * (kRows / kSlices) + i) * kPitch + c];
            __syncthreads();
            shared[slice * kPitch + c] = total;
            __syncthreads();
            if (slice == 0 && first + c < p.K) {
#pragma unroll
                for (int i = 1; i < kSlices; ++i) total += shared[i * kPitch + c];
                to[first + c] = total;
            }
        }
    }
};

// dx, and the workgroup's share of the weights' gradients, in one pass: WAVES wavefronts take a row, CHUNKS x 8 values a lane, rows part,
// part + parts, ..., the next row on its way while this one is summed and written.  What the workgroup's wavefronts added up is joined in
// LDS in their order and leaves as one partial sum.  16384 x 4096 bf16 70 us with the sums' join (4.8 TB/s), 65536 x 1024 64, fp32 118.
template <class T, int WAVES, int CHUNKS, bool WHOLE, int STREAMING>
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(const T* __restrict__ dy, const uint8_t* __restrict__ codes,
                                                             const uint8_t* __restrict__ scales, const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, const float* __restrict__ gamma, T* __restrict__ dx,
                                                             float* __restrict__ partial, float* __restrict__ dgamma, float* __restrict__ dbeta,
                                                             const NormGradParams p) {
    __shared__ float columns[ColumnGradients::kFloats];
    if ((int)blockIdx.x >= p.parts) {
        ColumnGradients::run(dy, codes, scales, mean, rstd, dgamma, dbeta, p, (int)(blockIdx.x - p.parts) * ColumnGradients::kColumns, columns);
        return;
    }
    constexpr int kRows = kWaves / WAVES, kSpan = WAVES * 512;
    __shared__ float sums[2][2][WAVES];
    __shared__ float joined[kRows > 1 ? kRows * CHUNKS * 512 : 1];
    const int wave = threadIdx.x >> 6, t = threadIdx.x & (WAVES * 64 - 1);
    const int64_t first = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? wave : 0), stride = (int64_t)p.parts * kRows;
    float g[CHUNKS][8], dg[CHUNKS][8] = {}, db[CHUNKS][8] = {};
    Place at[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        at[c] = place_of<WHOLE>(c * kSpan + 8 * t, p.K);
        load8(gamma + at[c].from, g[c]);
    }
    struct Held {
        Raw8<T> dy[CHUNKS];
        v2u x[CHUNKS];
        uint32_t scale[CHUNKS];
        float mean, rstd;
    };
    auto fetch = [&](Held& h, int64_t row) __attribute__((always_inline)) {
        row = row < p.rows ? row : p.rows - 1;               // (past the end: a row again, for nobody)
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            load_raw<STREAMING == kAll>(dy + row * p.ldy + at[c].from, h.dy[c]);
            __builtin_memcpy(&h.x[c], codes + row * p.code_pitch + at[c].from, 8);
            h.scale[c] = scales[row * p.scale_pitch + ((at[c].inside ? at[c].col : at[c].from) >> 5)];
        }
        h.mean = mean[row];
        h.rstd = rstd[row];
    };
    Held held;
    fetch(held, first);
    int turn = 0;
    for (int64_t row = first; row < p.rows; row += stride) {
        float d[CHUNKS][8], h[CHUNKS][8], s1 = 0.0f, s2 = 0.0f;
        const float mu = held.mean, r = held.rstd;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            values_of(held.dy[c], d[c]);
            values8_of(held.x[c], held.scale[c], h[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[c][i] = own<WHOLE>(at[c], i) ? (h[c][i] - mu) * r : 0.0f;
                const float e = own<WHOLE>(at[c], i) ? d[c][i] * g[c][i] : 0.0f;
                s1 += e;
                s2 += e * h[c][i];
            }
        }
        fetch(held, row + stride);
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) {
                sums[turn][0][wave] = s1;
                sums[turn][1][wave] = s2;
            }
            __syncthreads();
            s1 = sums[turn][0][0];
            s2 = sums[turn][1][0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) {
                s1 += sums[turn][0][i];
                s2 += sums[turn][1][i];
            }
            turn ^= 1;                                       // (the one after the next sum is written behind the next barrier)
        }
        s1 *= p.inv_K;
        s2 *= p.inv_K;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                o[i] = r * (d[c][i] * g[c][i] - s1 - h[c][i] * s2);
                dg[c][i] += d[c][i] * h[c][i];
                db[c][i] += d[c][i];
            }
            store_own<WHOLE, STREAMING == kAll>(dx + row * p.ldx, at[c], o);
        }
    }
    if (!partial) return;
    float* to = partial + (int64_t)blockIdx.x * 2 * p.K;
    if constexpr (kRows == 1) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            store_own<WHOLE>(to, at[c], dg[c]);
            store_own<WHOLE>(to + p.K, at[c], db[c]);
        }
    } else {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (which) __syncthreads();
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (own<WHOLE>(at[c], i)) joined[wave * CHUNKS * 512 + at[c].from + i] = which ? db[c][i] : dg[c][i];
            __syncthreads();
            for (int col = threadIdx.x; col < p.K; col += kThreads) {
                float s = joined[col];
#pragma unroll
                for (int w = 1; w < kRows; ++w) s += joined[w * CHUNKS * 512 + col];
                to[which * p.K + col] = s;
            }
        }
    }
}

// Rows too long for registers, or too short (4096 x 16384 bf16 141 us, 2.4 TB/s: dy and codes twice, three launches): their sums of d and d h first, one wavefront a row ...
template <class T>
__global__ __launch_bounds__(kThreads) void norm_grad_rows_kernel(const T* __restrict__ dy, const uint8_t* __restrict__ codes,
                                                                  const uint8_t* __restrict__ scales, const float* __restrict__ mean,
                                                                  const float* __restrict__ rstd, const float* __restrict__ gamma,
                                                                  v2f* __restrict__ sums, const NormGradParams p) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (row >= p.rows) return;
    const float mu = mean[row], r = rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int col = 8 * lane; col < p.K; col += 512) {
        const int n = p.K - col;
        float d[8], h[8], g[8];
        load_upto8(dy + row * p.ldy + col, n, d);
        load_upto8(gamma + col, n, g);
        values8_of(*reinterpret_cast<const v2u*>(codes + row * p.code_pitch + col), scales[row * p.scale_pitch + (col >> 5)], h);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = d[i] * g[i];                     // (zero past the row)
            s1 += e;
            s2 += e * ((h[i] - mu) * r);
        }
    }
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    if (lane == 0) sums[row] = v2f{s1 * p.inv_K, s2 * p.inv_K};
}

// ... then dx and the weights' shares, 2048 columns of rows part, part + parts, ... a workgroup.
template <class T>
__global__ __launch_bounds__(kThreads) void norm_grad_columns_kernel(const T* __restrict__ dy, const uint8_t* __restrict__ codes,
                                                                     const uint8_t* __restrict__ scales, const float* __restrict__ mean,
                                                                     const float* __restrict__ rstd, const float* __restrict__ gamma,
                                                                     const v2f* __restrict__ sums, T* __restrict__ dx,
                                                                     float* __restrict__ partial, const NormGradParams p) {
    const int col = (blockIdx.x * kThreads + threadIdx.x) * 8, n = p.K - col;
    if (n <= 0) return;
    float g[8], dg[8] = {}, db[8] = {};
    load_upto8(gamma + col, n, g);
    for (int64_t row = blockIdx.y; row < p.rows; row += p.parts) {
        const float mu = mean[row], r = rstd[row];
        const v2f s = sums[row];
        float d[8], h[8], o[8];
        load_upto8(dy + row * p.ldy + col, n, d);
        values8_of(*reinterpret_cast<const v2u*>(codes + row * p.code_pitch + col), scales[row * p.scale_pitch + (col >> 5)], h);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float hh = (h[i] - mu) * r;
            o[i] = r * (d[i] * g[i] - s[0] - hh * s[1]);
            dg[i] += d[i] * hh;
            db[i] += d[i];
        }
        store_upto8(dx + row * p.ldx + col, n, o);
    }
    if (partial) {
        float* at = partial + (int64_t)blockIdx.y * 2 * p.K + col;
        store_upto8(at, n, dg);
        store_upto8(at + p.K, n, db);
    }
}

// Rows are held in registers up to this length, one wavefront a row up to the other (four instead for 65536 x 1024: 66 -> 83 us, backward 65 ->
// 131).
constexpr int kHeldK = 8192, kWaveK = 1024;
static bool held_in_registers(int K) { return K >= 8 && K <= kHeldK; }
// Few rows: workgroups beside those of the rows make the weights' gradients, from dy and the codes read again, which is shorter than partial
// sums and the launch that joins them (us, with that -> beside: 130 x 1000 6.6 -> 3.8, 512 x 512 6.2 -> 5.0, 256 x 4096 10.7 -> 4.3,
// 1024 x 4096 17.3 -> 13.3; 1024 x 1024 7.6 -> 8.0, 2048 x 4096 17.3 -> 23.7).
static bool gradients_beside(int64_t rows, int K) { return held_in_registers(K) && rows <= (K <= kWaveK ? 512 : 1024); }
// Workgroups: enough that what they ask for hides the memory's latency, and no more, since each leaves a partial sum of both gradients.
static int norm_parts(int64_t rows, int K) {
    const int64_t most = !held_in_registers(K) ? 256 : 512, needed = held_in_registers(K) && K <= kWaveK ? (rows + kWaves - 1) / kWaves : rows;
    return (int)(needed < most ? needed : most);
}
static size_t norm_grad_bytes(int64_t rows, int K) {
    return (size_t)((held_in_registers(K) ? 0 : round_up(rows * 8, 256)) + round_up((int64_t)norm_parts(rows, K) * 2 * K * 4, 256));
}

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" sparq_status sparq_mx_norm(const void* x, int64_t ldx, const float* gamma, const float* beta, float eps, void* y, int64_t ldy,
                                      int32_t type, float* mean, float* rstd, void* codes, void* scales, int64_t rows, int32_t K,
                                      void* stream) {
    if (!sizes_ok(rows, K) || !type_valid(type) || !(eps >= 0.0f)) return SPARQ_EINVAL;
    if (rows == 0) return SPARQ_OK;
    if (!tensor_ok(x, type, ldx, K) || !tensor_ok(y, type, ldy, K) || !gamma || !aligned(gamma, 4) || !aligned(beta, 4)) return SPARQ_EINVAL;
    if (!extent_ok(rows, ldx) || !extent_ok(rows, ldy) || !extent_ok(rows, K) || !coded_ok_or_none(codes, scales)) return SPARQ_EINVAL;
    if ((mean != nullptr) != (rstd != nullptr) || !aligned(mean, 4) || !aligned(rstd, 4)) return SPARQ_EINVAL;
    if (rows >= (1ll << 31)) return SPARQ_EUNSUPPORTED;
    const NormParams p = {ldx, ldy, code_pitch(K, 8), scale_pitch(K), rows, K, (int)round_up(K, kCodeUnit), eps, (float)(1.0 / K)};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    sparq_status done = SPARQ_OK;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const auto launch = [&](auto kernel, int per_block, int per_cu) {
            const int64_t blocks = (rows + per_block - 1) / per_block, places = (int64_t)per_cu * device_cu_count();
            kernel<<<(unsigned)(blocks < places ? blocks : places), kThreads, 0, s>>>(
                static_cast<const T*>(x), gamma, beta, static_cast<T*>(y), mean, rstd, static_cast<uint8_t*>(codes),
                static_cast<uint8_t*>(scales), p);
            done = launch_status();
        };
        const auto held = [&](auto whole, auto streaming) {
            constexpr bool W = decltype(whole)::value;
            constexpr int S = decltype(streaming)::value;
            if (K <= 512) launch(norm_kernel<T, 1, 1, W, S>, 4, 8);
            else if (K <= kWaveK) launch(norm_kernel<T, 1, 2, W, S>, 4, 5);
            else if (K <= 2048) launch(norm_kernel<T, 4, 1, W, S>, 1, 8);
            else if (K <= 4096) launch(norm_kernel<T, 4, 2, W, S>, 1, 5);
            else launch(norm_kernel<T, 4, 4, W, S>, 1, 3);
        };
        if (!held_in_registers(K)) {
            done = in_launches(rows, kThreads, [&](int64_t first, int64_t n) {
                norm_long_kernel<T><<<(unsigned)n, kThreads, 0, s>>>(static_cast<const T*>(x) + first * ldx, gamma, beta, static_cast<T*>(y) + first * ldy,
                                                                     mean ? mean + first : nullptr, rstd ? rstd + first : nullptr,
                                                                     row_of(codes, first, p.code_pitch), row_of(scales, first, p.scale_pitch), p);
                return launch_status();
            });
        } else if (K % 8 == 0) {
            const int64_t result = rows * K * (int64_t)sizeof(T);
            with_streaming<T>(2 * result + (codes ? rows * K : 0), result, [&](auto streaming) { held(std::true_type{}, streaming); });
        } else held(std::false_type{}, std::integral_constant<int, kKept>{});
    });
    return done;
}

extern "C" size_t sparq_mx_norm_grad_workspace_bytes(int64_t rows, int32_t K) {
    return sizes_ok(rows, K) && extent_ok(rows, K) ? norm_grad_bytes(rows, K) : 0;
}

extern "C" sparq_status sparq_mx_norm_grad(const void* dy, int64_t lddy, const void* codes, const void* scales, const float* mean,
                                           const float* rstd, const float* gamma, void* dx, int64_t lddx, int32_t type, float* dgamma,
                                           float* dbeta, int64_t rows, int32_t K, void* workspace, size_t workspace_bytes, void* stream) {
    if (!sizes_ok(rows, K) || !type_valid(type) || !aligned(dgamma, 4) || !aligned(dbeta, 4)) return SPARQ_EINVAL;
    if (!extent_ok(rows, K)) return SPARQ_EINVAL;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (rows == 0) {
        return dgamma || dbeta ? launch_join_columns(nullptr, dgamma, dbeta, K, 2 * K, 0, s) : SPARQ_OK;
    }
    if (!tensor_ok(dy, type, lddy, K) || !tensor_ok(dx, type, lddx, K) || !coded_ok(codes, scales)) return SPARQ_EINVAL;
    if (!mean || !rstd || !gamma || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(gamma, 4)) return SPARQ_EINVAL;
    if (!extent_ok(rows, lddy) || !extent_ok(rows, lddx)) return SPARQ_EINVAL;
    if (rows >= (1ll << 31)) return SPARQ_EUNSUPPORTED;
    if (!workspace || !aligned(workspace, 256)) return SPARQ_EINVAL;
    if (workspace_bytes < norm_grad_bytes(rows, K)) return SPARQ_EWORKSPACE;
    v2f* sums = static_cast<v2f*>(workspace);
    const bool gradients = dgamma || dbeta, beside = gradients && gradients_beside(rows, K);
    float* partial = gradients && !beside ? reinterpret_cast<float*>(static_cast<char*>(workspace) + (held_in_registers(K) ? 0 : round_up(rows * 8, 256))) : nullptr;
    const NormGradParams p = {lddy, lddx, code_pitch(K, 8), scale_pitch(K), rows, K, (float)(1.0 / K), norm_parts(rows, K)};
    const uint8_t *c = static_cast<const uint8_t*>(codes), *sc = static_cast<const uint8_t*>(scales);
    sparq_status done = SPARQ_OK;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const T* from = static_cast<const T*>(dy);
        T* to = static_cast<T*>(dx);
        const auto launch = [&](auto kernel) {
            const unsigned further = beside ? (unsigned)((K + ColumnGradients::kColumns - 1) / ColumnGradients::kColumns) : 0;
            kernel<<<p.parts + further, kThreads, 0, s>>>(from, c, sc, mean, rstd, gamma, to, partial, dgamma, dbeta, p);
        };
        const auto held = [&](auto whole, auto streaming) {
            constexpr bool W = decltype(whole)::value;
            constexpr int S = decltype(streaming)::value == kAll ? kAll : kKept;      // (dx 2048 x 4096 past the caches: 17.1 -> 17.5 us)
            if (K <= 512) launch(norm_grad_kernel<T, 1, 1, W, S>);
            else if (K <= kWaveK) launch(norm_grad_kernel<T, 1, 2, W, S>);
            else if (K <= 2048) launch(norm_grad_kernel<T, 4, 1, W, S>);
            else if (K <= 4096) launch(norm_grad_kernel<T, 4, 2, W, S>);
            else launch(norm_grad_kernel<T, 4, 4, W, S>);
        };
        if (held_in_registers(K)) {
            const int64_t result = rows * K * (int64_t)sizeof(T);
            if (K % 8 == 0) with_streaming<T>(2 * result + rows * K, result, [&](auto streaming) { held(std::true_type{}, streaming); });
            else held(std::false_type{}, std::integral_constant<int, kKept>{});
        } else {
            done = in_launches(rows, 64, [&](int64_t first, int64_t n) {
                NormGradParams q = p;
                q.rows = n;
                norm_grad_rows_kernel<T><<<(unsigned)((n + kWaves - 1) / kWaves), kThreads, 0, s>>>(
                    from + first * lddy, row_of(c, first, p.code_pitch), row_of(sc, first, p.scale_pitch), mean + first, rstd + first, gamma, sums + first, q);
                return launch_status();
            });
            if (done != SPARQ_OK) return;
            norm_grad_columns_kernel<T><<<dim3((unsigned)((K + 8ll * kThreads - 1) / (8 * kThreads)), p.parts), kThreads, 0, s>>>(
                from, c, sc, mean, rstd, gamma, sums, to, partial, p);
        }
    });
    if (done != SPARQ_OK) return done;
    if (partial) return launch_join_columns(partial, dgamma, dbeta, K, 2 * K, p.parts, s);
    return launch_status();
}

// Rows to their experts and back, with the router's weights, and the gradients (include/sparq_mx_experts.h).
#include "sparq_mx_experts.h"

namespace sparq {
namespace mx {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// 16-bit results of what adds up and its gradient go past the caches: the rows these read have the caches to themselves, and what is written is not written back
// while the next kernel runs (8192 tokens of 4096, two rows each, left -> past, when it was chosen: 42 and 60 us -> 36 and 54).
// Times below: a call on the same tensors again, part of which the last-level cache still holds, and on four sets of them in turn, from memory.
template <class T> inline constexpr bool kPast = sizeof(T) == 2;

struct RouteParams {
    const int32_t* place;
    const float* weights;
    float* dweights;
    int64_t ldx, ldy, ldr;               // x, y and the residual (the gradient: x, dx and dy)
    int64_t code4_pitch, code8_pitch, scale_pitch;
    int64_t rows;                        // sorted rows there are
    int32_t K, K128, per;
    uint32_t items, chunks;              // wavefronts' worth of work: tokens x chunks of 512 values
    FastDiv div_chunks;
};

// A token's row is read once and stored at each of its places, a wavefront 512 values of it: what is read and written is what the formula names, in
// whole lines, whatever the order of the places.  Bound by memory: 8192 tokens of 4096, two places each, bf16 31 us and 40 (6.5 and 5.0 TB/s), to both coded forms of 2048
// 15 and 18.5; fp32 4096 of 2048, four places, 29 and 40.  (1024 values a wavefront: no change.)
template <class T, bool Y, bool F4, bool I8, int STREAMING>
__global__ __launch_bounds__(kThreads) void gather_kernel(const T* __restrict__ x, T* __restrict__ y, uint8_t* __restrict__ codes4, uint8_t* __restrict__ scales4,
                                                          uint8_t* __restrict__ codes8, uint8_t* __restrict__ scales8, const RouteParams p) {
    const int lane = threadIdx.x & 63;
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= p.items) return;
    const uint32_t token = fastdiv(item, p.div_chunks);
    const int col = (int)(item - token * p.chunks) * kScaleUnit + 8 * lane, n = p.K - col;
    const int32_t* const place = p.place + (int64_t)token * p.per;
    Raw8<T> raw;
    load_raw_upto8<STREAMING == kAll>(x + token * p.ldx + col, n, raw);
    uint32_t byte4 = 0, byte8 = 0, w4 = 0;
    v2u w8 = {};
    if constexpr (F4 || I8) {
        float v[8];
        values_of(raw, v);
        const uint32_t top = block_top(v);
        if constexpr (F4) {
            byte4 = scale4_of(top);
            w4 = codes4_of(v, byte4);
        }
        if constexpr (I8) {
            byte8 = scale8_of(top);
            w8 = codes8_of(v, byte8);
        }
    }
    for (int j = 0; j < p.per; ++j) {
        const int64_t row = place[j];
        if (row < 0 || row >= p.rows) continue;
        if constexpr (Y) {
            if (n > 0) store_raw_upto8<STREAMING != kKept>(y + row * p.ldy + col, n, raw);
        }
        const int64_t scale_at = row * p.scale_pitch + (col >> 5);
        if constexpr (F4) {
            if (col < p.K128) *reinterpret_cast<uint32_t*>(codes4 + row * p.code4_pitch + (col >> 1)) = w4;
            if ((lane & 3) == 0) scales4[scale_at] = (uint8_t)byte4;
        }
        if constexpr (I8) {
            if (col < p.K128) *reinterpret_cast<v2u*>(codes8 + row * p.code8_pitch + col) = w8;
            if ((lane & 3) == 0) scales8[scale_at] = (uint8_t)byte8;
        }
    }
}

// A wavefront makes 512 values of a token's row, or 1024, and the rows of four slots are on their way at a time.  (A slot without a row reads row 0 and leaves it
// out: a branch would have one row wait for another.)  Bound by memory: 8192 tokens of 4096, two rows each, bf16 30 us and 37.5 (6.7 and 5.4 TB/s), with a residual 39.5
// and 49; fp32 4096 of 2048, four rows, 25 and 36.
template <class T, int CHUNKS, bool NT>
__global__ __launch_bounds__(kThreads) void combine_kernel(const T* __restrict__ x, const T* __restrict__ residual, T* __restrict__ y, const RouteParams p) {
    const int lane = threadIdx.x & 63;
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= p.items) return;
    const uint32_t token = fastdiv(item, p.div_chunks);
    const int col = (int)(item - token * p.chunks) * (CHUNKS * kScaleUnit) + 8 * lane, n = p.K - col;
    const int64_t slot = (int64_t)token * p.per;
    float sum[CHUNKS][8] = {};
    for (int j0 = 0; j0 < p.per && p.rows > 0; j0 += 4) {
        Raw8<T> raw[4][CHUNKS];
        float w[4];
        bool there[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = j0 + i < p.per ? j0 + i : p.per - 1;
            const int64_t row = p.place[slot + j];
            there[i] = j0 + i < p.per && row >= 0 && row < p.rows;
            w[i] = p.weights ? p.weights[slot + j] : 1.0f;
            if (j0 + i < p.per) {
#pragma unroll
                for (int h = 0; h < CHUNKS; ++h) load_raw_upto8<false>(x + (there[i] ? row : 0) * p.ldx + col + h * kScaleUnit, n - h * kScaleUnit, raw[i][h]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (there[i]) {
#pragma unroll
                for (int h = 0; h < CHUNKS; ++h) {
                    float v[8];
                    values_of(raw[i][h], v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[h][e] = __builtin_fmaf(w[i], v[e], sum[h][e]);
                }
            }
        }
    }
#pragma unroll
    for (int h = 0; h < CHUNKS; ++h) {
        const int left = n - h * kScaleUnit;
        if (left <= 0) return;
        if (residual) {
            float r[8];
            load_upto8(residual + token * p.ldr + col + h * kScaleUnit, left, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[h][e] += r[e];
        }
        store_upto8<NT>(y + token * p.ldy + col + h * kScaleUnit, left, sum[h]);
    }
}

// W wavefronts take a token, every W-th 512 values of its row each and four slots at a time; dweights are sums within a lane, within a wavefront and over the
// wavefronts in their order.  Bound by memory: 8192 tokens of 4096, two rows each, bf16 50.5 us and 68 (6.65 and 4.9 TB/s); fp32 4096 of 2048, four rows, 61 and 69: a
// lane's 32 bytes leave as two stores, each half of every line.
template <class T, bool DX, bool DW, int W, bool NT>
__global__ __launch_bounds__(kThreads) void combine_grad_kernel(const T* __restrict__ dy, const T* __restrict__ x, T* __restrict__ dx, const RouteParams p) {
    __shared__ float sums[kWaves][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t at = blockIdx.x * (kWaves / W) + wave / W;
    const bool working = at < p.items;                       // (the others pass the barriers)
    const int64_t token = working ? at : p.items - 1, slot = token * p.per;
    for (int j0 = 0; j0 < p.per; j0 += 4) {
        int64_t row[4];
        bool there[4];
        float w[4], dot[4] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = j0 + i < p.per ? j0 + i : p.per - 1;
            row[i] = p.place[slot + j];
            there[i] = working && j0 + i < p.per && row[i] >= 0 && row[i] < p.rows;
            row[i] = there[i] ? row[i] : 0;
            if constexpr (DX) w[i] = p.weights[slot + j];
        }
        for (int chunk = wave % W; chunk < (int)p.chunks && p.rows > 0; chunk += W) {
            const int col = chunk * kScaleUnit + 8 * lane, n = p.K - col;
            Raw8<T> raw[4];
            float d[8];
            load_upto8(dy + token * p.ldr + col, n, d);
            if constexpr (DW) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (j0 + i < p.per) load_raw_upto8<false>(x + row[i] * p.ldx + col, n, raw[i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!there[i]) continue;
                if constexpr (DX) {
                    float o[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = w[i] * d[e];
                    if (n > 0) store_upto8<NT>(dx + row[i] * p.ldy + col, n, o);
                }
                if constexpr (DW) {
                    float v[8];
                    values_of(raw[i], v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot[i] = __builtin_fmaf(d[e], v[e], dot[i]);
                }
            }
        }
        if constexpr (DW) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int m = 1; m < 64; m <<= 1) dot[i] += __shfl_xor(dot[i], m);
                if (W > 1 && lane == 0) sums[wave][i] = dot[i];
            }
            if constexpr (W > 1) __syncthreads();
            if (working && wave % W == 0 && lane < 4 && j0 + lane < p.per) {
                float s = lane == 0 ? dot[0] : lane == 1 ? dot[1] : lane == 2 ? dot[2] : dot[3];
#pragma unroll
                for (int v = 1; v < W; ++v) s += sums[wave + v][lane];
                p.dweights[slot + j0 + lane] = s;
            }
            if constexpr (W > 1) __syncthreads();
        }
    }
}

constexpr int kMostSlots = 1 << 30;              // of a token: four at a time, they are counted in 32 bits
// false: more tokens or slots than a call counts
static bool route_params(int64_t tokens, int K, int per, const int32_t* place, int64_t rows, RouteParams* p) {
    const int64_t chunks = (K + kScaleUnit - 1) / kScaleUnit, items = tokens * chunks;
    if (tokens >= (1ll << 31) || items >= (1ll << 31) || per > kMostSlots || tokens * per >= (1ll << 40)) return false;
    *p = {};
    p->place = place;
    p->code4_pitch = code_pitch(K, 4);
    p->code8_pitch = code_pitch(K, 8);
    p->scale_pitch = scale_pitch(K);
    p->rows = rows;
    p->K = K;
    p->K128 = (int)round_up(K, kCodeUnit);
    p->per = per;
    p->items = (uint32_t)items;
    p->chunks = (uint32_t)chunks;
    p->div_chunks = make_fastdiv((uint32_t)chunks);
    return true;
}
// f(p, grid, first): launches for the tokens from `first` on, p of as many of them as a launch takes
template <class F>
static sparq_status in_route_launches(int64_t tokens, RouteParams p, F&& f) {
    return in_launches(tokens, 64ll * p.chunks, [&](int64_t first, int64_t n) {
        RouteParams q = p;
        q.items = (uint32_t)(n * p.chunks);
        q.place += first * p.per;
        if (q.weights) q.weights += first * p.per;
        f(q, (q.items + kWaves - 1) / kWaves, first);
        return launch_status();
    });
}
static bool route_sizes_ok(int64_t tokens, int64_t K, int64_t per, int64_t rows) { return sizes_ok(tokens, K) && per >= 1 && rows >= 0; }

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" sparq_status sparq_mx_gather(const void* x, int32_t type, int64_t ldx, int64_t tokens, int32_t K, const int32_t* place, int32_t per,
                                        void* y, int64_t ldy, void* codes4, void* scales4, void* codes8, void* scales8, int64_t rows, void* stream) {
    if (!route_sizes_ok(tokens, K, per, rows) || !type_valid(type)) return SPARQ_EINVAL;
    if (tokens == 0 || rows == 0) return SPARQ_OK;
    if (!tensor_ok(x, type, ldx, K) || !extent_ok(tokens, ldx) || !place || !aligned(place, 4)) return SPARQ_EINVAL;
    if ((y && (!tensor_ok(y, type, ldy, K) || !extent_ok(rows, ldy))) || !extent_ok(rows, K)) return SPARQ_EINVAL;
    if ((!y && !codes4 && !codes8) || !coded_ok_or_none(codes4, scales4) || !coded_ok_or_none(codes8, scales8)) return SPARQ_EINVAL;
    RouteParams p;
    if (!route_params(tokens, K, per, place, rows, &p)) return SPARQ_EUNSUPPORTED;
    p.ldx = ldx;
    p.ldy = ldy;
    sparq_status s = SPARQ_OK;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const int64_t slots = tokens * per, stored = slots < rows ? slots : rows;
        const int64_t result = y ? stored * K * (int64_t)sizeof(T) : 0;
        const int64_t bytes = tokens * K * (int64_t)sizeof(T) + result + stored * ((codes4 ? p.code4_pitch : 0) + (codes8 ? p.code8_pitch : 0));
        with_streaming<T>(bytes, y ? result : bytes, [&](auto streaming) {
            constexpr int S = decltype(streaming)::value;
            const auto launch = [&](auto kernel) {
                s = in_route_launches(tokens, p, [&](const RouteParams& q, uint32_t grid, int64_t first) {
                    kernel<<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
                        static_cast<const T*>(x) + first * ldx, static_cast<T*>(y), static_cast<uint8_t*>(codes4), static_cast<uint8_t*>(scales4),
                        static_cast<uint8_t*>(codes8), static_cast<uint8_t*>(scales8), q);
                });
            };
            if (y) {
                if (codes4) codes8 ? launch(gather_kernel<T, true, true, true, S>) : launch(gather_kernel<T, true, true, false, S>);
                else codes8 ? launch(gather_kernel<T, true, false, true, S>) : launch(gather_kernel<T, true, false, false, S>);
            } else {
                if (codes4) codes8 ? launch(gather_kernel<T, false, true, true, S>) : launch(gather_kernel<T, false, true, false, S>);
                else launch(gather_kernel<T, false, false, true, S>);
            }
        });
    });
    return s;
}

extern "C" sparq_status sparq_mx_combine(const void* x, int64_t ldx, int64_t rows, const int32_t* place, const float* weights, int32_t per,
                                         const void* residual, int64_t ldr, void* y, int64_t ldy, int32_t type, int64_t tokens, int32_t K,
                                         void* stream) {
    if (!route_sizes_ok(tokens, K, per, rows) || !type_valid(type)) return SPARQ_EINVAL;
    if (tokens == 0) return SPARQ_OK;
    if (rows > 0 && (!tensor_ok(x, type, ldx, K) || !extent_ok(rows, ldx))) return SPARQ_EINVAL;
    if (!tensor_ok(y, type, ldy, K) || !extent_ok(tokens, ldy) || !place || !aligned(place, 4) || !aligned(weights, 4)) return SPARQ_EINVAL;
    if (residual && (!tensor_ok(residual, type, ldr, K) || !extent_ok(tokens, ldr))) return SPARQ_EINVAL;
    RouteParams p;
    if (!route_params(tokens, K, per, place, rows, &p)) return SPARQ_EUNSUPPORTED;
    p.weights = weights;
    p.ldx = ldx;
    p.ldy = ldy;
    p.ldr = ldr;
    sparq_status s = SPARQ_OK;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const auto launch = [&](auto chunks) {
            constexpr int C = decltype(chunks)::value;
            RouteParams all = p;
            all.chunks = (p.chunks + C - 1) / C;
            all.div_chunks = make_fastdiv(all.chunks);
            s = in_route_launches(tokens, all, [&](const RouteParams& q, uint32_t grid, int64_t first) {
                combine_kernel<T, C, kPast<T>><<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
                    static_cast<const T*>(x), residual ? static_cast<const T*>(residual) + first * ldr : nullptr, static_cast<T*>(y) + first * ldy, q);
            });
        };
        // (more on its way at a time, where there is work for all CUs)
        if (p.chunks > 1 && p.items >= 8192) launch(std::integral_constant<int, 2>{});
        else launch(std::integral_constant<int, 1>{});
    });
    return s;
}

extern "C" sparq_status sparq_mx_combine_grad(const void* dy, int64_t lddy, const int32_t* place, const float* weights, int32_t per, void* dx,
                                              int64_t lddx, const void* x, int64_t ldx, int64_t rows, float* dweights, int32_t type,
                                              int64_t tokens, int32_t K, void* stream) {
    if (!route_sizes_ok(tokens, K, per, rows) || !type_valid(type)) return SPARQ_EINVAL;
    if (tokens == 0) return SPARQ_OK;
    if (rows == 0 && !dweights) return SPARQ_OK;
    if ((!dx && !dweights) || !tensor_ok(dy, type, lddy, K) || !extent_ok(tokens, lddy) || !place || !aligned(place, 4)) return SPARQ_EINVAL;
    if (dx && (!tensor_ok(dx, type, lddx, K) || !extent_ok(rows, lddx) || !weights || !aligned(weights, 4))) return SPARQ_EINVAL;
    if (!aligned(dweights, 4) || (dweights && rows > 0 && (!tensor_ok(x, type, ldx, K) || !extent_ok(rows, ldx)))) return SPARQ_EINVAL;
    RouteParams p;
    if (!route_params(tokens, K, per, place, rows, &p)) return SPARQ_EUNSUPPORTED;
    p.weights = weights;
    p.ldr = lddy;
    p.ldy = lddx;
    p.ldx = ldx;
    sparq_status s = SPARQ_OK;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const auto launch = [&](auto wavefronts) {
            constexpr int W = decltype(wavefronts)::value, kTokens = kWaves / W;
            constexpr bool NT = kPast<T>;
            const auto kernel = dx && dweights ? combine_grad_kernel<T, true, true, W, NT> : dx ? combine_grad_kernel<T, true, false, W, NT> : combine_grad_kernel<T, false, true, W, NT>;
            s = in_launches(tokens, kThreads / kTokens, [&](int64_t first, int64_t n) {
                RouteParams q = p;
                q.items = (uint32_t)n;
                q.place += first * per;
                if (q.weights) q.weights += first * per;
                q.dweights = dweights ? dweights + first * per : nullptr;
                kernel<<<(unsigned)((n + kTokens - 1) / kTokens), kThreads, 0, static_cast<hipStream_t>(stream)>>>(
                    static_cast<const T*>(dy) + first * lddy, static_cast<const T*>(x), static_cast<T*>(dx), q);
                return launch_status();
            });
        };
        // (two pieces of 512 a wavefront, while there are tokens for all CUs: 8192 tokens of 1003, two rows each, four wavefronts 32 us)
        if (p.chunks <= 2 && tokens >= 2048) launch(std::integral_constant<int, 1>{});
        else if (p.chunks <= 4 && tokens >= 2048) launch(std::integral_constant<int, 2>{});
        else launch(std::integral_constant<int, 4>{});
    });
    return s;
}

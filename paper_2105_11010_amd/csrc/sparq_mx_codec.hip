// Quantisation to the microscaled formats and back (include/sparq_mx.h).
#include "sparq_mx_common.h"

namespace sparq {
namespace mx {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

struct CodecParams {
    int64_t ld, code4_pitch, code8_pitch, scale_pitch;
    int32_t K, K128;
    uint32_t items, chunks;              // wavefronts' worth of work: rows x chunks of 512 values
    FastDiv div_chunks;
};

// A wavefront takes 512 values of one row, a lane eight of them, so that a block is four neighbouring lanes: the block's
// largest magnitude is two exchanges inside a quad, loads are 16 bytes a lane (fp32: twice), codes leave as 4 and 8 bytes a
// lane and the 16 scales as one byte of every fourth lane.  Bound by memory: 8192 x 8192 bf16 to 4 bits in 27 us (6.35 TB/s), to 8 in 32 (6.4), to
// both at once in 37 (6.5), fp32 to 4 bits in 52 (5.8); the way back 25.6 (6.6), 30.5 and 43 (7.0).  A large copy: 6.65 TB/s.
template <class T, bool F4, bool I8, int STREAMING>
__global__ __launch_bounds__(kThreads) void quantize_kernel(const T* __restrict__ x, uint8_t* __restrict__ codes4,
                                                            uint8_t* __restrict__ scales4, uint8_t* __restrict__ codes8,
                                                            uint8_t* __restrict__ scales8, const CodecParams p) {
    const int lane = threadIdx.x & 63;
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= p.items) return;
    const uint32_t row = fastdiv(item, p.div_chunks);
    const int col = (int)(item - row * p.chunks) * kScaleUnit + 8 * lane;
    float v[8];
    load_upto8<STREAMING == kAll>(x + row * p.ld + col, p.K - col, v);
    const uint32_t top = block_top(v);
    const int64_t scale_at = row * p.scale_pitch + (col >> 5);
    if constexpr (F4) {
        const uint32_t byte = scale4_of(top), w = codes4_of(v, byte);
        if (col < p.K128) *reinterpret_cast<uint32_t*>(codes4 + row * p.code4_pitch + (col >> 1)) = w;
        if ((lane & 3) == 0) scales4[scale_at] = (uint8_t)byte;
    }
    if constexpr (I8) {
        const uint32_t byte = scale8_of(top);
        const v2u w = codes8_of(v, byte);
        if (col < p.K128) *reinterpret_cast<v2u*>(codes8 + row * p.code8_pitch + col) = w;
        if ((lane & 3) == 0) scales8[scale_at] = (uint8_t)byte;
    }
}

template <class T, int BITS, int STREAMING>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                              T* __restrict__ y, const CodecParams p) {
    const int lane = threadIdx.x & 63;
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= p.items) return;
    const uint32_t row = fastdiv(item, p.div_chunks);
    if constexpr (sizeof(T) == 4) {
        // 32 bytes a lane would be two stores that each leave half of every line: four values of either half of the 512 instead.
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int col = (int)(item - row * p.chunks) * kScaleUnit + 256 * h + 4 * lane, n = p.K - col;
            if (n <= 0) return;
            const uint32_t byte = scales[row * p.scale_pitch + (col >> 5)];
            float v[8];
            if constexpr (BITS == 4) values4_of(*reinterpret_cast<const uint16_t*>(codes + row * p.code4_pitch + (col >> 1)), byte, v);
            else values8_of(v2u{*reinterpret_cast<const uint32_t*>(codes + row * p.code8_pitch + col), 0}, byte, v);
            T* to = y + row * p.ld + col;
            if (n >= 4) word_to<STREAMING != kKept>(to, v4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
            else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (i < n) to[i] = v[i];
            }
        }
        return;
    }
    const int col = (int)(item - row * p.chunks) * kScaleUnit + 8 * lane;
    if (col >= p.K) return;
    const uint32_t byte = scales[row * p.scale_pitch + (col >> 5)];
    float v[8];
    if constexpr (BITS == 4) values4_of(*reinterpret_cast<const uint32_t*>(codes + row * p.code4_pitch + (col >> 1)), byte, v);
    else values8_of(*reinterpret_cast<const v2u*>(codes + row * p.code8_pitch + col), byte, v);
    store_upto8<STREAMING != kKept>(y + row * p.ld + col, p.K - col, v);
}

// false: more rows than a call counts
static bool codec_params(int64_t rows, int K, int64_t ld, CodecParams* p) {
    const int64_t chunks = (K + kScaleUnit - 1) / kScaleUnit, items = rows * chunks;
    if (rows >= (1ll << 31) || items >= (1ll << 31)) return false;
    *p = {ld, code_pitch(K, 4), code_pitch(K, 8), scale_pitch(K), K, (int)round_up(K, kCodeUnit), (uint32_t)items, (uint32_t)chunks,
          make_fastdiv((uint32_t)chunks)};
    return true;
}

// f(p, grid, first): launches for the rows from `first` on, p of as many of them as a launch takes
template <class F>
static sparq_status in_codec_launches(int64_t rows, CodecParams p, F&& f) {
    return in_launches(rows, 64ll * p.chunks, [&](int64_t first, int64_t n) {
        p.items = (uint32_t)(n * p.chunks);
        f(p, (p.items + kWaves - 1) / kWaves, first);
        return launch_status();
    });
}

sparq_status launch_quantize(const void* x, int type, int64_t ldx, int64_t rows, int K, void* codes4, void* scales4, void* codes8,
                             void* scales8, hipStream_t stream) {
    CodecParams p;
    if (!codec_params(rows, K, ldx, &p)) return SPARQ_EUNSUPPORTED;
    sparq_status s = SPARQ_OK;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const int64_t bytes = rows * (K * (int64_t)sizeof(T) + (codes4 ? p.code4_pitch : 0) + (codes8 ? p.code8_pitch : 0));
        with_streaming<T>(bytes, bytes, [&](auto streaming) {
            constexpr int S = decltype(streaming)::value == kAll ? kAll : kKept;      // (codes are read soon)
            const auto kernel = codes4 && codes8 ? quantize_kernel<T, true, true, S> : codes4 ? quantize_kernel<T, true, false, S> : quantize_kernel<T, false, true, S>;
            s = in_codec_launches(rows, p, [&](const CodecParams& q, uint32_t grid, int64_t first) {
                kernel<<<grid, kThreads, 0, stream>>>(static_cast<const T*>(x) + first * ldx, row_of(codes4, first, p.code4_pitch),
                                                      row_of(scales4, first, p.scale_pitch), row_of(codes8, first, p.code8_pitch),
                                                      row_of(scales8, first, p.scale_pitch), q);
            });
        });
    });
    return s;
}

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" size_t sparq_mx_code_bytes(int32_t K, int32_t bits) {
    return sizes_ok(0, K) && (bits == 4 || bits == 8) ? (size_t)code_pitch(K, bits) : 0;
}
extern "C" size_t sparq_mx_scale_bytes(int32_t K) { return sizes_ok(0, K) ? (size_t)scale_pitch(K) : 0; }

extern "C" sparq_status sparq_mx_quantize(const void* x, int32_t type, int64_t ldx, int64_t rows, int32_t K, void* codes4,
                                          void* scales4, void* codes8, void* scales8, void* stream) {
    if (!sizes_ok(rows, K) || !type_valid(type)) return SPARQ_EINVAL;
    if (rows == 0) return SPARQ_OK;
    if (!tensor_ok(x, type, ldx, K) || !extent_ok(rows, ldx) || !extent_ok(rows, K)) return SPARQ_EINVAL;
    if ((!codes4 && !codes8) || !coded_ok_or_none(codes4, scales4) || !coded_ok_or_none(codes8, scales8)) return SPARQ_EINVAL;
    return launch_quantize(x, type, ldx, rows, K, codes4, scales4, codes8, scales8, static_cast<hipStream_t>(stream));
}

extern "C" sparq_status sparq_mx_dequantize(const void* codes, const void* scales, int32_t bits, void* y, int32_t type, int64_t ldy,
                                            int64_t rows, int32_t K, void* stream) {
    if (!sizes_ok(rows, K) || !type_valid(type) || (bits != 4 && bits != 8)) return SPARQ_EINVAL;
    if (rows == 0) return SPARQ_OK;
    if (!tensor_ok(y, type, ldy, K) || !extent_ok(rows, ldy) || !extent_ok(rows, K) || !coded_ok(codes, scales)) return SPARQ_EINVAL;
    CodecParams p;
    if (!codec_params(rows, K, ldy, &p)) return SPARQ_EUNSUPPORTED;
    const hipStream_t stream_ = static_cast<hipStream_t>(stream);
    sparq_status s = SPARQ_OK;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const int64_t result = rows * K * (int64_t)sizeof(T), bytes = result + rows * (int64_t)code_pitch(K, bits);
        const auto launch = [&](auto streaming) {
            constexpr int S = decltype(streaming)::value;
            const auto kernel = bits == 4 ? dequantize_kernel<T, 4, S> : dequantize_kernel<T, 8, S>;
            s = in_codec_launches(rows, p, [&](const CodecParams& q, uint32_t grid, int64_t first) {
                kernel<<<grid, kThreads, 0, stream_>>>(row_of(codes, first, code_pitch(K, bits)), row_of(scales, first, p.scale_pitch),
                                                       static_cast<T*>(y) + first * ldy, q);
            });
        };
        if (sizeof(T) == 4 && bytes >= kStreamedBytes) launch(std::integral_constant<int, kAll>{});      // (fp32 here in whole runs of 16 bytes a lane)
        else with_streaming<T>(bytes, result, launch);
    });
    return s;
}

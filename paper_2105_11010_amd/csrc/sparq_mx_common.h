// What the kernels of the microscaled formats share: element types, rows of codes and scales, both quantisers in
// registers, and the argument checks of their entry points.
#pragma once
#include <type_traits>

#include "../../include/sparq_mx.h"
#include "sparq_common.h"
#include "sparq_fastdiv.h"

namespace sparq {
namespace mx {

constexpr int kBlock = 32;           // values that share a scale
constexpr int kCodeUnit = 128;       // values: rows of codes are whole units (one step of the 16-row matrix instruction, two of the 32-row one)
constexpr int kScaleUnit = 512;      // ... and rows of scales (16 bytes)
constexpr int kMaxK = 1 << 28;

inline int64_t code_pitch(int K, int bits) { return round_up(K, kCodeUnit) * bits / 8; }
inline int64_t scale_pitch(int K) { return round_up(K, kScaleUnit) / kBlock; }

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef unsigned int v2u __attribute__((ext_vector_type(2)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

inline size_t type_bytes(int type) { return type == SPARQ_MX_F32 ? 4 : 2; }
inline bool type_valid(int type) { return type == SPARQ_MX_F32 || type == SPARQ_MX_F16 || type == SPARQ_MX_BF16; }
// A tensor argument: present, of whole elements, rows at least as far apart as they are long.
inline bool tensor_ok(const void* p, int type, int64_t ld, int64_t length) {
    return p && type_valid(type) && aligned(p, type_bytes(type)) && ld >= length && ld <= (INT64_MAX >> 4);
}
inline bool coded_ok(const void* codes, const void* scales) { return codes && scales && aligned(codes, 16) && aligned(scales, 16); }
inline bool coded_ok_or_none(const void* codes, const void* scales) { return codes || scales ? coded_ok(codes, scales) : true; }
inline bool sizes_ok(int64_t rows, int64_t K) { return rows >= 0 && K >= 1 && K <= kMaxK; }
// rows * pitch bytes and rows * ld elements stay inside 64 bits
inline bool extent_ok(int64_t rows, int64_t ld) { return rows == 0 || ld <= (INT64_MAX / 8) / rows; }

// A call that moves this many bytes streams them past the caches (us, kept -> streamed: 16384 x 8192 bf16 from 4-bit codes 72 -> 47, the gated
// activation of 8192 x 8192 94 -> 83; 16384 x 4096 bf16 to 4-bit codes, 174 MB, 27 -> 31, and what follows a smaller call finds it there).
// Not fp32 tensors, whose lanes' halves of 32 bytes go one after the other (16384 x 4096 from 4-bit codes 70 -> 104).
// Results of at most 16 MB go past them too (kResults): what a kernel leaves in the XCDs' caches is written back at its end, and with this, not then
// (us, left -> past, and with a quantiser that reads the result behind it: gated activation 1024 x 4096 7.5 -> 6.5, 10.4 -> 9.4; its gradient 6.8 -> 5.0,
// 13.4 -> 12.2; 8-bit codes to 2048 x 4096 5.1 -> 4.3, 8.9 -> 8.4; norm 2048 x 4096 9.2 -> 7.5, 17.7 -> 16.7; of larger ones the reader is slower than the
// writer gains: norm 4096 x 4096 14.5 -> 14.1, 23.4 -> 24.6).
enum Streaming { kKept, kResults, kAll };
template <class T, class F>
inline void with_streaming(int64_t bytes, int64_t results, F&& f) {
    if constexpr (sizeof(T) == 2) {
        if (bytes >= kStreamedBytes) return f(std::integral_constant<int, kAll>{});
        if (results <= 16 << 20) return f(std::integral_constant<int, kResults>{});
    }
    f(std::integral_constant<int, kKept>{});
}

// A launch has fewer than 2^32 threads along an axis, and of a larger grid only what is left over is run, without an error: f(first, rows) for as
// many rows at a time as make 2^31 threads.
template <class F>
inline sparq_status in_launches(int64_t rows, int64_t threads_a_row, F&& f) {
    const int64_t most = (1ll << 31) / threads_a_row;
    sparq_status s = SPARQ_OK;
    for (int64_t first = 0; first < rows && s == SPARQ_OK; first += most) s = f(first, rows - first < most ? rows - first : most);
    return s;
}

// Row `first` of codes or scales (NULL: none)
inline uint8_t* row_of(void* p, int64_t first, int64_t pitch) { return p ? static_cast<uint8_t*>(p) + first * pitch : nullptr; }
inline const uint8_t* row_of(const void* p, int64_t first, int64_t pitch) { return p ? static_cast<const uint8_t*>(p) + first * pitch : nullptr; }

template <class F>
inline void with_type(int type, F&& f) {
    if (type == SPARQ_MX_F32) f(float{});
    else if (type == SPARQ_MX_F16) f(_Float16{});
    else f(__bf16{});
}

#if defined(__HIPCC__)
// ---- eight neighbouring elements, from any address of an element -----------------
// (As members: as a template's argument a type loses its alignment, and the compiler would take such an address for a multiple of 16.)
template <int BYTES> struct Unaligned;
template <> struct Unaligned<4> { typedef v4u Word __attribute__((aligned(4))); };
template <> struct Unaligned<2> { typedef v4u Word __attribute__((aligned(2))); };

// NT: non-temporal, for what is streamed once and is not to stay in the caches (Streaming above).
template <bool NT, class T>
__device__ __forceinline__ v4u word_at(const T* p) {
    typedef const typename Unaligned<sizeof(T)>::Word V;
    if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<V*>(p));
    else return *reinterpret_cast<V*>(p);
}
template <bool NT, class T>
__device__ __forceinline__ void word_to(T* p, v4u w) {
    typedef typename Unaligned<sizeof(T)>::Word V;
    if constexpr (NT) __builtin_nontemporal_store(w, reinterpret_cast<V*>(p));
    else *reinterpret_cast<V*>(p) = w;
}
template <bool NT = false>
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const v4u a = word_at<NT>(p), b = word_at<NT>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = __uint_as_float(a[i]);
        v[4 + i] = __uint_as_float(b[i]);
    }
}
template <bool NT = false>
__device__ __forceinline__ void load8(const __bf16* p, float (&v)[8]) {
    const v4u a = word_at<NT>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    }
}
template <bool NT = false>
__device__ __forceinline__ void load8(const _Float16* p, float (&v)[8]) {
    const v4u a = word_at<NT>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = a[i];                     // (a copy: the bits of a vector's element cannot be taken in place)
        const v2h h = __builtin_bit_cast(v2h, w);
        v[2 * i] = (float)h[0];
        v[2 * i + 1] = (float)h[1];
    }
}
// ... of which the first n are there
template <bool NT = false, class T>
__device__ __forceinline__ void load_upto8(const T* p, int n, float (&v)[8]) {
    if (n >= 8) load8<NT>(p, v);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        if (n > 0) {                                         // (a branch an element would have one load wait for another)
            T e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = p[i < n ? i : 0];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)e[i] : 0.0f;
        }
    }
}

// Eight neighbouring elements as they lie in memory: what is on its way while something else is computed.
template <class T>
struct Raw8 {
    uint32_t w[2 * sizeof(T)];
};
template <bool NT, class T>
__device__ __forceinline__ void load_raw(const T* p, Raw8<T>& r) {
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
        const v4u w = word_at<NT>(p + 4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[4 * h + i] = w[i];
    }
}
template <class T>
__device__ __forceinline__ void values_of(const Raw8<T>& r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(r.w[i]);
        else {
            const uint16_t h = (uint16_t)(r.w[i >> 1] >> (16 * (i & 1)));
            v[i] = (float)__builtin_bit_cast(T, h);
        }
    }
}

// Rounded to nearest even by the conversion instructions.
__device__ __forceinline__ uint32_t pack2(float a, float b, __bf16) { return __builtin_bit_cast(uint32_t, v2bf{(__bf16)a, (__bf16)b}); }
__device__ __forceinline__ uint32_t pack2(float a, float b, _Float16) { return __builtin_bit_cast(uint32_t, v2h{(_Float16)a, (_Float16)b}); }
template <bool NT = false, class T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
    v4u a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = pack2(v[2 * i], v[2 * i + 1], T{});
    word_to<NT>(p, a);
}
template <bool NT = false>
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    v4u a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = __float_as_uint(v[i]);
        b[i] = __float_as_uint(v[4 + i]);
    }
    word_to<NT>(p, a);
    word_to<NT>(p + 4, b);
}
template <bool NT = false, class T>
__device__ __forceinline__ void store_upto8(T* p, int n, const float (&v)[8]) {
    if (n >= 8) store8<NT>(p, v);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (T)v[i];
    }
}

// ---- the formats: a lane holds eight values, four neighbouring lanes a block -------
// Largest magnitude of the block as the bits of a float: integer order is the order of magnitudes, and NaN and
// infinity lie above every number.
__device__ __forceinline__ uint32_t block_top(const float (&v)[8]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t m = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        top = m > top ? m : top;
    }
    const uint32_t b = (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true);       // lane ^ 1
    top = b > top ? b : top;
    const uint32_t c = (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, true);       // lane ^ 2
    return c > top ? c : top;
}
// The scale's byte.  The exponent field of the largest magnitude is floor(log2) + 127; 0 stands for zero and for
// everything below 2^-126, whose clamped exponent is -127 in both forms.
__device__ __forceinline__ uint32_t scale4_of(uint32_t top) {
    const uint32_t e = top >> 23;
    return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}
__device__ __forceinline__ uint32_t scale8_of(uint32_t top) { return top >> 23; }
// The scale as the 4-bit conversion instructions take it: they look at the exponent field alone, 0 standing for 2^-127 and 255 for
// NaN, which makes every value NaN.
__device__ __forceinline__ float scale_operand(uint32_t byte) { return __uint_as_float(byte << 23); }
// Eight 4-bit codes: the conversion instruction divides by the scale, rounds to nearest even and saturates at 6.
__device__ __forceinline__ uint32_t codes4_of(const float (&v)[8], uint32_t byte) {
    const float s = scale_operand(byte);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
    return byte == 255 ? 0u : w;
}
// 2^s / 64, the unit of the 8-bit codes (byte 255: NaN)
__device__ __forceinline__ float unit8_of(uint32_t byte) {
    return __builtin_amdgcn_ldexpf(byte == 255 ? __uint_as_float(0x7FC00000u) : 1.0f, (int)byte - 133);
}
// Eight 8-bit codes
__device__ __forceinline__ v2u codes8_of(const float (&v)[8], uint32_t byte) {
    const int up = 133 - (int)byte;                  // 64 / 2^s
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float r = __builtin_rintf(__builtin_amdgcn_ldexpf(v[i], up));
        q[i] = (uint32_t)(int)__builtin_amdgcn_fmed3f(r, -127.0f, 127.0f);
    }
    v2u w;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __builtin_amdgcn_perm(q[4 * h + 1], q[4 * h], 0x0C0C0400u);
        const uint32_t hi = __builtin_amdgcn_perm(q[4 * h + 3], q[4 * h + 2], 0x04000C0Cu);
        w[h] = byte == 255 ? 0u : lo | hi;
    }
    return w;
}
// The values of eight codes
__device__ __forceinline__ void values4_of(uint32_t w, uint32_t byte, float (&v)[8]) {
    const float s = scale_operand(byte);
    const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
    const v2f c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1]; v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
}
__device__ __forceinline__ void values8_of(v2u w, uint32_t byte, float (&v)[8]) {
    const float unit = unit8_of(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t h = w[i >> 2];
        v[i] = (float)(int8_t)(h >> (8 * (i & 3))) * unit;
    }
}
// Two neighbouring 4-bit values (of four pairs in a word) as bf16, exactly
__device__ __forceinline__ uint32_t pair4_of(uint32_t w, float scale, int pair) {
    const v2bf b = pair == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)
                   : pair == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)
                   : pair == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)
                               : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return __builtin_bit_cast(uint32_t, b);
}

// Tiles in an order that keeps what the workgroups of one XCD (every eighth) work on at a time close together: each XCD gets a run of
// tiles, eight columns of them wide.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_j, uint32_t tiles_k, uint32_t& tj, uint32_t& tk) {
    const uint32_t n = tiles_j * tiles_k, x = id & 7, per = n >> 3, more = n & 7;
    id = x * per + (x < more ? x : more) + (id >> 3);
    const uint32_t width = 8, group = id / (width * tiles_j), first = group * width, w = tiles_k - first < width ? tiles_k - first : width;
    const uint32_t in = id - group * width * tiles_j;
    tj = in / w;
    tk = first + in - tj * w;
}
#endif

// Implemented in sparq_mx_codec.hip: the arguments are checked already.
sparq_status launch_quantize(const void* x, int type, int64_t ldx, int64_t rows, int K, void* codes4, void* scales4, void* codes8,
                             void* scales8, hipStream_t stream);

// Implemented in sparq_mx_join.hip: out[j][k] = the sum over the parts of partial [parts][J][K], part after part, + bias[k]
// (NULL: none), rounded to the type.
sparq_status launch_join(const float* partial, const float* bias, void* out, int type, int64_t J, int K, int64_t ldo, int parts, hipStream_t stream);
// ... and of partial [parts][columns]: the columns before `split` into first, the others into second (NULL: not wanted).
sparq_status launch_join_columns(const float* partial, float* first, float* second, int split, int columns, int parts, hipStream_t stream);

typedef __attribute__((address_space(3))) void* LdsPtr;
// The wait instruction's operand for at most n loads and stores on their way; for that and no access to LDS.
constexpr int vmcnt(int n) { return (n & 15) | (n >> 4) << 14 | 0x0F70; }
constexpr int vmcnt_and_lds(int n) { return vmcnt(n) & ~0x0F00; }

}  // namespace mx
}  // namespace sparq

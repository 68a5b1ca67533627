// What the kernels' headers take from HIP and the compiler, for the host: device code compiled for the CPU, its index arithmetic as it is.  Lanes run as
// threads (gpu::run_workgroup), what they exchange is exchanged at barriers; loads by buffer go to gpu::load (the check's own); matrix instructions and conversions
// give nothing of use.  For checks of where a kernel reads and writes, not of what it computes.
#pragma once
#include <math.h>
#include <pthread.h>
#include <stddef.h>
#include <stdint.h>
#include <string.h>

#include <thread>
#include <vector>

#define __device__
#define __host__
#define __global__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __HIP_DEVICE_COMPILE__ 1

typedef struct Stream* hipStream_t;
typedef int hipError_t;
enum { hipSuccess = 0, hipFuncAttributeMaxDynamicSharedMemorySize = 0 };
struct hipDeviceProp_t {
    int multiProcessorCount;
};
inline hipError_t hipGetLastError() { return hipSuccess; }
inline hipError_t hipGetDevice(int* d) { return *d = 0, hipSuccess; }
inline hipError_t hipGetDeviceProperties(hipDeviceProp_t* p, int) { return p->multiProcessorCount = 256, hipSuccess; }
inline hipError_t hipFuncSetAttribute(const void*, int, int) { return hipSuccess; }
struct dim3 {
    unsigned x, y, z;
    dim3(unsigned x_ = 1, unsigned y_ = 1, unsigned z_ = 1) : x(x_), y(y_), z(z_) {}
};
extern "C" hipError_t __hipPushCallConfiguration(dim3, dim3, size_t, hipStream_t);       // (launches are read by the compiler, and never made)
inline thread_local dim3 threadIdx, blockIdx, gridDim;

namespace gpu {

typedef unsigned u2 __attribute__((ext_vector_type(2)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

// ---- lanes ----
struct Barrier {
    pthread_barrier_t b;
    explicit Barrier(unsigned n) { pthread_barrier_init(&b, nullptr, n); }
    ~Barrier() { pthread_barrier_destroy(&b); }
    void wait() { pthread_barrier_wait(&b); }
};
struct Wave {
    Barrier barrier{64};
    uint64_t slot[64];
};
inline thread_local Wave* wave;                  // NULL: a lane by itself, which gets back what it gives
inline thread_local Barrier* workgroup;
// What lane `from` gives
inline uint64_t exchange(uint64_t mine, int from) {
    if (!wave) return mine;
    wave->slot[threadIdx.x & 63] = mine;
    wave->barrier.wait();
    const uint64_t r = wave->slot[from & 63];
    wave->barrier.wait();
    return r;
}
inline uint64_t ballot(bool b) {
    if (!wave) return (uint64_t)b << (threadIdx.x & 63);
    wave->slot[threadIdx.x & 63] = b;
    wave->barrier.wait();
    uint64_t r = 0;
    for (int i = 0; i < 64; ++i) r |= wave->slot[i] << i;
    wave->barrier.wait();
    return r;
}
template <class F>
void run_workgroup(int threads, dim3 block, F&& kernel) {
    std::vector<Wave> waves((threads + 63) / 64);
    Barrier all(threads);
    std::vector<std::thread> t;
    for (int i = 0; i < threads; ++i)
        t.emplace_back([&, i] {
            threadIdx = dim3(i);
            blockIdx = block;
            wave = &waves[i / 64];
            workgroup = &all;
            kernel();
        });
    for (auto& x : t) x.join();
}
// A workgroup's threads one after the other, each by itself
template <class F>
void run_threads(int threads, dim3 block, F&& kernel) {
    blockIdx = block;
    for (int i = 0; i < threads; ++i) {
        threadIdx = dim3(i);
        kernel();
    }
}

// ---- loads by buffer ----
struct Buffer {
    const uint8_t* base;
    uint32_t bytes;
};
inline Buffer make_buffer(const void* p, int, int bytes, int) { return {static_cast<const uint8_t*>(p), (uint32_t)bytes}; }
void load(const Buffer& b, uint32_t vector, uint32_t scalar, int bytes);       // the check's
inline u4 load16(const Buffer& b, uint32_t v, uint32_t s, int) { return load(b, v, s, 16), u4{}; }
inline u2 load8(const Buffer& b, uint32_t v, uint32_t s, int) { return load(b, v, s, 8), u2{}; }
inline uint32_t load4(const Buffer& b, uint32_t v, uint32_t s, int) { return load(b, v, s, 4), 0; }
template <class P>
inline void load_lds(const Buffer& b, const P&, int bytes, uint32_t v, uint32_t s, int at, int) { load(b, v + at, s, bytes); }
inline uint8_t load1(const Buffer& b, uint32_t v, uint32_t s, int) { return load(b, v, s, 1), 0; }

struct Nothing {                                 // of any type
    template <class T>
    operator T() const { return T{}; }
};
template <class A, class B, class C, class... More>
inline C third(const A&, const B&, const C& c, const More&...) { return c; }
template <class... More>
inline u2 nothing2(const More&...) { return u2{}; }
template <class... More>
inline void ignore(const More&...) {}
template <class... More>
inline uint32_t zero(const More&...) { return 0; }

}  // namespace gpu

inline void __syncthreads() {
    if (gpu::workgroup) gpu::workgroup->wait();
}
template <class T>
inline T __shfl_up(T v, int d) {
    const int lane = threadIdx.x & 63;
    return (T)gpu::exchange((uint64_t)v, lane >= d ? lane - d : lane);
}
template <class T>
inline T __shfl_xor(T v, int) { return v; }
inline uint64_t __ballot(bool b) { return gpu::ballot(b); }
inline int __popcll(uint64_t v) { return __builtin_popcountll(v); }
inline uint32_t __float_as_uint(float v) { return __builtin_bit_cast(uint32_t, v); }
inline float __uint_as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
inline uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)((uint64_t)a * b >> 32); }
inline float __fmul_rn(float a, float b) { return a * b; }

#define __amdgpu_buffer_rsrc_t gpu::Buffer
#define __builtin_amdgcn_make_buffer_rsrc gpu::make_buffer
#define __builtin_amdgcn_raw_buffer_load_b128 gpu::load16
#define __builtin_amdgcn_raw_buffer_load_b64 gpu::load8
#define __builtin_amdgcn_raw_buffer_load_b32 gpu::load4
#define __builtin_amdgcn_raw_buffer_load_b8 gpu::load1
#define __builtin_amdgcn_raw_ptr_buffer_load_lds gpu::load_lds
#define __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4 gpu::third
#define __builtin_amdgcn_readlane(v, from) ((int)gpu::exchange((uint32_t)(v), from))
#define __builtin_amdgcn_readfirstlane(v) (v)
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16 gpu::third
#define __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4 gpu::third
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) (v4s{})
#define __builtin_amdgcn_cvt_scalef32_pk_fp4_f32 gpu::zero
#define __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(...) (v2f{})
#define __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(...) (v2bf{})
#define __builtin_amdgcn_permlane32_swap gpu::nothing2
#define __builtin_amdgcn_mov_dpp gpu::zero
#define __builtin_amdgcn_perm gpu::zero
#define __builtin_amdgcn_lerp gpu::zero
#define __builtin_amdgcn_bitop3_b32 gpu::zero
#define __builtin_amdgcn_cvt_pk_u8_f32 gpu::zero
#define __builtin_amdgcn_exp2f exp2f
#define __builtin_amdgcn_rcpf(v) (1.0f / (v))
#define __builtin_amdgcn_ldexpf ldexpf
#define __builtin_amdgcn_fmed3f(v, lo, hi) fminf(fmaxf(v, lo), hi)
#define __builtin_amdgcn_fence gpu::ignore
#define __builtin_amdgcn_s_barrier gpu::ignore
#define __builtin_amdgcn_s_waitcnt gpu::ignore
#define __builtin_amdgcn_sched_barrier gpu::ignore

// inner.cuh -- element access shared by the inner step's kernels: fp32 values in and out of the
// three element types, one element or 16 bytes at a time.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace isoloco {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// 16 bytes of elements
template <class T>
struct Vec {
    static constexpr int kN = 16 / static_cast<int>(sizeof(T));
    uint4 raw;
    __device__ __forceinline__ void unpack(float (&f)[kN]) const {
        if constexpr (sizeof(T) == 4) {
            f[0] = __uint_as_float(raw.x);
            f[1] = __uint_as_float(raw.y);
            f[2] = __uint_as_float(raw.z);
            f[3] = __uint_as_float(raw.w);
        } else {
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2 && __is_same(T, __half)) {
                    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                    f[2 * i] = v.x;
                    f[2 * i + 1] = v.y;
                } else {
                    f[2 * i] = __uint_as_float(w[i] << 16);
                    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                }
            }
        }
    }
    __device__ __forceinline__ void pack(const float (&f)[kN]) {
        if constexpr (sizeof(T) == 4) {
            raw = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (__is_same(T, __half)) {
                    const __half2 v = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t*>(&v);
                } else {
                    const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t*>(&v);
                }
            }
            raw = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
};

// Kernels of one call that follow one another: the next one's launch and first instructions pass behind the end
// of this one (next_may_start, then launch_next), up to its own after_previous(), which waits until the
// kernel before is complete and its writes are seen.
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <class... P, class... A>
inline cudaError_t launch_next(void (*kernel)(P...), dim3 grid, unsigned threads, cudaStream_t st, A... args) {
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

// Streaming accesses: read or written once, so they need not stay in L2.
__device__ __forceinline__ uint4 ld_stream(const void* p) { return __ldcs(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ void st_stream(void* p, uint4 v) { __stcs(reinterpret_cast<uint4*>(p), v); }

__host__ __device__ inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The token id at position t, or -1 where it is none of [0, vocab).
template <class I>
__device__ __forceinline__ int64_t token_at(const I* ids, int64_t t, int64_t vocab) {
    const int64_t v = static_cast<int64_t>(ids[t]);
    return (v >= 0 && v < vocab) ? v : -1;
}

}  // namespace isoloco

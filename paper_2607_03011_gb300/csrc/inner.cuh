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

// 16 bytes from an address that is a multiple of 2: the aligned pieces that hold them, shifted together.
__device__ __forceinline__ uint4 load16_any(const void* p) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const uint4* q = reinterpret_cast<const uint4*>(at & ~uintptr_t(15));
    const uint32_t off = static_cast<uint32_t>(at & 15u);
    const uint4 a = __ldg(q);
    if (off == 0) return a;
    const uint4 b = __ldg(q + 1);
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (off & 8u) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (off & 4u) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    const uint32_t bits = (off & 3u) * 8u;
    return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                      __funnelshift_r(w[3], w[4], bits));
}

// Rows whose addresses are no multiples of 16 bytes are written in pieces: piece 0 the elements before the row's first
// 16-byte boundary, piece j the j-th 16 bytes behind it, the last cut short by the row's end.
__host__ __device__ __forceinline__ uint32_t any_pieces(int64_t cols, int per_vec) { return static_cast<uint32_t>((cols + per_vec - 1) / per_vec + 1); }

// Piece j of dst[0 .. cols) = scale src[0 .. cols), zeros without src.
template <class T>
__device__ __forceinline__ void put_piece(const T* src, T* dst, int64_t cols, uint32_t j, float scale) {
    constexpr int V = Vec<T>::kN;
    const uint32_t mis = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(dst) & 15u);
    const int64_t head = min(cols, static_cast<int64_t>(mis ? (16u - mis) / sizeof(T) : 0u));
    const int64_t from = j ? head + static_cast<int64_t>(j - 1) * V : 0, to = j ? min(cols, from + V) : head;
    if (j && from + V <= cols) {
        Vec<T> v;
        v.raw = src ? load16_any(src + from) : make_uint4(0, 0, 0, 0);
        if (scale != 1.f && src) {
            float f[V];
            v.unpack(f);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] *= scale;
            v.pack(f);
        }
        st_stream(dst + from, v.raw);
    } else {
        for (int64_t i = from; i < to; ++i) dst[i] = !src ? from_f32<T>(0.f) : scale == 1.f ? src[i] : from_f32<T>(to_f32(src[i]) * scale);
    }
}

// The token id at position t, or -1 where it is none of [0, vocab).
template <class I>
__device__ __forceinline__ int64_t token_at(const I* ids, int64_t t, int64_t vocab) {
    const int64_t v = static_cast<int64_t>(ids[t]);
    return (v >= 0 && v < vocab) ? v : -1;
}

}  // namespace isoloco

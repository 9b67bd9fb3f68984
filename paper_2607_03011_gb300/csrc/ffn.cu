// ffn.cu -- gated feed-forward block, h = act(x Wg) * (x Wu), and its gradient.
#include <algorithm>

#include "inner.cuh"
#include "inner.h"

namespace isoloco {

namespace {

constexpr int kFt = 32;  // tile edge of the plain kernels

__device__ __forceinline__ float act_value(float g, int act) {
    if (act == ISOLOCO_SILU) return g / (1.f + expf(-g));
    return 0.5f * g * (1.f + tanhf(0.7978845608028654f * (g + 0.044715f * g * g * g)));
}
__device__ __forceinline__ float act_slope(float g, int act) {
    if (act == ISOLOCO_SILU) {
        const float s = 1.f / (1.f + expf(-g));
        return s * (1.f + g * (1.f - s));
    }
    const float t = tanhf(0.7978845608028654f * (g + 0.044715f * g * g * g));
    return 0.5f * (1.f + t) + 0.5f * g * (1.f - t * t) * 0.7978845608028654f * (1.f + 0.134145f * g * g);
}

// value clamped to the type's finite range: a saved product of inf would make NaN of 0 * inf
template <class T>
__device__ __forceinline__ T finite(float v) {
    const float most = __is_same(T, __half) ? 65504.f : 3.3895314e38f;
    return from_f32<T>(v > most ? most : v < -most ? -most : v);  // (NaN stays)
}

// acc(m, n) += sum_k A(m, k) B(k, n), element strides given; 32 x 32 outputs per CTA of 256 threads,
// 4 rows per thread.
template <class T>
__device__ __forceinline__ void tile_product(const T* A, int64_t sam, int64_t sak, const T* B, int64_t sbk, int64_t sbn, int64_t M,
                                             int64_t N, int64_t K, int64_t m0, int64_t n0, float (&acc)[4]) {
    __shared__ float as[kFt][kFt + 1], bs[kFt][kFt + 1];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    for (int64_t k0 = 0; k0 < K; k0 += kFt) {
        for (int i = ty; i < kFt; i += 8) {
            // the index along which memory is contiguous goes to the lanes
            const int am = sak == 1 ? i : tx, ak = sak == 1 ? tx : i;
            as[ak][am] = (m0 + am < M && k0 + ak < K) ? to_f32(A[(m0 + am) * sam + (k0 + ak) * sak]) : 0.f;
            const int bn = sbn == 1 ? tx : i, bk = sbn == 1 ? i : tx;
            bs[bk][bn] = (n0 + bn < N && k0 + bk < K) ? to_f32(B[(k0 + bk) * sbk + (n0 + bn) * sbn]) : 0.f;
        }
        __syncthreads();
#pragma unroll 8
        for (int k = 0; k < kFt; ++k) {
            const float b = bs[k][tx];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += as[k][ty * 4 + i] * b;
        }
        __syncthreads();
    }
}

template <class T>
__global__ void __launch_bounds__(256) k_ffn(FfnArgs a, T* h, int64_t ld_h, T* saved, int64_t fp) {
    const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kFt, n0 = static_cast<int64_t>(blockIdx.y) * kFt;
    float g[4] = {}, u[4] = {};
    const T* x = static_cast<const T*>(a.x);
    tile_product<T>(x, a.ld_x, 1, static_cast<const T*>(a.wg), a.ld_w, 1, a.tokens, a.ff, a.width, m0, n0, g);
    tile_product<T>(x, a.ld_x, 1, static_cast<const T*>(a.wu), a.ld_w, 1, a.tokens, a.ff, a.width, m0, n0, u);
    const int64_t n = n0 + (threadIdx.x & 31);
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + (threadIdx.x >> 5) * 4 + i;
        if (m >= a.tokens || n >= a.ff) continue;
        h[m * ld_h + n] = from_f32<T>(act_value(g[i], a.act) * u[i]);
        if (saved) {
            saved[m * 2 * fp + n] = finite<T>(g[i]);
            saved[m * 2 * fp + fp + n] = finite<T>(u[i]);
        }
    }
}

// d: tokens x 2 x fp, dg then du
template <class T>
__global__ void __launch_bounds__(256) k_ffn_dgu(FfnArgs a, const T* dh, int64_t ld_dh, const T* saved, T* d, int64_t fp) {
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (n >= a.ff) return;
    for (int64_t m = blockIdx.y; m < a.tokens; m += gridDim.y) {
        const float g = to_f32(saved[m * 2 * fp + n]), u = to_f32(saved[m * 2 * fp + fp + n]), v = to_f32(dh[m * ld_dh + n]);
        d[m * 2 * fp + n] = from_f32<T>(v * u * act_slope(g, a.act));
        d[m * 2 * fp + fp + n] = from_f32<T>(v * act_value(g, a.act));
    }
}

template <class T>
__global__ void __launch_bounds__(256) k_ffn_dx(FfnArgs a, const T* d, int64_t fp, T* dx, int64_t ld_dx) {
    const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kFt, n0 = static_cast<int64_t>(blockIdx.y) * kFt;
    float acc[4] = {};
    tile_product<T>(d, 2 * fp, 1, static_cast<const T*>(a.wg), 1, a.ld_w, a.tokens, a.width, a.ff, m0, n0, acc);
    tile_product<T>(d + fp, 2 * fp, 1, static_cast<const T*>(a.wu), 1, a.ld_w, a.tokens, a.width, a.ff, m0, n0, acc);
    const int64_t n = n0 + (threadIdx.x & 31);
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + (threadIdx.x >> 5) * 4 + i;
        if (m < a.tokens && n < a.width) dx[m * ld_dx + n] = from_f32<T>(acc[i]);
    }
}

template <class T>
__global__ void __launch_bounds__(256) k_ffn_dw(FfnArgs a, const T* d, int64_t fp, T* dwg, T* dwu, int64_t ld_dw) {
    const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kFt, n0 = static_cast<int64_t>(blockIdx.y) * kFt;
    T* dw = blockIdx.z ? dwu : dwg;
    float acc[4] = {};
    tile_product<T>(static_cast<const T*>(a.x), 1, a.ld_x, d + blockIdx.z * fp, 2 * fp, 1, a.width, a.ff, a.tokens, m0, n0, acc);
    const int64_t n = n0 + (threadIdx.x & 31);
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + (threadIdx.x >> 5) * 4 + i;
        if (m < a.width && n < a.ff) dw[m * ld_dw + n] = from_f32<T>(acc[i]);
    }
}

inline int64_t pitch_of(int64_t ff) { return (ff + 7) / 8 * 8; }
inline unsigned tiles(int64_t n) { return static_cast<unsigned>((n + kFt - 1) / kFt); }

template <class T>
cudaError_t grad_t(const FfnArgs& a, const void* dh, int64_t ld_dh, const void* saved, void* dx, int64_t ld_dx, void* dwg, void* dwu,
                   int64_t ld_dw, void* ws, cudaStream_t st) {
    const int64_t fp = pitch_of(a.ff);
    T* d = static_cast<T*>(ws);
    if (a.tokens) {
        k_ffn_dgu<T><<<dim3(static_cast<unsigned>((a.ff + 255) / 256), static_cast<unsigned>(std::min<int64_t>(a.tokens, 65535))), 256, 0,
                       st>>>(a, static_cast<const T*>(dh), ld_dh, static_cast<const T*>(saved), d, fp);
        if (dx) k_ffn_dx<T><<<dim3(tiles(a.tokens), tiles(a.width)), 256, 0, st>>>(a, d, fp, static_cast<T*>(dx), ld_dx);
    }
    if (dwg) k_ffn_dw<T><<<dim3(tiles(a.width), tiles(a.ff), 2), 256, 0, st>>>(a, d, fp, static_cast<T*>(dwg), static_cast<T*>(dwu), ld_dw);
    return cudaGetLastError();
}

}  // namespace

int64_t ffn_saved_bytes(int64_t tokens, int64_t ff) { return tokens * 2 * pitch_of(ff) * 2 + 16; }
int64_t ffn_workspace(int64_t tokens, int64_t, int64_t ff, bool backward) { return backward ? ffn_saved_bytes(tokens, ff) : 16; }

cudaError_t launch_ffn(const FfnArgs& a, void* h, int64_t ld_h, void* saved, void*, cudaStream_t st) {
    if (a.tokens == 0) return cudaSuccess;
    const dim3 grid(tiles(a.tokens), tiles(a.ff));
    if (a.dtype == ISOLOCO_BF16)
        k_ffn<__nv_bfloat16><<<grid, 256, 0, st>>>(a, static_cast<__nv_bfloat16*>(h), ld_h, static_cast<__nv_bfloat16*>(saved), pitch_of(a.ff));
    else
        k_ffn<__half><<<grid, 256, 0, st>>>(a, static_cast<__half*>(h), ld_h, static_cast<__half*>(saved), pitch_of(a.ff));
    return cudaGetLastError();
}

cudaError_t launch_ffn_grad(const FfnArgs& a, const void* dh, int64_t ld_dh, const void* saved, void* dx, int64_t ld_dx, void* dwg,
                            void* dwu, int64_t ld_dw, void* ws, cudaStream_t st) {
    if (a.dtype == ISOLOCO_BF16) return grad_t<__nv_bfloat16>(a, dh, ld_dh, saved, dx, ld_dx, dwg, dwu, ld_dw, ws, st);
    return grad_t<__half>(a, dh, ld_dh, saved, dx, ld_dx, dwg, dwu, ld_dw, ws, st);
}

}  // namespace isoloco

// logprob.cu -- log probabilities of given tokens, entropy, largest alternatives, and the gradient
// of the first two by the logits.
#include <algorithm>

#include "inner.cuh"
#include "inner.h"

namespace isoloco {

namespace {

constexpr int kLpThreads = 256;

template <class I>
__device__ __forceinline__ int64_t target_at(const I* t, int64_t r, int64_t vocab) { return token_at(t, r, vocab); }

__device__ __forceinline__ float cta_max(float v, float* sm) {
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
    __syncthreads();
    for (int i = 0; i < kLpThreads / 32; ++i) v = fmaxf(v, sm[i]);
    return v;
}
__device__ __forceinline__ float cta_sum(float v, float* sm) {
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < kLpThreads / 32; ++i) v += sm[i];
    return v;
}

// Greater logits first, then lower indices.
__device__ __forceinline__ bool before(float a, int64_t ia, float b, int64_t ib) { return a > b || (a == b && ia < ib); }

// One row per CTA, one pass over it for each of the maximum, the sums and every alternative.
template <class T, class I>
__global__ void __launch_bounds__(kLpThreads) k_logprobs(LogprobArgs a) {
    __shared__ float sm[kLpThreads / 32];
    __shared__ float sv[kLpThreads / 32];
    __shared__ int64_t si[kLpThreads / 32];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.logits) + r * a.ld;
        float m = -INFINITY;
        for (int64_t j = threadIdx.x; j < a.vocab; j += kLpThreads) m = fmaxf(m, to_f32(x[j]));
        m = cta_max(m, sm);
        float s = 0.f, w = 0.f;
        for (int64_t j = threadIdx.x; j < a.vocab; j += kLpThreads) {
            const float v = to_f32(x[j]);
            const float d = v == m ? 0.f : (v - m) * a.scale;
            const float e = expf(d);
            s += e;
            if (e != 0.f) w += e * d;
        }
        s = cta_sum(s, sm);
        w = cta_sum(w, sm);
        const bool none = m == -INFINITY && s == s;  // (s is NaN if an entry is)
        const float lse = none ? m : a.scale * m + logf(s);
        if (m == INFINITY) s = NAN;
        const float ent = none ? 0.f : logf(s) - w / s;
        const int64_t t = target_at(static_cast<const I*>(a.targets), r, a.vocab);
        if (threadIdx.x == 0) {
            if (a.logp) a.logp[r] = t < 0 ? 0.f : none ? m : (to_f32(x[t]) - m) * a.scale - logf(s);
            if (a.entropy) a.entropy[r] = ent;
            if (a.lse) a.lse[r] = m == INFINITY ? NAN : lse;
        }
        float pv = INFINITY;
        int64_t pi = -1;
        for (int k = 0; k < a.top; ++k) {
            float bv = -INFINITY;
            int64_t bi = a.vocab;
            for (int64_t j = threadIdx.x; j < a.vocab; j += kLpThreads) {
                const float v = to_f32(x[j]);
                if (before(pv, pi, v, j) && before(v, j, bv, bi)) {
                    bv = v;
                    bi = j;
                }
            }
            for (int o = 16; o; o >>= 1) {
                const float ov = __shfl_xor_sync(0xffffffffu, bv, o);
                const int64_t oi = __shfl_xor_sync(0xffffffffu, bi, o);
                if (before(ov, oi, bv, bi)) bv = ov, bi = oi;
            }
            __syncthreads();
            if ((threadIdx.x & 31) == 0) sv[threadIdx.x >> 5] = bv, si[threadIdx.x >> 5] = bi;
            __syncthreads();
            for (int i = 0; i < kLpThreads / 32; ++i)
                if (before(sv[i], si[i], bv, bi)) bv = sv[i], bi = si[i];
            if (bi >= a.vocab) bi = a.vocab - 1;  // fewer comparable logits than asked for (NaN)
            if (threadIdx.x == 0) {
                a.top_index[r * a.top + k] = bi;
                a.top_logp[r * a.top + k] = none ? m : (to_f32(x[bi]) - m) * a.scale - logf(s);
            }
            pv = bv;
            pi = bi;
        }
        if (a.grad_logits) {
            const float gl = (t >= 0 && a.grad_logp) ? a.grad_logp[r] : 0.f;
            const float ge = a.grad_entropy ? a.grad_entropy[r] : 0.f;
            const float ls = logf(s);
            T* o = static_cast<T*>(a.grad_logits) + r * a.ld_grad;
            __syncthreads();
            for (int64_t j = threadIdx.x; j < a.vocab; j += kLpThreads) {
                const float v = to_f32(x[j]);
                const float lp = (v == m ? 0.f : (v - m) * a.scale) - ls;
                const float p = expf(lp);
                float g = (j == t ? gl : 0.f) - gl * p;
                if (p != 0.f) g -= ge * p * (lp + ent);
                o[j] = from_f32<T>(none ? 0.f : g * a.scale);
            }
        }
        __syncthreads();
    }
}

template <class T, class I>
__global__ void __launch_bounds__(kLpThreads) k_logprobs_grad(LogprobArgs a) {
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.logits) + r * a.ld;
        T* o = static_cast<T*>(a.grad_logits) + r * a.ld_grad;
        const int64_t t = target_at(static_cast<const I*>(a.targets), r, a.vocab);
        const float lse = a.lse[r], ent = a.entropy ? a.entropy[r] : 0.f;
        const bool none = lse == -INFINITY;
        const float gl = (t >= 0 && a.grad_logp) ? a.grad_logp[r] : 0.f;
        const float ge = a.grad_entropy ? a.grad_entropy[r] : 0.f;
        for (int64_t j = threadIdx.x; j < a.vocab; j += kLpThreads) {
            const float lp = to_f32(x[j]) * a.scale - lse;
            const float p = expf(lp);
            float g = (j == t ? gl : 0.f) - gl * p;
            if (p != 0.f) g -= ge * p * (lp + ent);
            o[j] = from_f32<T>(none ? 0.f : g * a.scale);
        }
    }
}

template <class T>
cudaError_t run(const LogprobArgs& a, bool grad_only, cudaStream_t st) {
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(a.rows, 1 << 20));
    if (grad_only) {
        if (a.targets64) k_logprobs_grad<T, int64_t><<<grid, kLpThreads, 0, st>>>(a);
        else k_logprobs_grad<T, int32_t><<<grid, kLpThreads, 0, st>>>(a);
    } else {
        if (a.targets64) k_logprobs<T, int64_t><<<grid, kLpThreads, 0, st>>>(a);
        else k_logprobs<T, int32_t><<<grid, kLpThreads, 0, st>>>(a);
    }
    return cudaGetLastError();
}

cudaError_t dispatch(const LogprobArgs& a, bool grad_only, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    if (a.dtype == ISOLOCO_F32) return run<float>(a, grad_only, st);
    if (a.dtype == ISOLOCO_BF16) return run<__nv_bfloat16>(a, grad_only, st);
    return run<__half>(a, grad_only, st);
}

}  // namespace

int64_t logprob_workspace(int64_t, int64_t, int) { return 16; }

cudaError_t launch_logprobs(const LogprobArgs& a, void*, cudaStream_t st) { return dispatch(a, false, st); }
cudaError_t launch_logprobs_grad(const LogprobArgs& a, cudaStream_t st) { return dispatch(a, true, st); }

}  // namespace isoloco

// clip.cu -- the global norm of a gradient held in many tensors, and clipping by it.
//
//     n = sqrt(sum over all tensors and entries of g^2),   g' = g min(1, max_norm / n)
//
// The table of addresses and lengths travels in the kernel's parameters, so no copy to the device
// precedes the call.  Two launches per table (kMaxTensors tensors): the first sums squares over fixed chunks
// (fp32 within a thread, fp64 from there on) and leaves one fp64 partial per CTA; the second adds the
// partials, every CTA in the same order, so that all have the same bits, and scales.  A short list of
// small tensors takes one launch of one cluster (k_grad_small), whose CTAs exchange their sums in shared memory.
//
// Bound by HBM.  219.7 M fp32 entries in 110 tensors: squares 127 us (6.9 TB/s), scaling into other tensors
// 267 us (6.6 TB/s of the second read and the write; of the 64 MB that the first pass leaves in L2 it
// gains 2 us).
#include <algorithm>
#include <cmath>

#include "common.cuh"
#include "inner.cuh"
#include "inner.h"

namespace isoloco {

namespace {

constexpr int kClipThreads = 256;
constexpr int kMaxTensors = 512;       // of one table: 512 x 32 bytes of kernel parameters
constexpr int kFewTensors = 32;        // a short list's parameters are a 16th of that (launch and first reads)
constexpr int kChunkBytes = 32768;     // a CTA's unit of work: 8 16-byte loads per thread
constexpr int kCtasPerSm = 8;
constexpr int kSmallCluster = 8;       // CTAs of k_grad_small
constexpr int kSmallChunks = 64;       // 2 MB: what that takes, 8 chunks per CTA
constexpr int kKeepChunks = 2048;      // the last 64 MB stay in L2 for the scaling, which begins with them

struct ClipTensor {
    const void* in;
    void* out;
    int64_t n;
    int32_t dtype;
    int32_t first;  // chunk number of its first chunk
};

template <int N>
struct ClipTable {
    ClipTensor t[N];
    int count;
    int chunks;
};

// The chunk's elements [lo, hi) of tensor `t` and the first of them at a 16-byte address.  Chunk 0
// also holds the elements before the tensor's first 16-byte boundary.
struct ChunkSpan {
    int64_t lo, mid, hi;
};

template <class T>
__device__ __forceinline__ ChunkSpan chunk_span(const ClipTensor& t, int c) {
    constexpr int kElems = kChunkBytes / static_cast<int>(sizeof(T));
    const uint32_t mis = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(t.in) & 15u);
    const int64_t head = mis ? (16 - mis) / sizeof(T) : 0;
    ChunkSpan s;
    s.lo = c ? head + static_cast<int64_t>(c) * kElems : 0;
    s.mid = min(t.n, head + static_cast<int64_t>(c) * kElems);
    s.hi = min(t.n, head + static_cast<int64_t>(c + 1) * kElems);
    return s;
}

template <int N>
__device__ __forceinline__ int find_tensor(const ClipTable<N>& tab, int chunk) {
    int lo = 0, hi = tab.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.t[mid].first <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <class T>
__device__ __forceinline__ float chunk_squares(const ClipTensor& t, int c, bool keep) {
    const ChunkSpan s = chunk_span<T>(t, c);
    const T* p = static_cast<const T*>(t.in);
    constexpr int V = Vec<T>::kN;
    float acc = 0.f;
    for (int64_t i = s.lo + threadIdx.x; i < s.mid; i += kClipThreads) {
        const float v = to_f32(p[i]);
        acc += v * v;
    }
    const int64_t nvec = (s.hi - s.mid) / V;
    const T* q = p + s.mid;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < nvec; i += kClipThreads) {
        Vec<T> v;
        v.raw = keep ? __ldg(reinterpret_cast<const uint4*>(q + i * V)) : ld_stream(q + i * V);
        float f[V];
        v.unpack(f);
#pragma unroll
        for (int j = 0; j < V; ++j) acc += f[j] * f[j];
    }
    for (int64_t i = s.mid + nvec * V + threadIdx.x; i < s.hi; i += kClipThreads) {
        const float v = to_f32(p[i]);
        acc += v * v;
    }
    return acc;
}

template <class T>
__device__ __forceinline__ void chunk_scale(const ClipTensor& t, int c, float coef) {
    const ChunkSpan s = chunk_span<T>(t, c);
    const T* p = static_cast<const T*>(t.in);
    T* o = static_cast<T*>(t.out);
    constexpr int V = Vec<T>::kN;
    const bool vec = ((reinterpret_cast<uintptr_t>(t.in) ^ reinterpret_cast<uintptr_t>(t.out)) & 15u) == 0;
    const int64_t nvec = vec ? (s.hi - s.mid) / V : 0;
    for (int64_t i = s.lo + threadIdx.x; i < s.mid; i += kClipThreads) o[i] = coef == 1.f ? p[i] : from_f32<T>(to_f32(p[i]) * coef);
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < nvec; i += kClipThreads) {
        Vec<T> v;
        v.raw = ld_stream(p + s.mid + i * V);
        if (coef != 1.f) {  // (a copy keeps every bit, a NaN's too)
            float f[V];
            v.unpack(f);
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] *= coef;
            v.pack(f);
        }
        st_stream(o + s.mid + i * V, v.raw);
    }
    for (int64_t i = s.mid + nvec * V + threadIdx.x; i < s.hi; i += kClipThreads) o[i] = coef == 1.f ? p[i] : from_f32<T>(to_f32(p[i]) * coef);
}

// Sum over the CTA; every thread gets it.
__device__ __forceinline__ double cta_sum(double v) {
    __shared__ double part[kClipThreads / 32];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kClipThreads / 32; ++i) s += part[i];
    return s;
}

template <int N>
__device__ __forceinline__ float squares_of(const ClipTable<N>& tab, int c, bool keep) {
    const ClipTensor& t = tab.t[find_tensor(tab, c)];
    const int k = c - t.first;
    return t.dtype == ISOLOCO_F32 ? chunk_squares<float>(t, k, keep)
           : t.dtype == ISOLOCO_BF16 ? chunk_squares<__nv_bfloat16>(t, k, keep) : chunk_squares<__half>(t, k, keep);
}
template <int N>
__device__ __forceinline__ void scale_by(const ClipTable<N>& tab, int c, float coef) {
    const ClipTensor& t = tab.t[find_tensor(tab, c)];
    const int k = c - t.first;
    if (t.dtype == ISOLOCO_F32) chunk_scale<float>(t, k, coef);
    else if (t.dtype == ISOLOCO_BF16) chunk_scale<__nv_bfloat16>(t, k, coef);
    else chunk_scale<__half>(t, k, coef);
}

__device__ __forceinline__ float root_of(double s) {
    return s > 1e30 ? sqrtf(static_cast<float>(s * 0x1p-64)) * 0x1p32f : sqrtf(static_cast<float>(s));
}
// A norm that is not finite, or zero, scales nothing.
__device__ __forceinline__ float coef_of(float norm, float max_norm) { return norm > max_norm && norm < INFINITY ? max_norm / norm : 1.f; }

template <int N>
__global__ void __launch_bounds__(kClipThreads) k_grad_squares(const __grid_constant__ ClipTable<N> tab, double* part) {
    next_may_start();
    double acc = 0.0;
    for (int c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
        acc += static_cast<double>(squares_of(tab, c, tab.chunks - c <= kKeepChunks));
    }
    const double s = cta_sum(acc);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm from the partials, the same bits in every thread of every CTA.  (fp64 is slow here: warps without
// partials add nothing, and the root is fp32's, of a sum brought into its range.)
__device__ __forceinline__ float norm_of(const double* part, int nparts) {
    __shared__ double sum[kClipThreads / 32];
    const int warp = threadIdx.x >> 5, warps = min(kClipThreads / 32, (nparts + 31) / 32);
    if (warp < warps) {
        double s = 0.0;
        for (int i = threadIdx.x; i < nparts; i += kClipThreads) s += part[i];
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if ((threadIdx.x & 31) == 0) sum[warp] = s;
    }
    __syncthreads();
    double s = warps ? sum[0] : 0.0;
    for (int i = 1; i < warps; ++i) s += sum[i];
    return root_of(s);
}

// tab.chunks == 0: the norm only.
template <int N>
__global__ void __launch_bounds__(kClipThreads) k_grad_scale(const __grid_constant__ ClipTable<N> tab, const double* part,
                                                             int nparts, float max_norm, bool in_place, float* norm) {
    after_previous();
    const float n = norm_of(part, nparts);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = n;
    const float coef = coef_of(n, max_norm);
    if (in_place && coef == 1.f) return;
    // from the last chunk down: what the first pass read last is still in L2
    for (int c = tab.chunks - 1 - static_cast<int>(blockIdx.x); c >= 0; c -= gridDim.x) scale_by(tab, c, coef);
}

// (max_norm: negative for the norm alone)
__global__ void __cluster_dims__(kSmallCluster, 1, 1) __launch_bounds__(kClipThreads)
    k_grad_small(const __grid_constant__ ClipTable<kFewTensors> tab, float max_norm, bool in_place, float* norm) {
    __shared__ double sums[kSmallCluster];  // of every CTA, in every CTA
    const uint32_t rank = cluster_ctarank();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    double acc = 0.0;
    for (int c = rank; c < tab.chunks; c += kSmallCluster) acc += static_cast<double>(squares_of(tab, c, true));
    acc = cta_sum(acc);
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // every CTA runs: its shared memory may be written
    if (threadIdx.x < kSmallCluster)
        asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(mapa_shared(smem_u32(sums + rank), threadIdx.x)), "d"(acc) : "memory");
    cluster_sync();
    double s = 0.0;
    for (int i = 0; i < kSmallCluster; ++i) s += sums[i];
    const float n = root_of(s);
    if (rank == 0 && threadIdx.x == 0) norm[0] = n;
    const float coef = coef_of(n, max_norm);
    if (max_norm < 0.f || (in_place && coef == 1.f)) return;
    for (int c = rank; c < tab.chunks; c += kSmallCluster) scale_by(tab, c, coef);
}

int chunks_of(const isoloco_tensor_t& t) {
    const int es = t.dtype == ISOLOCO_F32 ? 4 : 2;
    const uint32_t mis = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(t.data) & 15u);
    const int64_t head = mis ? (16 - mis) / es : 0;
    const int64_t body = std::max<int64_t>(0, t.n - head), per = kChunkBytes / es;
    return static_cast<int>(std::max<int64_t>(1, (body + per - 1) / per));
}

}  // namespace

namespace {

bool is_small(const isoloco_tensor_t* in, int count) {
    if (count > kFewTensors) return false;
    int chunks = 0;
    for (int i = 0; i < count && chunks <= kSmallChunks; ++i)
        if (in[i].n) chunks += chunks_of(in[i]);
    return chunks <= kSmallChunks;
}

}  // namespace

// One table per kMaxTensors tensors, at most kCtasPerSm partials per SM each.
int64_t grad_norm_workspace(const isoloco_tensor_t* in, int count) {
    if (is_small(in, count)) return 0;
    const int64_t tables = (count + kMaxTensors - 1) / kMaxTensors;
    return tables * 1024 * kCtasPerSm * static_cast<int64_t>(sizeof(double));
}

namespace {

// Fills `tab` with the tensors from `i` on that have entries; returns the next one's place.
template <int N>
int fill_table(ClipTable<N>& tab, const isoloco_tensor_t* in, const isoloco_tensor_t* out, int i, int count) {
    tab.count = tab.chunks = 0;
    for (; i < count && tab.count < N; ++i) {
        if (in[i].n == 0) continue;
        ClipTensor& t = tab.t[tab.count++];
        t.in = in[i].data;
        t.out = out ? out[i].data : in[i].data;
        t.n = in[i].n;
        t.dtype = in[i].dtype;
        t.first = tab.chunks;
        tab.chunks += chunks_of(in[i]);  // (below 2^21 each: lengths are at most 2^33)
    }
    return i;
}

template <int N>
cudaError_t clip_n(const isoloco_tensor_t* in, const isoloco_tensor_t* out, int count, bool clip, float max_norm, float* norm, double* part,
                   int max_grid, cudaStream_t st) {
    int nparts = 0;
    cudaError_t e = cudaSuccess;
    ClipTable<N> tab;
    for (int i = 0; i < count;) {
        i = fill_table(tab, in, out, i, count);
        if (!tab.count) continue;
        const int grid = std::min(tab.chunks, max_grid);
        k_grad_squares<N><<<grid, kClipThreads, 0, st>>>(tab, part + nparts);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        nparts += grid;
    }
    const double* sums = part;
    bool written = false;
    for (int i = 0; clip && i < count;) {
        if (count > N || i > 0) i = fill_table(tab, in, out, i, count);  // (one table: it is the squares')
        else i = count;
        if (!tab.count) continue;
        const int grid = std::min(tab.chunks, max_grid);
        if ((e = launch_next(k_grad_scale<N>, grid, kClipThreads, st, tab, sums, nparts, max_norm, out == nullptr, norm)) != cudaSuccess) return e;
        written = true;
    }
    if (written) return e;
    tab.count = tab.chunks = 0;
    return launch_next(k_grad_scale<N>, 1, kClipThreads, st, tab, sums, nparts, 0.f, true, norm);
}

}  // namespace

cudaError_t launch_clip(const isoloco_tensor_t* in, const isoloco_tensor_t* out, int count, bool clip, float max_norm,
                        float* norm, void* ws, cudaStream_t st) {
    if (is_small(in, count)) {
        ClipTable<kFewTensors> tab;
        (void)fill_table(tab, in, out, 0, count);
        k_grad_small<<<kSmallCluster, kClipThreads, 0, st>>>(tab, clip ? max_norm : -1.f, out == nullptr, norm);
        return cudaGetLastError();
    }
    int sms = 0;
    const cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
    const int max_grid = std::min(1024, sms) * kCtasPerSm;
    double* part = static_cast<double*>(ws);
    return count <= kFewTensors ? clip_n<kFewTensors>(in, out, count, clip, max_norm, norm, part, max_grid, st)
                                : clip_n<kMaxTensors>(in, out, count, clip, max_norm, norm, part, max_grid, st);
}

}  // namespace isoloco

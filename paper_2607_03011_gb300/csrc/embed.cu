// embed.cu -- embedding lookup and its gradient.
//
//     y[t] = scale W[id_t]            dW[v] = scale sum_{t : id_t = v} dy[t]
//
// The gradient sorts the positions by token id (stable least-significant-digit radix sort in one
// thread-block cluster), so that a row's terms stand together, in the order of their positions:
//   k_embed_sort   cluster 0 sorts; the other CTAs meanwhile write the zeros of every row of dW.
//   k_embed_sum    a CTA adds kSpan consecutive sorted positions, in fp32, all columns; a row whose
//                  positions lie within one span is written at once, the sums at a span's ends
//                  that belong to a row shared with other spans go to the workspace.
//   k_embed_join   adds those, span by span in order, and writes their rows.
// Which terms are added in which order depends on the ids alone.
#include <algorithm>

#include "common.cuh"
#include "inner.cuh"
#include "inner.h"

namespace isoloco {

namespace {

constexpr int kRowThreads = 128;

// ------------------------------------------------------------------ lookup
// One row of y per CTA and step; 16 bytes per access when VEC.
template <class T, class I, bool VEC>
__global__ void __launch_bounds__(kRowThreads) k_embed(const T* __restrict__ w, int64_t ld_w, int64_t vocab, int64_t width,
                                                       const I* __restrict__ ids, int64_t tokens, float scale,
                                                       T* __restrict__ y, int64_t ld_y) {
    constexpr int V = VEC ? Vec<T>::kN : 1;
    const int64_t c = (static_cast<int64_t>(blockIdx.x) * kRowThreads + threadIdx.x) * V;
    if (c >= width) return;
    for (int64_t t = blockIdx.y; t < tokens; t += gridDim.y) {
        const int64_t id = token_at(ids, t, vocab);
        if constexpr (VEC) {
            Vec<T> v;
            v.raw = make_uint4(0, 0, 0, 0);
            if (id >= 0) {
                v.raw = __ldg(reinterpret_cast<const uint4*>(w + id * ld_w + c));
                float f[V];
                v.unpack(f);
#pragma unroll
                for (int j = 0; j < V; ++j) f[j] *= scale;
                v.pack(f);
            }
            *reinterpret_cast<uint4*>(y + t * ld_y + c) = v.raw;
        } else {
            y[t * ld_y + c] = id >= 0 ? from_f32<T>(to_f32(w[id * ld_w + c]) * scale) : from_f32<T>(0.f);
        }
    }
}

// ------------------------------------------------------------------ sort
constexpr int kSortCluster = 8;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kDigits = 256;

struct SortSmem {
    uint32_t warp[kSortWarps][kDigits];  // counts, then the next place of each warp's digit
    uint32_t total[kSortCluster][kDigits];  // every CTA's count of every digit
    uint32_t scan[kDigits];
};

// Positions of a cluster's keys: CTA r, warp w owns [begin, end), in order.
struct SortRange {
    int64_t begin, end;
};
__device__ __forceinline__ SortRange sort_range(int64_t n, uint32_t rank, int warp) {
    const int64_t per = (n + kSortCluster * kSortWarps - 1) / (kSortCluster * kSortWarps);
    const int64_t b = min(n, per * (static_cast<int64_t>(rank) * kSortWarps + warp));
    return {b, min(n, b + per)};
}

template <class I>
__device__ void sort_ids(SortSmem& sm, const I* ids, int64_t n, int64_t vocab, int bits, uint32_t* key[2], uint32_t* pos[2]) {
    const uint32_t rank = cluster_ctarank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const SortRange rg = sort_range(n, rank, warp);
    const int passes = (bits + 7) / 8, dbits = (bits + passes - 1) / passes;
    const uint32_t dmask = (1u << dbits) - 1u;
    cluster_sync();  // every CTA runs before another writes its shared memory
    for (int pass = 0; pass < passes; ++pass) {
        uint32_t* kdst = key[(passes - pass) & 1];  // key[1] in the last pass
        uint32_t* pdst = pos[(passes - pass) & 1];
        const uint32_t* ksrc = key[(passes - pass + 1) & 1];
        const uint32_t* psrc = pos[(passes - pass + 1) & 1];
        const int shift = pass * dbits;
        // a key that is no token sorts behind all others
        auto load = [&](int64_t i) -> uint32_t {
            if (pass) return ksrc[i];
            const int64_t v = token_at(ids, i, vocab);
            return static_cast<uint32_t>(v < 0 ? vocab : v);
        };
        for (int d = lane; d < kDigits; d += 32) sm.warp[warp][d] = 0;
        __syncwarp();
        for (int64_t i = rg.begin + lane; i < rg.end; i += 32) atomicAdd(&sm.warp[warp][(load(i) >> shift) & dmask], 1u);
        __syncthreads();
        // this CTA's total of each digit, to every CTA of the cluster
        if (threadIdx.x < kDigits) {
            uint32_t s = 0;
            for (int w = 0; w < kSortWarps; ++w) s += sm.warp[w][threadIdx.x];
            for (uint32_t r = 0; r < kSortCluster; ++r) {
                const uint32_t a = mapa_shared(smem_u32(&sm.total[rank][threadIdx.x]), r);
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(s) : "memory");
            }
        }
        cluster_sync();
        // places before this CTA's first of each digit: smaller digits anywhere, and the same
        // digit in earlier CTAs
        uint32_t all = 0, before = 0;
        if (threadIdx.x < kDigits) {
            for (uint32_t r = 0; r < kSortCluster; ++r) {
                const uint32_t v = sm.total[r][threadIdx.x];
                before += r < rank ? v : 0u;
                all += v;
            }
            // inclusive scan over the digits, warp by warp
            uint32_t s = all;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= o) s += u;
            }
            sm.scan[threadIdx.x] = s;
        }
        __syncthreads();
        if (threadIdx.x < kDigits) {
            uint32_t base = sm.scan[threadIdx.x] - all + before;
            for (int w = 0; w < warp; ++w) base += sm.scan[w * 32 + 31];
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = sm.warp[w][threadIdx.x];
                sm.warp[w][threadIdx.x] = base;
                base += c;
            }
        }
        __syncthreads();
        // stable: a warp places its keys 32 at a time, in order
        for (int64_t i0 = rg.begin; i0 < rg.end; i0 += 32) {
            const int64_t i = i0 + lane;
            const bool have = i < rg.end;
            const uint32_t k = have ? load(i) : 0u;
            const uint32_t d = have ? (k >> shift) & dmask : kDigits + lane;
            const uint32_t same = __match_any_sync(0xffffffffu, d);
            const uint32_t mine = __popc(same & ((1u << lane) - 1u));
            if (have) {
                const uint32_t at = sm.warp[warp][d] + mine;
                kdst[at] = k;
                pdst[at] = pass ? psrc[i] : static_cast<uint32_t>(i);
            }
            __syncwarp();
            if (have && mine == 0) sm.warp[warp][d] += __popc(same);
            __syncwarp();
        }
        __threadfence();
        cluster_sync();  // the pass's output is complete, and the totals may be overwritten
    }
}

// Cluster 0 sorts the positions by id into key[1], pos[1]; the others fill dw with zeros.
template <class I>
__global__ void __cluster_dims__(kSortCluster, 1, 1) __launch_bounds__(kSortThreads)
    k_embed_sort(const I* ids, int64_t n, int64_t vocab, int bits, uint32_t* k0, uint32_t* k1, uint32_t* p0, uint32_t* p1,
                 uint8_t* dw, int64_t row_bytes, int64_t ld_bytes) {
    __shared__ SortSmem sm;
    const int64_t cta = static_cast<int64_t>(blockIdx.x) - kSortCluster;
    if (cta < 0) {
        uint32_t* key[2] = {k0, k1};
        uint32_t* pos[2] = {p0, p1};
        sort_ids(sm, ids, n, vocab, bits, key, pos);
        return;
    }
    const int64_t ctas = static_cast<int64_t>(gridDim.x) - kSortCluster;
    if (ld_bytes == row_bytes && aligned16(dw)) {
        // one run of bytes
        const int64_t bytes = row_bytes * vocab, nvec = bytes / 16;
        for (int64_t i = cta * kSortThreads + threadIdx.x; i < nvec; i += ctas * kSortThreads)
            reinterpret_cast<uint4*>(dw)[i] = make_uint4(0, 0, 0, 0);
        if (cta == 0)
            for (int64_t i = nvec * 16 + threadIdx.x; i < bytes; i += kSortThreads) dw[i] = 0;
    } else {
        for (int64_t r = cta; r < vocab; r += ctas)
            for (int64_t i = threadIdx.x; i < row_bytes / 2; i += kSortThreads)
                reinterpret_cast<uint16_t*>(dw + r * ld_bytes)[i] = 0;
    }
}

// ------------------------------------------------------------------ sums
constexpr int kSpan = 32;  // sorted positions of one CTA

// part[span][0]: the sum of the span's first row, if that row began in an earlier span;
// part[span][1]: of its last row, if that goes on in a later span (and began here).
template <class T, class O, bool VEC>
__global__ void __launch_bounds__(kRowThreads) k_embed_sum(const T* __restrict__ dy, int64_t ld_dy, int64_t vocab, int64_t width,
                                                           const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos,
                                                           int64_t n, float scale, O* __restrict__ dw, int64_t ld_dw,
                                                           float* __restrict__ part) {
    constexpr int V = VEC ? Vec<T>::kN : 1;
    __shared__ uint32_t sk[kSpan + 2];  // keys from one before the span to one behind it
    __shared__ uint32_t sp[kSpan];
    const int64_t span = blockIdx.x;
    const int64_t first = span * kSpan;
    const int cnt = static_cast<int>(min(static_cast<int64_t>(kSpan), n - first));
    for (int i = threadIdx.x; i < cnt + 2; i += kRowThreads) {
        const int64_t j = first + i - 1;
        sk[i] = (j >= 0 && j < n) ? key[j] : 0xffffffffu;
    }
    for (int i = threadIdx.x; i < cnt; i += kRowThreads) sp[i] = pos[first + i];
    __syncthreads();
    const int64_t c = (static_cast<int64_t>(blockIdx.y) * kRowThreads + threadIdx.x) * V;
    if (c >= width) return;
    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    int begin = 0;  // of the row being added
    for (int i = 0; i < cnt; ++i) {
        const uint32_t k = sk[i + 1];
        if (k >= vocab) break;  // no token, nor are the later ones
        const T* src = dy + static_cast<int64_t>(sp[i]) * ld_dy + c;
        if constexpr (VEC) {
            Vec<T> v;
            v.raw = ld_stream(src);
            float f[V];
            v.unpack(f);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += f[j];
        } else {
            acc[0] += to_f32(src[0]);
        }
        const bool last = i + 1 == cnt;
        if (!last && sk[i + 2] == k) continue;
        const bool open_left = begin == 0 && sk[0] == k;
        const bool open_right = last && sk[i + 2] == k;
        if (open_left || open_right) {
            float* d = part + (span * 2 + (open_left ? 0 : 1)) * width + c;
#pragma unroll
            for (int j = 0; j < V; ++j) d[j] = acc[j];
        } else {
            O* d = dw + static_cast<int64_t>(k) * ld_dw + c;
#pragma unroll
            for (int j = 0; j < V; ++j) d[j] = from_f32<O>(acc[j] * scale);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
        begin = i + 1;
    }
}

// Rows that begin in span blockIdx.x and go on in later ones.
template <class O>
__global__ void __launch_bounds__(kRowThreads) k_embed_join(int64_t vocab, int64_t width, const uint32_t* __restrict__ key, int64_t n,
                                                            float scale, O* __restrict__ dw, int64_t ld_dw,
                                                            const float* __restrict__ part) {
    const int64_t span = blockIdx.x, first = span * kSpan, next = first + kSpan;
    if (next >= n) return;
    const uint32_t k = key[next - 1];
    if (k >= vocab || key[next] != k) return;       // nothing goes on behind this span
    if (first > 0 && key[first - 1] == k) return;   // it began earlier
    const int64_t c = static_cast<int64_t>(blockIdx.y) * kRowThreads + threadIdx.x;
    if (c >= width) return;
    float acc = part[(span * 2 + 1) * width + c];
    for (int64_t s = span + 1; s * kSpan < n && key[s * kSpan] == k; ++s) acc += part[s * 2 * width + c];
    dw[static_cast<int64_t>(k) * ld_dw + c] = from_f32<O>(acc * scale);
}

inline unsigned rows_grid(int64_t rows) { return static_cast<unsigned>(std::min<int64_t>(rows, 65535)); }

template <class T, class I>
cudaError_t embed_t(const void* w, int64_t ld_w, int64_t vocab, int64_t width, const void* ids, int64_t tokens, float scale,
                    void* y, int64_t ld_y, cudaStream_t st) {
    constexpr int64_t V = Vec<T>::kN;
    const bool vec = aligned16(w) && aligned16(y) && ld_w % V == 0 && ld_y % V == 0 && width % V == 0;
    const int64_t cols = vec ? width / V : width;
    const dim3 grid(static_cast<unsigned>((cols + kRowThreads - 1) / kRowThreads), rows_grid(tokens));
    if (vec)
        k_embed<T, I, true><<<grid, kRowThreads, 0, st>>>(static_cast<const T*>(w), ld_w, vocab, width,
                                                          static_cast<const I*>(ids), tokens, scale, static_cast<T*>(y), ld_y);
    else
        k_embed<T, I, false><<<grid, kRowThreads, 0, st>>>(static_cast<const T*>(w), ld_w, vocab, width,
                                                           static_cast<const I*>(ids), tokens, scale, static_cast<T*>(y), ld_y);
    return cudaGetLastError();
}

struct EmbedWs {
    uint32_t *k0, *k1, *p0, *p1;
    float* part;
};

int64_t r16(int64_t b) { return (b + 15) / 16 * 16; }

EmbedWs embed_ws(void* ws, int64_t tokens) {
    uint8_t* p = static_cast<uint8_t*>(ws);
    const int64_t s = r16(4 * tokens);
    return {reinterpret_cast<uint32_t*>(p), reinterpret_cast<uint32_t*>(p + s), reinterpret_cast<uint32_t*>(p + 2 * s),
            reinterpret_cast<uint32_t*>(p + 3 * s), reinterpret_cast<float*>(p + 4 * s)};
}

template <class T, class O>
cudaError_t embed_grad_t(const void* dy, int64_t ld_dy, int64_t vocab, int64_t width, const EmbedWs& w, int64_t n, float scale,
                         void* dw, int64_t ld_dw, cudaStream_t st) {
    constexpr int64_t V = Vec<T>::kN;
    const bool vec = aligned16(dy) && ld_dy % V == 0 && width % V == 0;
    const int64_t cols = vec ? width / V : width;
    const unsigned spans = static_cast<unsigned>((n + kSpan - 1) / kSpan);
    const dim3 grid(spans, static_cast<unsigned>((cols + kRowThreads - 1) / kRowThreads));
    if (vec)
        k_embed_sum<T, O, true><<<grid, kRowThreads, 0, st>>>(static_cast<const T*>(dy), ld_dy, vocab, width, w.k1, w.p1, n, scale,
                                                              static_cast<O*>(dw), ld_dw, w.part);
    else
        k_embed_sum<T, O, false><<<grid, kRowThreads, 0, st>>>(static_cast<const T*>(dy), ld_dy, vocab, width, w.k1, w.p1, n, scale,
                                                               static_cast<O*>(dw), ld_dw, w.part);
    const dim3 jgrid(spans, static_cast<unsigned>((width + kRowThreads - 1) / kRowThreads));
    k_embed_join<O><<<jgrid, kRowThreads, 0, st>>>(vocab, width, w.k1, n, scale, static_cast<O*>(dw), ld_dw, w.part);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_embed(const void* weight, int64_t ld_w, int dtype, int64_t vocab, int64_t width, const void* ids,
                         bool ids64, int64_t tokens, float scale, void* y, int64_t ld_y, cudaStream_t st) {
    if (tokens == 0) return cudaSuccess;
#define EMBED(T)                                                                                                    \
    return ids64 ? embed_t<T, int64_t>(weight, ld_w, vocab, width, ids, tokens, scale, y, ld_y, st)                  \
                 : embed_t<T, int32_t>(weight, ld_w, vocab, width, ids, tokens, scale, y, ld_y, st)
    if (dtype == ISOLOCO_F32) EMBED(float);
    if (dtype == ISOLOCO_BF16) EMBED(__nv_bfloat16);
    EMBED(__half);
#undef EMBED
}

int64_t embed_grad_workspace(int64_t vocab, int64_t width, int64_t tokens) {
    (void)vocab;
    return 4 * r16(4 * tokens) + (tokens + kSpan - 1) / kSpan * 2 * width * 4 + 16;
}

cudaError_t launch_embed_grad(const void* dy, int64_t ld_dy, int dtype, int64_t vocab, int64_t width, const void* ids,
                              bool ids64, int64_t tokens, float scale, void* dw, int64_t ld_dw, int dw_dtype, void* ws,
                              cudaStream_t st) {
    int sms = 0;
    cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
    const EmbedWs w = embed_ws(ws, tokens);
    int bits = 1;  // of the largest key, vocab
    while ((vocab >> bits) != 0) ++bits;
    const int es = dw_dtype == ISOLOCO_F32 ? 4 : 2;
    const unsigned grid = kSortCluster + std::max(1, (2 * sms) / kSortCluster) * kSortCluster;
    if (ids64)
        k_embed_sort<int64_t><<<grid, kSortThreads, 0, st>>>(static_cast<const int64_t*>(ids), tokens, vocab, bits, w.k0, w.k1, w.p0,
                                                             w.p1, static_cast<uint8_t*>(dw), width * es, ld_dw * es);
    else
        k_embed_sort<int32_t><<<grid, kSortThreads, 0, st>>>(static_cast<const int32_t*>(ids), tokens, vocab, bits, w.k0, w.k1, w.p0,
                                                             w.p1, static_cast<uint8_t*>(dw), width * es, ld_dw * es);
    if ((e = cudaGetLastError()) != cudaSuccess || tokens == 0) return e;
#define GRAD(T, O) return embed_grad_t<T, O>(dy, ld_dy, vocab, width, w, tokens, scale, dw, ld_dw, st)
    if (dtype == ISOLOCO_F32) GRAD(float, float);
    if (dtype == ISOLOCO_BF16) {
        if (dw_dtype == ISOLOCO_F32) GRAD(__nv_bfloat16, float);
        GRAD(__nv_bfloat16, __nv_bfloat16);
    }
    if (dw_dtype == ISOLOCO_F32) GRAD(__half, float);
    GRAD(__half, __half);
#undef GRAD
}

}  // namespace isoloco

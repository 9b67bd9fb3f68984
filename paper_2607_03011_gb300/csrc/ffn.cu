// ffn.cu -- gated feed-forward block and its gradient on tcgen05 tensor cores (sm_103a).
//
//     g = x Wg,  u = x Wu,  h = act(g) u                      (x: T x D, Wg and Wu: D x F)
//     dg = dh u act'(g),  du = dh act(g)
//     dx = dg Wg^T + du Wu^T,   dWg = x^T dg,   dWu = x^T du
//
// act(g) = g s(q(g)), s the logistic function: q = g for SiLU, and for GELU in its tanh form
// q = 2 sqrt(2/pi) (g + 0.044715 g^3), as (1 + tanh z) / 2 = s(2z).
//
// Forward and the two gradient products are one persistent kernel on CTA pairs, 256 x 256 output tiles
// (128 rows per CTA), 64-deep stages by TMA, accumulators double-buffered in tensor memory. Forward, a
// tile is 256 tokens by 128 columns of g beside the same 128 columns of u: CTA 0 of the pair brings
// Wg's columns and CTA 1 Wu's, so that each thread of the epilogue holds g and u of its token and
// writes h without either leaving the SM.  dx and the weights' gradients share one launch: dx's product
// is a sum over 2F, theirs over T, and tiles of one fill the SMs that the other's last wave leaves idle.
// Up to kGemvTokens tokens the block is bound by reading the weights and runs on k_ffn_few instead.
//
// Measured (bf16, 16384 tokens, 2048 x 5632; alone on the GPU): forward 418 us, 1.81 PFLOP/s; dg and du 151 us,
// 6.1 TB/s; the gradient's products 787 us, 1.92 PFLOP/s (cuBLAS's burst rate on 8192^3: 1.89; in a long run the power
// cap takes both to about nine tenths).  2047 x 1024 x 2816: 26, 13 and 33 us, where the last round of tiles and
// starting and draining the pipeline weigh.  One stage's 32 KB per SM arrive in about the time that its products take,
// so that a tile of half the columns takes 0.75 of the time, not 0.5.  The gradient of 33 tokens, whose dg and du go
// to the products as two values each (kSplitTokens): 34 us for 1024 x 2816, 58 for 2048 x 5632 (31 and 55 with one value).
#include <algorithm>

#include "common.cuh"
#include "ffn_gemm.cuh"
#include "inner.cuh"
#include "inner.h"
#include "per_device.h"
#include "tensor_map.h"

namespace isoloco {

namespace {

// ------------------------------------------------------------------ dg and du
// The rests of rounded values, rounded (none where the value has no finite form).
template <class T>
__device__ __forceinline__ void rests(const Vec<T>& rounded, float (&v)[8]) {
    float r[8];
    rounded.unpack(r);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = r[j] - r[j] == 0.f ? v[j] - r[j] : 0.f;
}

// d: tokens x 2 x pitch, dg then du of a token (SPLIT: x 4, their rests behind them).  8 columns per step; dh's rows may
// start anywhere.
template <class T, bool GELU, bool SPLIT>
__global__ void __launch_bounds__(256) k_ffn_dgu(const T* __restrict__ dh, int64_t ld_dh, bool dh_vec,
                                                 const typename Kept<T>::Store* __restrict__ saved, T* __restrict__ d, int64_t tokens,
                                                 int64_t ff, int64_t pitch) {
    next_may_start();
    after_previous();
    const uint32_t per_row = static_cast<uint32_t>(pitch >> 3);
    const int64_t total = tokens * per_row;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t m = total <= 0xffffffffll ? static_cast<int64_t>(static_cast<uint32_t>(i) / per_row) : i / per_row;
        const int64_t n = (i - m * per_row) * 8;
        const int cols = static_cast<int>(min(static_cast<int64_t>(8), ff - n));
        float g[8], u[8], v[8];
        const int64_t at = m * 2 * pitch + n;  // the pad behind a row's last column may be read, not used
        if constexpr (__is_same(T, __half)) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float4 a = __ldcs(reinterpret_cast<const float4*>(saved + at) + q);
                const float4 b = __ldcs(reinterpret_cast<const float4*>(saved + at + pitch) + q);
                g[4 * q] = a.x, g[4 * q + 1] = a.y, g[4 * q + 2] = a.z, g[4 * q + 3] = a.w;
                u[4 * q] = b.x, u[4 * q + 1] = b.y, u[4 * q + 2] = b.z, u[4 * q + 3] = b.w;
            }
        } else {
            const uint4 a = ld_stream(saved + at), b = ld_stream(saved + at + pitch);
            const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                g[2 * q] = Kept<T>::decode(aw[q] & 0xffffu), g[2 * q + 1] = Kept<T>::decode(aw[q] >> 16);
                u[2 * q] = Kept<T>::decode(bw[q] & 0xffffu), u[2 * q + 1] = Kept<T>::decode(bw[q] >> 16);
            }
        }
        if (dh_vec && cols == 8) {
            Vec<T> w;
            w.raw = ld_stream(dh + m * ld_dh + n);
            w.unpack(v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < cols ? to_f32(dh[m * ld_dh + n + j]) : 0.f;
        }
        float dg[8], du[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float a, s;
            act_both<GELU>(g[j], a, s);
            dg[j] = v[j] * u[j] * s;
            du[j] = v[j] * a;
        }
        T* out = d + (SPLIT ? at + m * 2 * pitch : at);
        Vec<T> w;
        w.pack(dg);
        *reinterpret_cast<uint4*>(out) = w.raw;
        if constexpr (SPLIT) {
            rests(w, dg);
            w.pack(dg);
            *reinterpret_cast<uint4*>(out + 2 * pitch) = w.raw;
        }
        w.pack(du);
        *reinterpret_cast<uint4*>(out + pitch) = w.raw;
        if constexpr (SPLIT) {
            rests(w, du);
            w.pack(du);
            *reinterpret_cast<uint4*>(out + 3 * pitch) = w.raw;
        }
    }
}

// dx of a split product: the sums over rounded values and over rests, kSplitTokens rows apart, added and rounded.
template <class T>
__global__ void __launch_bounds__(256) k_ffn_dx_join(const float* __restrict__ sums, int64_t pitch, T* __restrict__ dx, int64_t ld_dx,
                                                     int tokens, int width) {
    after_previous();
    const uint32_t per_row = static_cast<uint32_t>(pitch >> 2), i = blockIdx.x * 256u + threadIdx.x;
    const uint32_t t = i / per_row, c = (i - t * per_row) * 4u;
    if (t >= static_cast<uint32_t>(tokens)) return;
    const float4 a = *reinterpret_cast<const float4*>(sums + t * pitch + c);
    const float4 b = *reinterpret_cast<const float4*>(sums + (kSplitTokens + t) * pitch + c);
    const float v[4] = {a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w};
    T* out = dx + t * ld_dx + c;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (c + j < static_cast<uint32_t>(width)) out[j] = from_f32<T>(v[j]);
}

// ------------------------------------------------------------------ few tokens
constexpr int kGemvTokens = 2;    // (2048 x 5632 bf16: 14.9 us for 2 tokens, 21 for 4; the pair GEMM takes 18 for 9)
constexpr int kFewThreads = 256;
constexpr int kFewCols = 64;      // columns of F per cluster: 8 lanes of 16 bytes, whole 128-byte lines
constexpr int kFewMaxSplit = 8;   // CTAs of a cluster, each a share of D

// NT tokens.  One token through 2048 x 5632 bf16 takes 13.7 us, 3.4 TB/s.  All 352 CTAs are resident at once (42
// registers: 5 per SM fit) and wait for their loads (13.6 of the 21 cycles between a warp's instructions): a thread
// reads 16 rows of either matrix with a few loads in flight beside its 16 sums, and x's share, the sums over the
// warps and the cluster's barriers come before and behind.
// A cluster of `split` CTAs owns kFewCols columns; its CTAs share D's rows, a warp reads 4
// rows at a time (8 lanes each), and every thread keeps its 8 columns' sums for all tokens.  The sums meet by
// shuffles, shared memory and, for the cluster's first CTA, distributed shared memory, in fixed order.
template <class T, int NT, bool GELU>
__global__ void __launch_bounds__(kFewThreads) k_ffn_few(const T* __restrict__ x, int64_t ld_x, const T* __restrict__ wg,
                                                         const T* __restrict__ wu, int64_t ld_w, int width, int ff, T* __restrict__ h,
                                                         int64_t ld_h, typename Kept<T>::Store* __restrict__ saved, int64_t pitch,
                                                         int split) {
    extern __shared__ float fsm[];
    // [8 warps][2 NT][kFewCols] sums, then the CTA's [2 NT][kFewCols]; x's share [NT][rows] before that
    const uint32_t rank = cluster_ctarank();
    const int per = (width + split - 1) / split, d0 = static_cast<int>(rank) * per, rows = max(0, min(width - d0, per));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float* total = fsm;                              // [2 NT][kFewCols]
    float* part = total + 2 * NT * kFewCols;         // [8][2 NT][kFewCols]
    float* xs = part + 8 * 2 * NT * kFewCols;        // [rows][NT]
    for (int i = threadIdx.x; i < rows * NT; i += kFewThreads) xs[i] = to_f32(x[(i % NT) * ld_x + d0 + i / NT]);
    __syncthreads();
    const int n = static_cast<int>(blockIdx.x / split) * kFewCols + (lane & 7) * 8;
    float ag[NT][8], au[NT][8];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 8; ++j) ag[t][j] = au[t][j] = 0.f;
    if (n < ff) {  // (ff <= pitch, a multiple of 8: the last 16 bytes of a row exist)
        const T* pg = wg + static_cast<int64_t>(d0) * ld_w + n;
        const T* pu = wu + static_cast<int64_t>(d0) * ld_w + n;
#pragma unroll 8
        for (int r = warp * 4 + (lane >> 3); r < rows; r += 32) {
            Vec<T> a, b;
            a.raw = __ldg(reinterpret_cast<const uint4*>(pg + r * ld_w));
            b.raw = __ldg(reinterpret_cast<const uint4*>(pu + r * ld_w));
            float fa[8], fb[8];
            a.unpack(fa);
            b.unpack(fb);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float xv = xs[r * NT + t];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    ag[t][j] = fmaf(xv, fa[j], ag[t][j]);
                    au[t][j] = fmaf(xv, fb[j], au[t][j]);
                }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
#pragma unroll
            for (int o = 8; o <= 16; o <<= 1) {
                ag[t][j] += __shfl_xor_sync(0xffffffffu, ag[t][j], o);
                au[t][j] += __shfl_xor_sync(0xffffffffu, au[t][j], o);
            }
            if (lane < 8) {
                part[(warp * 2 * NT + t) * kFewCols + lane * 8 + j] = ag[t][j];
                part[(warp * 2 * NT + NT + t) * kFewCols + lane * 8 + j] = au[t][j];
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * NT * kFewCols; i += kFewThreads) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += part[w * 2 * NT * kFewCols + i];
        total[i] = s;
    }
    cluster_sync();
    if (rank == 0) {
        const int c0 = static_cast<int>(blockIdx.x / split) * kFewCols;
        for (int i = threadIdx.x; i < NT * kFewCols; i += kFewThreads) {
            const int t = i / kFewCols, col = c0 + i % kFewCols;
            float g = 0.f, u = 0.f;
            for (int r = 0; r < split; ++r) {
                float a, b;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(a) : "r"(mapa_shared(smem_u32(total + i), r)));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(b) : "r"(mapa_shared(smem_u32(total + NT * kFewCols + i), r)));
                g += a;
                u += b;
            }
            if (col < ff) {
                h[t * ld_h + col] = from_f32<T>(act_value<GELU>(g) * u);
                if (saved) {
                    if constexpr (__is_same(T, __half)) {
                        saved[t * 2 * pitch + col] = g;
                        saved[t * 2 * pitch + pitch + col] = u;
                    } else {
                        saved[t * 2 * pitch + col] = static_cast<uint16_t>(Kept<T>::encode2(g, 0.f));
                        saved[t * 2 * pitch + pitch + col] = static_cast<uint16_t>(Kept<T>::encode2(u, 0.f));
                    }
                }
            }
        }
    }
    cluster_sync();  // the other CTAs' sums stay until they have been read
}

// ------------------------------------------------------------------ pitches
// dst[r][0 .. cols) = src[r][0 .. cols), any pitches: operands that 16-byte accesses cannot read go through
// the workspace (an extra read and write of them), and outputs come back the same way.
__global__ void __launch_bounds__(256) k_repitch(const __nv_bfloat16* __restrict__ src, int64_t ld_s, __nv_bfloat16* __restrict__ dst, int64_t ld_d,
                                                 int64_t rows, int64_t cols, uint32_t pieces) {
    const int64_t total = rows * pieces;
#pragma unroll 4
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t r = total <= 0xffffffffll ? static_cast<int64_t>(static_cast<uint32_t>(i) / pieces) : i / pieces;
        put_piece(src + r * ld_s, dst + r * ld_d, cols, static_cast<uint32_t>(i - r * pieces), 1.f);
    }
}

cudaError_t repitch(const void* src, int64_t ld_s, void* dst, int64_t ld_d, int64_t rows, int64_t cols, cudaStream_t st) {
    if (rows == 0) return cudaSuccess;
    int sms = 0;
    const cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
    const uint32_t pieces = any_pieces(cols, 8);
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>((rows * pieces + 255) / 256, 32 * sms));
    k_repitch<<<grid, 256, 0, st>>>(static_cast<const __nv_bfloat16*>(src), ld_s, static_cast<__nv_bfloat16*>(dst), ld_d, rows, cols, pieces);
    return cudaGetLastError();
}

inline int64_t pitch_of(int64_t n) { return (n + 7) / 8 * 8; }
inline bool tma_ok(const void* p, int64_t ld) { return aligned16(p) && ld % 8 == 0; }
inline int64_t r256(int64_t b) { return (b + 255) / 256 * 256; }
inline int64_t copy_bytes(int64_t rows, int64_t cols) { return r256(rows * pitch_of(cols) * 2); }
inline bool splits(int64_t tokens) { return tokens > 0 && tokens <= kSplitTokens; }
inline int64_t split_bytes(int64_t width) { return r256(2 * kSplitTokens * pitch_of(width) * 4); }  // dx's sums
inline int slices_of(int64_t tokens) { return std::max(1, static_cast<int>((tokens + kSliceBlocks * kDepth - 1) / (kSliceBlocks * kDepth))); }
inline int64_t slice_rows(int64_t width) { return (width + 31) / 32 * 32; }  // (stores are of 32 rows)
inline int64_t slice_bytes(int64_t slices, int64_t width, int64_t ff) { return r256(2 * slices * slice_rows(width) * pitch_of(ff) * 4); }

// Pieces of the workspace, taken one after the other.
struct Arena {
    uint8_t* p;
    void* take(int64_t bytes) {
        void* r = p;
        p += r256(bytes);
        return r;
    }
};

// ------------------------------------------------------------------ tensor maps and launch
// rows x cols matrix of 2- or 4-byte elements, pitch in elements; boxes of 128 bytes x box_rows.
bool make_map2(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t pitch, int box_rows, int es = 2) {
    const EncodeTiledFn fn = tensor_map_encoder();
    if (!fn) return false;
    cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    cuuint64_t strides[1] = {static_cast<cuuint64_t>(pitch * es)};
    cuuint32_t box[2] = {static_cast<cuuint32_t>(128 / es), static_cast<cuuint32_t>(box_rows)}, step[2] = {1, 1};
    return fn(m, es == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims,
              strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaLaunchConfig_t cluster_config(unsigned grid, unsigned threads, size_t smem, int cluster, cudaStream_t st, cudaLaunchAttribute* at) {
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = static_cast<unsigned>(cluster);
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cfg;
}

// dw of sliced tokens: the slices' sums, in order, rounded.  blockIdx.y: which of the two matrices.
template <class T>
__global__ void __launch_bounds__(256) k_ffn_dw_join(const float* __restrict__ sums, int64_t pitch, int64_t slice_rows, int slices, T* __restrict__ dwg,
                                                     T* __restrict__ dwu, int64_t ld_dw, int64_t width, int64_t ff) {
    after_previous();
    const int64_t per_row = pitch >> 2, total = width * per_row, stride = 2 * slice_rows * pitch;
    T* dw = blockIdx.y ? dwu : dwg;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t r = i / per_row, c = (i - r * per_row) * 4;
        const float* from = sums + (blockIdx.y * slice_rows + r) * pitch + c;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int s = 0; s < slices; ++s) {
            const float4 a = __ldcs(reinterpret_cast<const float4*>(from + s * stride));
            v[0] += a.x, v[1] += a.y, v[2] += a.z, v[3] += a.w;
        }
        T* out = dw + r * ld_dw + c;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < ff) out[j] = from_f32<T>(v[j]);
    }
}

template <class T, bool FWD>
cudaError_t gemm_clusters(int* clusters) {
    using G = Geometry<FWD>;
    static PerDevice fit;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    return fit.get<cudaError_t>(dev, clusters, [&](int* n) {
        int sms = 0;
        cudaError_t r = device_sms(&sms);
        if (r == cudaSuccess) r = cudaFuncSetAttribute(k_ffn_gemm<T, FWD>, cudaFuncAttributeMaxDynamicSharedMemorySize, G::kSmemBytes);
        if (r != cudaSuccess) return r;
        cudaLaunchAttribute at[1];
        const cudaLaunchConfig_t cfg = cluster_config(static_cast<unsigned>(sms & ~1), G::kThreads, G::kSmemBytes, 2, nullptr, at);
        r = cudaOccupancyMaxActiveClusters(n, k_ffn_gemm<T, FWD>, &cfg);
        *n = std::max(1, std::min(*n, sms / 2));
        return r;
    });
}

// What a tile costs, in hundredths of a k-block of 256 columns: one of 128 columns takes 0.75 of its time (the
// bytes it loads: a k-block's arrive no faster than its products run), and starting and draining a tile about
// one k-block.  Narrow tiles pay only where they fill SMs that wide ones leave idle: 2047 x 1024 x 2816
// forward takes 26 us in 3 rounds of wide tiles, 29 in 5 of narrow ones; 33 tokens 12.4 and 11.8.
inline int64_t tile_cost(const Product& p) { return static_cast<int64_t>(p.kblocks) * (p.nh == 128 ? 100 : 75) + 100; }

// The rounds of p[1] that even out p[0]'s last (FfnTiles::extra) on C clusters, and the longest cluster's cost.
int64_t plan_rounds(const FfnTiles& g, int C, int* extra) {
    const int64_t c0 = tile_cost(g.p[0]), c1 = tile_cost(g.p[1]);
    const int full = g.n0 / C, rest = g.n0 % C, left = C - rest;
    int64_t best = INT64_MAX;
    for (int x = 0; x == 0 || (rest && x * left <= g.n1 + left && x < 4096); ++x) {
        const int after = std::max(0, g.n1 - x * left), rounds = after / C, more = after % C;
        // clusters without the extra tile of p[0] take the last round's tiles first
        const int64_t a = full * c0 + (x + rounds + (more > 0)) * c1;
        const int64_t b = rest ? (full + 1) * c0 + (rounds + (more > left)) * c1 : 0;
        if (std::max(a, b) < best) {
            best = std::max(a, b);
            *extra = x;
        }
    }
    return best;
}

template <class T, bool FWD>
cudaError_t launch_gemm2(FfnGemm<FWD>& g, int C, cudaStream_t st) {
    cudaError_t e = error_word(&g.err);
    if (e != cudaSuccess || g.n0 + g.n1 == 0) return e;
    C = std::min(C, g.n0 + g.n1);
    (void)plan_rounds(g, C, &g.extra);
    cudaLaunchAttribute at[2];
    cudaLaunchConfig_t cfg = cluster_config(static_cast<unsigned>(2 * C), Geometry<FWD>::kThreads, Geometry<FWD>::kSmemBytes, 2, st, at);
    if (!FWD) {
        at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.numAttrs = 2;
    }
    return cudaLaunchKernelEx(&cfg, k_ffn_gemm<T, FWD>, g);
}

inline int tiles(int64_t n, int per) { return static_cast<int>((n + per - 1) / per); }

// ------------------------------------------------------------------ entry points' bodies
template <class T, int NT, bool GELU>
cudaError_t few_n(const FfnArgs& a, const void* wg, const void* wu, int64_t ld_w, void* h, int64_t ld_h, void* saved, cudaStream_t st) {
    static PerDevice ready;
    int sms = 0, dev = 0, unused = 0;
    cudaError_t e = device_sms(&sms);
    if (e == cudaSuccess) e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const int blocks = tiles(a.ff, kFewCols);
    // split D until there are two CTAs for every SM, 64 of its rows each at least; a wide x needs the split for its
    // share in shared memory (few_fits)
    int split = 1;
    while (split < kFewMaxSplit && (blocks * split < 2 * sms || a.width / split > 4096) && a.width / (2 * split) >= 64) split *= 2;
    const size_t smem = sizeof(float) * (9 * 2 * NT * kFewCols + static_cast<size_t>((a.width + split - 1) / split) * NT);
    e = ready.get<cudaError_t>(dev, &unused, [&](int* v) {
        *v = 1;
        return cudaFuncSetAttribute(k_ffn_few<T, NT, GELU>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute at[1];
    const cudaLaunchConfig_t cfg = cluster_config(static_cast<unsigned>(blocks * split), kFewThreads, smem, split, st, at);
    return cudaLaunchKernelEx(&cfg, k_ffn_few<T, NT, GELU>, static_cast<const T*>(a.x), a.ld_x, static_cast<const T*>(wg),
                              static_cast<const T*>(wu), ld_w, static_cast<int>(a.width), static_cast<int>(a.ff), static_cast<T*>(h), ld_h,
                              static_cast<typename Kept<T>::Store*>(saved), pitch_of(a.ff), split);
}

// whether the shares of x and the sums fit shared memory
bool few_fits(int64_t tokens, int64_t width) {
    return tokens <= kGemvTokens && width <= 4096 * kFewMaxSplit;
}

template <class T, bool GELU>
cudaError_t few(const FfnArgs& a, const void* wg, const void* wu, int64_t ld_w, void* h, int64_t ld_h, void* saved, cudaStream_t st) {
    switch (a.tokens) {
        case 1: return few_n<T, 1, GELU>(a, wg, wu, ld_w, h, ld_h, saved, st);
        default: return few_n<T, 2, GELU>(a, wg, wu, ld_w, h, ld_h, saved, st);
    }
}

#define TRY(expr)                                  \
    do {                                           \
        const cudaError_t e_ = (expr);             \
        if (e_ != cudaSuccess) return e_;          \
    } while (0)

constexpr cudaError_t kNoMap = cudaErrorInvalidValue;  // a tensor map that the driver refuses

template <class T>
cudaError_t forward(const FfnArgs& a, void* h, int64_t ld_h, void* saved, void* ws, cudaStream_t st) {
    const bool f16 = __is_same(T, __half);
    const int64_t fp = pitch_of(a.ff);
    Arena arena = {static_cast<uint8_t*>(ws)};
    const void *wg = a.wg, *wu = a.wu, *x = a.x;
    int64_t ld_w = a.ld_w, ld_x = a.ld_x;
    if (!tma_ok(wg, ld_w) || !tma_ok(wu, ld_w)) {
        void *cg = arena.take(copy_bytes(a.width, a.ff)), *cu = arena.take(copy_bytes(a.width, a.ff));
        TRY(repitch(wg, ld_w, cg, fp, a.width, a.ff, st));
        TRY(repitch(wu, ld_w, cu, fp, a.width, a.ff, st));
        wg = cg, wu = cu, ld_w = fp;
    }
    if (few_fits(a.tokens, a.width))
        return a.act == ISOLOCO_SILU ? few<T, false>(a, wg, wu, ld_w, h, ld_h, saved, st) : few<T, true>(a, wg, wu, ld_w, h, ld_h, saved, st);
    if (!tma_ok(x, ld_x)) {
        void* cx = arena.take(copy_bytes(a.tokens, a.width));
        TRY(repitch(x, ld_x, cx, pitch_of(a.width), a.tokens, a.width, st));
        x = cx, ld_x = pitch_of(a.width);
    }
    const bool direct = tma_ok(h, ld_h);
    void* out = direct ? h : arena.take(copy_bytes(a.tokens, a.ff));
    FfnGemm<true> g;
    bool ok = make_map2(&g.x_k, x, a.tokens, a.width, ld_x, kTileRows) && make_map2(&g.wg_mn, wg, a.width, a.ff, ld_w, kDepth) &&
              make_map2(&g.wu_mn, wu, a.width, a.ff, ld_w, kDepth) && make_map2(&g.h, out, a.tokens, a.ff, direct ? ld_h : fp, 32);
    if (saved) {
        constexpr int es = sizeof(typename Kept<T>::Store);
        ok = ok && make_map2(&g.keep_g, saved, a.tokens, a.ff, 2 * fp, 32, es) &&
             make_map2(&g.keep_u, static_cast<uint8_t*>(saved) + fp * es, a.tokens, a.ff, 2 * fp, 32, es);
    }
    if (!ok) return kNoMap;
    const int kb = tiles(a.width, kDepth);
    int C = 0, unused;
    TRY((gemm_clusters<T, true>(&C)));
    g.n1 = 0;
    int64_t best = INT64_MAX;
    for (int nh = 128; nh >= 64; nh /= 2) {
        FfnTiles t = g;
        t.p[0] = t.p[1] = {kGated, tiles(a.tokens, 256), tiles(a.ff, nh), nh, kb, kb, 1, kb};
        t.n0 = t.p[0].tiles_m * t.p[0].tiles_n;
        const int64_t cost = plan_rounds(t, std::min(C, t.n0), &unused);
        if (cost < best) best = cost, static_cast<FfnTiles&>(g) = t;
    }
    g.tokens = static_cast<int>(a.tokens), g.width = static_cast<int>(a.width), g.ff = static_cast<int>(a.ff);
    g.f16 = f16, g.keep = saved != nullptr, g.gelu = a.act == ISOLOCO_GELU_TANH, g.split = false;
    g.slice_rows = 0;
    TRY((launch_gemm2<T, true>(g, C, st)));
    return direct ? cudaSuccess : repitch(out, fp, h, ld_h, a.tokens, a.ff, st);
}

template <class T>
cudaError_t backward(const FfnArgs& a, const void* dh, int64_t ld_dh, const void* saved, void* dx, int64_t ld_dx, void* dwg, void* dwu,
                     int64_t ld_dw, void* ws, cudaStream_t st) {
    const int64_t fp = pitch_of(a.ff), dp = pitch_of(a.width);
    if (a.tokens == 0) {
        if (dwg) {
            TRY(cudaMemset2DAsync(dwg, ld_dw * 2, 0, a.ff * 2, a.width, st));
            TRY(cudaMemset2DAsync(dwu, ld_dw * 2, 0, a.ff * 2, a.width, st));
        }
        return cudaSuccess;
    }
    Arena arena = {static_cast<uint8_t*>(ws)};
    const bool split = splits(a.tokens);
    const int planes = split ? 2 : 1, slices = slices_of(a.tokens);
    const int64_t dpitch = 2 * planes * fp;
    T* d = static_cast<T*>(arena.take(a.tokens * dpitch * 2));
    const bool dh_vec = tma_ok(dh, ld_dh);
    int sms = 0;
    TRY(device_sms(&sms));
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>((a.tokens * (fp / 8) + 255) / 256, 16 * sms));
    using Store = typename Kept<T>::Store;
    const auto dgu = a.act == ISOLOCO_SILU ? (split ? k_ffn_dgu<T, false, true> : k_ffn_dgu<T, false, false>)
                                           : (split ? k_ffn_dgu<T, true, true> : k_ffn_dgu<T, true, false>);
    TRY(launch_next(dgu, grid, 256, st, static_cast<const T*>(dh), ld_dh, dh_vec, static_cast<const Store*>(saved), d, a.tokens, a.ff, fp));
    FfnGemm<false> g;
    bool ok = true;
    int C = 0, unused;
    TRY((gemm_clusters<T, false>(&C)));
    int64_t best = INT64_MAX;
    for (int v = 0; v < 4; ++v) {  // tiles of 256 or 128 columns for either product
        const int nx = v & 1 ? 64 : 128, nw = v & 2 ? 64 : 128, seg = tiles(a.ff, kDepth), kw = tiles(a.tokens, kDepth);
        const Product pdx = {kDx, tiles(a.tokens, 256), tiles(a.width, 2 * nx), nx, 2 * seg, seg, 1, 2 * seg};
        const Product pdw = {kDw, tiles(a.width, 256), tiles(a.ff, 2 * nw), nw, std::min(planes * kw, kSliceBlocks), kw, 2 * slices, planes * kw};
        const int ndx = dx ? pdx.tiles_m * pdx.tiles_n : 0, ndw = dwg ? pdw.mats * pdw.tiles_m * pdw.tiles_n : 0;
        // the product with the longer tiles first
        const bool dw_first = !dx || (dwg && tile_cost(pdw) > tile_cost(pdx));
        FfnTiles t = g;
        t.p[0] = dw_first ? pdw : pdx, t.p[1] = dw_first ? pdx : pdw;
        t.n0 = dw_first ? ndw : ndx, t.n1 = dw_first ? ndx : ndw;
        if (t.n0 + t.n1 == 0) return cudaSuccess;
        const int64_t cost = plan_rounds(t, std::min(C, t.n0 + t.n1), &unused);
        if (cost < best) best = cost, static_cast<FfnTiles&>(g) = t;
    }
    const Product& pdx = g.p[0].kind == kDx ? g.p[0] : g.p[1];
    void *odx = dx, *odg = dwg, *odu = dwu;
    int64_t ldx = ld_dx, ldw = ld_dw;
    if (dx) {
        const void *wg = a.wg, *wu = a.wu;
        int64_t ld_w = a.ld_w;
        if (!tma_ok(wg, ld_w) || !tma_ok(wu, ld_w)) {
            void *cg = arena.take(copy_bytes(a.width, a.ff)), *cu = arena.take(copy_bytes(a.width, a.ff));
            TRY(repitch(wg, ld_w, cg, fp, a.width, a.ff, st));
            TRY(repitch(wu, ld_w, cu, fp, a.width, a.ff, st));
            wg = cg, wu = cu, ld_w = fp;
        }
        if (split) odx = arena.take(split_bytes(a.width)), ldx = dp;
        else if (!tma_ok(dx, ldx)) odx = arena.take(copy_bytes(a.tokens, a.width)), ldx = dp;
        ok = ok && make_map2(&g.dg_k, d, a.tokens, a.ff, dpitch, kTileRows) && make_map2(&g.du_k, d + fp, a.tokens, a.ff, dpitch, kTileRows) &&
             make_map2(&g.wg_k, wg, a.width, a.ff, ld_w, pdx.nh) && make_map2(&g.wu_k, wu, a.width, a.ff, ld_w, pdx.nh) &&
             make_map2(&g.dx, odx, split ? 2 * kSplitTokens : a.tokens, a.width, ldx, 32, split ? 4 : 2);
        if (split)
            ok = ok && make_map2(&g.dg_lo_k, d + 2 * fp, a.tokens, a.ff, dpitch, kTileRows) &&
                 make_map2(&g.du_lo_k, d + 3 * fp, a.tokens, a.ff, dpitch, kTileRows);
    }
    if (dwg) {
        const void* x = a.x;
        int64_t ld_x = a.ld_x;
        if (!tma_ok(x, ld_x)) {
            void* cx = arena.take(copy_bytes(a.tokens, a.width));
            TRY(repitch(x, ld_x, cx, dp, a.tokens, a.width, st));
            x = cx, ld_x = dp;
        }
        if (slices > 1) {
            odg = arena.take(slice_bytes(slices, a.width, a.ff)), odu = nullptr, ldw = fp;
        } else if (!tma_ok(dwg, ldw) || !tma_ok(dwu, ldw)) {
            odg = arena.take(copy_bytes(a.width, a.ff)), odu = arena.take(copy_bytes(a.width, a.ff));
            ldw = fp;
        }
        ok = ok && make_map2(&g.x_mn, x, a.tokens, a.width, ld_x, kDepth) && make_map2(&g.dg_mn, d, a.tokens, a.ff, dpitch, kDepth) &&
             make_map2(&g.du_mn, d + fp, a.tokens, a.ff, dpitch, kDepth);
        if (slices > 1) ok = ok && make_map2(&g.dwg, odg, 2 * slices * slice_rows(a.width), a.ff, fp, 32, 4);
        else ok = ok && make_map2(&g.dwg, odg, a.width, a.ff, ldw, 32) && make_map2(&g.dwu, odu, a.width, a.ff, ldw, 32);
        if (split)
            ok = ok && make_map2(&g.dg_lo_mn, d + 2 * fp, a.tokens, a.ff, dpitch, kDepth) &&
                 make_map2(&g.du_lo_mn, d + 3 * fp, a.tokens, a.ff, dpitch, kDepth);
    }
    if (!ok) return kNoMap;
    g.tokens = static_cast<int>(a.tokens), g.width = static_cast<int>(a.width), g.ff = static_cast<int>(a.ff);
    g.f16 = __is_same(T, __half), g.keep = false, g.gelu = false, g.split = split;
    g.slice_rows = slices > 1 ? static_cast<int>(slice_rows(a.width)) : 0;
    TRY((launch_gemm2<T, false>(g, C, st)));
    if (dx && split)
        TRY(launch_next(k_ffn_dx_join<T>, static_cast<unsigned>((a.tokens * (dp / 4) + 255) / 256), 256, st, static_cast<const float*>(odx), dp,
                        static_cast<T*>(dx), ld_dx, static_cast<int>(a.tokens), static_cast<int>(a.width)));
    else if (odx != dx) TRY(repitch(odx, ldx, dx, ld_dx, a.tokens, a.width, st));
    if (dwg && slices > 1) {
        const dim3 blocks(static_cast<unsigned>(std::min<int64_t>((a.width * (fp / 4) + 255) / 256, 16 * sms)), 2);
        TRY(launch_next(k_ffn_dw_join<T>, blocks, 256, st, static_cast<const float*>(odg), fp, slice_rows(a.width), slices, static_cast<T*>(dwg),
                        static_cast<T*>(dwu), ld_dw, a.width, a.ff));
    } else if (odg != dwg) {
        TRY(repitch(odg, ldw, dwg, ld_dw, a.width, a.ff, st));
        TRY(repitch(odu, ldw, dwu, ld_dw, a.width, a.ff, st));
    }
    return cudaSuccess;
}

}  // namespace

int64_t ffn_saved_bytes(int64_t tokens, int64_t ff, int dtype) {
    return tokens * 2 * pitch_of(ff) * (dtype == ISOLOCO_F16 ? 4 : 2) + 16;
}

// `aligned`: no operand needs a copy with another pitch.
int64_t ffn_workspace(int64_t tokens, int64_t width, int64_t ff, bool backward, bool aligned) {
    int64_t n = 0;
    if (backward) n += r256(tokens * (splits(tokens) ? 4 : 2) * pitch_of(ff) * 2) + (splits(tokens) ? split_bytes(width) : 0) +
                       (slices_of(tokens) > 1 ? slice_bytes(slices_of(tokens), width, ff) : 0);
    // the weights and x; h, or dx and the weights' gradients
    if (!aligned) n += (backward ? 4 : 2) * copy_bytes(width, ff) + (backward ? 2 : 1) * copy_bytes(tokens, width) +
                       (backward ? 0 : copy_bytes(tokens, ff));
    return n;
}

cudaError_t launch_ffn(const FfnArgs& a, void* h, int64_t ld_h, void* saved, void* ws, cudaStream_t st) {
    if (a.tokens == 0) return cudaSuccess;
    return a.dtype == ISOLOCO_BF16 ? forward<__nv_bfloat16>(a, h, ld_h, saved, ws, st) : forward<__half>(a, h, ld_h, saved, ws, st);
}

cudaError_t launch_ffn_grad(const FfnArgs& a, const void* dh, int64_t ld_dh, const void* saved, void* dx, int64_t ld_dx, void* dwg,
                            void* dwu, int64_t ld_dw, void* ws, cudaStream_t st) {
    return a.dtype == ISOLOCO_BF16 ? backward<__nv_bfloat16>(a, dh, ld_dh, saved, dx, ld_dx, dwg, dwu, ld_dw, ws, st)
                                   : backward<__half>(a, dh, ld_dh, saved, dx, ld_dx, dwg, dwu, ld_dw, ws, st);
}

}  // namespace isoloco

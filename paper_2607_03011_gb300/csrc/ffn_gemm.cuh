// ffn_gemm.cuh -- the gated block's products on CTA pairs (see ffn.cu): activation, the form g and u are kept
// in, and the persistent tcgen05 kernel with its two epilogues.
#pragma once
#include "common.cuh"
#include "inner.cuh"
#include "inner.h"

namespace isoloco {

namespace {

// ------------------------------------------------------------------ activation
// act(g) and act'(g).  The reciprocal is good to a unit in fp32's last place, e^-q to about 1 + |q| units (its
// argument q log2 e is rounded): 2^-17 at |q| = 80, far below every rounding to 16 bits that follows (e^-q
// past fp32's range gives s = 0).
__device__ __forceinline__ float logistic(float q) {
    float e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(q * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.f + e));
    return s;
}

template <bool GELU>
__device__ __forceinline__ float act_value(float g) {
    return g * logistic(GELU ? 1.5957691216057308f * g * fmaf(0.044715f * g, g, 1.f) : g);
}
template <bool GELU>
__device__ __forceinline__ void act_both(float g, float& a, float& slope) {
    if constexpr (GELU) {
        const float g2 = g * g;
        const float q = 1.5957691216057308f * g * fmaf(0.044715f, g2, 1.f);
        const float s = logistic(q);
        a = g * s;
        // s is 0 or 1 to fp32 beyond |g| = 20, where g^3 may be infinite
        const float t = fabsf(g) < 20.f ? 1.5957691216057308f * g * fmaf(0.134145f, g2, 1.f) * (1.f - s) : 0.f;
        slope = s * (1.f + t);
    } else {
        const float s = logistic(g);
        a = g * s;
        slope = s * (1.f + g * (1.f - s));
    }
}

// ------------------------------------------------------------------ g and u kept for the gradient
// With fp16 operands they stay fp32.  With bf16 they take 16 bits that cover fp32's exponents up to 2^33: 10
// significant bits from 2^-22 to 2^10 (9 fraction bits, so four codes for each of bf16's) and bf16's 8 on either side.
// What lies past 2^33, like NaN, comes back as NaN.  Two bits more than bf16 has keep their rounding below that of dg
// and du: for entries of ordinary size the gradients' error against 64 bits is 1.45 times that of one rounding to
// bf16, where bf16 here gave 1.85; fp16's 11 bits would end at 65504.
template <class T>
struct Kept;
template <>
struct Kept<__half> {
    using Store = float;
};
template <>
struct Kept<__nv_bfloat16> {
    using Store = uint16_t;
    // |v|'s bits b: b >> 16 below kLow and, shifted on, from kHigh, b >> 14 between
    static constexpr uint32_t kLow = 105u << 23, kHigh = 137u << 23, kWide = kHigh - kLow;  // 2^-22, 2^10
    // the code (and v's sign) in the upper half
    static __device__ __forceinline__ uint32_t upper(float v) {
        const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
        const uint32_t s = b + (0x8000u - 3u * kLow) + 3u * min(max(b, kLow), kHigh);
        return min(s, 0x7fffffffu) | (__float_as_uint(v) & 0x80000000u);
    }
    // two values, a's code in the low half
    static __device__ __forceinline__ uint32_t encode2(float a, float b) { return __byte_perm(upper(a), upper(b), 0x7632); }
    static __device__ __forceinline__ float decode(uint32_t c) {
        const uint32_t s = (c & 0x7fffu) << 16, t = min(max(s, kLow), kLow + 4u * kWide) - kLow;
        const uint32_t b = s >= 0x7fff0000u ? 0x7fc00000u : s - t + (t >> 2);
        return __uint_as_float(b | ((c & 0x8000u) << 16));
    }
};

// ------------------------------------------------------------------ the pair GEMM
constexpr int kTileRows = 128;                 // of A per CTA
constexpr int kDepth = 64;                     // K of a stage
constexpr int kABytes = kTileRows * kDepth * 2;
constexpr int kBBytes = 128 * kDepth * 2;      // at most 128 rows of B per CTA
constexpr int kStageBytes = kABytes + kBBytes;
constexpr int kStagingBytes = 4096;            // of an epilogue warp: 32 rows of 128 bytes
constexpr int kMaxStages = 6;
// Forward, 16 epilogue warps: 8 for the even and 8 for the odd tiles of a cluster, so that a tile's epilogue
// (two special functions and three stores per entry) may take as long as two tiles' products.  Backward, 8
// warps suffice and the shared memory is another stage's.
template <bool FWD>
struct Geometry {
    static constexpr int kEpiWarps = FWD ? 16 : 8;
    static constexpr int kStages = FWD ? 5 : 6;
    static constexpr int kThreads = 32 * (2 + kEpiWarps);
    static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kEpiWarps * kStagingBytes + 256;
};
constexpr int kTileWarps = 8;                  // that drain one accumulator
constexpr int kAccCols = 256;                  // tensor-memory columns of one accumulator

// A product of the launch: `tiles` = tiles_m x tiles_n tiles of 256 x 2 nh.
struct Product {
    int kind;       // kGated, kDx or kDw
    int tiles_m, tiles_n, nh;
    int kblocks;    // of one tile, over all segments
    int seg;        // k-blocks of one segment (kDx: dg's F, then du's; kDw: the tokens, with `split` once more)
    int mats;       // kDw: 2 (dWg's tiles, then dWu's) for every slice of the tokens, else 1
    int all;        // k-blocks of all slices
};
enum { kGated = 0, kDx = 1, kDw = 2 };

// The tensor core adds a k-block's products to the sum by cutting off what lies below its last places: a sum of one sign
// loses some 6e-9 of itself with every product, 4e-4 over 2^16 tokens, 6.6e-3 over 2^20.  More than 2^16 tokens are
// summed in slices of as many, each to fp32 sums in memory, which are added in order (1.4e-3 in all, one rounding to
// bf16, at any length; the gradient of 131072 x 1024 x 2816 takes 2.28 ms, in one slice 2.21).
constexpr int kSliceBlocks = 65536 / kDepth;

template <bool FWD>
struct FfnGemm;
struct FfnTiles {
    Product p[2];
    int n0, n1;       // tiles of p[0] and p[1]
    int extra;        // rounds of p[1] that the clusters without a tile in p[0]'s last round run first
    int tokens, width, ff;
    bool f16, keep, gelu;
    bool split;       // dg and du come as sums of two 16-bit values (kDx, kDw; see kSplitTokens)
    int slice_rows;   // kDw in slices of the tokens (kSliceBlocks): rows of one slice's fp32 sums of a matrix; 0: one slice
    uint32_t* err;
};
template <>
struct FfnGemm<true> : FfnTiles {
    CUtensorMap x_k, wg_mn, wu_mn, h, keep_g, keep_u;
};
template <>
struct FfnGemm<false> : FfnTiles {
    CUtensorMap dg_k, du_k, wg_k, wu_k, dx, x_mn, dg_mn, du_mn, dwg, dwu;
    CUtensorMap dg_lo_k, du_lo_k, dg_lo_mn, du_lo_mn;  // with `split`: the lower values
};

// Up to so many tokens dg and du go to the tensor cores as the sum of two 16-bit values, the rounded one and the rounded
// rest: dx and the weights' gradients of few tokens are sums of few roundings, and came out up to 1.6 times as far
// from 64 bits as one rounding of the output is (1.05 times with the rest; 1.45 where many tokens' roundings average
// out).  It costs few tokens little: dx's 128 rows of lower values are the second CTA's, which has no tokens of
// its own, and the weights' gradients sum over one or two k-blocks more.
constexpr int kSplitTokens = kTileRows;

__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                     reinterpret_cast<uint64_t>(map)),
                 "r"(src), "r"(c0), "r"(c1)
                 : "memory");
}

// The i-th tile of cluster c of C: p[0]'s tiles go round the clusters; p[1]'s fill the clusters that
// p[0]'s last round left out for `extra` rounds and then go round all, those clusters first.
struct TileAt {
    const Product* p;
    int m0, n0, mat;  // first row of the pair's 256, first column, matrix (kDw: 2 slice + which)
    int k0, nkb;      // its k-blocks
    bool valid;
};
__device__ __forceinline__ TileAt tile_at(const FfnTiles& g, int c, int C, int i) {
    const int full = g.n0 / C, rest = g.n0 % C, left = C - rest;  // clusters < rest run one more tile of p[0]
    const int mine = full + (c < rest ? 1 : 0);
    TileAt r;
    r.valid = true;
    int t;
    if (i < mine) {
        r.p = &g.p[0];
        t = i * C + c;
    } else {
        r.p = &g.p[1];
        const int j = i - mine;
        if (c >= rest && j < g.extra) {
            t = j * left + (c - rest);
        } else {
            const int round = c >= rest ? j - g.extra : j;
            const int order = c >= rest ? c - rest : c + left;
            t = g.extra * left + round * C + order;
        }
        if (t >= g.n1) {
            r.valid = false;
            return r;
        }
    }
    const int per = r.p->tiles_m * r.p->tiles_n;
    r.mat = t / per;
    t -= r.mat * per;
    r.k0 = r.p->kind == kDw ? (r.mat >> 1) * r.p->kblocks : 0;
    r.nkb = min(r.p->kblocks, r.p->all - r.k0);
    // panels of up to 8 tile rows, column by column: the clusters of one round share rows and columns
    const int panel = t / (8 * r.p->tiles_n), in = t - panel * 8 * r.p->tiles_n;
    const int rows = min(8, r.p->tiles_m - panel * 8);
    r.m0 = (panel * 8 + in % rows) * 2 * kTileRows;
    r.n0 = (in / rows) * (r.p->kind == kGated ? r.p->nh : 2 * r.p->nh);
    return r;
}

__device__ __forceinline__ uint64_t k_desc(uint32_t a) { return make_sdesc(a, 16, 8 * kDepth * 2, 2); }
__device__ __forceinline__ uint64_t mn_desc(uint32_t a) { return make_sdesc(a, kDepth * 128, 1024, 2); }

// Two pieces of 16 columns of the warp's tensor-memory lanes, one wait for both.
__device__ __forceinline__ void tmem_ld16x2(uint32_t at_a, uint32_t at_b, uint32_t (&a)[16], uint32_t (&b)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%32];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%33];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]), "=r"(a[4]), "=r"(a[5]), "=r"(a[6]), "=r"(a[7]), "=r"(a[8]), "=r"(a[9]),
          "=r"(a[10]), "=r"(a[11]), "=r"(a[12]), "=r"(a[13]), "=r"(a[14]), "=r"(a[15]), "=r"(b[0]), "=r"(b[1]), "=r"(b[2]),
          "=r"(b[3]), "=r"(b[4]), "=r"(b[5]), "=r"(b[6]), "=r"(b[7]), "=r"(b[8]), "=r"(b[9]), "=r"(b[10]), "=r"(b[11]),
          "=r"(b[12]), "=r"(b[13]), "=r"(b[14]), "=r"(b[15])
        : "r"(at_a), "r"(at_b)
        : "memory");
}

// A block of 32 rows of 128 bytes goes to memory through the warp's staging block, in the 128-byte swizzle:
// the block before has left (begin), each lane writes its row's eight 16-byte chunks (chunk), one TMA
// store takes it to (col, row) (end).
struct Staging {
    uint32_t stg, row_at;
    __device__ __forceinline__ Staging(uint32_t s, int lane) : stg(s), row_at(s + lane * 128 + ((lane & 7) << 4)) {}
    __device__ __forceinline__ void begin() const {
        if (elect_one()) bulk_wait_read0();
        __syncwarp();
    }
    __device__ __forceinline__ void chunk(int q, uint32_t a, uint32_t b, uint32_t c, uint32_t d) const {
        st_shared4(row_at ^ (q << 4), a, b, c, d);
    }
    __device__ __forceinline__ void end(const CUtensorMap* map, int col, int row) const {
        fence_proxy_async_smem();
        __syncwarp();
        if (elect_one()) {
            tma_store_2d(map, stg, col, row);
            bulk_commit();
        }
    }
};

// One warp's 32 rows of a forward tile: columns [c0, c0 + 64) of g and u.  The accumulators are read again for
// each output: keeping them would take 128 registers.
template <class T, bool GELU>
__device__ __forceinline__ void gated_block(const FfnGemm<true>& p, uint32_t tacc, int nh, int c0, int col, int row, const Staging& st) {
    constexpr bool kF16 = __is_same(T, __half);
    uint32_t g[16], u[16];
    st.begin();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        tmem_ld16x2(tacc + c0 + q * 16, tacc + nh + c0 + q * 16, g, u);
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float g0 = __uint_as_float(g[2 * j]), g1 = __uint_as_float(g[2 * j + 1]);
            w[j] = round16x2(act_value<GELU>(g0) * __uint_as_float(u[2 * j]), act_value<GELU>(g1) * __uint_as_float(u[2 * j + 1]), kF16);
        }
        st.chunk(2 * q, w[0], w[1], w[2], w[3]);
        st.chunk(2 * q + 1, w[4], w[5], w[6], w[7]);
    }
    st.end(&p.h, col, row);
    if (!p.keep) return;
#pragma unroll 1
    for (int m = 0; m < 2; ++m) {
        const uint32_t from = tacc + (m ? nh : 0) + c0;
        const CUtensorMap* map = m ? &p.keep_u : &p.keep_g;
        if constexpr (kF16) {
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {  // fp32: 32 columns are 128 bytes
                if (col + half * 32 >= p.ff) break;
                st.begin();
                tmem_ld16x2(from + half * 32, from + half * 32 + 16, g, u);
#pragma unroll
                for (int q = 0; q < 4; ++q) st.chunk(q, g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]);
#pragma unroll
                for (int q = 0; q < 4; ++q) st.chunk(4 + q, u[4 * q], u[4 * q + 1], u[4 * q + 2], u[4 * q + 3]);
                st.end(map, col + half * 32, row);
            }
        } else {
            st.begin();
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                tmem_ld16x2(from + half * 32, from + half * 32 + 16, g, u);
                uint32_t w[16];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    w[j] = Kept<T>::encode2(__uint_as_float(g[2 * j]), __uint_as_float(g[2 * j + 1]));
                    w[8 + j] = Kept<T>::encode2(__uint_as_float(u[2 * j]), __uint_as_float(u[2 * j + 1]));
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) st.chunk(4 * half + q, w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
            }
            st.end(map, col, row);
        }
    }
}

template <class T>
__device__ __forceinline__ void plain_block(uint32_t tacc, int c0, const CUtensorMap* map, int col, int row, const Staging& st) {
    st.begin();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint32_t v[32], w[16];
        tmem_ld32(tacc + c0 + half * 32, v);
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] = round16x2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]), __is_same(T, __half));
#pragma unroll
        for (int q = 0; q < 4; ++q) st.chunk(4 * half + q, w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
    }
    st.end(map, col, row);
}

// The same of fp32 sums (128 bytes are 32 columns).
__device__ __forceinline__ void sums_block(uint32_t tacc, int c0, const CUtensorMap* map, int col, int cols, int row, const Staging& st) {
#pragma unroll 1
    for (int half = 0; half < 2 && col + half * 32 < cols; ++half) {
        uint32_t v[32];
        st.begin();
        tmem_ld32(tacc + c0 + half * 32, v);
#pragma unroll
        for (int q = 0; q < 8; ++q) st.chunk(q, v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        st.end(map, col + half * 32, row);
    }
}

// Persistent, clusters of two CTAs; cluster c runs tile_at(c, 0), tile_at(c, 1), ...  Warp 0 loads, warp 1
// of CTA 0 issues the pair's MMAs, the other warps of both drain the accumulators.  `full` / `empty` hand
// stages over, `tfull` / `tempty` accumulators, as the TMA bytes and MMA commits complete.
template <class T, bool FWD>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Geometry<FWD>::kThreads, 1) k_ffn_gemm(const __grid_constant__ FfnGemm<FWD> p) {
    constexpr int kStages = Geometry<FWD>::kStages, kEpiWarps = Geometry<FWD>::kEpiWarps;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* staging = smem + kStages * kStageBytes;
    uint64_t* full = reinterpret_cast<uint64_t*>(staging + kEpiWarps * kStagingBytes);
    uint64_t* empty = full + kStages;
    uint64_t* tfull = empty + kStages;  // [2]
    uint64_t* tempty = tfull + 2;       // [2]
    uint64_t* drain = tempty + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    static_assert(8 * (2 * kMaxStages + 5) + 8 <= 256, "barriers behind the staging blocks");

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const uint32_t crank = cluster_ctarank();
    const bool leader = crank == 0;
    const int c = static_cast<int>(blockIdx.x >> 1), C = static_cast<int>(gridDim.x >> 1);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&tfull[i], 1);
            mbar_init(&tempty[i], kTileWarps * 2);
        }
        mbar_init(drain, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc_pair(tmem_slot, 2 * kAccCols);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    if (FWD) next_may_start();
    else after_previous();  // dg and du are complete

    if (warp == 0) {
        // ================= loads (one thread of each CTA)
        if (elect_one()) {
            const uint32_t sbase = smem_u32(smem);
            const uint32_t fbar0 = mapa_shared(smem_u32(full), 0);
            int stage = 0;
            uint32_t phase = 0;
            bool wrapped = false;
            for (int i = 0; !*abort_flag; ++i) {
                const TileAt t = tile_at(p, c, C, i);
                if (!t.valid) break;
                const Product& q = *t.p;
                const int m0 = t.m0 + static_cast<int>(crank) * kTileRows;
                const uint32_t pair_bytes = 2u * (kABytes + static_cast<uint32_t>(q.nh) * kDepth * 2u);
                for (int kb = 0; kb < t.nkb; ++kb) {
                    if (!mbar_wait(&empty[stage], phase ^ 1u)) {
                        *abort_flag = 1;
                        atomicOr(p.err, kErrTimeout);
                        break;
                    }
                    if (leader) mbar_arrive_expect_tx(&full[stage], pair_bytes);
                    const uint32_t bar = fbar0 + 8u * stage;
                    const uint32_t sa = sbase + stage * kStageBytes, sb = sa + kABytes;
                    if constexpr (FWD) {
                        const int k0 = kb * kDepth;
                        tma_load_2d_pair(sa, &p.x_k, bar, k0, m0);
                        const CUtensorMap* w = leader ? &p.wg_mn : &p.wu_mn;
                        for (int n = 0; n < q.nh; n += 64) tma_load_2d_pair(sb + n * kDepth * 2, w, bar, t.n0 + n, k0);
                    } else if (q.kind == kDx) {
                        const bool up = kb >= q.seg, lo = p.split && !leader;
                        const int k0 = (up ? kb - q.seg : kb) * kDepth;
                        const CUtensorMap* d = lo ? (up ? &p.du_lo_k : &p.dg_lo_k) : (up ? &p.du_k : &p.dg_k);
                        tma_load_2d_pair(sa, d, bar, k0, p.split ? t.m0 : m0);
                        tma_load_2d_pair(sb, up ? &p.wu_k : &p.wg_k, bar, k0, t.n0 + static_cast<int>(crank) * q.nh);
                    } else {
                        const int k = t.k0 + kb;
                        const bool lo = k >= q.seg;
                        const int k0 = (lo ? k - q.seg : k) * kDepth, n0 = t.n0 + static_cast<int>(crank) * q.nh;
                        for (int m = 0; m < kTileRows; m += 64) tma_load_2d_pair(sa + m * kDepth * 2, &p.x_mn, bar, m0 + m, k0);
                        const bool up = t.mat & 1;
                        const CUtensorMap* d = lo ? (up ? &p.du_lo_mn : &p.dg_lo_mn) : (up ? &p.du_mn : &p.dg_mn);
                        for (int n = 0; n < q.nh; n += 64) tma_load_2d_pair(sb + n * kDepth * 2, d, bar, n0 + n, k0);
                    }
                    if (++stage == kStages) {
                        stage = 0;
                        phase ^= 1u;
                        wrapped = true;
                    }
                }
            }
            if (*abort_flag) {
                // copies in flight land before the CTA exits: rank 0's barriers count both CTAs' copies, and rank 1
                // gives up only here, by a wait of kWaitTimeoutNs behind its last copy, which has landed by then
                if (leader) {
                    drain_barriers(kStages, [&](int s, uint64_t*& bar, uint32_t& parity) {
                        bar = &full[s];
                        parity = s < stage ? phase : phase ^ 1u;
                        return s < stage || wrapped;
                    });
                }
            }
        }
    } else if (warp == 1) {
        // ================= MMAs (one thread of CTA 0)
        if (leader && elect_one()) {
            const uint32_t sbase = smem_u32(smem);
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int i = 0; ok && !*abort_flag; ++i) {
                const TileAt t = tile_at(p, c, C, i);
                if (!t.valid) break;
                const Product& q = *t.p;
                const bool a_mn = q.kind == kDw, b_mn = q.kind != kDx;
                const uint32_t idesc = make_idesc_16bit(2 * kTileRows, 2 * q.nh, a_mn, b_mn, p.f16);
                const uint64_t da = a_mn ? mn_desc(sbase) : k_desc(sbase);
                const uint64_t db = b_mn ? mn_desc(sbase + kABytes) : k_desc(sbase + kABytes);
                const uint32_t a_lo = static_cast<uint32_t>(da), a_hi = static_cast<uint32_t>(da >> 32);
                const uint32_t b_lo = static_cast<uint32_t>(db), b_hi = static_cast<uint32_t>(db >> 32);
                const uint32_t step_a = a_mn ? 2048 >> 4 : 32 >> 4, step_b = b_mn ? 2048 >> 4 : 32 >> 4;
                const uint32_t buf = i & 1;
                if (!mbar_wait(&tempty[buf], ((i >> 1) & 1) ^ 1u)) {
                    *abort_flag = 1;
                    atomicOr(p.err, kErrTimeout);
                    break;
                }
                tc_fence_after();
                const uint32_t tacc = tmem_base + buf * kAccCols;
                uint32_t acc = 0;
                const int nkb = t.nkb;
                bool ready = mbar_test(&full[stage], phase);
#pragma unroll 1
                for (int kb = 0; kb < nkb; ++kb) {
                    const int s = stage;
                    if (!ready && !mbar_wait(&full[s], phase)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t so = s * (kStageBytes >> 4);
                    if (++stage == kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
#pragma unroll
                    for (int ks = 0; ks < kDepth / 16; ++ks) {
                        umma_16bit_pair(tacc, a_lo + so + ks * step_a, a_hi, b_lo + so + ks * step_b, b_hi, idesc, acc);
                        acc = 1u;
                        // the next stage's barrier is tested behind queued MMAs
                        if (ks == kDepth / 16 - 2) ready = mbar_test(&full[stage], phase);
                    }
                    umma_commit_pair_mc(&empty[s], 0x3);
                }
                if (!ok) {
                    *abort_flag = 1;
                    atomicOr(p.err, kErrTimeout);
                }
                umma_commit_pair_mc(&tfull[buf], 0x3);
            }
            umma_commit_pair(drain);
            (void)mbar_wait(drain, 0);
        }
    } else {
        // ================= epilogue: warp w reads tensor-memory lanes 32 (w % 4) ..; of the tile's blocks of
        // 64 columns one set of four warps takes the even, the next the odd ones; forward, warps 2..9 take the
        // even and warps 10..17 the odd tiles
        const int eg = warp & 3, half = ((warp - 2) >> 2) & 1;
        const Staging st(smem_u32(staging) + (warp - 2) * kStagingBytes, lane);
        constexpr int kSets = kEpiWarps / kTileWarps;
        for (int i = (warp - 2) / kTileWarps;; i += kSets) {
            const TileAt t = tile_at(p, c, C, i);
            if (!t.valid) break;
            const Product& q = *t.p;
            const uint32_t buf = i & 1;
            // (a k-block takes 0.2 to 0.8 us, and a tile has at most 2^15 of them)
            if (!__all_sync(0xffffffffu, mbar_wait(&tfull[buf], (i >> 1) & 1))) {
                if (lane == 0) atomicOr(p.err, kErrTimeout);
                break;
            }
            tc_fence_after();
            const uint32_t tacc = tmem_base + buf * kAccCols + (static_cast<uint32_t>(eg * 32) << 16);
            const int row = t.m0 + static_cast<int>(crank) * kTileRows + eg * 32;
            if constexpr (FWD) {
                if (row < p.tokens)
                    for (int c0 = half * 64; c0 < q.nh && t.n0 + c0 < p.ff; c0 += 128) {
                        if (p.gelu) gated_block<T, true>(p, tacc, q.nh, c0, t.n0 + c0, row, st);
                        else gated_block<T, false>(p, tacc, q.nh, c0, t.n0 + c0, row, st);
                    }
            } else {
                const int rows = q.kind == kDx ? p.tokens : p.width, cols = q.kind == kDx ? p.width : p.ff;
                const CUtensorMap* map = q.kind == kDx ? &p.dx : t.mat ? &p.dwu : &p.dwg;
                if (q.kind == kDx && p.split) {
                    // one tile of rows: either CTA's are the same tokens
                    if (eg * 32 < rows)
                        for (int c0 = half * 64; c0 < 2 * q.nh && t.n0 + c0 < cols; c0 += 128)
                            sums_block(tacc, c0, map, t.n0 + c0, cols, row, st);
                } else if (q.kind == kDw && p.slice_rows) {
                    if (row < rows)
                        for (int c0 = half * 64; c0 < 2 * q.nh && t.n0 + c0 < cols; c0 += 128)
                            sums_block(tacc, c0, &p.dwg, t.n0 + c0, cols, t.mat * p.slice_rows + row, st);
                } else if (row < rows)
                    for (int c0 = half * 64; c0 < 2 * q.nh && t.n0 + c0 < cols; c0 += 128)
                        plain_block<T>(tacc, c0, map, t.n0 + c0, row, st);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (leader) mbar_arrive(&tempty[buf]);
                else mbar_arrive_cluster(mapa_shared(smem_u32(&tempty[buf]), 0));
            }
        }
        if (elect_one()) bulk_wait0();
        __syncwarp();
    }

    // neither CTA leaves, or frees tensor memory, while the pair's MMAs could still read its shared memory
    // or write its accumulators (the issuing thread has waited for them)
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, 2 * kAccCols);
    }
}

}  // namespace

}  // namespace isoloco

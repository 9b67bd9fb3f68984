// rows.cuh -- what the kernels over rows of logits share: powers of two, packed fp32 arithmetic, largest entries and their
// order.
#pragma once
#include <cfloat>

#include "inner.cuh"
#include "inner.h"

namespace isoloco {

constexpr float kLowest = -1000.f;  // 2^d is 0 there
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// max(d, kLowest); NaN stays
__device__ __forceinline__ float cut(float d) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(d), "f"(kLowest));
    return y;
}

// Two fp32 operations per instruction (sm_100's packed forms; each rounds as its scalar form does).
struct F2 {
    unsigned long long v;
};
__device__ __forceinline__ F2 pair(float a, float b) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(F2 a, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(a.v)); }
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// The sum of 2^((f - m) c), of even and odd entries apart, added up as a tree (a sum that takes them one by one rounds
// more often, and waits for itself).
template <int N>
__device__ __forceinline__ F2 powers(const float (&f)[N], F2 minus_m, F2 c2) {
    F2 p[N / 2];
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
        float d0, d1;
        unpair(mul2(add2(pair(f[2 * j], f[2 * j + 1]), minus_m), c2), d0, d1);
        p[j] = pair(ex2(d0), ex2(d1));
    }
#pragma unroll
    for (int n = N / 4; n; n /= 2)
#pragma unroll
        for (int j = 0; j < n; ++j) p[j] = add2(p[j], p[j + n]);
    return p[0];
}

// Largest entries of vectors: pairs of 16-bit entries (or four fp32 ones) are compared at once.
template <class T>
struct Largest {
    uint32_t w[4];
    __device__ __forceinline__ void set(const Vec<T>& v) { w[0] = v.raw.x, w[1] = v.raw.y, w[2] = v.raw.z, w[3] = v.raw.w; }
    static __device__ __forceinline__ uint32_t more(uint32_t a, uint32_t b) {
        if constexpr (sizeof(T) == 4) {
            return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
        } else if constexpr (__is_same(T, __half)) {
            const __half2 h = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
            return *reinterpret_cast<const uint32_t*>(&h);
        } else {
            const __nv_bfloat162 h = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
            return *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    __device__ __forceinline__ void take(const Largest& o) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = more(w[i], o.w[i]);
    }
    __device__ __forceinline__ float value() const {
        const uint32_t m = more(more(w[0], w[1]), more(w[2], w[3]));
        if constexpr (sizeof(T) == 4) return __uint_as_float(m);
        else if constexpr (__is_same(T, __half)) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&m));
            return fmaxf(f.x, f.y);
        } else {
            return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
        }
    }
};

// Order of (value, index): greater values first, then lower indices; -0 and 0 are equal.
__device__ __forceinline__ uint64_t rank_key(float v, uint32_t idx) {
    const uint32_t u = __float_as_uint(v + 0.f);
    const uint32_t o = (u & 0x80000000u) ? ~u : u | 0x80000000u;
    return (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~idx);
}

constexpr int kGroups = 64;  // of threads, at least 2 ISOLOCO_MAX_TOP
// Entries a CTA ranks: all that a row of equal logits gives, a vector of up to 8 of each thread of `top` groups.
constexpr int candidates_of(int threads) { return ISOLOCO_MAX_TOP * 8 * (threads > 256 ? threads : 256) / kGroups; }

// What the search for the largest entries of a CTA of THREADS (or of up to 256) needs, and LISTS results.
template <int LISTS, int THREADS = 256>
struct TopSmem {
    uint64_t group[kGroups];
    uint64_t bound;
    int count, threads;
    uint16_t thread[THREADS];  // those whose entries may reach the bound
    uint64_t cand[candidates_of(THREADS)];
    uint64_t best[LISTS][ISOLOCO_MAX_TOP];
};

// sm.bound: the k-th largest of the groups' largest g.
template <int THREADS, class Smem>
__device__ __forceinline__ void make_bound(Smem& sm, int k, uint64_t g) {
    constexpr int kPer = THREADS / kGroups;
#pragma unroll
    for (int o = 1; o < kPer; o <<= 1) {
        const uint64_t other = __shfl_xor_sync(0xffffffffu, g, o);
        g = other > g ? other : g;
    }
    if (threadIdx.x % kPer == 0) sm.group[threadIdx.x / kPer] = g;
    __syncthreads();
    {
        // ranks of the groups: kPer threads each count a share of the greater ones
        const int own_at = threadIdx.x / kPer, sub = threadIdx.x % kPer;
        const uint64_t own = sm.group[own_at];
        int r = 0;
#pragma unroll
        for (int j = 0; j < kGroups / kPer; ++j) {
            const uint64_t v = sm.group[j * kPer + sub];
            r += (v > own || (v == own && j * kPer + sub < own_at)) ? 1 : 0;  // (equal keys: groups without entries)
        }
#pragma unroll
        for (int o = 1; o < kPer; o <<= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
        if (r == k - 1) sm.bound = own;
    }
    __syncthreads();
}

// The CTA's k largest entries, in order, to best[0 .. k) (keys; 0 where there are fewer).  bv, bi: this
// thread's largest value and an index not below its first place.
template <class T, int THREADS, class Smem, class Share>
__device__ __forceinline__ void top_of_cta(Smem& sm, const Share& sh, int k, float bv, uint32_t bi, float second, uint64_t* best) {
    constexpr int V = Vec<T>::kN, kCandidates = candidates_of(THREADS);
    // keys not above and not below that of the thread's largest entry, which lies within a vector of bi
    const bool any = bi != 0xffffffffu;
    const uint64_t least = any ? rank_key(bv, sh.first + bi) : 0, most = any ? rank_key(bv, sh.first + (bi >= V - 1 ? bi - (V - 1) : 0)) : 0;
    if (threadIdx.x == 0) sm.count = sm.threads = 0;
    if (threadIdx.x < k) best[threadIdx.x] = 0;
    make_bound<THREADS>(sm, k, least);
    const uint64_t bound = sm.bound;
    auto look = [&](float v, uint32_t i) {
        if (v != v) return;  // NaN ranks nowhere
        const uint64_t key = rank_key(v, sh.first + i);
        if (key >= bound) {
            const int at = atomicAdd(&sm.count, 1);
            if (at < kCandidates) sm.cand[at] = key;
        }
    };
    auto look_at = [&](uint32_t i) {
        Vec<T> v;
        v.raw = sh.load(i);
        float f[V];
        v.unpack(f);
#pragma unroll
        for (int j = 0; j < V; ++j) look(f[j], sh.head + i * V + j);
    };
    static_assert(sizeof(sm.thread) >= 2 * THREADS && sizeof(sm.cand) >= 8 * kCandidates, "TopSmem");
    if (any && most >= bound) {
        // the vector with the thread's largest entry, or, where another of its vectors may reach the bound, all of them
        if (rank_key(second, 0) >= bound) sm.thread[atomicAdd(&sm.threads, 1)] = static_cast<uint16_t>(threadIdx.x);
        else if (bi >= sh.head && bi < sh.tail()) look_at((bi - sh.head) / V);
    }
    __syncthreads();
    // those threads' vectors, dealt to all
    const uint32_t found = sm.threads, each = (sh.nvec + THREADS - 1) / THREADS;
    for (uint32_t e = threadIdx.x; e < found * each; e += THREADS) {
        const uint32_t i = sm.thread[e / each] + (e % each) * THREADS;
        if (i < sh.nvec) look_at(i);
    }
    if (threadIdx.x < sh.head) look(to_f32(sh.x[threadIdx.x]), threadIdx.x);
    if (threadIdx.x < sh.n - sh.tail()) look(to_f32(sh.x[sh.tail() + threadIdx.x]), sh.tail() + threadIdx.x);
    __syncthreads();
    int n = sm.count;
    if constexpr (THREADS > 256)
        if (n > kGroups * 4 && n <= kCandidates) {
            // Many equal entries (all tokens masked but a few): a bound once more, from the candidates (k groups or more have some, in any order).
            // 1 x 4 x 50021 fp16, 8 tokens left, 32 kept: 20 us, 108 where all candidates are ranked against each other, 72 one at a time; 17 unmasked.
            constexpr int kOwn = kCandidates / THREADS;
            uint64_t own[kOwn], most_own = 0;
#pragma unroll
            for (int u = 0; u < kOwn; ++u) {
                own[u] = threadIdx.x + u * THREADS < n ? sm.cand[threadIdx.x + u * THREADS] : 0;
                most_own = own[u] > most_own ? own[u] : most_own;
            }
            make_bound<THREADS>(sm, k, most_own);
            if (threadIdx.x == 0) sm.count = 0;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kOwn; ++u)
                if (own[u] && own[u] >= sm.bound) sm.cand[atomicAdd(&sm.count, 1)] = own[u];
            __syncthreads();
            n = sm.count;
        }
    if (n <= kCandidates) {
        for (int i = threadIdx.x; i < n; i += THREADS) {
            const uint64_t own = sm.cand[i];
            int r = 0;
            for (int j = 0; j < n; ++j) r += sm.cand[j] > own ? 1 : 0;
            if (r < k) best[r] = own;
        }
    } else {
        // more entries above the bound than fit (most of the row's largest lie in few threads' shares):
        // one at a time, the largest below the one before
        uint64_t below = ~uint64_t(0);
        for (int q = 0; q < k; ++q) {
            uint64_t b = 0;
            for (uint32_t i = threadIdx.x; i < sh.n; i += THREADS) {
                const float v = to_f32(sh.x[i]);
                const uint64_t key = v == v ? rank_key(v, sh.first + i) : 0;
                if (key < below && key > b) b = key;
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                const uint64_t other = __shfl_xor_sync(0xffffffffu, b, o);
                b = other > b ? other : b;
            }
            __syncthreads();
            if ((threadIdx.x & 31) == 0) sm.group[threadIdx.x >> 5] = b;
            __syncthreads();
            b = 0;
            for (int i = 0; i < THREADS / 32; ++i) b = sm.group[i] > b ? sm.group[i] : b;
            if (threadIdx.x == 0) best[q] = b;
            below = b;
        }
    }
    __syncthreads();
}

// The largest logit that counts as masked: the type's lowest value.
template <class T>
__device__ __forceinline__ float masked_at() { return -FLT_MAX; }
template <>
__device__ __forceinline__ float masked_at<__nv_bfloat16>() { return __uint_as_float(0xff7f0000u); }
template <>
__device__ __forceinline__ float masked_at<__half>() { return -65504.f; }

}  // namespace isoloco

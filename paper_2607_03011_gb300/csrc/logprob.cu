// logprob.cu -- log probabilities of given tokens, entropy, largest alternatives, and the gradient
// of the first two by the logits.
//
// With M the row's largest logit and d = (x - M) scale / ln 2:
//     s = sum 2^d,  w = sum d 2^d:   lse = scale M + ln s,  entropy = ln s - ln 2 w / s
// in one pass with a running maximum (s and w are rescaled when it rises).  The difference comes first,
// so that the largest entry's power is 1 exactly and nothing overflows at the types' ends (folding it
// into one multiply-add, x c - M c, needs both handled apart).  d is cut off at kLowest, where 2^d
// is 0 and d 2^d must be, too (masked logits; max.NaN keeps a NaN's row NaN).
//
// A row belongs to a cluster of `split` CTAs, each a contiguous share: one CTA where there are many
// rows, up to 8 where few would leave SMs idle.  The gradient's second pass finds its row in L2.
//
// Measured: 8192 x 32000 bf16 with gradient 176 us (6.0 TB/s of logits read once and gradient written; about 8
// instructions per 32 entries and pass at 2.5 per cycle and SM: loads' latency and issue share the bound); 2049 x
// 50021 bf16 with 5 alternatives 48 us (4.3 TB/s: a row's reductions and alternatives weigh against its few
// hundred entries per thread, and 2049 rows are 1.5 rounds of the 1368 that the SMs hold); 4 x 32000 fp32 with 20
// alternatives 11.9 us on 16 CTAs.  The gradient alone (k_logprobs_grad): 184 us for 8192 x 32000 bf16, 703 for
// 8192 x 50021, whose rows off 16-byte boundaries it reads and writes one entry at a time (with the
// statistics, from scalar heads and tails, 330).
//
// The `top` largest: the threads' own maxima, taken by groups, bound the top-th largest from below
// (the top-th largest of kGroups group maxima); only threads whose maximum reaches the bound look again,
// at the vector that holds it and, if another of theirs reaches the bound, at all of them, and the few
// entries found are ranked by counting.
#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "inner.cuh"
#include "inner.h"

namespace isoloco {

namespace {

constexpr float kLowest = -1000.f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kGroups = 64;         // of threads, at least 2 ISOLOCO_MAX_TOP
constexpr int kCandidates = 1024;   // entries a CTA ranks: all that a row of equal logits gives, 32 per group and `top`
constexpr int kMaxSplit = 8;
// A row's share of a CTA with gradient: 760 of them at once are 73 MB (4096 x 128000 fp32: 721 us in shares of 64 KB,
// 957 in shares of 128, 1029 in whole rows).
constexpr int64_t kShareBytes = 98304;
constexpr int kUnroll = 4;
// Threads per SM the registers are cut for.  5 CTAs of 256 (8192 x 32000 bf16 with gradient 180 us; 4 CTAs, with 64
// registers, 194; 6, with 40, 188; 8 of 128 threads 229); with alternatives 9 of 128 threads (8192 x 40000 bf16,
// 20 alternatives: 142 us; 10 CTAs 151, 8 148, 5 of 256 threads 160).
constexpr int threads_per_sm(bool top) { return top ? 1152 : 1280; }
constexpr int ctas_per_sm(int threads, bool top) { return threads_per_sm(top) / threads > 32 ? 32 : threads_per_sm(top) / threads; }

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
// d of two logits, from -M and c
__device__ __forceinline__ F2 exponents(float x0, float x1, F2 minus_m, F2 c2, float& d0, float& d1) {
    unpair(mul2(add2(pair(x0, x1), minus_m), c2), d0, d1);
    d0 = cut(d0);
    d1 = cut(d1);
    return pair(d0, d1);
}

// Running sums about the largest logit so far (no logit: the least number, with sums of 0).
struct Stat {
    float m, s, w;
    __device__ __forceinline__ void clear() { m = -3.402823466e38f, s = w = 0.f; }
    // the same sums about `to` >= m
    __device__ __forceinline__ void raise(float to, float c) {
        const float d = cut((m - to) * c), f = ex2(d);
        w = fmaf(s, d, w) * f;
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void add(float x, float c) {
        const float d = cut((x - m) * c), p = ex2(d);
        s += p;
        w = fmaf(d, p, w);
    }
};

// A thread's running sums, of even and odd entries apart.
struct Stat2 {
    float m;
    F2 s, w;
    __device__ __forceinline__ void raise(float to, float c) {
        const float d = cut((m - to) * c), f = ex2(d);
        w = mul2(fma2(s, pair(d, d), w), pair(f, f));
        s = mul2(s, pair(f, f));
        m = to;
    }
    __device__ __forceinline__ void add(float x0, float x1, F2 minus_m, F2 c2) {
        float d0, d1;
        const F2 d = exponents(x0, x1, minus_m, c2, d0, d1), p = pair(ex2(d0), ex2(d1));
        s = add2(s, p);
        w = fma2(d, p, w);
    }
};

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

struct TopSmem {
    uint64_t group[kGroups];
    uint64_t bound;
    int count, threads;
    uint16_t thread[256];  // those whose entries may reach the bound
    uint64_t cand[kCandidates];
    uint64_t best[kMaxSplit][ISOLOCO_MAX_TOP];  // of every CTA of the cluster (read in the first)
};

// A CTA's share of a row: entries before the first 16-byte boundary, vectors, entries behind.
template <class T>
struct Share {
    static constexpr int V = Vec<T>::kN;
    const T* x;      // the share's first entry
    uint32_t first;  // its index in the row
    uint32_t n, head, nvec;
    __device__ __forceinline__ Share(const T* row, uint32_t vocab, uint32_t rank, uint32_t split) {
        const uint32_t per = ((vocab + split - 1) / split + 63u) & ~63u;
        const uint64_t b = static_cast<uint64_t>(per) * rank;
        first = b < vocab ? static_cast<uint32_t>(b) : vocab;
        n = min(per, vocab - first);
        x = row + first;
        const uint32_t mis = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(x) & 15u);
        head = min(n, mis ? (16u - mis) / static_cast<uint32_t>(sizeof(T)) : 0u);
        nvec = (n - head) / V;
    }
    __device__ __forceinline__ uint32_t tail() const { return head + nvec * V; }
    __device__ __forceinline__ const uint4* vec(uint32_t i) const { return reinterpret_cast<const uint4*>(x + head) + i; }
};

// Sums over W lanes (every lane gets them): first the common maximum, then one rescaling.
template <int W>
__device__ __forceinline__ void merge_lanes(Stat& st, float c) {
    float m = st.m;
#pragma unroll
    for (int o = W / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    st.raise(m, c);
#pragma unroll
    for (int o = W / 2; o; o >>= 1) {
        st.s += __shfl_xor_sync(0xffffffffu, st.s, o);
        st.w += __shfl_xor_sync(0xffffffffu, st.w, o);
    }
}

// Over the CTA; every thread gets the sums.
template <int THREADS>
__device__ __forceinline__ void merge_cta(Stat& st, float c, Stat* sm) {
    merge_lanes<32>(st, c);
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = st;
    __syncthreads();
    constexpr int W = THREADS / 32;
    st = sm[threadIdx.x & (W - 1)];
    merge_lanes<W>(st, c);
}

// The CTA's k largest entries, in order, to best[0 .. k) (keys; 0 where there are fewer).  bv, bi: this
// thread's largest value and an index not below its first place.
template <class T, int THREADS>
__device__ __forceinline__ void top_of_cta(TopSmem& sm, const Share<T>& sh, int k, float bv, uint32_t bi, float second, uint64_t* best) {
    constexpr int kPer = THREADS / kGroups, V = Vec<T>::kN;
    // keys not above and not below that of the thread's largest entry, which lies within a vector of bi
    const bool any = bi != 0xffffffffu;
    const uint64_t least = any ? rank_key(bv, sh.first + bi) : 0, most = any ? rank_key(bv, sh.first + (bi >= V - 1 ? bi - (V - 1) : 0)) : 0;
    uint64_t g = least;
#pragma unroll
    for (int o = 1; o < kPer; o <<= 1) {
        const uint64_t other = __shfl_xor_sync(0xffffffffu, g, o);
        g = other > g ? other : g;
    }
    if (threadIdx.x % kPer == 0) sm.group[threadIdx.x / kPer] = g;
    if (threadIdx.x == 0) sm.count = sm.threads = 0;
    if (threadIdx.x < k) best[threadIdx.x] = 0;
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
        v.raw = *sh.vec(i);
        float f[V];
        v.unpack(f);
#pragma unroll
        for (int j = 0; j < V; ++j) look(f[j], sh.head + i * V + j);
    };
    static_assert(THREADS <= 256, "TopSmem::thread");
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
    const int n = sm.count;
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

template <class T, class I, int THREADS, bool TOP, bool GRAD>
__global__ void __launch_bounds__(THREADS, ctas_per_sm(THREADS, TOP)) k_logprobs(LogprobArgs a, uint32_t split) {
    constexpr int V = Vec<T>::kN;
    __shared__ Stat sm[THREADS / 32];
    __shared__ Stat peer[kMaxSplit];  // the sums of every CTA of the cluster
    __shared__ typename std::conditional<TOP, TopSmem, int>::type top_sm;
    const uint32_t rank = split > 1 ? cluster_ctarank() : 0u;
    const float c = a.scale * kLog2e;
    const uint32_t vocab = static_cast<uint32_t>(a.vocab);
    bool started = split == 1;  // every CTA of the cluster runs (before its shared memory is written)
    if (!started) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    for (int64_t r = blockIdx.x / split; r < a.rows; r += gridDim.x / split) {
        const T* row = static_cast<const T*>(a.logits) + r * a.ld;
        const Share<T> sh(row, vocab, rank, split);
        const int64_t t = token_at(static_cast<const I*>(a.targets), r, a.vocab);
        const float xt = t >= 0 ? to_f32(row[t]) : 0.f;  // (early: its latency passes behind the row's)
        Stat st;
        st.clear();
        float bv = -INFINITY, second = -INFINITY;  // the largest entry, and of the other vectors (and single entries)
        uint32_t bi = 0xffffffffu;
        if (threadIdx.x < sh.head) {
            const float v = to_f32(sh.x[threadIdx.x]);
            if (v > st.m) st.raise(v, c);
            st.add(v, c);
            if (TOP) bi = threadIdx.x, bv = v == v ? v : -INFINITY;
        }
        Stat2 two = {st.m, pair(st.s, 0.f), pair(st.w, 0.f)};
        const F2 c2 = pair(c, c);
        // kUnroll vectors in flight per thread; ALL: every one of them exists
        auto batch = [&](uint32_t i, auto all) {
            constexpr bool ALL = decltype(all)::value;
            Vec<T> v[kUnroll];
#pragma unroll
            for (int q = 0; q < kUnroll; ++q)
                if (ALL || i + q * THREADS < sh.nvec) {
                    // (read again below: plain loads, which stay in L2; the gradient may overwrite the logits)
                    if constexpr (GRAD || TOP) v[q].raw = *sh.vec(i + q * THREADS);
                    else v[q].raw = ld_stream(sh.vec(i + q * THREADS));
                }
            float vm[kUnroll], most = -INFINITY;
            if constexpr (TOP) {
#pragma unroll
                for (int q = 0; q < kUnroll; ++q)
                    if (ALL || i + q * THREADS < sh.nvec) {
                        Largest<T> l;
                        l.set(v[q]);
                        vm[q] = l.value();
                        most = fmaxf(most, vm[q]);
                    }
            } else {
                Largest<T> l, o;
                l.set(v[0]);
#pragma unroll
                for (int q = 1; q < kUnroll; ++q)
                    if (ALL || i + q * THREADS < sh.nvec) {
                        o.set(v[q]);
                        l.take(o);
                    }
                most = l.value();
            }
            if (most > two.m) two.raise(most, c);
            const F2 minus_m = pair(-two.m, -two.m);
#pragma unroll
            for (int q = 0; q < kUnroll; ++q)
                if (ALL || i + q * THREADS < sh.nvec) {
                    float f[V];
                    v[q].unpack(f);
#pragma unroll
                    for (int j = 0; j < V; j += 2) two.add(f[j], f[j + 1], minus_m, c2);
                    if (TOP) second = fmaxf(second, fminf(vm[q], bv));
                    if (TOP && (vm[q] > bv || bi == 0xffffffffu)) {
                        bv = fmaxf(vm[q], bv);
                        bi = sh.head + (i + q * THREADS) * V + V - 1;
                    }
                }
        };
        uint32_t i = threadIdx.x;
        for (; i + (kUnroll - 1) * THREADS < sh.nvec; i += kUnroll * THREADS) batch(i, std::true_type());
        if (i < sh.nvec) batch(i, std::false_type());
        {
            float a0, a1, b0, b1;
            unpair(two.s, a0, a1);
            unpair(two.w, b0, b1);
            st = {two.m, a0 + a1, b0 + b1};
        }
        if (threadIdx.x < sh.n - sh.tail()) {
            const float v = to_f32(sh.x[sh.tail() + threadIdx.x]);
            if (v > st.m) st.raise(v, c);
            st.add(v, c);
            if (TOP) second = fmaxf(second, fminf(v, bv));
            if (TOP && (v > bv || bi == 0xffffffffu)) bv = fmaxf(v, bv), bi = sh.tail() + threadIdx.x;
        }
        merge_cta<THREADS>(st, c, sm);
        if (split > 1) {
            if (!started) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
            started = true;
            if (threadIdx.x < split) {
                const uint32_t at = mapa_shared(smem_u32(peer + rank), threadIdx.x);
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(st.m) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 4), "f"(st.s) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 8), "f"(st.w) : "memory");
            }
        }
        if constexpr (TOP) {
            // every CTA's largest go to the first CTA's shared memory
            top_of_cta<T, THREADS>(top_sm, sh, a.top, bv, bi, second, top_sm.best[rank]);
            if (split > 1 && rank > 0 && threadIdx.x < a.top) {
                const uint32_t at = mapa_shared(smem_u32(&top_sm.best[rank][threadIdx.x]), 0);
                asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(at), "l"(top_sm.best[rank][threadIdx.x]) : "memory");
            }
        }
        if (split > 1) {
            cluster_sync();
            st.clear();
            for (uint32_t q = 0; q < split; ++q) {
                Stat o = peer[q];
                const float m = fmaxf(st.m, o.m);
                st.raise(m, c);
                o.raise(m, c);
                st.s += o.s, st.w += o.w;
            }
        }
        const bool none = st.s == 0.f;  // every logit is -inf
        const float lns = logf(st.s), ent = none ? 0.f : lns - kLn2 * (st.w / st.s);
        auto logp_of = [&](float x) { return none ? -INFINITY : fmaf(x - st.m, a.scale, -lns); };
        if (rank == 0 && threadIdx.x == 0) {
            if (a.logp) a.logp[r] = t < 0 ? 0.f : logp_of(xt);
            if (a.entropy) a.entropy[r] = ent;
            if (a.lse) a.lse[r] = none ? -INFINITY : fmaf(st.m, a.scale, lns);
        }
        if constexpr (TOP) {
            if (rank == 0) {
                auto put = [&](int q, uint64_t key) {
                    const uint32_t o = static_cast<uint32_t>(key >> 32);
                    const float v = key ? __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o) : NAN;
                    a.top_index[r * a.top + q] = key ? static_cast<int64_t>(static_cast<uint32_t>(~key)) : 0;
                    a.top_logp[r * a.top + q] = logp_of(v);
                };
                if (split == 1) {
                    if (threadIdx.x < a.top) put(threadIdx.x, top_sm.best[0][threadIdx.x]);
                } else {
                    // ranks among all CTAs' largest (equal keys: places that hold none, key 0)
                    const int n = static_cast<int>(split) * a.top;
                    for (int e = threadIdx.x; e < n; e += THREADS) {
                        const uint64_t own = top_sm.best[e / a.top][e % a.top];
                        int rk = 0;
                        for (int j = 0; j < n; ++j) {
                            const uint64_t v = top_sm.best[j / a.top][j % a.top];
                            rk += (v > own || (v == own && j < e)) ? 1 : 0;
                        }
                        if (rk < a.top) put(rk, own);
                    }
                }
            }
        }
        if constexpr (GRAD) {
            const float gl = (t >= 0 && !none && a.grad_logp) ? a.grad_logp[r] : 0.f;
            const float ge = (!none && a.grad_entropy) ? a.grad_entropy[r] : 0.f;
            // scale (-gl p - ge p (ln p + entropy)) = 2^d (A + B d)
            const float inv = none ? 0.f : 1.f / st.s;
            const float A = -a.scale * inv * (gl + ge * (ent - (none ? 0.f : lns))), B = -a.scale * inv * ge * kLn2;
            const float hot = gl * a.scale;
            T* out = static_cast<T*>(a.grad_logits) + r * a.ld_grad + sh.first;
            const uint32_t tt = t >= static_cast<int64_t>(sh.first) && t < static_cast<int64_t>(sh.first) + sh.n
                                    ? static_cast<uint32_t>(t) - sh.first : 0xffffffffu;
            const bool vec_out = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(sh.x)) & 15u) == 0;
            const F2 A2 = pair(A, A), B2 = pair(B, B), minus_m = pair(-st.m, -st.m);
            auto grad = [&](float x) {
                const float d = cut((x - st.m) * c);
                return ex2(d) * fmaf(B, d, A);
            };
            // (a NaN among the gradients or logits spreads by itself)
            if (threadIdx.x < sh.head) out[threadIdx.x] = from_f32<T>(grad(to_f32(sh.x[threadIdx.x])));
            auto body = [&](auto vector_out) {
                T* o = out + sh.head;
#pragma unroll 4
                for (uint32_t v = threadIdx.x; v < sh.nvec; v += THREADS) {
                    Vec<T> x;
                    x.raw = *sh.vec(v);
                    float f[V];
                    x.unpack(f);
#pragma unroll
                    for (int j = 0; j < V; j += 2) {
                        float d0, d1;
                        const F2 d = exponents(f[j], f[j + 1], minus_m, c2, d0, d1);
                        unpair(mul2(pair(ex2(d0), ex2(d1)), fma2(B2, d, A2)), f[j], f[j + 1]);
                    }
                    if constexpr (decltype(vector_out)::value) {
                        x.pack(f);
                        st_stream(o + v * V, x.raw);
                    } else {
#pragma unroll
                        for (int j = 0; j < V; ++j) o[v * V + j] = from_f32<T>(f[j]);
                    }
                }
            };
            if (vec_out) body(std::true_type());
            else body(std::false_type());
            const uint32_t e = sh.tail() + threadIdx.x;
            if (e < sh.n) out[e] = from_f32<T>(grad(to_f32(sh.x[e])));
            // the target's entry once more, with its own term, by the thread that wrote it
            if (tt != 0xffffffffu) {
                const uint32_t by = tt < sh.head ? tt : tt < sh.tail() ? (tt - sh.head) / V % THREADS : tt - sh.tail();
                if (threadIdx.x == by) out[tt] = from_f32<T>(grad(xt) + hot);
            }
        }
        // the next row's sums overwrite shared memory that this row's threads (and CTAs) may still read
        if (r + gridDim.x / split < a.rows) {
            if (split > 1) cluster_sync();
            else __syncthreads();
        }
    }
}

template <class T, class I>
__global__ void __launch_bounds__(256) k_logprobs_grad(LogprobArgs a) {
    constexpr int V = Vec<T>::kN;
    for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const T* row = static_cast<const T*>(a.logits) + r * a.ld;
        T* out = static_cast<T*>(a.grad_logits) + r * a.ld_grad;
        const int64_t t = token_at(static_cast<const I*>(a.targets), r, a.vocab);
        const float lse = a.lse[r], ent = a.grad_entropy ? a.entropy[r] : 0.f;
        const bool none = lse == -INFINITY;
        const float gl = (t >= 0 && !none && a.grad_logp) ? a.grad_logp[r] : 0.f;
        const float ge = (!none && a.grad_entropy) ? a.grad_entropy[r] : 0.f;
        const float A = -a.scale * fmaf(ge, ent, gl), B = -a.scale * ge * kLn2;
        auto grad = [&](float x, int64_t j) {
            const float lp = cut(none ? kLowest : fmaf(x, a.scale, -lse) * kLog2e), p = ex2(lp);
            return fmaf(p, fmaf(B, lp, A), j == t ? gl * a.scale : 0.f);
        };
        const bool vec = aligned16(row) && aligned16(out);
        const int64_t nvec = vec ? a.vocab / V : 0;
        for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < nvec; i += static_cast<int64_t>(gridDim.x) * 256) {
            Vec<T> v;
            v.raw = ld_stream(row + i * V);
            float f[V];
            v.unpack(f);
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = grad(f[j], i * V + j);
            v.pack(f);
            st_stream(out + i * V, v.raw);
        }
        for (int64_t i = nvec * V + static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < a.vocab; i += static_cast<int64_t>(gridDim.x) * 256)
            out[i] = from_f32<T>(grad(to_f32(row[i]), i));
    }
}

template <class T, class I, int THREADS, bool TOP, bool GRAD>
cudaError_t launch_rows(const LogprobArgs& a, int sms, cudaStream_t st) {
    // a row to one CTA where rows fill the GPU; else a cluster of up to 8, at least 4096 entries each.  With the
    // gradient also where the rows that are under way at once would not stay in L2 for its second pass: shares of
    // kShareBytes
    uint32_t split = 1;
    while (split < kMaxSplit && ((a.rows * split * 2 <= 2 * sms && a.vocab / (2 * split) >= 4096) ||
                                 (GRAD && a.vocab * static_cast<int64_t>(sizeof(T)) > split * kShareBytes)))
        split *= 2;
    const int64_t rows = std::min<int64_t>(a.rows, int64_t(1) << 24);
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows * split));
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = split > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, k_logprobs<T, I, THREADS, TOP, GRAD>, a, split);
}

template <class T, class I>
cudaError_t run(const LogprobArgs& a, cudaStream_t st) {
    int sms = 0;
    const cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
#define ROWS(N)                                                                                   \
    (a.grad_logits ? (a.top ? launch_rows<T, I, N, true, true>(a, sms, st) : launch_rows<T, I, N, false, true>(a, sms, st)) \
                   : (a.top ? launch_rows<T, I, N, true, false>(a, sms, st) : launch_rows<T, I, N, false, false>(a, sms, st)))
    // A short row is a few vectors per thread and its reductions weigh more: smaller CTAs, more rows at once (8192
    // bf16 rows without / with gradient: of 8000 32 / 62 us with 64 threads, 36 / 64 with 128; of 16000 52 / 103
    // with 128, 64 / 116 with 256; of 32000 with gradient 229 with 128, 180 with 256).
    // With alternatives, whose search weighs as much, 128 threads wherever rows fill the GPU.
    if (a.vocab <= 8192) return ROWS(64);
    return a.vocab <= 16384 || (a.top && a.rows > sms) ? ROWS(128) : ROWS(256);
#undef ROWS
}

template <class T, class I>
cudaError_t run_grad(const LogprobArgs& a, cudaStream_t st) {
    const unsigned rows = static_cast<unsigned>(std::min<int64_t>(a.rows, 65535));
    const unsigned cols = static_cast<unsigned>(std::min<int64_t>((a.vocab + 8191) / 8192, 64));
    k_logprobs_grad<T, I><<<dim3(cols, rows), 256, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_logprobs(const LogprobArgs& a, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    if (a.dtype == ISOLOCO_F32) return a.targets64 ? run<float, int64_t>(a, st) : run<float, int32_t>(a, st);
    if (a.dtype == ISOLOCO_BF16) return a.targets64 ? run<__nv_bfloat16, int64_t>(a, st) : run<__nv_bfloat16, int32_t>(a, st);
    return a.targets64 ? run<__half, int64_t>(a, st) : run<__half, int32_t>(a, st);
}

cudaError_t launch_logprobs_grad(const LogprobArgs& a, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    if (a.dtype == ISOLOCO_F32) return a.targets64 ? run_grad<float, int64_t>(a, st) : run_grad<float, int32_t>(a, st);
    if (a.dtype == ISOLOCO_BF16) return a.targets64 ? run_grad<__nv_bfloat16, int64_t>(a, st) : run_grad<__nv_bfloat16, int32_t>(a, st);
    return a.targets64 ? run_grad<__half, int64_t>(a, st) : run_grad<__half, int32_t>(a, st);
}

}  // namespace isoloco

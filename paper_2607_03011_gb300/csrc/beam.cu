// beam.cu -- a beam search's selection over beams and tokens, and what is kept for the beams moved along.
//
// Selection: with M the largest logit of beam w's row and S = sum e^{scale (x - M)}, a continuation by t has the total
// score_w + scale (x_t - M) - ln S.  Within a beam the totals rank as the logits do, so each row gives its `keep` largest logits
// (found as token_logprobs finds them) and its two sums, in one pass, and the batch entry's best are merged from those lists.
// What bounds it: HBM where there are many rows, else the chain of reductions in a row's search.
//
// Every row is cut in the same places, counted from its first entry, wherever that lies: beams with equal logits and
// scores get equal totals to the last bit, and rank by their numbers.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "common.cuh"
#include "inner.cuh"
#include "inner.h"
#include "rows.cuh"

namespace isoloco {

namespace {

constexpr int kMaxKeep = ISOLOCO_MAX_TOP;
constexpr int kMaxLists = ISOLOCO_MAX_BEAMS;  // of a batch entry: rows, or shares of rows
constexpr int kMaxCtas = 8;    // of a batch entry
constexpr int kUnroll = 4;

__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t o = static_cast<uint32_t>(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint32_t index_of(uint64_t key) { return static_cast<uint32_t>(~key); }

// The place of the n-th bit that is set (there are more than n).
__device__ __forceinline__ int nth_bit(uint32_t bits, int n) {
    int at = 0;
#pragma unroll
    for (int half = 16; half; half >>= 1) {
        const int low = __popc(bits >> at & ((1u << half) - 1));
        if (n >= low) n -= low, at += half;
    }
    return at;
}

enum Kind : int { kLive, kDead, kNan, kFinished };

__device__ __forceinline__ Kind kind_of(float score, bool finished) {
    if (!(score < INFINITY)) return kNan;
    if (score == -INFINITY) return kDead;
    return finished ? kFinished : kLive;
}

// A share of a row, as vectors counted from the share's first entry (which may lie at any address) and entries behind them.
template <class T>
struct Part {
    static constexpr uint32_t V = Vec<T>::kN;
    const T* x;
    uint32_t first, n, nvec, head = 0;
    bool aligned;
    __device__ __forceinline__ Part(const T* row, uint32_t vocab, uint32_t part, uint32_t per) {
        const uint64_t b = static_cast<uint64_t>(per) * part;
        first = b < vocab ? static_cast<uint32_t>(b) : vocab;
        n = min(per, vocab - first);
        x = row + first;
        nvec = n / V;
        aligned = aligned16(x);
    }
    __device__ __forceinline__ uint32_t tail() const { return nvec * V; }
    __device__ __forceinline__ uint4 load(uint32_t i) const {
        return aligned ? __ldg(reinterpret_cast<const uint4*>(x) + i) : load16_any(x + i * V);
    }
};

// What one list says: the continuations of a live beam's share by their logits, or (made, not read) of another beam.
struct Lists {
    uint64_t best[kMaxLists][kMaxKeep];
    float m[kMaxLists], s[kMaxLists];
};

struct Sum {
    float m, s;
    __device__ __forceinline__ void raise(float to, float c) { s *= ex2((m - to) * c), m = to; }
};

// A share's sums and its k largest entries, to list `at` of the cluster's first CTA.
template <class T, int THREADS>
__device__ __forceinline__ void search(const Part<T>& sh, int k, float c, TopSmem<1>& sm, Sum* sums, Lists& lists, int at, bool remote) {
    constexpr int V = Vec<T>::kN;
    float m = -FLT_MAX, bv = -INFINITY, second = -INFINITY;  // the largest entry, and of the other vectors (and single entries)
    uint32_t bi = 0xffffffffu;
    const F2 c2 = pair(c, c);
    F2 s2 = pair(0.f, 0.f);
    auto raise = [&](float big) {
        if (big > m) {
            const float f = ex2((m - big) * c);
            s2 = mul2(s2, pair(f, f));
            m = big;
        }
    };
    auto batch = [&](uint32_t i, auto all) {
        constexpr bool ALL = decltype(all)::value;
        Vec<T> v[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (ALL || i + u * THREADS < sh.nvec) v[u].raw = sh.load(i + u * THREADS);
        float vm[kUnroll], most = -INFINITY;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (ALL || i + u * THREADS < sh.nvec) {
                Largest<T> l;
                l.set(v[u]);
                vm[u] = l.value();
                most = fmaxf(most, vm[u]);
            }
        raise(most);
        const F2 minus = pair(-m, -m);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (ALL || i + u * THREADS < sh.nvec) {
                float f[V];
                v[u].unpack(f);
#pragma unroll
                for (int j = 0; j < V; j += 2) {
                    float d0, d1;
                    unpair(mul2(add2(pair(f[j], f[j + 1]), minus), c2), d0, d1);
                    s2 = add2(s2, pair(ex2(d0), ex2(d1)));
                }
                second = fmaxf(second, fminf(vm[u], bv));
                if (vm[u] > bv || bi == 0xffffffffu) {
                    bv = fmaxf(vm[u], bv);
                    bi = (i + u * THREADS) * V + V - 1;
                }
            }
    };
    uint32_t i = threadIdx.x;
    for (; i + (kUnroll - 1) * THREADS < sh.nvec; i += kUnroll * THREADS) batch(i, std::true_type());
    if (i < sh.nvec) batch(i, std::false_type());
    float s0, s1;
    if (threadIdx.x < sh.n - sh.tail()) {
        const float v = to_f32(sh.x[sh.tail() + threadIdx.x]);
        raise(v);
        unpair(s2, s0, s1);
        s2 = pair(s0 + ex2((v - m) * c), s1);
        second = fmaxf(second, fminf(v, bv));
        if (v > bv || bi == 0xffffffffu) bv = fmaxf(v, bv), bi = sh.tail() + threadIdx.x;
    }
    unpair(s2, s0, s1);
    Sum o = {m, s0 + s1};
    float to = o.m;
#pragma unroll
    for (int q = 16; q; q >>= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, q));
    o.raise(to, c);
#pragma unroll
    for (int q = 16; q; q >>= 1) o.s += __shfl_xor_sync(0xffffffffu, o.s, q);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = o;
    top_of_cta<T, THREADS>(sm, sh, k, bv, bi, second, sm.best[0]);  // (barriers within order `sums`, too)
    if (threadIdx.x < 32) {
        constexpr int W = THREADS / 32;
        o = sums[threadIdx.x & (W - 1)];
        to = o.m;
#pragma unroll
        for (int q = W / 2; q; q >>= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, q));
        o.raise(to, c);
#pragma unroll
        for (int q = W / 2; q; q >>= 1) o.s += __shfl_xor_sync(0xffffffffu, o.s, q);
        const uint64_t key = threadIdx.x < k ? sm.best[0][threadIdx.x] : 0;
        if (!remote) {
            lists.best[at][threadIdx.x] = key;
            if (threadIdx.x == 0) lists.m[at] = o.m, lists.s[at] = o.s;
        } else {
            asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(mapa_shared(smem_u32(&lists.best[at][threadIdx.x]), 0)), "l"(key) : "memory");
            if (threadIdx.x == 0) {
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_shared(smem_u32(&lists.m[at]), 0)), "f"(o.m) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_shared(smem_u32(&lists.s[at]), 0)), "f"(o.s) : "memory");
            }
        }
    }
    __syncthreads();
}

// Totals as whole numbers of the same order.
__device__ __forceinline__ uint64_t ordered(double v) {
    const uint64_t u = static_cast<uint64_t>(__double_as_longlong(v + 0.0));
    return (u >> 63) ? ~u : u | (uint64_t(1) << 63);
}

// The `keep` best of a batch entry from its lists, by one warp: a lane per list, each at its next continuation.  Lists: `split` of every live
// beam, in the beams' order, then one of every other beam.
template <class T>
__device__ __forceinline__ void merge(const BeamArgs& a, int64_t b, uint32_t live, Kind kind_of_lane, float score_of_lane, int split, int per, Lists& lists) {
    const int lane = threadIdx.x, count = __popc(live), shares = count * split;
    const uint32_t beams = a.beams == 32 ? 0xffffffffu : (1u << a.beams) - 1;
    // this lane's list: of which beam, and of which share of it
    const bool read = lane < shares;
    const uint32_t others = beams & ~live;
    const bool made = !read && lane < shares + __popc(others);
    const int nth = read ? lane / split : lane - shares;
    const int w = read ? nth_bit(live, nth) : made ? nth_bit(others, nth) : 0;
    const float score = __shfl_sync(0xffffffffu, score_of_lane, w);
    Kind kind = static_cast<Kind>(__shfl_sync(0xffffffffu, static_cast<int>(kind_of_lane), w));
    // a live beam's sums over its shares
    const double scale = a.scale;
    float m = -FLT_MAX;
    double base = 0.0;
    if (read) {
        for (int q = 0; q < split; ++q) m = fmaxf(m, lists.m[nth * split + q]);
        float s = 0.f;
        for (int q = 0; q < split; ++q) s += lists.s[nth * split + q] * ex2((lists.m[nth * split + q] - m) * (a.scale * kLog2e));
        if (!(s < INFINITY)) kind = kNan;
        else if (m <= masked_at<T>()) kind = kDead;
        // ln s: the exponent's part in 64 bits, so that what is rounded is ln of 1 .. 2
        const uint32_t bits = __float_as_uint(s);
        const double ln = static_cast<double>(static_cast<int>(bits >> 23) - 127) * 0.69314718055994531 +
                          static_cast<double>(logf(__uint_as_float((bits & 0x7fffffu) | 0x3f800000u)));
        base = static_cast<double>(score) - ln;
    }
    int left = (read && (kind == kLive || lane % split == 0)) || made ? per : 0;
    if (read && kind == kLive) {
        // (a share may be shorter than `per`)
        int have = 0;
        while (have < per && lists.best[lane][have]) ++have;
        left = have;
    }
    const uint32_t end = static_cast<uint32_t>(a.end);
    int p = 0;
    double total = 0.0;
    uint64_t key = 0, order = 0;
    uint32_t token = 0;
    auto next = [&] {
        total = -INFINITY;
        if (p >= left) return;
        if (kind == kLive) {
            key = lists.best[lane][p];
            const float x = value_of(key);
            token = index_of(key);
            if (x > masked_at<T>()) total = base + (static_cast<double>(x) - m) * scale;
        } else if (kind == kFinished && p == 0) {
            token = end, total = score;
        } else {
            token = static_cast<uint32_t>(p);
            if (kind == kFinished) token = token - 1 < end ? token - 1 : token;
        }
        order = ordered(total);
    };
    next();
    for (int q = 0; q < a.keep; ++q) {
        const bool in = p < left;
        const uint32_t hi = in ? static_cast<uint32_t>(order >> 32) : 0u, most_hi = __reduce_max_sync(0xffffffffu, hi);
        const uint32_t lo = in && hi == most_hi ? static_cast<uint32_t>(order) : 0u, most_lo = __reduce_max_sync(0xffffffffu, lo);
        bool best = in && hi == most_hi && lo == most_lo;
        uint32_t have = __ballot_sync(0xffffffffu, best);
        if (have & (have - 1)) {
            // equal totals: the lower beam, then the larger logit, then the lower token
            const uint32_t least = __reduce_min_sync(0xffffffffu, best ? static_cast<uint32_t>(w) : 0xffffffffu);
            best = best && static_cast<uint32_t>(w) == least;
            const uint64_t k = best ? (kind == kLive ? key : 1) : 0;
            const uint32_t khi = static_cast<uint32_t>(k >> 32), mhi = __reduce_max_sync(0xffffffffu, khi);
            const uint32_t klo = best && khi == mhi ? static_cast<uint32_t>(k) : 0u, mlo = __reduce_max_sync(0xffffffffu, klo);
            best = best && khi == mhi && klo == mlo;
            have = __ballot_sync(0xffffffffu, best);
        }
        if (lane == __ffs(have) - 1) {
            const int64_t at = b * a.keep + q;
            a.out_scores[at] = kind == kNan ? NAN : static_cast<float>(total);
            a.out_beams[at] = w;
            a.out_tokens[at] = token;
            if (a.out_finished) a.out_finished[at] = (a.finished && a.finished[b * a.beams + w]) || static_cast<int64_t>(token) == a.end;
            ++p;
            next();
        }
    }
}

// A cluster of `ctas` CTAs per batch entry: the live beams' rows, each in `split` shares of `per_share` entries (a multiple of 64), are dealt
// among them, and the first merges.
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS, 4) k_beam_select(BeamArgs a, int ctas, int split, uint32_t per_share) {
    __shared__ TopSmem<1> sm;
    __shared__ Lists lists;
    __shared__ Sum sums[THREADS / 32];
    const int rank = ctas > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    if (ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int64_t b = blockIdx.x / ctas;
    const float c = a.scale * kLog2e;
    const int per = static_cast<int>(min(static_cast<int64_t>(a.keep), a.vocab)), lane = threadIdx.x & 31;
    Kind kind = kDead;
    float score = 0.f;
    if (lane < a.beams) {
        score = a.scores[b * a.beams + lane];
        kind = kind_of(score, a.finished && a.finished[b * a.beams + lane]);
    }
    const uint32_t live = __ballot_sync(0xffffffffu, lane < a.beams && kind == kLive);
    const int units = __popc(live) * split;
    bool started = false;  // every CTA of the cluster runs (before its shared memory is written)
    for (int u = rank; u < units; u += ctas) {
        const int w = nth_bit(live, u / split);
        const Part<T> sh(static_cast<const T*>(a.logits) + (b * a.beams + w) * a.ld, static_cast<uint32_t>(a.vocab), u % split, per_share);
        if (ctas > 1 && !started) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        started = true;
        search<T, THREADS>(sh, static_cast<int>(min(static_cast<uint32_t>(per), sh.n)), c, sm, sums, lists, u, rank > 0);
    }
    if (ctas > 1) {
        if (!started) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        cluster_sync();
    }
    if (rank == 0 && threadIdx.x < 32) merge<T>(a, b, live, kind, score, split, per, lists);
}

// ---- states

struct StateArgs {
    const char* src;
    char* dst;
    int64_t src_batch, src_beam, src_outer, dst_batch, dst_beam, dst_outer;
    uint64_t units, run;   // of a beam, of a piece
    uint64_t tiles;        // of a beam
    bool in_place;
};
constexpr int kStates = 32;  // of a launch
struct ReorderArgs {
    StateArgs state[kStates];
    uint64_t first[kStates + 1];  // tiles before each state's
    int count, width;
    const void* beams;
};

// A thread moves one unit of all beams: it has read all that are needed before it writes any.
template <class U, class I, int W>
__global__ void __launch_bounds__(256) k_beam_reorder(const __grid_constant__ ReorderArgs a) {
    __shared__ int from[W];
    for (uint64_t tile = blockIdx.x; tile < a.first[a.count]; tile += gridDim.x) {
        int i = 0;
        while (tile >= a.first[i + 1]) ++i;
        const StateArgs& s = a.state[i];
        const uint64_t at = tile - a.first[i], b = at / s.tiles, u = (at % s.tiles) * 256 + threadIdx.x;
        __syncthreads();
        if (threadIdx.x < a.width) {
            const int64_t f = static_cast<const I*>(a.beams)[b * a.width + threadIdx.x];
            from[threadIdx.x] = f >= 0 && f < a.width ? static_cast<int>(f) : threadIdx.x;
        }
        __syncthreads();
        if (u >= s.units) continue;
        const uint64_t piece = u / s.run, in = u % s.run;
        const char* src = s.src + b * s.src_batch + piece * s.src_outer + in * sizeof(U);
        char* dst = s.dst + b * s.dst_batch + piece * s.dst_outer + in * sizeof(U);
        U v[W];
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (w < a.width && !(s.in_place && from[w] == w)) v[w] = *reinterpret_cast<const U*>(src + from[w] * s.src_beam);
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (w < a.width && !(s.in_place && from[w] == w)) *reinterpret_cast<U*>(dst + w * s.dst_beam) = v[w];
    }
}

template <class U, class I>
cudaError_t reorder(const ReorderArgs& a, cudaStream_t st) {
    const unsigned grid = static_cast<unsigned>(std::min<uint64_t>(a.first[a.count], uint64_t(1) << 30));
    if (a.width <= 4) k_beam_reorder<U, I, 4><<<grid, 256, 0, st>>>(a);
    else if (a.width <= 8) k_beam_reorder<U, I, 8><<<grid, 256, 0, st>>>(a);
    else if (a.width <= 16) k_beam_reorder<U, I, 16><<<grid, 256, 0, st>>>(a);
    else k_beam_reorder<U, I, 32><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
}

template <class I>
cudaError_t reorder(const ReorderArgs& a, int unit, cudaStream_t st) {
    if (unit == 16) return reorder<uint4, I>(a, st);
    if (unit == 8) return reorder<uint2, I>(a, st);
    if (unit == 4) return reorder<uint32_t, I>(a, st);
    if (unit == 2) return reorder<uint16_t, I>(a, st);
    return reorder<uint8_t, I>(a, st);
}

// The largest unit that divides a state's addresses, strides and runs.
int unit_of(const isoloco_state_t& s, int64_t batch, int width) {
    uint64_t bits = reinterpret_cast<uint64_t>(s.src) | reinterpret_cast<uint64_t>(s.dst) | static_cast<uint64_t>(s.run) | 16u;
    if (batch > 1) bits |= s.src_batch | s.dst_batch;
    if (width > 1) bits |= s.src_beam | s.dst_beam;
    if (s.outer > 1) bits |= s.src_outer | s.dst_outer;
    return static_cast<int>(bits & (~bits + 1));
}

}  // namespace

namespace {

template <class T>
cudaError_t select(const BeamArgs& a, cudaStream_t st) {
    constexpr int THREADS = 256;
    int sms = 0;
    const cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
    // rows in two, four or eight shares while that leaves every SM less than two CTAs, and shares of 4096 entries
    int split = 1;
    while (split < kMaxCtas && a.beams * split * 2 <= kMaxLists && a.batch * a.beams * split * 2 <= 2 * sms && a.vocab / (2 * split) >= 4096) split *= 2;
    const int ctas = std::min(kMaxCtas, a.beams * split);
    const uint32_t per = static_cast<uint32_t>(((a.vocab + split - 1) / split + 63) & ~int64_t(63));
    const int64_t most = int64_t(1) << 27;  // batch entries of a grid
    for (int64_t from = 0; from < a.batch; from += most) {
        BeamArgs p = a;
        p.batch = std::min(most, a.batch - from);
        p.logits = static_cast<const T*>(a.logits) + from * a.beams * a.ld;
        p.scores += from * a.beams;
        if (p.finished) p.finished += from * a.beams;
        p.out_scores += from * a.keep, p.out_beams += from * a.keep, p.out_tokens += from * a.keep;
        if (p.out_finished) p.out_finished += from * a.keep;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = static_cast<unsigned>(ctas);
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>(p.batch * ctas));
        cfg.blockDim = dim3(THREADS);
        cfg.stream = st;
        cfg.attrs = at;
        cfg.numAttrs = ctas > 1 ? 1 : 0;
        const cudaError_t x = cudaLaunchKernelEx(&cfg, k_beam_select<T, THREADS>, p, ctas, split, per);
        if (x != cudaSuccess) return x;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_beam_select(const BeamArgs& a, cudaStream_t st) {
    return a.dtype == ISOLOCO_F32 ? select<float>(a, st) : a.dtype == ISOLOCO_BF16 ? select<__nv_bfloat16>(a, st) : select<__half>(a, st);
}

cudaError_t launch_beam_reorder(const isoloco_state_t* states, int count, int64_t batch, int width, const void* beams,
                                bool ids64, cudaStream_t st) {
    if (batch == 0) return cudaSuccess;
    for (int unit = 16; unit; unit >>= 1) {
        ReorderArgs a;
        a.count = 0;
        a.width = width;
        a.beams = beams;
        a.first[0] = 0;
        auto flush = [&] {
            const cudaError_t e = a.count == 0 ? cudaSuccess : ids64 ? reorder<int64_t>(a, unit, st) : reorder<int32_t>(a, unit, st);
            a.count = 0;
            return e;
        };
        for (int i = 0; i < count; ++i) {
            const isoloco_state_t& s = states[i];
            if (s.outer == 0 || s.run == 0 || unit_of(s, batch, width) != unit) continue;
            StateArgs& t = a.state[a.count];
            t.src = static_cast<const char*>(s.src);
            t.dst = static_cast<char*>(s.dst);
            t.src_batch = s.src_batch, t.src_beam = s.src_beam, t.src_outer = s.src_outer;
            t.dst_batch = s.dst_batch, t.dst_beam = s.dst_beam, t.dst_outer = s.dst_outer;
            t.run = static_cast<uint64_t>(s.run) / unit;
            t.units = t.run * static_cast<uint64_t>(s.outer);
            t.tiles = (t.units + 255) / 256;
            t.in_place = s.src == s.dst;
            a.first[a.count + 1] = a.first[a.count] + static_cast<uint64_t>(batch) * t.tiles;
            if (++a.count == kStates) {
                const cudaError_t e = flush();
                if (e != cudaSuccess) return e;
            }
        }
        const cudaError_t e = flush();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace isoloco

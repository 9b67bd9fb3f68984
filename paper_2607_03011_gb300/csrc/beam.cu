// beam.cu -- a beam search's selection over beams and tokens, and what is kept for the beams moved along.
//
// Selection: with M the largest logit of beam w's row and S = sum e^{scale (x - M)}, a continuation by t has the total
// score_w + scale (x_t - M) - ln S.  Within a beam the totals rank as the logits do, so each row gives its `keep` largest logits
// (found as token_logprobs finds them) and its two sums, in one pass, and the batch entry's best are merged from those lists.
// What bounds it: for few rows the chain of loads, reductions and barriers (1 x 4 x 32000 bf16 10.3 us: 2.2 thousand cycles for the row,
// 4 for its search, 4 for the cluster's barrier, 5 for the merging); for many the loads in flight and what SMs have left to do when
// others are done (64 x 16 x 128000 bf16 60 us, 3.9 TB/s: the 922 rows that are read are 6.07 to an SM, in CTAs of two).  The
// merging in a launch of its own, with a CTA per row, took 63.  (Calls in graphs of their own, one after the other; "in a row" below: of many
// calls in one graph, where a call takes some 3 us less.)
//
// Every row is cut in the same places, counted from its first entry, wherever that lies: beams with equal logits and
// scores get equal totals to the last bit, and rank by their numbers.
#include <algorithm>
#include <atomic>
#include <cfloat>
#include <type_traits>

#include "common.cuh"
#include "inner.cuh"
#include "inner.h"
#include "per_device.h"
#include "rows.cuh"

namespace isoloco {

namespace {

constexpr int kMaxKeep = ISOLOCO_MAX_TOP;
constexpr int kMaxLists = ISOLOCO_MAX_BEAMS;  // of a batch entry: rows, or shares of rows
constexpr int kMaxCtas = 16;                  // of a batch entry
constexpr int kUnroll = 4;  // (6 or 8 vectors in flight: 63 and 65 us for 60)

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
        return aligned ? load_aligned(i) : load16_any(x + i * V);
    }
    __device__ __forceinline__ uint4 load_aligned(uint32_t i) const { return __ldg(reinterpret_cast<const uint4*>(x) + i); }
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
__device__ __forceinline__ void search(const Part<T>& sh, int k, float c, TopSmem<1, THREADS>& sm, Sum* sums, Lists& lists, int at, bool remote, bool& wait) {
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
    auto batch = [&](uint32_t i, auto all, auto aligned) {
        constexpr bool ALL = decltype(all)::value, ALIGNED = decltype(aligned)::value;
        Vec<T> v[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (ALL || i + u * THREADS < sh.nvec) v[u].raw = ALIGNED ? sh.load_aligned(i + u * THREADS) : load16_any(sh.x + (i + u * THREADS) * V);
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
    auto pass = [&](auto aligned) {
        uint32_t i = threadIdx.x;
        for (; i + (kUnroll - 1) * THREADS < sh.nvec; i += kUnroll * THREADS) batch(i, std::true_type(), aligned);
        if (i < sh.nvec) batch(i, std::false_type(), aligned);
    };
    if (sh.aligned) pass(std::true_type());
    else pass(std::false_type());
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
    if (wait) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // (the first CTA runs: its shared memory may be written)
    wait = false;
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

// The `keep` best of a batch entry from its lists: `split` of every live beam, in the beams' order, then one of every other beam.
template <class T, int THREADS>
__device__ __forceinline__ void merge(const BeamArgs& a, int64_t b, uint32_t live, Kind kind_of_lane, float score_of_lane, int split, int per, Lists& lists) {
    __shared__ double base[kMaxLists];
    __shared__ float top[kMaxLists];
    __shared__ int beam[kMaxLists], kinds[kMaxLists];
    __shared__ uint64_t order[kMaxLists * kMaxKeep];
    const int shares = __popc(live) * split;
    const uint32_t others = (a.beams == 32 ? 0xffffffffu : (1u << a.beams) - 1) & ~live;
    const int count = shares + __popc(others), n = count * per;
    const double scale = a.scale;
    if (threadIdx.x < 32) {
        // this lane's list: of which beam, and a live beam's sums over its shares
        const int lane = threadIdx.x;
        const bool read = lane < shares;
        const int nth = read ? lane / split : lane - shares;
        const int w = read ? nth_bit(live, nth) : lane < count ? nth_bit(others, nth) : 0;
        const float score = __shfl_sync(0xffffffffu, score_of_lane, w);
        Kind kind = static_cast<Kind>(__shfl_sync(0xffffffffu, static_cast<int>(kind_of_lane), w));
        float m = -FLT_MAX;
        if (read) {
            for (int q = 0; q < split; ++q) m = fmaxf(m, lists.m[nth * split + q]);
            float s = 0.f;
            for (int q = 0; q < split; ++q) s += lists.s[nth * split + q] * ex2((lists.m[nth * split + q] - m) * (a.scale * kLog2e));
            if (!(s < INFINITY)) kind = kNan;
            else if (m <= masked_at<T>()) kind = kDead;
            // ln s: the exponent's part in 64 bits, so that what is rounded is ln of 1 .. 2
            const uint32_t bits = __float_as_uint(s);
            base[lane] = static_cast<double>(score) - (static_cast<double>(static_cast<int>(bits >> 23) - 127) * 0.69314718055994531 +
                                                       static_cast<double>(logf(__uint_as_float((bits & 0x7fffffu) | 0x3f800000u))));
        } else {
            base[lane] = score;
        }
        top[lane] = m;
        beam[lane] = w;
        kinds[lane] = kind;
    }
    __syncthreads();
    // the p-th continuation of list l: its total in order (0: there is none), and its token
    auto token_of = [&](int l, int p) -> uint32_t {
        if (kinds[l] == kLive) return index_of(lists.best[l][p]);
        const uint32_t t = static_cast<uint32_t>(p), end = static_cast<uint32_t>(a.end);
        return kinds[l] != kFinished ? t : p == 0 ? end : t - 1 < end ? t - 1 : t;
    };
    auto total_of = [&](int l, int p) -> double {
        if (kinds[l] == kFinished) return p == 0 ? base[l] : -INFINITY;
        if (kinds[l] != kLive) return -INFINITY;
        const float x = value_of(lists.best[l][p]);
        return x > masked_at<T>() ? base[l] + (static_cast<double>(x) - top[l]) * scale : -INFINITY;
    };
    for (int e = threadIdx.x; e < n; e += THREADS) {
        const int l = e / per, p = e - l * per;
        // (a live beam's share may be shorter than `per`; of a beam that is not, one list is made)
        const bool there = kinds[l] == kLive ? lists.best[l][p] != 0 : l >= shares || l % split == 0;
        order[e] = there ? ordered(total_of(l, p)) : 0;
    }
    __syncthreads();
    if (threadIdx.x >= 32) return;
    // one warp, a lane per list, each at its next continuation; the q-th answer is kept by lane q
    const int lane = threadIdx.x;
    int p = 0, from = 0, at_p = 0;
    uint64_t own = lane < count ? order[lane * per] : 0;
#pragma unroll 1
    for (int q = 0; q < a.keep; ++q) {
        const uint32_t hi = static_cast<uint32_t>(own >> 32), most = __reduce_max_sync(0xffffffffu, hi);
        const uint32_t lo = hi == most ? static_cast<uint32_t>(own) : 0u, least = __reduce_max_sync(0xffffffffu, lo);
        bool best = hi == most && lo == least;
        uint32_t have = __ballot_sync(0xffffffffu, best);
        if (have & (have - 1)) {
            // equal totals: the lower beam, then (in shares of one row) the larger logit, then the lower token
            const uint32_t w = best ? static_cast<uint32_t>(beam[lane]) : 0xffffffffu, lowest = __reduce_min_sync(0xffffffffu, w);
            best = best && w == lowest;
            have = __ballot_sync(0xffffffffu, best);
            if (have & (have - 1)) {
                const uint64_t key = best ? lists.best[lane][p] : 0;
                const uint32_t khi = static_cast<uint32_t>(key >> 32), mhi = __reduce_max_sync(0xffffffffu, khi);
                const uint32_t klo = best && khi == mhi ? static_cast<uint32_t>(key) : 0u, mlo = __reduce_max_sync(0xffffffffu, klo);
                have = __ballot_sync(0xffffffffu, best && khi == mhi && klo == mlo);
            }
        }
        const int winner = __ffs(have) - 1, p_there = __shfl_sync(0xffffffffu, p, winner);
        if (lane == q) from = winner, at_p = p_there;
        if (lane == winner) {
            ++p;
            own = p < per ? order[lane * per + p] : 0;
        }
    }
    if (lane >= a.keep) return;
    const int64_t at = b * a.keep + lane;
    const uint32_t token = token_of(from, at_p);
    const int w = beam[from];
    const bool was = a.finished && a.finished[b * a.beams + w];
    __syncwarp(a.keep == 32 ? 0xffffffffu : (1u << a.keep) - 1);  // (out_finished may be finished)
    a.out_scores[at] = kinds[from] == kNan ? NAN : static_cast<float>(total_of(from, at_p));
    a.out_beams[at] = w;
    a.out_tokens[at] = token;
    if (a.out_finished) a.out_finished[at] = was || static_cast<int64_t>(token) == a.end;
}

// A cluster of `ctas` CTAs per batch entry: the live beams' rows, each in `split` shares of `per_share` entries (a multiple of 64), are dealt
// among them, and the first merges.
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_beam_select(BeamArgs a, int ctas, int split, uint32_t per_share) {
    __shared__ TopSmem<1, THREADS> sm;
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
    bool wait = ctas > 1;
    for (int u = rank; u < units; u += ctas) {
        const int w = nth_bit(live, u / split);
        const Part<T> sh(static_cast<const T*>(a.logits) + (b * a.beams + w) * a.ld, static_cast<uint32_t>(a.vocab), u % split, per_share);
        search<T, THREADS>(sh, static_cast<int>(min(static_cast<uint32_t>(per), sh.n)), c, sm, sums, lists, u, rank > 0, wait);
    }
    if (ctas > 1) {
        if (wait) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        cluster_sync();
    }
    if (rank == 0) merge<T, THREADS>(a, b, live, kind, score, split, per, lists);
}

// ---- states
//
// Moving states along is a copy: bytes read of every beam that is continued, once, and bytes written of every beam that
// changes.  A thread moves one place of all beams of a batch entry: it has read all that are needed before it writes
// any, so that a state may be its own destination, and a beam that several continue is read from HBM once.

constexpr int kStates = 32;               // of a launch
constexpr double kShiftLeast = 1 << 20;  // bytes
// CTAs per SM that the registers are cut for, us with 5, 4, 3 and 2 of them (GB read and written in 16-byte units): four beams (4.73) 786, 866, 865, 865; eight
// (4.68) 703, 690, 776, 985, half as much again where every beam's address has registers of its own; twelve (4.66) 883, 816, 705, 851; sixteen (4.96)
// 916, 831, 728, 850; twenty-four (4.71) 1442, 1215, 1137, 881; thirty-two (4.96) 1497, 1263, 1122, 893.  At these cuts the beams' units do not all
// stay in registers: of 4, 8, 16 and 32 beams a thread spills 24, 104, 320 and 752 bytes, and moves 64 to 512.  8 and 16 beams reach 6.8 TB/s, 17
// to 32 5.3 to 5.5.
constexpr int reorder_ctas(int width) { return width <= 4 ? 5 : width <= 8 ? 4 : width <= 16 ? 3 : 2; }
struct StateArgs {
    const char* src;
    char* dst;
    int64_t src_batch, src_beam, src_outer, dst_batch, dst_beam, dst_outer;
    uint64_t units, run;  // of a beam, of a piece (shifted: bytes)
    uint64_t tiles;       // of a beam
    int unit;             // bytes that addresses, strides and runs are multiples of, 1 .. 16
    bool in_place;
};
struct ReorderArgs {
    StateArgs state[kStates];
    uint64_t first[kStates + 1];  // tiles before each state's
    int count, width;
    bool ids64;
    const void* beams;
};

__device__ __forceinline__ uint64_t quotient(uint64_t a, uint64_t b) {
    return (a | b) >> 32 ? a / b : static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
}

template <class U, int W>
__device__ __forceinline__ void move_unit(const StateArgs& s, uint64_t b, uint64_t u, int width, const int* from) {
    const uint64_t piece = quotient(u, s.run), in = u - piece * s.run;
    const char* src = s.src + b * s.src_batch + piece * s.src_outer + in * sizeof(U);
    char* dst = s.dst + b * s.dst_batch + piece * s.dst_outer + in * sizeof(U);
    U v[W];
#pragma unroll
    for (int w = 0; w < W; ++w)
        if (w < width && !(s.in_place && from[w] == w)) v[w] = *reinterpret_cast<const U*>(src + from[w] * s.src_beam);
#pragma unroll
    for (int w = 0; w < W; ++w)
        if (w < width && !(s.in_place && from[w] == w)) {
            if constexpr (sizeof(U) == 16) st_stream(dst + w * s.dst_beam, v[w]);
            else *reinterpret_cast<U*>(dst + w * s.dst_beam) = v[w];
        }
}

// Runs that lie at any address, into other memory: piece 0 is what lies before a run's first 16-byte boundary of the destination, piece j the j-th 16
// bytes behind it, put together from the two aligned pieces of the source that hold them.
template <int W>
__device__ __forceinline__ void move_shifted(const StateArgs& s, uint64_t b, uint64_t u, int width, const int* from) {
    const uint32_t run = static_cast<uint32_t>(s.run), pieces = (run + 15) / 16 + 1;
    const uint64_t piece = quotient(u, pieces);
    const int j = static_cast<int>(u - piece * pieces);
    const char* src = s.src + b * s.src_batch + piece * s.src_outer;
    char* dst = s.dst + b * s.dst_batch + piece * s.dst_outer;
    // where this piece of beam w begins, from its run's start (piece 0: before it)
    auto place = [&](int w) { return (j - 1) * 16 + static_cast<int>(-reinterpret_cast<uintptr_t>(dst + w * s.dst_beam) & 15u); };
    constexpr int kGroup = 4;
#pragma unroll 1
    for (int g = 0; g < width; g += kGroup) {
        uint4 v[kGroup];
#pragma unroll
        for (int i = 0; i < kGroup; ++i)
            if (g + i < width) {
                const int at = place(g + i);
                if (at >= 0 && at + 16 <= static_cast<int>(run)) v[i] = load16_any(src + from[g + i] * s.src_beam + at);
            }
#pragma unroll
        for (int i = 0; i < kGroup; ++i)
            if (g + i < width) {
                const int at = place(g + i);
                char* to = dst + (g + i) * s.dst_beam;
                if (at >= 0 && at + 16 <= static_cast<int>(run)) {
                    st_stream(to + at, v[i]);
                } else {
                    const char* p = src + from[g + i] * s.src_beam;
                    const int stop = min(at + 16, static_cast<int>(run));
                    if (s.unit >= 4) {
                        for (int k = max(at, 0); k < stop; k += 4) *reinterpret_cast<uint32_t*>(to + k) = *reinterpret_cast<const uint32_t*>(p + k);
                    } else {
                        for (int k = max(at, 0); k < stop; ++k) to[k] = p[k];
                    }
                }
            }
    }
}

template <int W, bool SHIFTED>
__global__ void __launch_bounds__(256, reorder_ctas(W)) k_beam_reorder(const __grid_constant__ ReorderArgs a) {
    __shared__ int from[W];
    for (uint64_t tile = blockIdx.x; tile < a.first[a.count]; tile += gridDim.x) {
        int i = 0;
        while (tile >= a.first[i + 1]) ++i;
        const StateArgs& s = a.state[i];
        const uint64_t at = tile - a.first[i], b = quotient(at, s.tiles), u = (at - b * s.tiles) * 256 + threadIdx.x;
        __syncthreads();
        if (threadIdx.x < a.width) {
            const int64_t e = b * a.width + threadIdx.x;
            const int64_t f = a.ids64 ? static_cast<const int64_t*>(a.beams)[e] : static_cast<const int32_t*>(a.beams)[e];
            from[threadIdx.x] = f >= 0 && f < a.width ? static_cast<int>(f) : threadIdx.x;
        }
        __syncthreads();
        if (u >= s.units) continue;
        if constexpr (SHIFTED) {
            move_shifted<W>(s, b, u, a.width, from);
        } else {
            if (s.unit == 16) move_unit<uint4, W>(s, b, u, a.width, from);
            else if (s.unit == 8) move_unit<uint2, W>(s, b, u, a.width, from);
            else if (s.unit == 4) move_unit<uint32_t, W>(s, b, u, a.width, from);
            else if (s.unit == 2) move_unit<uint16_t, W>(s, b, u, a.width, from);
            else move_unit<uint8_t, W>(s, b, u, a.width, from);
        }
    }
}

template <bool SHIFTED>
cudaError_t reorder(const ReorderArgs& a, cudaStream_t st) {
    if (a.count == 0) return cudaSuccess;
    const unsigned grid = static_cast<unsigned>(std::min<uint64_t>(a.first[a.count], uint64_t(1) << 30));
    if (a.width <= 4) k_beam_reorder<4, SHIFTED><<<grid, 256, 0, st>>>(a);
    else if (a.width <= 8) k_beam_reorder<8, SHIFTED><<<grid, 256, 0, st>>>(a);
    else if (a.width <= 16) k_beam_reorder<16, SHIFTED><<<grid, 256, 0, st>>>(a);
    else k_beam_reorder<32, SHIFTED><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
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

std::atomic<int> g_refuse_clusters{0};

// Whether clusters of kMaxCtas CTAs can run on the current device (a restricted share of a GPU may not have room for them).
template <class T, int THREADS>
cudaError_t large_clusters(bool* fit) {
    static PerDevice known;
    int dev = 0, n = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess)
        e = known.get<cudaError_t>(dev, &n, [](int* clusters) {
            *clusters = 0;
            cudaLaunchAttribute at[1];
            at[0].id = cudaLaunchAttributeClusterDimension;
            at[0].val.clusterDim.x = kMaxCtas;
            at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(kMaxCtas);
            cfg.blockDim = dim3(THREADS);
            cfg.attrs = at;
            cfg.numAttrs = 1;
            cudaError_t r = cudaFuncSetAttribute(k_beam_select<T, THREADS>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
            if (r == cudaSuccess) r = cudaOccupancyMaxActiveClusters(clusters, k_beam_select<T, THREADS>, &cfg);
            if (r != cudaSuccess) {  // (refused altogether: smaller ones are made; what else is wrong shows at the launch)
                *clusters = 0;
                cudaGetLastError();
            }
            return cudaSuccess;
        });
    *fit = n > 0 && g_refuse_clusters.load(std::memory_order_relaxed) == 0;
    return e;
}

template <class T, int THREADS>
cudaError_t launch_select(const BeamArgs& a, int split, int ctas, cudaStream_t st) {
    if (ctas > 8) {
        bool fit = false;
        const cudaError_t e = large_clusters<T, THREADS>(&fit);
        if (e != cudaSuccess) return e;
        if (!fit) ctas = 8;  // (which every device runs; the rows are cut in the same places)
    }
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
        const cudaError_t e = cudaLaunchKernelEx(&cfg, k_beam_select<T, THREADS>, p, ctas, split, per);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <class T>
cudaError_t select(const BeamArgs& a, cudaStream_t st) {
    int sms = 0;
    const cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
    // A row in two, four, eight or sixteen shares while a batch entry's CTAs have one each, all run at once, and shares have
    // 4096 entries (in a row: 64 x 4 x 32000 fp32 11.4 us, 12.9 in whole rows; 1 x 4 x 128000 bf16 7.8 and 11.2; 16 x 8 x 50021 fp16 15.2 and 16.7).
    int split = 1;
    while (a.beams * split * 2 <= kMaxCtas && a.batch * a.beams * split * 2 <= 4 * sms && a.vocab / (2 * split) >= 4096) split *= 2;
    // Clusters of up to 16 while all of their CTAs run at once, or where CTAs of 8 would have unequal shares (in a row: 32 x 16 x 128000
    // bf16 34 us, 43 with clusters of 8; 100 x 10 x 32000 26 and 36); else of 8 (64 x 16 x 128000 57 us, 70 with 16).
    const int units = a.beams * split;
    const int ctas = units <= 8 || (units % 8 == 0 && a.batch * units > 4 * sms) ? std::min(8, units) : std::min(kMaxCtas, units);
    // 512 threads where an SM has no more than one CTA, for long shares (in a row, with 512 and 256 threads: 9 x 16 x 128000 bf16 19.6 and 23.2, fp32 24.6
    // and 32.8; 4 x 32 x 128000 25.9 and 34.3; 8 x 8 x 50021 fp16 13.5 with either; short ones lose, 9 x 16 x 32000 bf16 12.2 and 11.5, 8 x 16 x 1000
    // 10.6 and 9.2); 256 where it has more (64 x 5 x 32000 fp32 19.9 and 15.2; 16 x 8 x 50021 19.3 and 15.2).
    return a.batch * ctas <= sms ? launch_select<T, 512>(a, split, ctas, st) : launch_select<T, 256>(a, split, ctas, st);
}

}  // namespace

cudaError_t launch_beam_select(const BeamArgs& a, cudaStream_t st) {
    return a.dtype == ISOLOCO_F32 ? select<float>(a, st) : a.dtype == ISOLOCO_BF16 ? select<__nv_bfloat16>(a, st) : select<__half>(a, st);
}

void refuse_large_clusters(bool refuse) { g_refuse_clusters = refuse; }

cudaError_t launch_beam_reorder(const isoloco_state_t* states, int count, int64_t batch, int width, const void* beams,
                                bool ids64, cudaStream_t st) {
    if (batch == 0) return cudaSuccess;
    ReorderArgs args[2];  // by whole units, and shifted
    for (ReorderArgs& a : args) {
        a.count = 0;
        a.width = width;
        a.ids64 = ids64;
        a.beams = beams;
        a.first[0] = 0;
    }
    // By shifted pieces, where there is enough of it to pay for a launch of its own (4 us), what no 16-byte unit divides: 3 x 5 beams, 55 MB of fp32 rows
    // of 33 written, 27 us (3.6 TB/s read and written: beams go in groups of four, so five take two rounds of loads and stores), by units of 4 73.  In
    // place by units, 62: a thread's places of two beams, cut at their own boundaries, would not be the same.
    auto may_shift = [](const isoloco_state_t& s, int unit) { return s.src != s.dst && unit < 16 && s.run >= 64 && s.run < (1 << 30); };
    double large = 0.0;
    for (int i = 0; i < count; ++i)
        if (states[i].outer > 0 && may_shift(states[i], unit_of(states[i], batch, width)))
            large += static_cast<double>(states[i].run) * static_cast<double>(states[i].outer) * static_cast<double>(batch) * width;
    const bool shift = large >= kShiftLeast;
    for (int i = 0; i < count; ++i) {
        const isoloco_state_t& s = states[i];
        if (s.outer == 0 || s.run == 0) continue;
        const int unit = unit_of(s, batch, width);
        const bool shifted = shift && may_shift(s, unit);
        ReorderArgs& a = args[shifted];
        StateArgs& t = a.state[a.count];
        t.src = static_cast<const char*>(s.src);
        t.dst = static_cast<char*>(s.dst);
        t.src_batch = s.src_batch, t.src_beam = s.src_beam, t.src_outer = s.src_outer;
        t.dst_batch = s.dst_batch, t.dst_beam = s.dst_beam, t.dst_outer = s.dst_outer;
        t.unit = unit;
        t.in_place = s.src == s.dst;
        t.run = static_cast<uint64_t>(shifted ? s.run : s.run / unit);
        t.units = (shifted ? (t.run + 15) / 16 + 1 : t.run) * static_cast<uint64_t>(s.outer);
        t.tiles = (t.units + 255) / 256;
        a.first[a.count + 1] = a.first[a.count] + static_cast<uint64_t>(batch) * t.tiles;
        if (++a.count == kStates) {
            const cudaError_t e = shifted ? reorder<true>(a, st) : reorder<false>(a, st);
            if (e != cudaSuccess) return e;
            a.count = 0;
        }
    }
    const cudaError_t e = reorder<false>(args[0], st);
    return e == cudaSuccess ? reorder<true>(args[1], st) : e;
}

}  // namespace isoloco

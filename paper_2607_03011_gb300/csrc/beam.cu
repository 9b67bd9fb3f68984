// beam.cu -- a beam search's selection over beams and tokens, and what is kept for the beams moved along.
#include <algorithm>
#include <cfloat>

#include "inner.cuh"
#include "inner.h"

namespace isoloco {

namespace {

constexpr int kMaxBeams = ISOLOCO_MAX_BEAMS, kMaxKeep = ISOLOCO_MAX_TOP;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <class T>
__device__ __forceinline__ float masked_at() { return -FLT_MAX; }
template <>
__device__ __forceinline__ float masked_at<__nv_bfloat16>() { return __uint_as_float(0xff7f0000u); }
template <>
__device__ __forceinline__ float masked_at<__half>() { return -65504.f; }

// Order of (value, index): greater values first, then lower indices; -0 and 0 are equal.
__device__ __forceinline__ uint64_t rank_key(float v, uint32_t idx) {
    const uint32_t u = __float_as_uint(v + 0.f);
    const uint32_t o = (u & 0x80000000u) ? ~u : u | 0x80000000u;
    return (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~idx);
}
__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t o = static_cast<uint32_t>(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint32_t index_of(uint64_t key) { return static_cast<uint32_t>(~key); }

enum Kind : int { kLive, kDead, kNan, kFinished };

__device__ __forceinline__ Kind kind_of(float score, bool finished) {
    if (!(score < INFINITY)) return kNan;
    if (score == -INFINITY) return kDead;
    return finished ? kFinished : kLive;
}

// A beam's continuations in its own order.
struct Beam {
    Kind kind;
    float m;       // largest logit
    double base;   // score - ln sum e^{scale (x - m)}
};

struct Choice {
    double total;  // -inf for what ranks last
    uint32_t token;
};

// The p-th continuation; key: of the p-th largest logit (of a live beam).
template <class T>
__device__ __forceinline__ Choice choice(const Beam& b, int p, uint64_t key, float score, uint32_t end, double scale) {
    if (b.kind == kLive) {
        const float x = value_of(key);
        return {x <= masked_at<T>() ? -INFINITY : b.base + (static_cast<double>(x) - b.m) * scale, index_of(key)};
    }
    if (b.kind == kFinished) {
        if (p == 0) return {score, end};
        const uint32_t t = static_cast<uint32_t>(p - 1);
        return {-INFINITY, t < end ? t : t + 1};
    }
    return {-INFINITY, static_cast<uint32_t>(p)};
}

// One CTA per batch entry; every row is read once for its sums and once for each of its continuations.
template <class T>
__global__ void __launch_bounds__(256) k_beam_select(BeamArgs a) {
    constexpr int THREADS = 256;
    __shared__ uint64_t best[kMaxBeams][kMaxKeep];
    __shared__ Beam beam[kMaxBeams];
    __shared__ uint64_t part[THREADS / 32];
    __shared__ float fpart[THREADS / 32];
    const float c = a.scale * kLog2e;
    const uint32_t vocab = static_cast<uint32_t>(a.vocab);
    const int per = static_cast<int>(min(static_cast<int64_t>(a.keep), a.vocab));
    for (int64_t b = blockIdx.x; b < a.batch; b += gridDim.x) {
        for (int w = 0; w < a.beams; ++w) {
            const float score = a.scores[b * a.beams + w];
            Beam me = {kind_of(score, a.finished && a.finished[b * a.beams + w]), 0.f, 0.0};
            if (me.kind == kLive) {
                const T* row = static_cast<const T*>(a.logits) + (b * a.beams + w) * a.ld;
                uint64_t below = ~uint64_t(0);
                for (int q = 0; q < per; ++q) {
                    uint64_t top = 0;
                    for (uint32_t j = threadIdx.x; j < vocab; j += THREADS) {
                        const float x = to_f32(row[j]);
                        const uint64_t key = x == x ? rank_key(x, j) : 0;
                        if (key < below && key > top) top = key;
                    }
#pragma unroll
                    for (int o = 16; o; o >>= 1) {
                        const uint64_t other = __shfl_xor_sync(0xffffffffu, top, o);
                        top = other > top ? other : top;
                    }
                    __syncthreads();
                    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
                    __syncthreads();
                    for (int i = 0; i < THREADS / 32; ++i) top = part[i] > top ? part[i] : top;
                    if (threadIdx.x == 0) best[w][q] = top;
                    below = top;
                    if (q == 0) me.m = top ? value_of(top) : NAN;
                }
                me.m = fmaxf(me.m, -FLT_MAX);
                float s = 0.f;
                for (uint32_t j = threadIdx.x; j < vocab; j += THREADS) s += ex2((to_f32(row[j]) - me.m) * c);
#pragma unroll
                for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                if ((threadIdx.x & 31) == 0) fpart[threadIdx.x >> 5] = s;
                __syncthreads();
                s = 0.f;
                for (int i = 0; i < THREADS / 32; ++i) s += fpart[i];
                if (!(s < INFINITY)) me.kind = kNan;
                else if (me.m <= masked_at<T>()) me.kind = kDead;
                me.base = static_cast<double>(score) - log(static_cast<double>(s));
            }
            if (threadIdx.x == 0) beam[w] = me;
        }
        __syncthreads();
        if (threadIdx.x < 32) {
            // one lane per beam, each at its next continuation
            const int w = threadIdx.x;
            int p = w < a.beams ? 0 : per;
            const float score = w < a.beams ? a.scores[b * a.beams + w] : 0.f;
            for (int q = 0; q < a.keep; ++q) {
                Choice mine = {-INFINITY, 0};
                if (p < per) mine = choice<T>(beam[w], p, best[w][p], score, static_cast<uint32_t>(a.end), a.scale);
                double most = p < per ? mine.total : -INFINITY;
#pragma unroll
                for (int o = 16; o; o >>= 1) most = fmax(most, __shfl_xor_sync(0xffffffffu, most, o));
                const uint32_t have = __ballot_sync(0xffffffffu, p < per && mine.total == most);
                if (w == __ffs(have) - 1) {
                    const int64_t at = b * a.keep + q;
                    a.out_scores[at] = beam[w].kind == kNan ? NAN : static_cast<float>(mine.total);
                    a.out_beams[at] = w;
                    a.out_tokens[at] = mine.token;
                    if (a.out_finished) a.out_finished[at] = (a.finished && a.finished[b * a.beams + w]) || static_cast<int64_t>(mine.token) == a.end;
                    ++p;
                }
            }
        }
        __syncthreads();
    }
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

cudaError_t launch_beam_select(const BeamArgs& a, cudaStream_t st) {
    if (a.batch == 0) return cudaSuccess;
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(a.batch, 1 << 24));
    if (a.dtype == ISOLOCO_F32) k_beam_select<float><<<grid, 256, 0, st>>>(a);
    else if (a.dtype == ISOLOCO_BF16) k_beam_select<__nv_bfloat16><<<grid, 256, 0, st>>>(a);
    else k_beam_select<__half><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
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

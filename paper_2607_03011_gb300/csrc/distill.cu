// distill.cu -- distillation from a teacher's top logits: the loss of every row and its gradient by the logits.
//
// With z = scale x, M the row's largest logit, c = scale / ln 2 and the row's tokens parted into those of the teacher's list
// and the others:
//     others: Mr their largest logit, Sr = sum 2^((x - Mr) c)          list: Ml, Sl the same
//     S = Sl 2^((Ml - M) c) + Sr 2^((Mr - M) c),   lse = scale M + ln S,   P = Sr 2^((Mr - M) c) / S
//     loss = sum q (ln q - z + lse) + r (ln r - ln P),  Q = sum q + r
//     gradient: others 2^((x - Mr) c) (P Q - r) / Sr,  list 2^((x - M) c) / S Q - q
// The others are summed by themselves and about their own largest: a student that has learned the list leaves them a small
// share, which a difference (S less the list's) would lose, and one so small that it is 0 about M still has its logarithm.
#include <cfloat>

#include "inner.cuh"
#include "inner.h"

namespace isoloco {

namespace {

constexpr int kList = ISOLOCO_MAX_LIST;
constexpr float kLowest = -1000.f;  // 2^d is 0 there
constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kNone = 0xffffffffu;

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
// 2^((x - m) c)
__device__ __forceinline__ float power(float x, float m, float c) { return ex2(cut((x - m) * c)); }

// The largest logit that counts as masked.
template <class T>
__device__ __forceinline__ float masked_at() { return -FLT_MAX; }
template <>
__device__ __forceinline__ float masked_at<__nv_bfloat16>() { return __uint_as_float(0xff7f0000u); }
template <>
__device__ __forceinline__ float masked_at<__half>() { return -65504.f; }

__device__ __forceinline__ float element(const void* p, int64_t i, int dtype) {
    if (dtype == ISOLOCO_F32) return static_cast<const float*>(p)[i];
    if (dtype == ISOLOCO_BF16) return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
    return to_f32(static_cast<const __half*>(p)[i]);
}

// A row's list as its CTA holds it.
struct ListSmem {
    uint32_t index[kList];  // kNone: not there, or the same token as an earlier entry
    float logp[kList], q[kList], x[kList];
    float part[8][32];  // of the warps' reductions
};

// What the list gives for the row's loss: sums over its entries, and over its different tokens.
struct List {
    bool any;           // there are entries that count
    float weight;       // sum q
    float rest;         // 1 - sum q, at least 0 (DROP: 0)
    float terms;        // sum q (ln q - scale (x - m))
    float m, s;         // largest logit and sum of powers about it
};

template <int THREADS>
__device__ __forceinline__ float sum_cta(float v, float* part) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) v += part[i];
    return v;
}
template <int THREADS>
__device__ __forceinline__ float max_cta(float v, float* part) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < THREADS / 32; ++i) v = fmaxf(v, part[i]);
    return v;
}

// Reads row r's list and the student's logits for it.
template <class T, int THREADS>
__device__ __forceinline__ List load_list(const DistillArgs& a, int64_t r, const T* row, float c, ListSmem& sm) {
    float top = -FLT_MAX, m = -FLT_MAX, there = 0.f;
    for (int e = threadIdx.x; e < a.k; e += THREADS) {
        const int64_t at = r * a.ld_index + e;
        const int64_t id = a.index64 ? static_cast<const int64_t*>(a.top_index)[at] : static_cast<const int32_t*>(a.top_index)[at];
        const bool here = id >= 0 && id < a.vocab;
        float x = 0.f, v = -INFINITY;
        if (here) {
            v = element(a.top_logp, r * a.ld_logp + e, a.logp_dtype);
            x = to_f32(row[id]);
            if (x <= masked_at<T>()) x = -INFINITY;
            top = fmaxf(top, v);
            m = fmaxf(m, x);
            there = 1.f;
        }
        sm.index[e] = here ? static_cast<uint32_t>(id) : kNone;
        sm.logp[e] = v;
        sm.x[e] = x;
    }
    List l;
    top = max_cta<THREADS>(top, sm.part[0]);
    l.m = max_cta<THREADS>(m, sm.part[1]);
    there = max_cta<THREADS>(there, sm.part[2]);  // (its barriers order what was written above, too)
    const float about = a.rest ? 0.f : top;
    // entries of one token: the first of them stands for all, with the sum of their weights
    float w = 0.f, terms = 0.f, s = 0.f;
    uint32_t first[kList / THREADS > 0 ? kList / THREADS : 1];
    float weight[kList / THREADS > 0 ? kList / THREADS : 1];
#pragma unroll
    for (int n = 0; n < (kList / THREADS > 0 ? kList / THREADS : 1); ++n) {
        const int e = threadIdx.x + n * THREADS;
        first[n] = kNone;
        weight[n] = 0.f;
        if (e >= a.k || sm.index[e] == kNone) continue;
        const uint32_t id = sm.index[e];
        const float x = sm.x[e], we = expf(sm.logp[e] - about);
        w += we;
        if (we != 0.f) terms += we * ((sm.logp[e] - about) - (x - l.m) * a.scale);
        bool earlier = false;
        float total = 0.f;
        for (int j = 0; j < a.k; ++j)
            if (sm.index[j] == id) {
                earlier |= j < e;
                total += expf(sm.logp[j] - about);
            }
        weight[n] = total;
        if (!earlier) {
            first[n] = id;
            s += power(x, l.m, c);
        }
    }
    l.weight = sum_cta<THREADS>(w, sm.part[3]);
    l.terms = sum_cta<THREADS>(terms, sm.part[4]);
    l.s = sum_cta<THREADS>(s, sm.part[5]);
    const float scale = a.rest ? 1.f : 1.f / l.weight;
#pragma unroll
    for (int n = 0; n < (kList / THREADS > 0 ? kList / THREADS : 1); ++n) {
        const int e = threadIdx.x + n * THREADS;
        if (e < a.k) {
            sm.index[e] = first[n];
            sm.q[e] = weight[n] * scale;
        }
    }
    l.any = there != 0.f && (a.rest || l.weight != 0.f);
    l.rest = 0.f;
    if (a.rest) {
        const float rest = 1.f - l.weight;
        l.rest = rest < 0.f ? 0.f : rest;
        if (!(l.weight < INFINITY)) l.weight = l.rest = NAN;
    } else {
        l.terms = l.terms * scale - logf(l.weight);
        l.weight = l.weight == l.weight ? 1.f : l.weight;
    }
    __syncthreads();
    return l;
}

// Sums about the largest logit so far (no logit: s = 0).
struct Sum {
    float m, s;
    __device__ __forceinline__ void add(float x, float c) {
        if (x > m) s *= power(m, x, c), m = x;
        s += power(x, m, c);
    }
    __device__ __forceinline__ void take(const Sum& o, float c) {
        const float to = fmaxf(m, o.m);
        s = s * power(m, to, c) + o.s * power(o.m, to, c);
        m = to;
    }
};

// The row from its list and the others' sums.
struct Row {
    float m, s, loss;
    bool none;     // no gradient
    float others;  // gradient / (scale grad_loss) of an entry outside the list: others 2^((x - Mr) c)
    float list;    // and of one in it: list 2^((x - m) c) - q
    template <class T>
    __device__ __forceinline__ void find(const DistillArgs& a, const List& l, Sum o, float c) {
        if (o.m <= masked_at<T>() && o.s == o.s) o.s = 0.f;  // (a NaN stays)
        m = fmaxf(l.m, o.m);
        const float so = o.s * power(o.m, m, c);
        s = l.s * power(l.m, m, c) + so;
        const float rest = o.s == 0.f ? 0.f : l.rest, Q = l.weight + rest, lns = logf(s);
        none = !l.any || s == 0.f;
        loss = l.terms;
        if (l.weight != 0.f) loss += l.weight * fmaf(m - l.m, a.scale, lns);
        if (rest != 0.f) loss += rest * (logf(rest) + fmaf(m - o.m, a.scale, lns - logf(o.s)));
        if (s == 0.f) loss = l.weight != 0.f ? INFINITY * l.weight : 0.f;
        if (!l.any) loss = 0.f;
        list = none ? 0.f : Q / s;
        others = none || o.s == 0.f ? 0.f : (so / s * Q - rest) / o.s;
    }
};

// One CTA per row; two passes over it.
template <class T, bool GIVEN>
__global__ void __launch_bounds__(256) k_distill(DistillArgs a) {
    constexpr int THREADS = 256;
    __shared__ ListSmem sm;
    __shared__ uint32_t marks[256];  // of the list's tokens, by their index modulo 8192
    __shared__ Sum sums[THREADS / 32];
    const float c = a.scale * kLog2e;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* row = static_cast<const T*>(a.logits) + r * a.ld;
        const List l = load_list<T, THREADS>(a, r, row, c, sm);
        marks[threadIdx.x] = 0;
        __syncthreads();
        for (int e = threadIdx.x; e < a.k; e += THREADS)
            if (sm.index[e] != kNone) atomicOr(&marks[(sm.index[e] & 8191) >> 5], 1u << (sm.index[e] & 31));
        __syncthreads();
        auto listed = [&](uint32_t j) {
            if (!(marks[(j & 8191) >> 5] >> (j & 31) & 1)) return false;
            for (int e = 0; e < a.k; ++e)
                if (sm.index[e] == j) return true;
            return false;
        };
        Sum o = {-FLT_MAX, 0.f};
        if (GIVEN) {
            o = {a.saved[2 * r], a.saved[2 * r + 1]};
        } else {
            for (uint32_t j = threadIdx.x; j < a.vocab; j += THREADS)
                if (!listed(j)) o.add(to_f32(row[j]), c);
#pragma unroll
            for (int s = 16; s; s >>= 1) o.take({__shfl_xor_sync(0xffffffffu, o.m, s), __shfl_xor_sync(0xffffffffu, o.s, s)}, c);
            if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = o;
            __syncthreads();
            o = sums[0];
            for (int i = 1; i < THREADS / 32; ++i) o.take(sums[i], c);
        }
        Row f;
        f.find<T>(a, l, o, c);
        if (!GIVEN && threadIdx.x == 0) {
            a.loss[r] = f.loss;
            if (a.saved) a.saved[2 * r] = o.m, a.saved[2 * r + 1] = o.s;
        }
        if (a.grad_logits) {
            T* out = static_cast<T*>(a.grad_logits) + r * a.ld_grad;
            const float g = f.none ? 0.f : a.scale * a.grad_loss[r];
            for (uint32_t j = threadIdx.x; j < a.vocab; j += THREADS)
                if (!listed(j)) out[j] = from_f32<T>(f.none ? 0.f : g * f.others * power(to_f32(row[j]), o.m, c));
            for (int e = threadIdx.x; e < a.k; e += THREADS)
                if (sm.index[e] != kNone) out[sm.index[e]] = from_f32<T>(f.none ? 0.f : g * (f.list * power(sm.x[e], f.m, c) - sm.q[e]));
        }
        __syncthreads();
    }
}

template <class T>
cudaError_t run(const DistillArgs& a, bool given, cudaStream_t st) {
    const unsigned grid = static_cast<unsigned>(a.rows < (1 << 24) ? a.rows : (1 << 24));
    if (given) k_distill<T, true><<<grid, 256, 0, st>>>(a);
    else k_distill<T, false><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch(const DistillArgs& a, bool given, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    if (a.dtype == ISOLOCO_F32) return run<float>(a, given, st);
    if (a.dtype == ISOLOCO_BF16) return run<__nv_bfloat16>(a, given, st);
    return run<__half>(a, given, st);
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, cudaStream_t st) { return launch(a, false, st); }
cudaError_t launch_distill_grad(const DistillArgs& a, cudaStream_t st) { return launch(a, true, st); }

}  // namespace isoloco

// distill.cu -- distillation from a teacher's top logits: the loss of every row and its gradient by the logits.
//
// With z = scale x, M the row's largest logit, c = scale / ln 2 and the row's tokens parted into those of the teacher's list
// and the others:
//     others: Mr their largest logit, Sr = sum 2^((x - Mr) c)          list: Ml, Sl the same
//     S = Sl 2^((Ml - M) c) + Sr 2^((Mr - M) c),   lse = scale M + ln S,   P = Sr 2^((Mr - M) c) / S
//     loss = sum q (ln q - z + lse) + r (ln r - ln P),  Q = sum q + r    (q of a token: the sum over its entries)
//     gradient: others 2^((x - Mr) c) (P Q - r) / Sr,  list 2^((x - M) c) / S Q - q
// The others are summed by themselves and about their own largest: a student that has learned the list leaves them a small
// share, which a difference (S less the list's) would lose, and one so small that it is 0 about M still has its logarithm.
// Without a rest (r = 0) the parting is not needed: the sums are over all tokens, and Mr = M, Sr = S above.
//
// What bounds it: HBM (8192 x 32000 bf16 with gradient 173 us, 6.1 TB/s of logits read and gradient written; the copy's rate
// allows 157).  Issue slots are half used, the pipe of the powers, two to an entry, a third.  The list (k tokens scattered over the row,
// equal ones added up) is a chain of dependent loads and small reductions; a warp of its own goes through it beside the pass over the row (before
// it: 22 us more).
#include <algorithm>

#include "common.cuh"
#include "inner.cuh"
#include "inner.h"
#include "per_device.h"
#include "rows.cuh"

namespace isoloco {

namespace {

constexpr int kList = ISOLOCO_MAX_LIST;
constexpr int kSaved = 6;  // floats of a row for the gradient by itself
constexpr int kMaxSplit = 8;
constexpr int kUnroll = 4;
constexpr uint32_t kNone = 0xffffffffu;

// ---- which kernel, and how many threads to how much of a row (8192 rows unless said otherwise, us)
// With gradient a row is held in shared memory (k_distill_held): 32000 bf16 173, where reading it again from L2 takes 195
// (loss and list in the same threads) and persistent CTAs that start together 247: they stay in step, so that loads, powers and
// stores do not overlap.
// In one CTA up to kHeldBytes (two of 512 threads to an SM above kWideHeld, three of 256 below): 50021 fp16 258, in two CTAs that wait for each
// other 289; 4096 x 54000 bf16 151 and 180; 4096 x 25000 fp32 137 and 141.
// 16-bit rows of more (kHeldMost entries) are read again from L2, in shares of kShareBytes: 4096 x 64000 bf16 186, held in two shares 198; 128000
// bf16 904, held in four 1205 (in shares of 140000 bytes, which L2 does not keep, 985; of 40000 1070).  fp32 rows have half the
// entries to a byte: 2048 x 128000 378 held, 400 from L2.
// Without gradient nothing is held: 4096 x 32000 fp32 79 to 82, held 131.
constexpr int64_t kHeldBytes = 108 * 1024;
constexpr int64_t kWideHeld = 72 * 1024;
constexpr int64_t kMostHeldBytes = 216 * 1024;  // (where few rows are long)
constexpr int64_t kHeldMost = 55000;
constexpr int64_t kShareBytes = 98304;
// 64 threads: held 4000 bf16 43 us, 54 with 128; 8000 60 and 66.  128: held fp32 2048 x 128000 (shares of 16000) 378, 397 with 256.
constexpr int64_t kSmallHeld = 8192, kMediumHeld = 16384;
constexpr int64_t kSmall = 8192, kMedium = 16384;
// CTAs per SM that the registers are cut for
constexpr int held_ctas(int threads) { return threads == 64 ? 11 : threads == 128 ? 7 : threads == 256 ? 4 : 2; }
constexpr int stream_ctas(int threads) { return threads == 64 ? 14 : threads == 128 ? 8 : 5; }
// Entries of a share whose marks (of the list's tokens) are kept apart.
constexpr uint32_t marks_of(int threads) { return threads <= 128 ? 16384 : 65536; }
constexpr uint64_t kLostNs = 20000000;  // the limit of a wait for a row whose copy is not started (DistillArgs::lost)
constexpr float kSmallRest = 0.0625f;  // rests of a teacher below this are made good (left_of)
// Vectors per thread of the gradient by itself: 8192 x 128000 bf16 657 us (the copy rate allows 628); 16 667, 8 769, 4 869 (a list for
// every span).
constexpr int kSpan = 32;

// 2^((x - m) c)
__device__ __forceinline__ float power(float x, float m, float c) { return ex2((x - m) * c); }

__device__ __forceinline__ float element(const void* p, int64_t i, int dtype) {
    if (dtype == ISOLOCO_F32) return static_cast<const float*>(p)[i];
    if (dtype == ISOLOCO_BF16) return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
    return to_f32(static_cast<const __half*>(p)[i]);
}

__device__ __forceinline__ uint32_t index_at(const DistillArgs& a, int64_t r, int e) {
    const int64_t at = r * a.ld_index + e;
    const int64_t id = a.index64 ? static_cast<const int64_t*>(a.top_index)[at] : static_cast<const int32_t*>(a.top_index)[at];
    return id >= 0 && id < a.vocab ? static_cast<uint32_t>(id) : kNone;
}

// A row's list as its CTA holds it.
struct ListSmem {
    uint4 index[kList / 4];  // of tokens; kNone: no entry
    float logp[kList], x[kList];
    float q[kList];          // of the first entry of a token, times 1 / inv; -1 of others
    __device__ __forceinline__ uint32_t* ids() { return reinterpret_cast<uint32_t*>(index); }
};

// Whether entry e is the first of its token, and the sum of f(entry) over all entries of that token, in their order.
template <class F>
__device__ __forceinline__ bool first_of_token(ListSmem& sm, int k, int e, uint32_t id, float& total, F f) {
    bool first = true;
    total = 0.f;
    for (int j = 0; j < k; j += 4) {
        const uint4 w = sm.index[j / 4];
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (v[i] == id) {
                first = first && j + i >= e;
                total += f(j + i);
            }
    }
    return first;
}

struct List {
    bool any;           // there are entries that count
    float weight;       // sum q
    float rest;         // 1 - sum q, at least 0 (DROP: 0)
    float terms;        // sum over its tokens of q (ln q - scale (x - m))
    float m, s;         // largest logit of its tokens, and the sum of powers about it
    float about, inv;   // q = e^(logp - about) inv

    // Entry e of row r: its token (kNone: none) and log probability.
    static __device__ __forceinline__ void fetch(const DistillArgs& a, int64_t r, int e, uint32_t& id, float& v) {
        id = e < a.k ? index_at(a, r, e) : kNone;
        v = e < a.k ? element(a.top_logp, r * a.ld_logp + e, a.logp_dtype) : 0.f;
    }
    // The student's logit for it.
    template <class T>
    static __device__ __forceinline__ float logit(const T* row, uint32_t id) {
        const float x = id != kNone ? to_f32(row[id]) : 0.f;
        return x <= masked_at<T>() ? -INFINITY : x;
    }
    // The rest of it, from the sums of the weights e^(logp - about) and of their terms, and what they leave of 1.
    __device__ __forceinline__ void finish(const DistillArgs& a, float w, float t, float left) {
        any = any && (a.rest || w != 0.f);
        if (a.rest) {
            inv = 1.f;
            weight = w < INFINITY ? w : NAN;
            rest = w < INFINITY ? fmaxf(left, 0.f) : NAN;
            terms = t;
        } else {
            inv = 1.f / w;
            weight = w == w ? 1.f : w;
            rest = 0.f;
            terms = t * inv - logf(w);
        }
    }
};

// Sums of powers about the largest logit so far (no logit: s = 0).
struct Sum {
    float m, s;
    __device__ __forceinline__ void raise(float to, float c) { s *= power(m, to, c), m = to; }
    __device__ __forceinline__ void add(float x, float c) {
        if (x > m) raise(x, c);
        s += power(x, m, c);
    }
    __device__ __forceinline__ void take(Sum o, float c) {
        const float to = fmaxf(m, o.m);
        raise(to, c);
        o.raise(to, c);
        s += o.s;
    }
    // over W lanes: the common maximum, then one rescaling
    template <int W>
    __device__ __forceinline__ void lanes(float c) {
        float to = m;
#pragma unroll
        for (int o = W / 2; o; o >>= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, o));
        raise(to, c);
#pragma unroll
        for (int o = W / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    }
};

// A thread's sums, of even and odd entries apart, about m.
__device__ __forceinline__ void raise_to(float big, float& m, F2& s2, float c) {
    if (big > m) {
        const float f = power(m, big, c);
        s2 = mul2(s2, pair(f, f));
        m = big;
    }
}
template <class T>
__device__ __forceinline__ void add_powers(const Vec<T>& v, float m, F2 c2, F2& s2) {
    const F2 minus = pair(-m, -m);
    float f[Vec<T>::kN];
    v.unpack(f);
    s2 = add2(s2, powers(f, minus, c2));
}
__device__ __forceinline__ float both(F2 s2) {
    float a, b;
    unpair(s2, a, b);
    return a + b;
}
// G 2^((x - m) c) in place of x.
template <class T>
__device__ __forceinline__ void gradients(Vec<T>& v, F2 minus_m, F2 c2, F2 G2) {
    float d[Vec<T>::kN];
    v.unpack(d);
#pragma unroll
    for (int j = 0; j < Vec<T>::kN; j += 2) {
        float d0, d1;
        unpair(mul2(add2(pair(d[j], d[j + 1]), minus_m), c2), d0, d1);
        unpair(mul2(pair(ex2(d0), ex2(d1)), G2), d[j], d[j + 1]);
    }
    v.pack(d);
}

// The row from its list and the others' sums.
struct Row {
    float m, loss;
    bool none;     // no gradient
    float others;  // gradient / (scale grad_loss) of an entry outside the list: others 2^((x - Mr) c)
    float list;    // and of one in it: list 2^((x - m) c) - q
};
// o: the sums over the others, or (DROP) over all.
template <class T>
__device__ __forceinline__ Row row_of(const DistillArgs& a, const List& l, Sum o, float c) {
    if (o.m <= masked_at<T>() && o.s == o.s) o.s = 0.f;  // (a NaN stays)
    float m = o.m, so = o.s, s = o.s;
    if (a.rest) {
        m = fmaxf(l.m, o.m);
        so = o.s * power(o.m, m, c);
        s = l.s * power(l.m, m, c) + so;
    }
    const float rest = o.s == 0.f ? 0.f : l.rest, Q = l.weight + rest, lns = logf(s);
    const bool none = !l.any || s == 0.f;
    float loss = l.terms;
    if (l.weight != 0.f) loss += l.weight * fmaf(m - l.m, a.scale, lns);
    if (rest != 0.f) loss += rest * (logf(rest) + fmaf(m - o.m, a.scale, lns - logf(o.s)));
    if (s == 0.f) loss = l.weight != 0.f ? INFINITY * l.weight : 0.f;
    if (!l.any) loss = 0.f;
    return {m, loss, none, none || o.s == 0.f ? 0.f : (so / s * Q - rest) / o.s, none ? 0.f : Q / s};
}

// out = G 2^((x - m) c) (none: 0) for a CTA's n entries.
template <class T, int THREADS>
__device__ __forceinline__ void put_gradient(const T* x, T* out, uint32_t n, float m, float c, float G, bool none) {
    constexpr uint32_t V = Vec<T>::kN;
    auto grad = [&](float v) { return none ? 0.f : G * power(v, m, c); };
    const uint32_t mis = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(x) & 15u);
    if (((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(x)) & 15u) != 0) {
        for (uint32_t i = threadIdx.x; i < n; i += THREADS) out[i] = from_f32<T>(grad(to_f32(x[i])));
        return;
    }
    const uint32_t head = min(n, mis ? (16u - mis) / static_cast<uint32_t>(sizeof(T)) : 0u), nvec = (n - head) / V, tail = head + nvec * V;
    if (threadIdx.x < head) out[threadIdx.x] = from_f32<T>(grad(to_f32(x[threadIdx.x])));
    const F2 c2 = pair(c, c), G2 = pair(G, G), minus = pair(-m, -m);
    const uint4* src = reinterpret_cast<const uint4*>(x + head);
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < nvec; i += THREADS) {
        Vec<T> v;
        v.raw = src[i];
        gradients(v, minus, c2, G2);
        if (none) v.raw = make_uint4(0, 0, 0, 0);  // (whatever the logits are)
        st_stream(out + head + i * V, v.raw);
    }
    if (threadIdx.x < n - tail) out[tail + threadIdx.x] = from_f32<T>(grad(to_f32(x[tail + threadIdx.x])));
}

// Row::others and Row::none alone, which a second pass over the row waits for: without logarithms, and with quotients good to two
// units in the last place.
template <class T>
__device__ __forceinline__ float others_of(const DistillArgs& a, const List& l, Sum o, float c, bool& none) {
    if (o.m <= masked_at<T>() && o.s == o.s) o.s = 0.f;
    if (!a.rest) {
        none = !l.any || o.s == 0.f;
        return none ? 0.f : __fdividef(l.weight, o.s);
    }
    const float m = fmaxf(l.m, o.m), so = o.s * power(o.m, m, c), s = l.s * power(l.m, m, c) + so;
    const float rest = o.s == 0.f ? 0.f : l.rest;
    none = !l.any || s == 0.f;
    return none || o.s == 0.f ? 0.f : __fdividef(__fdividef(so, s) * (l.weight + rest) - rest, o.s);
}

__device__ __forceinline__ void save_row(float* to, const Sum& o, const Row& f, const List& l) {
    to[0] = o.m, to[1] = f.others, to[2] = f.m, to[3] = f.list, to[4] = l.about, to[5] = f.none ? -1.f : l.inv;
}

// A CTA's share of a row: entries before the first 16-byte boundary, vectors, entries behind.
template <class T>
struct Share {
    static constexpr uint32_t V = Vec<T>::kN;
    const T* x;      // the share's first entry
    uint32_t first;  // its index in the row
    uint32_t n, head, nvec;
    __device__ __forceinline__ Share(const T* row, uint32_t vocab, uint32_t rank, uint32_t per) {
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

// The vector's entries whose bits are set, masked.
template <class T>
__device__ __forceinline__ void mask_entries(uint4& raw, uint32_t bits) {
    uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            if (bits >> i & 1) w[i] = 0xff800000u;
        } else {
            constexpr uint32_t ninf = __is_same(T, __half) ? 0xfc00u : 0xff80u;
            if (bits >> (2 * i) & 1) w[i] = (w[i] & 0xffff0000u) | ninf;
            if (bits >> (2 * i + 1) & 1) w[i] = (w[i] & 0xffffu) | ninf << 16;
        }
    }
    raw = make_uint4(w[0], w[1], w[2], w[3]);
}

// A bulk copy of `bytes` (a multiple of 16; both addresses, too) into this CTA's shared memory.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src),
                 "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// A barrier of the first `threads` threads, and one that is passed by some and waited at by others.
template <int ID>
__device__ __forceinline__ void bar_sync(int threads) { asm volatile("bar.sync %0, %1;" ::"n"(ID), "r"(threads) : "memory"); }
template <int ID>
__device__ __forceinline__ void bar_arrive(int threads) { asm volatile("bar.arrive %0, %1;" ::"n"(ID), "r"(threads) : "memory"); }

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// A row's list in one warp.
template <class T>
__device__ __forceinline__ void warp_read(const DistillArgs& a, int64_t r, ListSmem& sm) {
    const T* row = static_cast<const T*>(a.logits) + r * a.ld;
#pragma unroll 2
    for (int e = threadIdx.x & 31; e < (a.k + 3) / 4 * 4; e += 32) {
        uint32_t id;
        float v;
        List::fetch(a, r, e, id, v);
        sm.ids()[e] = id;
        sm.logp[e] = id == kNone ? -INFINITY : v;
        sm.x[e] = List::logit(row, id);
    }
    __syncwarp();
}
// 1 - sum e^logp, w the sum in fp32.  That is off by some 2^-22, which is nothing beside a large rest, but all of one that a teacher
// leaves whose list holds nearly everything; rests below kSmallRest are made good to 2^-43 for each entry.  e^v - 1 = hi + lo, two fp32 numbers:
// Taylor's series at v / 1024, then ten times (1 + p)^2 - 1 = 2 p + p^2, with the roundings of hi + hi + hi^2 kept in lo (off by 2^-44 at most over
// 800000 numbers tried); the sums as whole numbers of 2^-22 and 2^-45.  8192 x 32000 bf16, lists of 32: 185 us where all rests are small, 180 where
// none is; with 64-bit floating point, of which an SM makes two operations a cycle, 193.
__device__ __forceinline__ float left_of(const DistillArgs& a, float w, ListSmem& sm) {
    if (!(1.f - w < kSmallRest)) return 1.f - w;
    constexpr int kTimes = 10;
    constexpr float kCoarse = 1 << 22, kFine = 35184372088832.f;
    int coarse = 0, fine = 0;  // (of 256 entries: at most 2^30 each)
#pragma unroll 1
    for (int e = threadIdx.x & 31; e < a.k; e += 32) {
        const float v = fminf(sm.logp[e], 0.f);  // (one above 0 leaves nothing as it is)
        if (v < -40.f) continue;                 // nothing in these units (no entry: -inf)
        const float x = v * (1.f / (1 << kTimes)), xx = __fmul_rn(x, x), half = 0.5f * xx;
        const float more = x * xx * fmaf(x, fmaf(x, 1.f / 120.f, 1.f / 24.f), 1.f / 6.f);
        float hi = __fadd_rn(x, half), lo = __fadd_rn(__fadd_rn(x, -hi), half) + fmaf(0.5f, __fmaf_rn(x, x, -xx), more);
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            const float two = hi + hi, sq = __fmul_rn(hi, hi), low = fmaf(two, lo, __fmaf_rn(hi, hi, -sq));
            const float top = __fadd_rn(two, sq), l = __fadd_rn(__fadd_rn(two, -top), sq) + fmaf(2.f, lo, low);
            hi = __fadd_rn(top, l);
            lo = __fadd_rn(__fadd_rn(top, -hi), l);
        }
        const int n = __float2int_rn(hi * kCoarse);
        coarse += n + (1 << 22);
        fine += __float2int_rn((fmaf(static_cast<float>(n), -1.f / kCoarse, hi) + lo) * kFine);
    }
    coarse = __reduce_add_sync(0xffffffffu, coarse);
    fine = __reduce_add_sync(0xffffffffu, fine);
    const long long units = static_cast<long long>((1 << 22) - coarse) * (1 << 23) - fine;
    return __ll2float_rn(units) * (1.f / kFine);
}
template <bool REST>
__device__ __forceinline__ List warp_sums(const DistillArgs& a, float c, ListSmem& sm) {
    const int lane = threadIdx.x & 31;
    List l;
    float top = -INFINITY, m = -FLT_MAX, w = 0.f, t = 0.f, s = 0.f;
    for (int e = lane; e < a.k; e += 32)
        if (sm.ids()[e] != kNone) top = fmaxf(top, fmaxf(sm.logp[e], -FLT_MAX)), m = fmaxf(m, sm.x[e]);
    top = warp_max(top);
    l.m = m = warp_max(m);
    l.any = top != -INFINITY;  // (there are entries)
    const float about = l.about = a.rest ? 0.f : top;
    for (int e = lane; e < a.k; e += 32) {
        const uint32_t id = sm.ids()[e];
        sm.q[e] = -1.f;
        if (id == kNone) continue;
        const float v = sm.logp[e], x = sm.x[e], we = expf(v - about);
        w += we;
        float total;
        if (first_of_token(sm, a.k, e, id, total, [&](int j) { return j == e ? we : expf(sm.logp[j] - about); })) {
            sm.q[e] = total;
            s += power(x, m, c);
            // (its only entry of a weight above 0: the logarithm as it was given)
            if (total != 0.f) t += total * ((total == we ? v - about : logf(total)) - (x - m) * a.scale);
        }
    }
    l.s = warp_sum(s);
    w = warp_sum(w);
    l.finish(a, w, warp_sum(t), REST ? left_of(a, w, sm) : 0.f);
    return l;
}

// A cluster of `split` CTAs per row, each with `per` of its entries, which go past in registers; a gradient reads them again (rows that
// no shared memory holds).  One warp more than the THREADS does what the list needs meanwhile.
template <class T, int THREADS, bool REST, bool GRAD>
__global__ void __launch_bounds__(THREADS + 32, stream_ctas(THREADS)) k_distill(DistillArgs a, uint32_t split, uint32_t per) {
    constexpr uint32_t V = Vec<T>::kN;
    constexpr int kAll = THREADS + 32;
    enum { kMasked = 1, kSums, kListed, kDone };  // barriers
    __shared__ ListSmem sm;
    __shared__ List list_out;
    __shared__ Sum sums[THREADS / 32], peer[kMaxSplit], sum_out;
    constexpr uint32_t kMarks = marks_of(THREADS);
    __shared__ uint32_t marks[REST ? kMarks / 32 : 1];  // of the list's tokens: bit (place behind the head) modulo kMarks
    const uint32_t rank = split > 1 ? cluster_ctarank() : 0u;
    if (split > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int64_t r = blockIdx.x / split;
    const T* row = static_cast<const T*>(a.logits) + r * a.ld;
    const Share<T> sh(row, static_cast<uint32_t>(a.vocab), rank, per);
    T* out = GRAD ? static_cast<T*>(a.grad_logits) + r * a.ld_grad + sh.first : nullptr;
    const float c = a.scale * kLog2e;
    if (threadIdx.x >= THREADS) {
        const uint32_t lane = threadIdx.x & 31;
        if (REST) {
            for (uint32_t i = lane; i < min(kMarks / 32, (sh.n + 31) / 32); i += 32) marks[i] = 0;
            __syncwarp();
        }
        warp_read<T>(a, r, sm);
        if (REST) {
            for (int e = lane; e < a.k; e += 32) {
                const uint32_t j = sm.ids()[e] - sh.first - sh.head;
                if (sm.ids()[e] != kNone && sm.ids()[e] >= sh.first + sh.head && j < sh.nvec * V) atomicOr(&marks[j % kMarks / 32], 1u << (j & 31));
            }
            __syncwarp();
            bar_arrive<kMasked>(kAll);
        }
        const List l = warp_sums<REST>(a, c, sm);
        if (lane == 0) list_out = l;
        __syncwarp();
        if (GRAD) bar_arrive<kListed>(kAll);
        if (split > 1) {
            asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
            cluster_sync();
        }
        bar_sync<kDone>(kAll);
        const Sum o = sum_out;
        const Row f = row_of<T>(a, l, o, c);
        if (rank == 0 && lane == 0) {
            a.loss[r] = f.loss;
            if (a.saved) save_row(a.saved + kSaved * r, o, f, l);
        }
        if (GRAD) {  // the list's entries once more
            const float g = a.scale * a.grad_loss[r];
            for (int e = lane; e < a.k; e += 32)
                if (sm.ids()[e] != kNone && sm.q[e] != -1.f && sm.ids()[e] - sh.first < sh.n)
                    out[sm.ids()[e] - sh.first] = from_f32<T>(f.none ? 0.f : g * (f.list * power(sm.x[e], f.m, c) - sm.q[e] * l.inv));
        }
        return;
    }
    const F2 c2 = pair(c, c);
    // whether the share's j-th entry is in the list
    auto listed = [&](uint32_t j) {
        for (int e = 0; e < a.k; ++e)
            if (sm.ids()[e] == sh.first + j) return true;
        return false;
    };
    const bool exact_marks = sh.n <= kMarks;
    // the bits of vector i
    auto marked = [&](uint32_t i) -> uint32_t {
        const uint32_t j = i * V, at = j % kMarks;
        uint32_t bits = reinterpret_cast<const uint8_t*>(marks)[at / 8];
        if (V == 4) bits = bits >> (at & 4) & 15u;
        if (bits && !exact_marks) {
            uint32_t sure = 0;
            for (uint32_t b = 0; b < V; ++b)
                if (bits >> b & 1 && listed(sh.head + j + b)) sure |= 1u << b;
            bits = sure;
        }
        return bits;
    };
    float m = -FLT_MAX;
    F2 s2 = pair(0.f, 0.f);
    Vec<T> v[kUnroll];
    auto load = [&](uint32_t i, auto all) {
        constexpr bool ALL = decltype(all)::value;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (ALL || i + u * THREADS < sh.nvec) {
                // (read again below: plain loads, which stay in L2; the gradient may overwrite the logits)
                if constexpr (GRAD) v[u].raw = *sh.vec(i + u * THREADS);
                else v[u].raw = ld_stream(sh.vec(i + u * THREADS));
            }
    };
    auto add = [&](uint32_t i, auto all) {
        constexpr bool ALL = decltype(all)::value;
        Largest<T> most, other;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (ALL || i + u * THREADS < sh.nvec) {
                if constexpr (REST) {
                    const uint32_t bits = marked(i + u * THREADS);
                    if (bits) mask_entries<T>(v[u].raw, bits);
                }
                other.set(v[u]);
                if (u == 0) most = other;
                else most.take(other);
            }
        raise_to(most.value(), m, s2, c);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (ALL || i + u * THREADS < sh.nvec) add_powers(v[u], m, c2, s2);
    };
    uint32_t i = threadIdx.x;
    // the first vectors are on their way while the marks are made
    if (i < sh.nvec) load(i, std::false_type());
    __syncwarp();
    if (REST) bar_sync<kMasked>(kAll);
    if (i < sh.nvec) add(i, std::false_type());
    i += kUnroll * THREADS;
    for (; i + (kUnroll - 1) * THREADS < sh.nvec; i += kUnroll * THREADS) {
        load(i, std::true_type());
        add(i, std::true_type());
    }
    if (i < sh.nvec) {
        load(i, std::false_type());
        add(i, std::false_type());
    }
    Sum o = {m, both(s2)};
    if (threadIdx.x < sh.head && !(REST && listed(threadIdx.x))) o.add(to_f32(sh.x[threadIdx.x]), c);
    if (threadIdx.x < sh.n - sh.tail() && !(REST && listed(sh.tail() + threadIdx.x))) o.add(to_f32(sh.x[sh.tail() + threadIdx.x]), c);
    __syncwarp();
    o.lanes<32>(c);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = o;
    __syncwarp();
    bar_sync<kSums>(THREADS);
    o = sums[threadIdx.x & (THREADS / 32 - 1)];
    o.lanes<THREADS / 32>(c);
    if (split > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // (every CTA of the cluster runs)
        if (threadIdx.x < split) {
            const uint32_t to = mapa_shared(smem_u32(peer + rank), threadIdx.x);
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(o.m) : "memory");
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4), "f"(o.s) : "memory");
        }
        __syncwarp();
        cluster_sync();
        o = peer[0];
        for (uint32_t q = 1; q < split; ++q) o.take(peer[q], c);
    }
    if (threadIdx.x == 0) sum_out = o;
    __syncwarp();
    if constexpr (GRAD) {
        bar_sync<kListed>(kAll);
        bool none;
        const float others = others_of<T>(a, list_out, o, c, none);
        put_gradient<T, THREADS>(sh.x, out, sh.n, o.m, c, none ? 0.f : a.scale * a.grad_loss[r] * others, none);
        __syncwarp();
    }
    bar_sync<kDone>(kAll);
}

// The gradient by itself: a CTA takes `span` entries (a multiple of 64) of a row, whose statistics are known.
template <class T>
__global__ void __launch_bounds__(256, 5) k_distill_grad(DistillArgs a, uint32_t span, uint32_t spans) {
    constexpr uint32_t V = Vec<T>::kN, THREADS = 256;
    __shared__ ListSmem sm;
    const int64_t r = blockIdx.x / spans;
    const uint32_t first = blockIdx.x % spans * span, n = min(span, static_cast<uint32_t>(a.vocab) - first);
    const T* x = static_cast<const T*>(a.logits) + r * a.ld + first;
    T* out = static_cast<T*>(a.grad_logits) + r * a.ld_grad + first;
    // the first vectors are on their way while the list is read
    const uint32_t mis = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(x) & 15u);
    const bool vec_out = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(x)) & 15u) == 0;
    const uint32_t head = min(n, mis ? (16u - mis) / static_cast<uint32_t>(sizeof(T)) : 0u), nvec = vec_out ? (n - head) / V : 0u;
    const uint4* src = reinterpret_cast<const uint4*>(x + head);
    Vec<T> v[kUnroll];
    auto load = [&](uint32_t i) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (i + u * THREADS < nvec) v[u].raw = ld_stream(src + i + u * THREADS);
    };
    load(threadIdx.x);
    const float* st = a.saved + kSaved * r;
    const float mo = st[0], others = st[1], m = st[2], list = st[3], about = st[4], inv = st[5];
    const bool none = inv == -1.f;
    const float c = a.scale * kLog2e, g = none ? 0.f : a.scale * a.grad_loss[r], G = g * others;
    static_assert(kList <= THREADS, "one entry per thread");
    const int e = threadIdx.x;
    uint32_t id = kNone;
    bool here = false;
    float xe = 0.f;
    if (e < a.k) {
        float lp;
        List::fetch(a, r, e, id, lp);
        here = id != kNone && id - first < n;
        if (here) xe = to_f32(x[id - first]);
        sm.logp[e] = lp;
    }
    if (e < (a.k + 3) / 4 * 4) sm.ids()[e] = id;
    __syncthreads();  // (the list's logits are read before the gradient may overwrite them)
    const F2 c2 = pair(c, c), G2 = pair(G, G), minus = pair(-mo, -mo);
    for (uint32_t i = threadIdx.x; i < nvec;) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (i + u * THREADS < nvec) {
                gradients(v[u], minus, c2, G2);
                if (none) v[u].raw = make_uint4(0, 0, 0, 0);  // (whatever the logits are)
                st_stream(out + head + (i + u * THREADS) * V, v[u].raw);
            }
        i += kUnroll * THREADS;
        load(i);
    }
    // the entries around the vectors; all of them where the two rows lie apart differently
    auto one = [&](uint32_t i) { out[i] = from_f32<T>(none ? 0.f : G * power(to_f32(x[i]), mo, c)); };
    if (vec_out && threadIdx.x < head) one(threadIdx.x);
    for (uint32_t i = (vec_out ? head + nvec * V : 0u) + threadIdx.x; i < n; i += THREADS) one(i);
    __syncthreads();  // the list's entries once more
    if (here) {
        if (xe <= masked_at<T>()) xe = -INFINITY;
        float q;
        if (first_of_token(sm, a.k, e, id, q, [&](int j) { return expf(sm.logp[j] - about); }))
            out[id - first] = from_f32<T>(none ? 0.f : g * (list * power(xe, m, c) - q * inv));
    }
}

// Loss and gradient in one.  A cluster of `split` CTAs holds a row in shared memory, each `per` entries of it (a multiple of 64), as the
// 16-byte pieces that hold them; those of its neighbours in the first and last piece, and with a rest the list's
// tokens, are masked there.  One warp more than the THREADS that go through the row brings it there and does what the list
// needs meanwhile.
template <class T, int THREADS, bool REST>
__global__ void __launch_bounds__(THREADS + 32, held_ctas(THREADS)) k_distill_held(DistillArgs a, uint32_t split, uint32_t per, uint32_t* err) {
    constexpr uint32_t V = Vec<T>::kN;
    constexpr int kAll = THREADS + 32;
    enum { kMasked = 1, kSums, kListed, kDone };  // barriers
    extern __shared__ uint4 held[];
    __shared__ ListSmem sm;
    __shared__ List list_out;
    __shared__ Sum sums[THREADS / 32], peer[kMaxSplit], sum_out;
    __shared__ alignas(8) uint64_t bar;
    const uint32_t rank = split > 1 ? cluster_ctarank() : 0u;
    if (split > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int64_t r = blockIdx.x / split;
    const uint32_t vocab = static_cast<uint32_t>(a.vocab), first = min(per * rank, vocab), n = min(per, vocab - first);
    const T* x = static_cast<const T*>(a.logits) + r * a.ld + first;
    const uint32_t lead = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(x) & 15u) / static_cast<uint32_t>(sizeof(T));
    const uint32_t end = lead + n, nvec = (end + V - 1) / V;
    T* out = static_cast<T*>(a.grad_logits) + r * a.ld_grad + first;
    if (threadIdx.x == THREADS) {
        mbar_init(&bar, 1);
        fence_mbar_init();
        mbar_arrive_expect_tx(&bar, nvec * 16u);
        if (!a.lost) bulk_load(held, x - lead, nvec * 16u, &bar);
    }
    __syncthreads();  // (nobody waits for a barrier that is not set up)
    const float c = a.scale * kLog2e;
    const float grad_loss = a.grad_loss[r];
    // whether the row is there; where it is not, what is summed is NaN, and so the row's results are
    auto wait_row = [&]() -> bool {
        const bool there = mbar_wait(&bar, 0u, a.lost ? kLostNs : kWaitTimeoutNs);
        if (!there) {
            atomicOr(err, kErrTimeout);
            drain_barriers(1, [&](int, uint64_t*& b, uint32_t& parity) { return b = &bar, parity = 0u, !a.lost; });
        }
        __syncwarp();  // (barriers are passed by whole warps)
        return there;
    };
    if (threadIdx.x >= THREADS) {
        const uint32_t lane = threadIdx.x & 31;
        warp_read<T>(a, r, sm);
        const bool there = __all_sync(0xffffffffu, wait_row());
        T* mine = reinterpret_cast<T*>(held);
        if (REST)
            for (int e = lane; e < a.k; e += 32)
                if (sm.ids()[e] != kNone && sm.ids()[e] - first < n) mine[sm.ids()[e] - first + lead] = from_f32<T>(-INFINITY);
        if (lane < lead) mine[lane] = from_f32<T>(-INFINITY);
        if (lane < nvec * V - end) mine[end + lane] = from_f32<T>(-INFINITY);
        __syncwarp();
        bar_arrive<kMasked>(kAll);
        List l = warp_sums<REST>(a, c, sm);
        if (!there) l.weight = NAN;
        if (lane == 0) list_out = l;
        __syncwarp();
        bar_arrive<kListed>(kAll);
        if (split > 1) {
            asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
            cluster_sync();
        }
        bar_sync<kDone>(kAll);
        // the row's loss, and the list's entries once more
        const Sum o = sum_out;
        const Row f = row_of<T>(a, l, o, c);
        if (rank == 0 && lane == 0) {
            a.loss[r] = f.loss;
            if (a.saved) save_row(a.saved + kSaved * r, o, f, l);
        }
        const float g = a.scale * grad_loss;
        for (int e = lane; e < a.k; e += 32)
            if (sm.ids()[e] != kNone && sm.q[e] != -1.f && sm.ids()[e] - first < n)
                out[sm.ids()[e] - first] = from_f32<T>(f.none ? 0.f : g * (f.list * power(sm.x[e], f.m, c) - sm.q[e] * l.inv));
        return;
    }
    const F2 c2 = pair(c, c);
    const bool there = wait_row();
    bar_sync<kMasked>(kAll);
    float m = -FLT_MAX;
    F2 s2 = pair(0.f, 0.f);
    auto batch = [&](uint32_t i, auto all) {
        constexpr bool ALL = decltype(all)::value;
        Vec<T> w[kUnroll];
        Largest<T> most, other;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (ALL || i + u * THREADS < nvec) w[u].raw = held[i + u * THREADS];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (ALL || i + u * THREADS < nvec) {
                other.set(w[u]);
                if (u == 0) most = other;
                else most.take(other);
            }
        raise_to(most.value(), m, s2, c);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (ALL || i + u * THREADS < nvec) add_powers(w[u], m, c2, s2);
    };
    uint32_t i = threadIdx.x;
    for (; i + (kUnroll - 1) * THREADS < nvec; i += kUnroll * THREADS) batch(i, std::true_type());
    if (i < nvec) batch(i, std::false_type());
    Sum o = {m, there ? both(s2) : NAN};
    __syncwarp();
    o.lanes<32>(c);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = o;
    __syncwarp();
    bar_sync<kSums>(THREADS);
    o = sums[threadIdx.x & (THREADS / 32 - 1)];
    o.lanes<THREADS / 32>(c);
    if (split > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // (every CTA of the cluster runs)
        if (threadIdx.x < split) {
            const uint32_t to = mapa_shared(smem_u32(peer + rank), threadIdx.x);
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(o.m) : "memory");
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4), "f"(o.s) : "memory");
        }
        __syncwarp();
        cluster_sync();
        o = peer[0];
        for (uint32_t q = 1; q < split; ++q) o.take(peer[q], c);
    }
    if (threadIdx.x == 0) sum_out = o;
    __syncwarp();
    bar_sync<kListed>(kAll);
    bool none;
    const float others = others_of<T>(a, list_out, o, c, none), G = none ? 0.f : a.scale * grad_loss * others;
    const bool vec_out = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(x)) & 15u) == 0;
    const F2 G2 = pair(G, G), minus = pair(-o.m, -o.m);
#pragma unroll 4
    for (uint32_t w = threadIdx.x; w < nvec; w += THREADS) {
        Vec<T> p;
        p.raw = held[w];
        gradients(p, minus, c2, G2);
        if (none) p.raw = make_uint4(0, 0, 0, 0);  // (whatever the logits are)
        if (vec_out && w * V >= lead && (w + 1) * V <= end) {
            st_stream(out + (w * V - lead), p.raw);
        } else {
            const T* e = reinterpret_cast<const T*>(&p.raw);
#pragma unroll
            for (uint32_t j = 0; j < V; ++j)
                if (w * V + j >= lead && w * V + j < end) out[w * V + j - lead] = e[j];
        }
    }
    __syncwarp();
    bar_sync<kDone>(kAll);
}

// `rows` rows of a, from row `from` on.
DistillArgs part(DistillArgs a, int64_t from, int64_t rows) {
    auto bytes = [](int dtype) { return dtype == ISOLOCO_F32 ? 4 : 2; };
    a.logits = static_cast<const char*>(a.logits) + from * a.ld * bytes(a.dtype);
    a.top_logp = static_cast<const char*>(a.top_logp) + from * a.ld_logp * bytes(a.logp_dtype);
    a.top_index = static_cast<const char*>(a.top_index) + from * a.ld_index * (a.index64 ? 8 : 4);
    if (a.loss) a.loss += from;
    if (a.saved) a.saved += from * kSaved;
    if (a.grad_logits) {
        a.grad_loss += from;
        a.grad_logits = static_cast<char*>(a.grad_logits) + from * a.ld_grad * bytes(a.dtype);
    }
    a.rows = rows;
    return a;
}

// A grid's first dimension: rows times a cluster's CTAs.
constexpr int64_t kMostRows = int64_t(1) << 27;

template <class T, int THREADS, bool REST, bool GRAD>
cudaError_t launch_rows(const DistillArgs& a, uint32_t split, cudaStream_t st) {
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.rows * split));
    cfg.blockDim = dim3(THREADS + 32);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = split > 1 ? 1 : 0;
    const uint32_t per = static_cast<uint32_t>(((a.vocab + split - 1) / split + 63) & ~int64_t(63));
    return cudaLaunchKernelEx(&cfg, k_distill<T, THREADS, REST, GRAD>, a, split, per);
}

template <class T, int THREADS>
cudaError_t launch_rows(const DistillArgs& a, uint32_t split, cudaStream_t st) {
    if (a.rest) return a.grad_logits ? launch_rows<T, THREADS, true, true>(a, split, st) : launch_rows<T, THREADS, true, false>(a, split, st);
    return a.grad_logits ? launch_rows<T, THREADS, false, true>(a, split, st) : launch_rows<T, THREADS, false, false>(a, split, st);
}

template <class T, int THREADS, bool REST>
cudaError_t launch_held(const DistillArgs& a, uint32_t split, uint32_t* err, cudaStream_t st) {
    static PerDevice ready;
    int dev = 0, set = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess)
        e = ready.get<cudaError_t>(dev, &set, [](int*) {
            return cudaFuncSetAttribute(k_distill_held<T, THREADS, REST>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                        static_cast<int>(kMostHeldBytes) + 16);
        });
    if (e != cudaSuccess) return e;
    const int64_t per = ((a.vocab + split - 1) / split + 63) & ~int64_t(63), bytes = per * static_cast<int64_t>(sizeof(T)) + 16;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.rows * split));
    cfg.blockDim = dim3(THREADS + 32);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = split > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, k_distill_held<T, THREADS, REST>, a, split, static_cast<uint32_t>(per), err);
}

template <class T>
cudaError_t run_held(const DistillArgs& a, int sms, cudaStream_t st) {
    uint32_t* err = nullptr;
    const cudaError_t e = error_word(&err);
    if (e != cudaSuccess) return e;
    uint32_t split = 1;
    while (split < kMaxSplit && (a.vocab * static_cast<int64_t>(sizeof(T)) > split * kHeldBytes ||
                                 (a.rows * split <= sms && a.vocab / (2 * split) >= 4096)))
        split *= 2;
    const int64_t share = a.vocab / split;
#define HELD(N) (a.rest ? launch_held<T, N, true>(a, split, err, st) : launch_held<T, N, false>(a, split, err, st))
    if (share <= kSmallHeld) return HELD(64);
    if (share * static_cast<int64_t>(sizeof(T)) > kWideHeld) return HELD(512);
    return share <= kMediumHeld ? HELD(128) : HELD(256);
#undef HELD
}

template <class T>
cudaError_t run(const DistillArgs& a, cudaStream_t st) {
    int sms = 0;
    const cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
    const int64_t least = (a.vocab / kMaxSplit + 64) * static_cast<int64_t>(sizeof(T));
    if (a.grad_logits && (sizeof(T) == 4 || a.vocab <= kHeldMost) && least <= kMostHeldBytes) return run_held<T>(a, sms, st);
    // CTAs per row: more than one where rows leave SMs idle (of at least 4096 entries each), where the rows that are under way
    // at once would not stay in L2 for the gradient, and where marks would meet
    uint32_t split = 1;
    while (split < kMaxSplit && ((a.rows * split <= sms && a.vocab / (2 * split) >= 4096) ||
                                 (a.grad_logits && a.vocab * static_cast<int64_t>(sizeof(T)) > split * kShareBytes) ||
                                 (a.rest && a.vocab > split * int64_t(marks_of(256)))))
        split *= 2;
    const int64_t share = a.vocab / split;
    if (share <= kSmall) return launch_rows<T, 64>(a, split, st);
    return share <= kMedium ? launch_rows<T, 128>(a, split, st) : launch_rows<T, 256>(a, split, st);
}

template <class T>
cudaError_t run_grad(const DistillArgs& a, cudaStream_t st) {
    const uint32_t span = kSpan * 256 * Vec<T>::kN, spans = static_cast<uint32_t>((a.vocab + span - 1) / span);
    const int64_t most = std::max<int64_t>(1, (int64_t(1) << 30) / spans);  // rows of a grid
    for (int64_t from = 0; from < a.rows; from += most) {
        const int64_t rows = std::min(most, a.rows - from);
        k_distill_grad<T><<<static_cast<unsigned>(rows * spans), 256, 0, st>>>(part(a, from, rows), span, spans);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <class F>
cudaError_t by_parts(const DistillArgs& a, F f) {
    for (int64_t from = 0; from < a.rows; from += kMostRows) {
        const cudaError_t e = f(part(a, from, std::min(kMostRows, a.rows - from)));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, cudaStream_t st) {
    return by_parts(a, [&](const DistillArgs& p) {
        return p.dtype == ISOLOCO_F32 ? run<float>(p, st) : p.dtype == ISOLOCO_BF16 ? run<__nv_bfloat16>(p, st) : run<__half>(p, st);
    });
}

cudaError_t launch_distill_grad(const DistillArgs& a, cudaStream_t st) {
    return by_parts(a, [&](const DistillArgs& p) {
        return p.dtype == ISOLOCO_F32 ? run_grad<float>(p, st) : p.dtype == ISOLOCO_BF16 ? run_grad<__nv_bfloat16>(p, st) : run_grad<__half>(p, st);
    });
}

}  // namespace isoloco

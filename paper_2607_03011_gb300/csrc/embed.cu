// embed.cu -- embedding lookup and its gradient.
//
//     y[t] = scale W[id_t]            dW[v] = scale sum_{t : id_t = v} dy[t]
//
// The gradient sorts the positions by token id (stable least-significant-digit radix sort in one
// thread-block cluster), so that a row's terms stand together, in the order of their positions:
//   k_embed_sort   cluster 0 sorts; the other CTAs meanwhile write the zeros of every row of dW.
//   k_embed_sum    a CTA adds a span of consecutive sorted positions in fp32.  A row whose positions lie in one
//                  span, or in two neighbouring ones, is added by the CTA it begins in and written at
//                  once; what each span adds to a row that lies in three or more goes to the workspace.
//   k_embed_join   adds those shares in the order of their spans and writes their rows.
// Which terms are added in which order depends on the ids alone.
//
// Measured: the lookup of 65533 x 2048 fp32 rows 118 us (537 MB written, 165 MB of table rows read); its gradient
// over 128000 rows 166 to 175 us for the zeros (6.2 TB/s; the sort's 31 us pass behind them), 98 us for the sums
// (537 MB read) and 14 us to join.  8192 x 1024 bf16 over 32000 rows: 6.7 us, and 13.5 (the sort's own
// 12.7 us, mostly its cluster barriers and trips to L2), 9.6 and 6.3 us.  One cluster sorts however many positions there
// are: up to 65536 the keys stay in registers over a pass, beyond that each pass reads them twice.  The whole
// gradient of T x 64 bf16 rows over 32000: 28 us for 8192, 48 for 65536, 120 for 262144, 386 for 2^20, 1437 for 2^22.
#include <algorithm>

#include "common.cuh"
#include "inner.cuh"
#include "inner.h"

namespace isoloco {

namespace {

constexpr int kRowThreads = 128;

// ------------------------------------------------------------------ lookup
// Pieces (16 bytes when VEC, else put_piece's) of all rows of y in one sequence; a thread takes N of them,
// kLookThreads apart, so that N rows' ids and then N pieces of the table are in flight.
constexpr int kLookThreads = 256;

template <class T, class I, bool VEC, int N>
__global__ void __launch_bounds__(kLookThreads) k_embed(const T* __restrict__ w, int64_t ld_w, int64_t vocab, int64_t width, uint32_t pieces,
                                                        const I* __restrict__ ids, int64_t tokens, float scale, T* __restrict__ y,
                                                        int64_t ld_y) {
    constexpr int V = Vec<T>::kN;
    const int64_t total = tokens * pieces;
    for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * (kLookThreads * N) + threadIdx.x; i0 < total;
         i0 += static_cast<int64_t>(gridDim.x) * (kLookThreads * N)) {
        int64_t t[N], id[N];
        uint32_t c[N];
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int64_t i = min(i0 + q * kLookThreads, total - 1);
            t[q] = total <= 0xffffffffll ? static_cast<int64_t>(static_cast<uint32_t>(i) / pieces) : i / pieces;
            c[q] = static_cast<uint32_t>(i - t[q] * pieces);
            id[q] = token_at(ids, t[q], vocab);
        }
        if constexpr (VEC) {
            Vec<T> v[N];
#pragma unroll
            for (int q = 0; q < N; ++q) {
                v[q].raw = make_uint4(0, 0, 0, 0);
                if (id[q] >= 0) v[q].raw = __ldg(reinterpret_cast<const uint4*>(w + id[q] * ld_w + static_cast<int64_t>(c[q]) * V));
            }
#pragma unroll
            for (int q = 0; q < N; ++q) {
                if (i0 + q * kLookThreads >= total) break;
                if (scale != 1.f && id[q] >= 0) {
                    float f[V];
                    v[q].unpack(f);
#pragma unroll
                    for (int j = 0; j < V; ++j) f[j] *= scale;
                    v[q].pack(f);
                }
                st_stream(y + t[q] * ld_y + static_cast<int64_t>(c[q]) * V, v[q].raw);
            }
        } else {
#pragma unroll
            for (int q = 0; q < N; ++q) {
                if (i0 + q * kLookThreads >= total) break;
                put_piece(id[q] >= 0 ? w + id[q] * ld_w : nullptr, y + t[q] * ld_y, width, c[q], scale);
            }
        }
    }
}

// ------------------------------------------------------------------ sort
constexpr int kSortCluster = 8;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kDigits = 256;

// The warp's lanes with the same 8-bit digit (match.any in its place: 46.7 us for the gradient of 65533 narrow rows,
// so 44.5).
__device__ __forceinline__ uint32_t same_digit(uint32_t d) {
    uint32_t same = 0xffffffffu;
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const uint32_t v = __ballot_sync(0xffffffffu, (d >> b) & 1u);
        same &= (d >> b) & 1u ? v : ~v;
    }
    return same;
}

constexpr int kSortItems = 8;                     // keys of a lane in registers at once
constexpr int kSortBatch = 32 * kSortItems;
constexpr int kQuadWarps = kSortWarps / 4;

struct SortSmem {
    uint32_t warp[kSortWarps][kDigits + 1];  // counts, then the next place of each warp's digit (rows apart by a bank)
    uint32_t total[kSortCluster][kDigits];   // every CTA's count of every digit
    uint32_t before[kDigits];                // places before this CTA's first of each digit
    uint32_t ends[kDigits / 32];
};
static_assert(kSortThreads == 4 * kDigits, "four threads per digit");

// Sorts (id, position) into kp[1].  A pass over a digit: every warp counts the digits of its keys (a
// contiguous run of them), the CTA and then the cluster add the counts up to the places where each warp's keys of
// each digit begin, and every warp places its keys 32 at a time, in order.  Up to kSortBatch keys per warp (65536
// in all) stay in registers over a pass.
template <class I>
__device__ __forceinline__ void sort_ids(SortSmem& sm, const I* ids, int64_t n, int64_t vocab, int bits, uint2* const (&kp)[2]) {
    const uint32_t rank = cluster_ctarank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t per = (n + kSortCluster * kSortWarps - 1) / (kSortCluster * kSortWarps);
    const int64_t begin = min(n, per * (static_cast<int64_t>(rank) * kSortWarps + warp)), end = min(n, begin + per);
    const int passes = (bits + 7) / 8, dbits = (bits + passes - 1) / passes;
    const uint32_t dmask = (1u << dbits) - 1u;
    const int d = threadIdx.x >> 2, q = threadIdx.x & 3;  // digit, and which quarter of the warps
    const bool once = per <= kSortBatch;
    cluster_sync();  // every CTA runs before another writes its shared memory
    for (int pass = 0; pass < passes; ++pass) {
        uint2* dst = kp[(passes - pass) & 1];  // kp[1] in the last pass
        const uint2* src = kp[(passes - pass + 1) & 1];
        const int shift = pass * dbits;
        uint2 k[kSortItems];
        auto load = [&](int64_t i0) {
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                const int64_t i = i0 + j * 32 + lane;
                if (i >= end) continue;
                if (pass) {
                    k[j] = src[i];
                } else {
                    const int64_t v = token_at(ids, i, vocab);
                    k[j] = make_uint2(static_cast<uint32_t>(v < 0 ? vocab : v), static_cast<uint32_t>(i));  // no token: behind all others
                }
            }
        };
        for (int i = lane; i < kDigits; i += 32) sm.warp[warp][i] = 0;
        __syncwarp();
        for (int64_t i0 = begin; i0 < end; i0 += kSortBatch) {
            load(i0);
#pragma unroll
            for (int j = 0; j < kSortItems; ++j)
                if (i0 + j * 32 + lane < end) atomicAdd(&sm.warp[warp][(k[j].x >> shift) & dmask], 1u);
        }
        __syncthreads();
        uint32_t c[kQuadWarps], mine = 0;
#pragma unroll
        for (int i = 0; i < kQuadWarps; ++i) {
            c[i] = sm.warp[q * kQuadWarps + i][d];
            mine += c[i];
        }
        uint32_t upto = mine;
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, upto, o, 4);
            if (q >= o) upto += u;
        }
        // this CTA's total of the digit, to every CTA of the cluster
        const uint32_t total = __shfl_sync(0xffffffffu, upto, 3, 4);
#pragma unroll
        for (uint32_t r = 0; r < kSortCluster / 4; ++r)
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa_shared(smem_u32(&sm.total[rank][d]), q * (kSortCluster / 4) + r)),
                         "r"(total)
                         : "memory");
        cluster_sync();
        // places before this CTA's first of each digit: smaller digits anywhere, and the same digit in earlier CTAs
        uint32_t all = 0, before = 0, scan = 0;
        if (threadIdx.x < kDigits) {
#pragma unroll
            for (uint32_t r = 0; r < kSortCluster; ++r) {
                const uint32_t v = sm.total[r][threadIdx.x];
                before += r < rank ? v : 0u;
                all += v;
            }
            scan = all;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, scan, o);
                if (lane >= o) scan += u;
            }
            if (lane == 31) sm.ends[warp] = scan;
        }
        __syncthreads();
        if (threadIdx.x < kDigits) {
            uint32_t base = scan - all + before;
#pragma unroll
            for (int w = 0; w < kDigits / 32; ++w) base += w < warp ? sm.ends[w] : 0u;
            sm.before[threadIdx.x] = base;
        }
        __syncthreads();
        uint32_t place = sm.before[d] + upto - mine;
#pragma unroll
        for (int i = 0; i < kQuadWarps; ++i) {
            sm.warp[q * kQuadWarps + i][d] = place;
            place += c[i];
        }
        __syncthreads();
        for (int64_t i0 = begin; i0 < end; i0 += kSortBatch) {
            if (!once) load(i0);
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                if (i0 + j * 32 >= end) break;  // (the whole warp)
                const bool have = i0 + j * 32 + lane < end;
                const uint32_t dg = (k[j].x >> shift) & dmask;
                const uint32_t same = same_digit(dg) & __ballot_sync(0xffffffffu, have);
                const uint32_t lower = __popc(same & ((1u << lane) - 1u));
                uint32_t at = 0;
                if (have) at = sm.warp[warp][dg] + lower;
                __syncwarp();
                if (have && lower == 0) sm.warp[warp][dg] = at + __popc(same);
                __syncwarp();
                if (have) dst[at] = k[j];
            }
        }
        __threadfence();
        cluster_sync();  // the pass's output is complete, and the totals may be overwritten
    }
}

// Cluster 0 sorts (id, position) into kp1; the others fill dw with zeros.
template <class I>
__global__ void __cluster_dims__(kSortCluster, 1, 1) __launch_bounds__(kSortThreads)
    k_embed_sort(const I* ids, int64_t n, int64_t vocab, int bits, uint2* kp0, uint2* kp1,
                 uint32_t* nchains, uint8_t* dw, int64_t row_bytes, int64_t ld_bytes) {
    __shared__ SortSmem sm;
    next_may_start();
    const int64_t cta = static_cast<int64_t>(blockIdx.x) - kSortCluster;
    if (cta < 0) {
        if (blockIdx.x == 0 && threadIdx.x == 0) *nchains = 0;
        uint2* const kp[2] = {kp0, kp1};
        sort_ids(sm, ids, n, vocab, bits, kp);
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
constexpr int kMaxSpan = 32;  // sorted positions of one CTA, at most (its last row's may be as many more)
constexpr int kBatch = 8;     // rows of dy in flight per thread

// chains: the spans in which a row begins that lies in three spans or more (in any order); part[span][1] is its
// sum there, part[s][0] its sum in each of the later spans s.
template <class T, class O, bool VEC>
__global__ void __launch_bounds__(kRowThreads) k_embed_sum(const T* __restrict__ dy, int64_t ld_dy, int64_t vocab, int64_t width,
                                                           const uint2* __restrict__ kp, int64_t n, int len, float scale, O* __restrict__ dw, int64_t ld_dw,
                                                           float* __restrict__ part, uint32_t* nchains,
                                                           uint32_t* __restrict__ chains) {
    constexpr int V = VEC ? Vec<T>::kN : 1;
    __shared__ uint32_t sk[2 * kMaxSpan + 2];  // keys from one before the span to one behind the next
    __shared__ uint32_t sp[2 * kMaxSpan];
    after_previous();
    const int64_t span = blockIdx.x, first = span * len;
    auto key_at = [&](int64_t j) { return j >= 0 && j < n ? kp[j].x : 0xffffffffu; };
    for (int i = threadIdx.x; i < 2 * len + 2; i += kRowThreads) sk[i] = key_at(first + i - 1);
    for (int i = threadIdx.x; i < 2 * len; i += kRowThreads) sp[i] = first + i < n ? kp[first + i].y : 0u;
    const uint32_t before = key_at(first - len - 1);
    __syncthreads();
    const int64_t c = (static_cast<int64_t>(blockIdx.y) * kRowThreads + threadIdx.x) * V;
    if (c >= width) return;
    // positions [from, to) are added here: without the end of a row that the span before adds as a whole, with
    // the rest of a row that begins here and ends in the next span
    const int cnt = static_cast<int>(min(static_cast<int64_t>(len), n - first));
    int from = 0, to = cnt;
    bool shared = sk[0] == sk[1];  // the first row began in an earlier span, and its share here is one of many
    if (shared && before != sk[1] && sk[len + 1] != sk[1]) {
        shared = false;
        while (from < cnt && sk[from + 1] == sk[1]) ++from;
    }
    const uint32_t end_key = sk[cnt];
    if (sk[cnt + 1] == end_key && sk[0] != end_key && sk[2 * len + 1] != end_key)
        while (sk[to + 1] == end_key) ++to;  // (ends by sk[2 len + 1])
    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    for (int i0 = from; i0 < to; i0 += kBatch) {
        Vec<T> v[kBatch];
        T one[kBatch];
#pragma unroll
        for (int q = 0; q < kBatch; ++q) {
            if (i0 + q >= to || sk[i0 + q + 1] >= vocab) continue;  // (no token sorts last)
            const T* src = dy + static_cast<int64_t>(sp[i0 + q]) * ld_dy + c;
            if constexpr (VEC) v[q].raw = ld_stream(src);
            else one[q] = src[0];
        }
#pragma unroll
        for (int q = 0; q < kBatch; ++q) {
            const int i = i0 + q;
            if (i >= to) break;
            const uint32_t k = sk[i + 1];
            if (k >= vocab) break;
            if constexpr (VEC) {
                float f[V];
                v[q].unpack(f);
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] += f[j];
            } else {
                acc[0] += to_f32(one[q]);
            }
            const bool last = i + 1 == to, goes_on = sk[i + 2] == k;
            if (!last && goes_on) continue;
            if (shared || goes_on) {
                if (!shared && blockIdx.y == 0 && threadIdx.x == 0) chains[atomicAdd(nchains, 1u)] = static_cast<uint32_t>(span);
                float* d = part + (span * 2 + (shared ? 0 : 1)) * width + c;
#pragma unroll
                for (int j = 0; j < V; ++j) d[j] = acc[j];
            } else {
                O* d = dw + static_cast<int64_t>(k) * ld_dw + c;
                bool whole = false;  // 16 bytes at once where the output's type and address allow
                if constexpr (VEC && sizeof(O) == sizeof(T)) {
                    whole = (reinterpret_cast<uintptr_t>(d) & 15u) == 0;
                    if (whole) {
                        float f[V];
#pragma unroll
                        for (int j = 0; j < V; ++j) f[j] = acc[j] * scale;
                        Vec<O> w;
                        w.pack(f);
                        *reinterpret_cast<uint4*>(d) = w.raw;
                    }
                }
                if (!whole) {
#pragma unroll
                    for (int j = 0; j < V; ++j) d[j] = from_f32<O>(acc[j] * scale);
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = 0.f;
            shared = false;
        }
    }
}

// Rows that lie in many spans (a frequent token's in hundreds): kJoinCols columns of one of them per CTA step,
// its spans in kJoinParts runs, each added by a group of threads.
constexpr int kJoinCols = 128, kJoinParts = 4, kJoinThreads = kJoinCols * kJoinParts;

template <class O>
__global__ void __launch_bounds__(kJoinThreads) k_embed_join(int64_t width, const uint2* __restrict__ kp, int64_t n, int len,
                                                             float scale, O* __restrict__ dw, int64_t ld_dw,
                                                             const float* __restrict__ part, const uint32_t* nchains,
                                                             const uint32_t* __restrict__ chains) {
    __shared__ float sum[kJoinParts][kJoinCols];
    after_previous();
    const uint32_t blocks = static_cast<uint32_t>((width + kJoinCols - 1) / kJoinCols);
    const int64_t items = static_cast<int64_t>(*nchains) * blocks;
    const int run = threadIdx.x / kJoinCols, col = threadIdx.x % kJoinCols;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t span = chains[item / blocks], c = item % blocks * kJoinCols + col;
        const uint32_t k = kp[(span + 1) * len].x;
        // later spans that begin with this row's key
        int64_t more = 0;
        for (;;) {
            const int64_t at = (span + 1 + more + threadIdx.x) * len;
            const int got = __syncthreads_count(at < n && kp[at].x == k);
            more += got;
            if (got < kJoinThreads) break;
        }
        const int64_t each = (more + kJoinParts - 1) / kJoinParts;
        const int64_t lo = span + 1 + min(more, run * each), hi = span + 1 + min(more, (run + 1) * each);
        float acc = 0.f;
        if (c < width) {
            if (run == 0) acc = part[(span * 2 + 1) * width + c];
#pragma unroll 8
            for (int64_t s = lo; s < hi; ++s) acc += part[s * 2 * width + c];
        }
        sum[run][col] = acc;
        __syncthreads();
        if (run == 0 && c < width) {
#pragma unroll
            for (int q = 1; q < kJoinParts; ++q) acc += sum[q][col];
            dw[static_cast<int64_t>(k) * ld_dw + c] = from_f32<O>(acc * scale);
        }
        __syncthreads();
    }
}

template <class T, class I, bool VEC, int N>
cudaError_t embed_n(const void* w, int64_t ld_w, int64_t vocab, int64_t width, int64_t pieces, const void* ids, int64_t tokens, float scale, void* y,
                    int64_t ld_y, cudaStream_t st) {
    const int64_t blocks = (tokens * pieces + kLookThreads * N - 1) / (kLookThreads * N);
    k_embed<T, I, VEC, N><<<static_cast<unsigned>(std::min<int64_t>(blocks, int64_t(1) << 30)), kLookThreads, 0, st>>>(
        static_cast<const T*>(w), ld_w, vocab, width, static_cast<uint32_t>(pieces), static_cast<const I*>(ids), tokens, scale, static_cast<T*>(y),
        ld_y);
    return cudaGetLastError();
}

template <class T, class I>
cudaError_t embed_t(const void* w, int64_t ld_w, int64_t vocab, int64_t width, const void* ids, int64_t tokens, float scale,
                    void* y, int64_t ld_y, cudaStream_t st) {
    constexpr int64_t V = Vec<T>::kN;
    int sms = 0;
    const cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
    const bool vec = aligned16(w) && aligned16(y) && ld_w % V == 0 && ld_y % V == 0 && width % V == 0;
    const int64_t pieces = vec ? width / V : any_pieces(width, V);
    // four pieces per thread once that still leaves every SM a few CTAs
    const bool many = tokens * pieces >= int64_t(4) * 4 * kLookThreads * sms;
#define LOOK(VEC, N) embed_n<T, I, VEC, N>(w, ld_w, vocab, width, pieces, ids, tokens, scale, y, ld_y, st)
    return vec ? (many ? LOOK(true, 4) : LOOK(true, 1)) : (many ? LOOK(false, 4) : LOOK(false, 1));
#undef LOOK
}

// Positions per CTA of k_embed_sum: a short batch is cut finer, so that every SM has a few CTAs; a long one
// leaves less at the spans' ends.
int span_of(int64_t tokens) { return tokens <= 16384 ? 16 : kMaxSpan; }

struct EmbedWs {
    uint2 *kp0, *kp1;
    uint32_t *nchains, *chains;
    float* part;
};

int64_t r16(int64_t b) { return (b + 15) / 16 * 16; }

EmbedWs embed_ws(void* ws, int64_t tokens) {
    uint8_t* p = static_cast<uint8_t*>(ws);
    const int64_t s = r16(8 * tokens), spans = (tokens + span_of(tokens) - 1) / span_of(tokens);
    return {reinterpret_cast<uint2*>(p), reinterpret_cast<uint2*>(p + s), reinterpret_cast<uint32_t*>(p + 2 * s),
            reinterpret_cast<uint32_t*>(p + 2 * s + 16), reinterpret_cast<float*>(p + 2 * s + 16 + r16(4 * spans))};
}

template <class T, class O>
cudaError_t embed_grad_t(const void* dy, int64_t ld_dy, int64_t vocab, int64_t width, const EmbedWs& w, int64_t n, float scale,
                         void* dw, int64_t ld_dw, int sms, cudaStream_t st) {
    constexpr int64_t V = Vec<T>::kN;
    const bool vec = aligned16(dy) && ld_dy % V == 0 && width % V == 0;
    const int64_t cols = vec ? width / V : width;  // (16 bytes put together from two pieces: 149 us where single columns take 122)
    const int len = span_of(n);
    const unsigned spans = static_cast<unsigned>((n + len - 1) / len);
    const dim3 grid(spans, static_cast<unsigned>((cols + kRowThreads - 1) / kRowThreads));
    cudaError_t e;
    if (vec)
        e = launch_next(k_embed_sum<T, O, true>, grid, kRowThreads, st, static_cast<const T*>(dy), ld_dy, vocab, width,
                        static_cast<const uint2*>(w.kp1), n, len, scale, static_cast<O*>(dw), ld_dw, w.part, w.nchains, w.chains);
    else
        e = launch_next(k_embed_sum<T, O, false>, grid, kRowThreads, st, static_cast<const T*>(dy), ld_dy, vocab, width,
                        static_cast<const uint2*>(w.kp1), n, len, scale, static_cast<O*>(dw), ld_dw, w.part, w.nchains, w.chains);
    if (e != cudaSuccess) return e;
    if (spans < 3) return cudaSuccess;  // no row lies in three
    return launch_next(k_embed_join<O>, 4 * sms, kJoinThreads, st, width, static_cast<const uint2*>(w.kp1), n, len,
                       scale, static_cast<O*>(dw), ld_dw, static_cast<const float*>(w.part), static_cast<const uint32_t*>(w.nchains),
                       static_cast<const uint32_t*>(w.chains));
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
    const int64_t spans = (tokens + span_of(tokens) - 1) / span_of(tokens);
    return 2 * r16(8 * tokens) + 16 + r16(4 * spans) + spans * 2 * width * 4;
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
        k_embed_sort<int64_t><<<grid, kSortThreads, 0, st>>>(static_cast<const int64_t*>(ids), tokens, vocab, bits, w.kp0, w.kp1,
                                                             w.nchains, static_cast<uint8_t*>(dw), width * es, ld_dw * es);
    else
        k_embed_sort<int32_t><<<grid, kSortThreads, 0, st>>>(static_cast<const int32_t*>(ids), tokens, vocab, bits, w.kp0, w.kp1,
                                                             w.nchains, static_cast<uint8_t*>(dw), width * es, ld_dw * es);
    if ((e = cudaGetLastError()) != cudaSuccess || tokens == 0) return e;
#define GRAD(T, O) return embed_grad_t<T, O>(dy, ld_dy, vocab, width, w, tokens, scale, dw, ld_dw, sms, st)
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

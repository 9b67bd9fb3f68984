// inner_api.cu -- C entry points of the inner step's operators: argument checks, then the launchers.
#include <algorithm>
#include <atomic>
#include <climits>
#include <string>
#include <vector>

#include "common.cuh"
#include "inner.h"
#include "per_device.h"

namespace isoloco {

cudaError_t device_sms(int* sms) {
    static PerDevice known;
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    return known.get<cudaError_t>(dev, sms, [&](int* n) { return cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev); });
}

static __device__ uint32_t g_error_word;

static __global__ void k_raise(uint32_t* word, uint32_t bits) { atomicOr(word, bits); }
static __global__ void k_clear(uint32_t* word, uint32_t bits) { atomicAnd(word, ~bits); }

cudaError_t error_word(uint32_t** word) {
    return cudaGetSymbolAddress(reinterpret_cast<void**>(word), g_error_word);
}

}  // namespace isoloco

using namespace isoloco;

namespace {

std::atomic<int> g_lose_rows{0};  // calls still to be made without their rows' copies (isoloco_debug_lose_rows)

constexpr int64_t kMaxSize = INT_MAX;
// No exception passes an entry point: what may be thrown here is for want of memory (a message's text).
constexpr int kNoMemory = ISOLOCO_ERR_OOM;

int invalid(const char* what) { return set_error(ISOLOCO_ERR_INVALID, what); }

int cuda_status(cudaError_t e) { return e == cudaSuccess ? ISOLOCO_OK : set_error(ISOLOCO_ERR_CUDA, cudaGetErrorString(e)); }

int elem_size(int dtype) { return dtype == ISOLOCO_F32 ? 4 : 2; }
bool any_dtype(int d) { return d == ISOLOCO_F32 || d == ISOLOCO_BF16 || d == ISOLOCO_F16; }
bool half_dtype(int d) { return d == ISOLOCO_BF16 || d == ISOLOCO_F16; }
bool size_ok(int64_t n, int64_t least) { return n >= least && n <= kMaxSize; }
// a matrix of `rows` rows (none may be NULL unless empty) whose elements are `bytes` long
bool matrix_ok(const void* p, int64_t rows, int64_t cols, int64_t ld, int bytes) {
    if (rows == 0) return true;
    return p && reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld >= cols && ld <= (int64_t(1) << 40);
}
// (NULL is)
bool aligned_to(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
bool array_ok(const void* p, int64_t n, int bytes) { return n == 0 || (p && aligned_to(p, bytes)); }

int workspace_ok(const void* ws, int64_t have, int64_t need) {
    if (need == 0) return ISOLOCO_OK;
    if (!ws || have < need) return set_error(ISOLOCO_ERR_INVALID, ("workspace of " + std::to_string(need) + " bytes needed").c_str());
    if (reinterpret_cast<uintptr_t>(ws) & 15u) return set_error(ISOLOCO_ERR_ALIGN, "workspace is not 16-byte aligned");
    return ISOLOCO_OK;
}

// rows of 16-bit elements that all start at multiples of 16 bytes
bool rows16(const void* p, int64_t ld, int64_t rows) { return rows == 0 || ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % 8 == 0); }

cudaStream_t stream_of(void* s) { return static_cast<cudaStream_t>(s); }

const char* embed_sizes_problem(int64_t vocab, int64_t width, int64_t tokens) {
    return size_ok(vocab, 1) && size_ok(width, 1) && width <= (1 << 20) && size_ok(tokens, 0)
               ? nullptr : "vocab must be in 1 .. 2^31 - 1, width in 1 .. 2^20, tokens in 0 .. 2^31 - 1";
}

const char* embed_problem(int dtype, int64_t vocab, int64_t width, const void* ids, int id_bytes, int64_t tokens) {
    if (!any_dtype(dtype)) return "bad element type";
    if (const char* p = embed_sizes_problem(vocab, width, tokens)) return p;
    if (id_bytes != 4 && id_bytes != 8) return "id_bytes must be 4 or 8";
    if (!array_ok(ids, tokens, id_bytes)) return "ids is NULL or misaligned";
    return nullptr;
}

const char* ffn_sizes_problem(int64_t tokens, int64_t width, int64_t ff) {
    return tokens >= 0 && tokens <= (1 << 30) && width >= 1 && ff >= 1 && width <= (1 << 20) && ff <= (1 << 20)
               ? nullptr : "tokens must be in 0 .. 2^30, width and ff in 1 .. 2^20";
}

const char* ffn_problem(const FfnArgs& a) {
    if (!half_dtype(a.dtype)) return "the gated block takes BF16 or F16";
    if (a.act != ISOLOCO_SILU && a.act != ISOLOCO_GELU_TANH) return "bad activation";
    if (const char* p = ffn_sizes_problem(a.tokens, a.width, a.ff)) return p;
    if (!matrix_ok(a.x, a.tokens, a.width, a.ld_x, 2)) return "x is NULL, misaligned or its pitch too small";
    if (!matrix_ok(a.wg, a.width, a.ff, a.ld_w, 2) || !matrix_ok(a.wu, a.width, a.ff, a.ld_w, 2))
        return "w_gate or w_up is NULL, misaligned or its pitch too small";
    return nullptr;
}

const char* logprob_problem(const LogprobArgs& a, int target_bytes) {
    if (!any_dtype(a.dtype)) return "bad element type";
    if (!size_ok(a.rows, 0) || !size_ok(a.vocab, 1)) return "rows must be in 0 .. 2^31 - 1, vocab in 1 .. 2^31 - 1";
    const int es = elem_size(a.dtype);
    if (!matrix_ok(a.logits, a.rows, a.vocab, a.ld, es)) return "logits is NULL, misaligned or its pitch too small";
    if (target_bytes != 4 && target_bytes != 8) return "target_bytes must be 4 or 8";
    if (!array_ok(a.targets, a.rows, target_bytes)) return "targets is NULL or misaligned";
    if (!(a.scale > 0.f) || a.scale > 1e30f) return "scale must be positive and finite";
    if (a.grad_logits && !matrix_ok(a.grad_logits, a.rows, a.vocab, a.ld_grad, es)) return "grad_logits is misaligned or its pitch too small";
    if (!aligned_to(a.logp, 4) || !aligned_to(a.entropy, 4) || !aligned_to(a.lse, 4)) return "logp, entropy or lse is misaligned";
    if (!aligned_to(a.grad_logp, 4) || !aligned_to(a.grad_entropy, 4)) return "grad_logp or grad_entropy is misaligned";
    return nullptr;
}

// n of a tensor: chunk numbers of a table of tensors fit 32 bits
constexpr int64_t kMaxTensorElems = int64_t(1) << 33;

const char* tensors_problem(const isoloco_tensor_t* t, int count) {
    if (count < 0 || (count > 0 && !t)) return "bad tensor list";
    for (int i = 0; i < count; ++i) {
        if (!any_dtype(t[i].dtype)) return "bad element type in the tensor list";
        if (t[i].n < 0 || t[i].n > kMaxTensorElems) return "a tensor's length must be in 0 .. 2^33";
        if (!array_ok(t[i].data, t[i].n, elem_size(t[i].dtype))) return "a tensor's data is NULL or misaligned";
    }
    return nullptr;
}

const char* distill_problem(const DistillArgs& a, int index_bytes, int tail) {
    if (!any_dtype(a.dtype) || !any_dtype(a.logp_dtype)) return "bad element type";
    if (!size_ok(a.rows, 0) || !size_ok(a.vocab, 1)) return "rows must be in 0 .. 2^31 - 1, vocab in 1 .. 2^31 - 1";
    if (a.k < 1 || a.k > ISOLOCO_MAX_LIST) return "k must be in 1 .. 256";
    if (!matrix_ok(a.logits, a.rows, a.vocab, a.ld, elem_size(a.dtype))) return "logits is NULL, misaligned or its pitch too small";
    if (!matrix_ok(a.top_logp, a.rows, a.k, a.ld_logp, elem_size(a.logp_dtype))) return "top_logp is NULL, misaligned or its pitch too small";
    if (index_bytes != 4 && index_bytes != 8) return "index_bytes must be 4 or 8";
    if (!matrix_ok(a.top_index, a.rows, a.k, a.ld_index, index_bytes)) return "top_index is NULL, misaligned or its pitch too small";
    if (!(a.scale > 0.f) || a.scale > 1e30f) return "scale must be positive and finite";
    if (tail != ISOLOCO_TAIL_DROP && tail != ISOLOCO_TAIL_REST) return "bad tail";
    if (a.grad_logits) {
        if (!matrix_ok(a.grad_logits, a.rows, a.vocab, a.ld_grad, elem_size(a.dtype))) return "grad_logits is misaligned or its pitch too small";
        if (!array_ok(a.grad_loss, a.rows, 4)) return "grad_loss is NULL or misaligned";
        if (a.grad_logits == a.logits && a.rows > 1 && a.ld_grad != a.ld) return "a gradient over the logits needs their pitch";
    }
    if (!aligned_to(a.saved, 4)) return "saved is misaligned";
    return nullptr;
}

// Whether outputs of a selection share memory with one another or with scores or finished; where as many continuations are kept as there are
// beams, a batch entry writes the same places of scores and finished that it alone has read.
bool selection_shares(const BeamArgs& a) {
    struct Range {
        const void* p;
        int64_t bytes;
        bool meets(const Range& o) const {
            const uint64_t at = reinterpret_cast<uint64_t>(p), other = reinterpret_cast<uint64_t>(o.p);
            return p && o.p && at < other + static_cast<uint64_t>(o.bytes) && other < at + static_cast<uint64_t>(bytes);
        }
    };
    const int64_t read = a.batch * a.beams, made = a.batch * a.keep;
    const Range in[2] = {{a.scores, read * 4}, {a.finished, read}};
    const Range out[4] = {{a.out_scores, made * 4}, {a.out_finished, made}, {a.out_beams, made * 8}, {a.out_tokens, made * 8}};
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < 2; ++j)
            if (out[i].meets(in[j]) && !(i == j && out[i].p == in[j].p && a.keep == a.beams)) return true;
        for (int j = 0; j < i; ++j)
            if (out[i].meets(out[j])) return true;
    }
    return false;
}

// ---- states that are reordered: what they may share

// The addresses of one side of a state.
struct Places {
    uint64_t at;
    uint64_t batch, beam, outer;  // strides
    uint64_t pieces, run;
    bool written;
    uint64_t block() const { return (pieces - 1) * outer + run; }  // a beam's
};

// Whether the strides, each over the extent of the smaller ones, keep all pieces apart; their extent.
bool nested(const Places& p, uint64_t batch, uint64_t beams, uint64_t* extent) {
    std::pair<uint64_t, uint64_t> dim[3] = {{p.outer, p.pieces}, {p.beam, beams}, {p.batch, batch}};
    std::sort(dim, dim + 3);
    uint64_t e = p.run;
    bool apart = true;
    for (const auto& d : dim)
        if (d.second > 1) {
            apart = apart && d.first >= e;
            e += (d.second - 1) * d.first;
        }
    *extent = e;
    return apart;
}

// Whether two ranges of addresses overlap that lie `delta` apart (the second behind the first).
bool ranges_meet(int64_t delta, uint64_t first, uint64_t second) {
    return delta < 0 ? static_cast<uint64_t>(-delta) < second : static_cast<uint64_t>(delta) < first;
}

// Whether no piece of one is known to meet a piece of the other: equal strides of batch and beam, between which the
// distance of the two leaves room for both beams' blocks, or, with equal strides of pieces too, for both runs.
bool apart(const Places& a, const Places& b, uint64_t batch, uint64_t beams) {
    if ((batch > 1 && a.batch != b.batch) || (beams > 1 && a.beam != b.beam)) return false;
    const bool same_outer = a.outer == b.outer || (a.pieces == 1 && b.pieces == 1);
    struct Dim {
        uint64_t stride, n;
    } dim[3] = {{a.batch, batch}, {a.beam, beams}, {a.outer, same_outer ? std::max(a.pieces, b.pieces) : 1}};
    uint64_t first = same_outer ? a.run : a.block(), second = same_outer ? b.run : b.block();
    std::sort(dim, dim + 3, [](const Dim& x, const Dim& y) { return x.stride > y.stride; });
    // nested strides: the distance less a multiple of the largest, rounded down or up, and so on
    uint64_t e = std::max(first, second);
    for (int i = 2; i >= 0; --i)
        if (dim[i].n > 1) {
            if (dim[i].stride < e) return false;
            e += (dim[i].n - 1) * dim[i].stride;
        }
    const int64_t delta = static_cast<int64_t>(b.at - a.at);
    for (int pick = 0; pick < 8; ++pick) {
        int64_t d = delta;
        bool there = true;
        for (int i = 0; i < 3 && there; ++i) {
            const bool up = pick >> i & 1;
            if (dim[i].n < 2) {
                there = !up;
                continue;
            }
            const int64_t s = static_cast<int64_t>(dim[i].stride);
            int64_t q = d / s - (d % s < 0 ? 1 : 0) + (up ? 1 : 0);
            const int64_t most = static_cast<int64_t>(dim[i].n) - 1;
            q = std::min(std::max(q, -most), most);
            d -= q * s;
        }
        if (there && ranges_meet(d, first, second)) return false;
    }
    return true;
}

const char* states_problem(const isoloco_state_t* t, int count, int64_t batch, int64_t width, const void* beams, int id_bytes) {
    constexpr int64_t kFar = int64_t(1) << 46;  // no byte of a state is further from its start
    if (count < 0 || (count > 0 && !t)) return "bad list of states";
    std::vector<Places> all;
    all.reserve(2 * static_cast<size_t>(count) + 1);
    for (int i = 0; i < count; ++i) {
        const isoloco_state_t& s = t[i];
        if (s.outer < 0 || s.run < 0 || s.outer > kFar || s.run > kFar) return "a state's pieces and their length must not be negative";
        if (s.outer == 0 || s.run == 0 || batch == 0) continue;
        if (!s.src || !s.dst) return "a state's address is NULL";
        for (const int64_t v : {s.src_batch, s.src_beam, s.src_outer, s.dst_batch, s.dst_beam, s.dst_outer})
            if (v < 0 || v > kFar) return "a state's strides must be in 0 .. 2^46";
        const double far = static_cast<double>(batch) * std::max(s.src_batch, s.dst_batch) +
                           static_cast<double>(width) * std::max(s.src_beam, s.dst_beam) +
                           static_cast<double>(s.outer) * std::max(s.src_outer, s.dst_outer) + s.run;
        if (far > static_cast<double>(kFar)) return "a state must lie within 2^46 bytes";
        const Places src = {reinterpret_cast<uint64_t>(s.src), static_cast<uint64_t>(s.src_batch), static_cast<uint64_t>(s.src_beam),
                            static_cast<uint64_t>(s.src_outer), static_cast<uint64_t>(s.outer), static_cast<uint64_t>(s.run), false};
        const Places dst = {reinterpret_cast<uint64_t>(s.dst), static_cast<uint64_t>(s.dst_batch), static_cast<uint64_t>(s.dst_beam),
                            static_cast<uint64_t>(s.dst_outer), static_cast<uint64_t>(s.outer), static_cast<uint64_t>(s.run), true};
        const bool in_place = src.at == dst.at && (batch < 2 || src.batch == dst.batch) && (width < 2 || src.beam == dst.beam) &&
                              (s.outer < 2 || src.outer == dst.outer);
        uint64_t extent;
        if (!nested(dst, batch, width, &extent)) return "a state's destination overlaps itself";
        all.push_back(dst);
        if (!in_place) all.push_back(src);
    }
    if (beams && batch > 0 && !all.empty()) {
        const uint64_t id = static_cast<uint64_t>(id_bytes);
        all.push_back({reinterpret_cast<uint64_t>(beams), id * static_cast<uint64_t>(width), id, 0, 1, id, false});
    }
    std::sort(all.begin(), all.end(), [](const Places& a, const Places& b) { return a.at < b.at; });
    for (size_t i = 0; i < all.size(); ++i) {
        uint64_t extent;
        nested(all[i], batch, width, &extent);
        for (size_t j = i + 1; j < all.size() && all[j].at < all[i].at + extent; ++j)
            if ((all[i].written || all[j].written) && !apart(all[i], all[j], batch, width))
                return "a state's destination shares memory with another state, its own source or beams, or may";
    }
    return nullptr;
}

}  // namespace

extern "C" {

int isoloco_embed(const void* weight, int64_t ld_weight, isoloco_dtype_t dtype, int64_t vocab, int64_t width,
                  const void* ids, int id_bytes, int64_t tokens, float scale, void* y, int64_t ld_y, void* stream) try {
    if (const char* p = embed_problem(dtype, vocab, width, ids, id_bytes, tokens)) return invalid(p);
    const int es = elem_size(dtype);
    if (!matrix_ok(weight, vocab, width, ld_weight, es)) return invalid("weight is NULL, misaligned or its pitch too small");
    if (!matrix_ok(y, tokens, width, ld_y, es)) return invalid("y is NULL, misaligned or its pitch too small");
    return cuda_status(launch_embed(weight, ld_weight, dtype, vocab, width, ids, id_bytes == 8, tokens, scale, y, ld_y, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int64_t isoloco_embed_grad_workspace(int64_t vocab, int64_t width, int64_t tokens) try {
    if (const char* p = embed_sizes_problem(vocab, width, tokens)) return invalid(p);
    return embed_grad_workspace(vocab, width, tokens);
} catch (...) {
    return kNoMemory;
}

int isoloco_embed_grad(const void* dy, int64_t ld_dy, isoloco_dtype_t dtype, int64_t vocab, int64_t width,
                       const void* ids, int id_bytes, int64_t tokens, float scale, void* dw, int64_t ld_dw,
                       isoloco_dtype_t dw_dtype, void* workspace, int64_t workspace_bytes, void* stream) try {
    if (const char* p = embed_problem(dtype, vocab, width, ids, id_bytes, tokens)) return invalid(p);
    if (dw_dtype != dtype && dw_dtype != ISOLOCO_F32) return invalid("dw is of dy's type or F32");
    if (!matrix_ok(dy, tokens, width, ld_dy, elem_size(dtype))) return invalid("dy is NULL, misaligned or its pitch too small");
    if (!matrix_ok(dw, vocab, width, ld_dw, elem_size(dw_dtype))) return invalid("dw is NULL, misaligned or its pitch too small");
    const int rc = workspace_ok(workspace, workspace_bytes, embed_grad_workspace(vocab, width, tokens));
    if (rc != ISOLOCO_OK) return rc;
    return cuda_status(launch_embed_grad(dy, ld_dy, dtype, vocab, width, ids, id_bytes == 8, tokens, scale, dw, ld_dw, dw_dtype,
                                         workspace, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int64_t isoloco_gated_ffn_saved_bytes(int64_t tokens, int64_t ff, isoloco_dtype_t dtype) try {
    if (!half_dtype(dtype)) return invalid("the gated block takes BF16 or F16");
    if (const char* p = ffn_sizes_problem(tokens, 1, ff)) return invalid(p);
    return ffn_saved_bytes(tokens, ff, dtype);
} catch (...) {
    return kNoMemory;
}

int64_t isoloco_gated_ffn_workspace(int64_t tokens, int64_t width, int64_t ff, int aligned) try {
    if (const char* p = ffn_sizes_problem(tokens, width, ff)) return invalid(p);
    return ffn_workspace(tokens, width, ff, false, aligned != 0);
} catch (...) {
    return kNoMemory;
}

int64_t isoloco_gated_ffn_grad_workspace(int64_t tokens, int64_t width, int64_t ff, int aligned) try {
    if (const char* p = ffn_sizes_problem(tokens, width, ff)) return invalid(p);
    return ffn_workspace(tokens, width, ff, true, aligned != 0);
} catch (...) {
    return kNoMemory;
}

int isoloco_gated_ffn(const void* x, int64_t ld_x, const void* w_gate, const void* w_up, int64_t ld_w,
                      isoloco_dtype_t dtype, int64_t tokens, int64_t width, int64_t ff, isoloco_act_t act, void* h,
                      int64_t ld_h, void* saved, void* workspace, int64_t workspace_bytes, void* stream) try {
    const FfnArgs a = {x, w_gate, w_up, ld_x, ld_w, tokens, width, ff, dtype, act};
    if (const char* p = ffn_problem(a)) return invalid(p);
    if (!matrix_ok(h, tokens, ff, ld_h, 2)) return invalid("h is NULL, misaligned or its pitch too small");
    if (reinterpret_cast<uintptr_t>(saved) & 15u) return set_error(ISOLOCO_ERR_ALIGN, "saved is not 16-byte aligned");
    const int rc = workspace_ok(workspace, workspace_bytes, ffn_workspace(tokens, width, ff, false,
        rows16(x, ld_x, tokens) && rows16(w_gate, ld_w, width) && rows16(w_up, ld_w, width) && rows16(h, ld_h, tokens)));
    if (rc != ISOLOCO_OK) return rc;
    return cuda_status(launch_ffn(a, h, ld_h, saved, workspace, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int isoloco_gated_ffn_grad(const void* dh, int64_t ld_dh, const void* x, int64_t ld_x, const void* w_gate,
                           const void* w_up, int64_t ld_w, isoloco_dtype_t dtype, int64_t tokens, int64_t width,
                           int64_t ff, isoloco_act_t act, const void* saved, void* dx, int64_t ld_dx, void* dw_gate,
                           void* dw_up, int64_t ld_dw, void* workspace, int64_t workspace_bytes, void* stream) try {
    const FfnArgs a = {x, w_gate, w_up, ld_x, ld_w, tokens, width, ff, dtype, act};
    if (const char* p = ffn_problem(a)) return invalid(p);
    if (!matrix_ok(dh, tokens, ff, ld_dh, 2)) return invalid("dh is NULL, misaligned or its pitch too small");
    if (tokens > 0 && !saved) return invalid("saved is NULL");
    if (reinterpret_cast<uintptr_t>(saved) & 15u) return set_error(ISOLOCO_ERR_ALIGN, "saved is not 16-byte aligned");
    if (dx && !matrix_ok(dx, tokens, width, ld_dx, 2)) return invalid("dx is misaligned or its pitch too small");
    if (!dw_gate != !dw_up) return invalid("dw_gate and dw_up are given together");
    if (dw_gate && (!matrix_ok(dw_gate, width, ff, ld_dw, 2) || !matrix_ok(dw_up, width, ff, ld_dw, 2)))
        return invalid("dw_gate or dw_up is misaligned or its pitch too small");
    const int rc = workspace_ok(workspace, workspace_bytes, ffn_workspace(tokens, width, ff, true,
        rows16(x, ld_x, tokens) && rows16(w_gate, ld_w, width) && rows16(w_up, ld_w, width) && (!dx || rows16(dx, ld_dx, tokens)) &&
        (!dw_gate || (rows16(dw_gate, ld_dw, width) && rows16(dw_up, ld_dw, width)))));
    if (rc != ISOLOCO_OK) return rc;
    return cuda_status(launch_ffn_grad(a, dh, ld_dh, saved, dx, ld_dx, dw_gate, dw_up, ld_dw, workspace, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int isoloco_token_logprobs(const void* logits, int64_t ld_logits, isoloco_dtype_t dtype, int64_t rows, int64_t vocab,
                           const void* targets, int target_bytes, float scale, float* logp, float* entropy, float* lse,
                           int top, float* top_logp, int64_t* top_index, const float* grad_logp,
                           const float* grad_entropy, void* grad_logits, int64_t ld_grad, void* stream) try {
    const LogprobArgs a = {logits, ld_logits, rows, vocab, dtype, targets, target_bytes == 8, scale, logp, entropy, lse, top,
                           top_logp, top_index, grad_logp, grad_entropy, grad_logits, ld_grad};
    if (const char* p = logprob_problem(a, target_bytes)) return invalid(p);
    if (top < 0 || top > ISOLOCO_MAX_TOP || top > vocab) return invalid("top must be in 0 .. min(vocab, 32)");
    if (top && (!array_ok(top_logp, rows, 4) || !array_ok(top_index, rows, 8))) return invalid("top_logp or top_index is NULL or misaligned");
    return cuda_status(launch_logprobs(a, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int isoloco_token_logprobs_grad(const void* logits, int64_t ld_logits, isoloco_dtype_t dtype, int64_t rows,
                                int64_t vocab, const void* targets, int target_bytes, float scale, const float* lse,
                                const float* entropy, const float* grad_logp, const float* grad_entropy,
                                void* grad_logits, int64_t ld_grad, void* stream) try {
    const LogprobArgs a = {logits, ld_logits, rows, vocab, dtype, targets, target_bytes == 8, scale, nullptr,
                           const_cast<float*>(entropy), const_cast<float*>(lse), 0, nullptr, nullptr, grad_logp, grad_entropy,
                           grad_logits, ld_grad};
    if (const char* p = logprob_problem(a, target_bytes)) return invalid(p);
    if (!array_ok(lse, rows, 4)) return invalid("lse is NULL or misaligned");
    if (rows > 0 && !grad_logits) return invalid("grad_logits is NULL");
    if (grad_entropy && !array_ok(entropy, rows, 4)) return invalid("entropy is NULL or misaligned");
    return cuda_status(launch_logprobs_grad(a, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int isoloco_distill(const void* logits, int64_t ld_logits, isoloco_dtype_t dtype, int64_t rows, int64_t vocab,
                    const void* top_logp, int64_t ld_logp, isoloco_dtype_t logp_dtype, const void* top_index,
                    int64_t ld_index, int index_bytes, int k, float scale, isoloco_tail_t tail, float* loss, float* saved,
                    const float* grad_loss, void* grad_logits, int64_t ld_grad, void* stream) try {
    DistillArgs a = {logits, ld_logits, rows, vocab, dtype, top_logp, ld_logp, logp_dtype, top_index, ld_index,
                     index_bytes == 8, k, scale, tail == ISOLOCO_TAIL_REST, loss, saved, grad_loss, grad_logits, ld_grad, false};
    if (const char* p = distill_problem(a, index_bytes, tail)) return invalid(p);
    if (!array_ok(loss, rows, 4)) return invalid("loss is NULL or misaligned");
    a.lost = g_lose_rows.load(std::memory_order_relaxed) > 0 && g_lose_rows.fetch_sub(1) > 0;
    return cuda_status(launch_distill(a, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int isoloco_distill_grad(const float* grad_loss, const void* logits, int64_t ld_logits, isoloco_dtype_t dtype, int64_t rows,
                         int64_t vocab, const void* top_logp, int64_t ld_logp, isoloco_dtype_t logp_dtype,
                         const void* top_index, int64_t ld_index, int index_bytes, int k, float scale, isoloco_tail_t tail,
                         const float* saved, void* grad_logits, int64_t ld_grad, void* stream) try {
    const DistillArgs a = {logits, ld_logits, rows, vocab, dtype, top_logp, ld_logp, logp_dtype, top_index, ld_index,
                           index_bytes == 8, k, scale, tail == ISOLOCO_TAIL_REST, nullptr, const_cast<float*>(saved), grad_loss,
                           grad_logits, ld_grad, false};
    if (rows > 0 && !grad_logits) return invalid("grad_logits is NULL");
    if (const char* p = distill_problem(a, index_bytes, tail)) return invalid(p);
    if (!array_ok(saved, rows, 4)) return invalid("saved is NULL or misaligned");
    return cuda_status(launch_distill_grad(a, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int isoloco_beam_select(const void* logits, int64_t ld_logits, isoloco_dtype_t dtype, int64_t batch, int64_t beams,
                        int64_t vocab, const float* scores, const uint8_t* finished, int64_t end, float scale, int keep,
                        float* out_scores, int64_t* out_beams, int64_t* out_tokens, uint8_t* out_finished, void* stream) try {
    if (!any_dtype(dtype)) return invalid("bad element type");
    if (beams < 1 || beams > ISOLOCO_MAX_BEAMS) return invalid("beams must be in 1 .. 32");
    if (!size_ok(batch, 0) || !size_ok(batch * beams, 0) || !size_ok(vocab, 1)) return invalid("batch * beams must be in 0 .. 2^31 - 1, vocab in 1 .. 2^31 - 1");
    if (keep < 1 || keep > ISOLOCO_MAX_TOP || keep > beams * vocab) return invalid("keep must be in 1 .. min(beams * vocab, 32)");
    if (!matrix_ok(logits, batch * beams, vocab, ld_logits, elem_size(dtype))) return invalid("logits is NULL, misaligned or its pitch too small");
    if (!(scale > 0.f) || scale > 1e30f) return invalid("scale must be positive and finite");
    if (!array_ok(scores, batch, 4)) return invalid("scores is NULL or misaligned");
    if (end >= vocab) return invalid("end is no token");
    if (finished && end < 0) return invalid("finished beams need a token to continue with");
    if (!array_ok(out_scores, batch, 4) || !array_ok(out_beams, batch, 8) || !array_ok(out_tokens, batch, 8))
        return invalid("out_scores, out_beams or out_tokens is NULL or misaligned");
    const BeamArgs a = {logits, ld_logits, batch, vocab, end < 0 ? -1 : end, dtype, static_cast<int>(beams), keep, scores, finished, scale,
                        out_scores, out_beams, out_tokens, out_finished};
    if (selection_shares(a)) return invalid("outputs share memory with one another, or with scores or finished otherwise than in place");
    return cuda_status(launch_beam_select(a, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int isoloco_beam_reorder(const isoloco_state_t* states, int count, int64_t batch, int64_t width, const void* beams,
                         int id_bytes, void* stream) try {
    if (width < 1 || width > ISOLOCO_MAX_BEAMS) return invalid("width must be in 1 .. 32");
    if (!size_ok(batch, 0) || !size_ok(batch * width, 0)) return invalid("batch * width must be in 0 .. 2^31 - 1");
    if (id_bytes != 4 && id_bytes != 8) return invalid("id_bytes must be 4 or 8");
    if (const char* p = states_problem(states, count, batch, width, beams, id_bytes)) return invalid(p);
    if (!array_ok(beams, batch, id_bytes)) return invalid("beams is NULL or misaligned");
    return cuda_status(launch_beam_reorder(states, count, batch, static_cast<int>(width), beams, id_bytes == 8, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int64_t isoloco_grad_norm_workspace(const isoloco_tensor_t* tensors, int count) try {
    if (const char* p = tensors_problem(tensors, count)) return invalid(p);
    return grad_norm_workspace(tensors, count);
} catch (...) {
    return kNoMemory;
}

int isoloco_grad_norm(const isoloco_tensor_t* tensors, int count, float* norm, void* workspace,
                      int64_t workspace_bytes, void* stream) try {
    if (const char* p = tensors_problem(tensors, count)) return invalid(p);
    if (!array_ok(norm, 1, 4)) return invalid("norm is NULL or misaligned");
    const int rc = workspace_ok(workspace, workspace_bytes, grad_norm_workspace(tensors, count));
    if (rc != ISOLOCO_OK) return rc;
    return cuda_status(launch_clip(tensors, nullptr, count, false, 0.f, norm, workspace, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int isoloco_clip_grads(const isoloco_tensor_t* tensors, const isoloco_tensor_t* outs, int count, float max_norm,
                       float* norm, void* workspace, int64_t workspace_bytes, void* stream) try {
    if (const char* p = tensors_problem(tensors, count)) return invalid(p);
    if (outs) {
        if (const char* p = tensors_problem(outs, count)) return invalid(p);
        for (int i = 0; i < count; ++i)
            if (outs[i].n != tensors[i].n || outs[i].dtype != tensors[i].dtype) return invalid("an output's length or type is not its input's");
    }
    if (!(max_norm > 0.f)) return invalid("max_norm must be positive");
    if (!array_ok(norm, 1, 4)) return invalid("norm is NULL or misaligned");
    const int rc = workspace_ok(workspace, workspace_bytes, grad_norm_workspace(tensors, count));
    if (rc != ISOLOCO_OK) return rc;
    return cuda_status(launch_clip(tensors, outs, count, true, max_norm, norm, workspace, stream_of(stream)));
} catch (...) {
    return kNoMemory;
}

int isoloco_inner_status(void* stream) try {
    uint32_t *word = nullptr, bits = 0;
    cudaStream_t st = stream_of(stream);
    cudaError_t e = error_word(&word);
    if (e == cudaSuccess) e = cudaMemcpyAsync(&bits, word, sizeof(bits), cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e == cudaSuccess && bits) {
        // only what this call reports: a kernel on another stream may have raised an error since
        k_clear<<<1, 1, 0, st>>>(word, bits);
        e = cudaGetLastError();
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    }
    if (e != cudaSuccess) return cuda_status(e);
    return (bits & kErrTimeout) ? set_error(ISOLOCO_ERR_TIMEOUT, "a wait in an inner-step kernel gave up") : ISOLOCO_OK;
} catch (...) {
    return kNoMemory;
}

int isoloco_debug_lose_rows(int calls) {
    if (calls < 0) return ISOLOCO_ERR_INVALID;
    g_lose_rows = calls;
    return ISOLOCO_OK;
}

int isoloco_debug_refuse_clusters(int refuse) {
    if (refuse != 0 && refuse != 1) return ISOLOCO_ERR_INVALID;
    refuse_large_clusters(refuse == 1);
    return ISOLOCO_OK;
}

int isoloco_debug_raise_inner(void* stream) try {
    uint32_t* word = nullptr;
    cudaError_t e = error_word(&word);
    if (e != cudaSuccess) return cuda_status(e);
    k_raise<<<1, 1, 0, stream_of(stream)>>>(word, kErrTimeout);
    return cuda_status(cudaGetLastError());
} catch (...) {
    return kNoMemory;
}

}  // extern "C"

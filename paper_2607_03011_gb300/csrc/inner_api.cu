// inner_api.cu -- C entry points of the inner step's operators: argument checks, then the launchers.
#include <climits>
#include <string>

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

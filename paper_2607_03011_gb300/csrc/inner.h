// inner.h -- launchers of the inner step's operators (checked arguments; see include/isoloco.h).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "isoloco.h"

namespace isoloco {

// The message isoloco_last_error() gives on this thread; returns `code`.
int set_error(int code, const char* msg);

// SMs of the current device.
cudaError_t device_sms(int* sms);

// The current device's word that collects kErr* bits until isoloco_inner_status reads it.
cudaError_t error_word(uint32_t** word);

cudaError_t launch_embed(const void* weight, int64_t ld_w, int dtype, int64_t vocab, int64_t width, const void* ids,
                         bool ids64, int64_t tokens, float scale, void* y, int64_t ld_y, cudaStream_t st);

int64_t embed_grad_workspace(int64_t vocab, int64_t width, int64_t tokens);
cudaError_t launch_embed_grad(const void* dy, int64_t ld_dy, int dtype, int64_t vocab, int64_t width, const void* ids,
                              bool ids64, int64_t tokens, float scale, void* dw, int64_t ld_dw, int dw_dtype, void* ws,
                              cudaStream_t st);

struct FfnArgs {
    const void *x, *wg, *wu;
    int64_t ld_x, ld_w, tokens, width, ff;
    int dtype, act;
};
int64_t ffn_saved_bytes(int64_t tokens, int64_t ff, int dtype);
// aligned: every matrix's address and pitch are multiples of 16 bytes
int64_t ffn_workspace(int64_t tokens, int64_t width, int64_t ff, bool backward, bool aligned);
cudaError_t launch_ffn(const FfnArgs& a, void* h, int64_t ld_h, void* saved, void* ws, cudaStream_t st);
cudaError_t launch_ffn_grad(const FfnArgs& a, const void* dh, int64_t ld_dh, const void* saved, void* dx,
                            int64_t ld_dx, void* dwg, void* dwu, int64_t ld_dw, void* ws, cudaStream_t st);

struct LogprobArgs {
    const void* logits;
    int64_t ld, rows, vocab;
    int dtype;
    const void* targets;
    bool targets64;
    float scale;
    float *logp, *entropy, *lse;
    int top;
    float* top_logp;
    int64_t* top_index;
    const float *grad_logp, *grad_entropy;
    void* grad_logits;
    int64_t ld_grad;
};
cudaError_t launch_logprobs(const LogprobArgs& a, cudaStream_t st);
// a.lse and a.entropy are read
cudaError_t launch_logprobs_grad(const LogprobArgs& a, cudaStream_t st);

int64_t grad_norm_workspace(const isoloco_tensor_t* in, int count);
// clip: false writes the norm only
cudaError_t launch_clip(const isoloco_tensor_t* in, const isoloco_tensor_t* out, int count, bool clip, float max_norm,
                        float* norm, void* ws, cudaStream_t st);

}  // namespace isoloco

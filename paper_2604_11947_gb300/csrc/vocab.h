// vocab.h -- host-side interface of the vocabulary's losses to the rest of the library.
#pragma once

#include "internal.h"

namespace resbm {

// Reads (and optionally clears) the error word of their tensor-core kernels; synchronizing.
cudaError_t vocab_device_error(unsigned int *code, bool clear);
// Scratch bytes of the embedding's gradient.
size_t embed_bwd_ws_bytes(int64_t T, int64_t d);


// The losses over the vocabulary for up to kFewTokens tokens (vocab_few.cu). Shapes it takes, its CTAs (each has a slot of
// the forward's partial sums, or of dX), and the kernels (the targets' lists before them and the join are the caller's).
constexpr int kFewTokens = 8, kFewSlots = 304;
struct FewArgs {
    bool bwd;
    const void *X, *W;
    int64_t ldx, ldw, V;
    int T, d, dp;               // dp: d rounded up to 8
    const int64_t *label;       // or null: the lists
    const int32_t *list, *count;
    const float *weight, *bad;
    int K;
    float c, tau;               // log2(e) / tau
    float2 *stat;               // forward: slot, token (tp a slot)
    float *zt;
    int64_t tp;
    const float *lse, *dloss;   // backward
    int dloss_step;
    void *dX, *dW;
    float *slots;               // slot, token, dp columns
};
bool few_tokens(int64_t T, int64_t d, int64_t es, bool bwd);
int few_slots(int64_t V, bool bwd, int sms);
cudaError_t few_run(const FewArgs &a, bool f32, const Ctx &c, int *launches);

}  // namespace resbm

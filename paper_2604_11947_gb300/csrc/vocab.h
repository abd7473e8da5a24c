// vocab.h -- host-side interface of the vocabulary's losses to the rest of the library.
#pragma once

#include "internal.h"

namespace resbm {

// Reads (and optionally clears) the error word of their tensor-core kernels; synchronizing.
cudaError_t vocab_device_error(unsigned int *code, bool clear);
// The embedding's sizes and type: valid and supported.
resbm_status embed_check_shape(int64_t T, int64_t V, int64_t d, int32_t dtype);
// Scratch bytes of the embedding's gradient.
size_t embed_bwd_ws_bytes(int64_t T, int64_t d);

}  // namespace resbm

// The feed-forward projections on the tensor cores (hla_ffn_sm103.cu), as hla_ffn.cu calls them: bf16.
#pragma once

#include "hla_internal.h"

namespace hla {

size_t ffn_tc_forward_scratch_bytes(int M, int K, int F);
size_t ffn_tc_backward_scratch_bytes(int M, int K, int F);
cudaError_t ffn_tc_forward(const Ffn &p, cudaStream_t stream);
cudaError_t ffn_tc_backward(const FfnBwd &p, cudaStream_t stream);

}  // namespace hla

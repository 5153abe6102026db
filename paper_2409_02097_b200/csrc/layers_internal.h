// What the sources of include/linfusion_layers.h share.
#pragma once

#include <cuda_runtime.h>

namespace lf {
// How many waits of linear_kernel have expired on the current device, copied in the order of the stream.
cudaError_t read_linear_expired(unsigned int* n, cudaStream_t s);
}  // namespace lf

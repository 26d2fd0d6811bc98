// mcd_sample_rows' kernels for bf16 logits (mcd_sample.cuh).
#include "mcd_sample.cuh"

template cudaError_t mcd::rows::launch_sample<uint16_t>(mcd::rows::SampleArgs, int, cudaStream_t);

// mcd_sample_rows' checks, and its kernels for fp32 logits (mcd_sample.cuh).
#include "mcd_sample.cuh"

template cudaError_t mcd::rows::launch_sample<float>(mcd::rows::SampleArgs, int, cudaStream_t);

using namespace mcd;

extern "C" mcd_status mcd_sample_rows(int32_t n_rows, int32_t vocab, const void* logits, int64_t stride, int32_t dtype,
                                      const float* temperature, const int32_t* top_k, const float* top_p,
                                      const float* min_p, const double* u, int32_t* ids, float* probs, int32_t* kept,
                                      int32_t* err, void* stream) {
  using namespace rows;
  if (n_rows < 0 || vocab <= 0 || !err) return MCD_ERR_INVALID_ARG;
  if (dtype != MCD_WEIGHT_F32 && dtype != MCD_WEIGHT_BF16) return MCD_ERR_UNSUPPORTED;
  if (vocab > kMaxVocabRows || n_rows > (1 << 27)) return MCD_ERR_UNSUPPORTED;
  if (n_rows == 0) return MCD_OK;
  if (!logits || !u || !ids || stride < vocab) return MCD_ERR_INVALID_ARG;
  const Block in{logits, stride, n_rows, vocab, bytes_of(dtype)};
  if (!in.aligned() || !in.fits() || !aligned_to(u, 8)) return MCD_ERR_UNSUPPORTED;
  const void* const fours[] = {temperature, top_k, top_p, min_p, ids, probs, kept, err};
  for (const void* p : fours)
    if (!aligned_to(p, 4)) return MCD_ERR_UNSUPPORTED;
  const Block read[] = {in, values(temperature, n_rows, 4), values(top_k, n_rows, 4), values(top_p, n_rows, 4), values(min_p, n_rows, 4),
                        values(u, n_rows, 8)};
  const Block written[] = {values(ids, n_rows, 4), values(probs, n_rows, 4), values(kept, n_rows, 4), values(err, 1, 4)};
  for (int i = 0; i < 4; ++i) {
    for (const Block& r : read)
      if (overlap(written[i], r)) return MCD_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (overlap(written[i], written[j])) return MCD_ERR_INVALID_ARG;
  }
  const SampleArgs a{logits, stride, vocab, 1, n_rows, 0, temperature, top_k, top_p, min_p, u, ids, probs, kept, err};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return cuda_status(dtype == MCD_WEIGHT_F32 ? launch_sample<float>(a, n_rows, st) : launch_sample<uint16_t>(a, n_rows, st));
}

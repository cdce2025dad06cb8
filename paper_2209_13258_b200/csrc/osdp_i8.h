// The int8 product of a few tokens (osdp_i8.cu), called by the entry point that also owns the tile kernel's path.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace osdp {

constexpr int64_t OSDP_I8_MAX_K = 131071;   // 2^31 / 128^2 = 131072 products of the largest magnitude would overflow

int launch_i8_quantize(const void *x, int64_t M, int64_t K, void *q, float *scale, cudaStream_t stream);
// Whether launch_i8_few_tokens takes this product (64 tokens at most).
bool i8_few_tokens(int64_t M, int64_t N, int64_t K);
int launch_i8_few_tokens(const void *x8, const float *x_scale, const void *w8, const float *w_scale, const float *bias, int64_t M, int64_t N,
                         int64_t K, int act, void *out, cudaStream_t stream);

}  // namespace osdp

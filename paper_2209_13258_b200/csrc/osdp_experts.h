// The plan of the experts' rows, shared by the translation units that write and read it.  Not part of the C ABI.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace osdp {

// int32 words of a plan for E experts.  What the ABI documents comes first: where the experts' rows start (E + 1) and how
// many there are (E).  Then what the products' kernels walk: tiles of 128 and of 256 rows before each expert (E + 1 each), the
// experts that have rows (E) and their number.
constexpr int PLAN_OFFSETS = 0;
__host__ __device__ constexpr int plan_counts(int E) { return E + 1; }
__host__ __device__ constexpr int plan_tiles128(int E) { return 2 * E + 1; }
__host__ __device__ constexpr int plan_tiles256(int E) { return 3 * E + 2; }
__host__ __device__ constexpr int plan_live(int E) { return 4 * E + 3; }
__host__ __device__ constexpr int plan_n_live(int E) { return 5 * E + 3; }
__host__ __device__ constexpr int plan_length(int E) { return (5 * E + 4 + 3) / 4 * 4; }

// Rows that are enough however the choices fall.
int64_t expert_rows(int64_t T, int top_k, int E);
// The checks that every call over the experts' rows makes of T, top_k and E.
int expert_check(int64_t T, int top_k, int E);
// The products of few rows for each expert (osdp_expert_few.cu): whether they go there, and the launch.
bool expert_few_rows(int64_t T, int top_k, int E, int64_t N, int64_t K);
int launch_expert_few(const void *rows, const int32_t *plan, const void *w, const float *bias, int64_t T, int top_k, int E, int64_t N, int64_t K, int act,
                      void *out, void *z_save, cudaStream_t stream);

}  // namespace osdp

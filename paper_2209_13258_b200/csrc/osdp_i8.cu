// int8 operands of the serving path: the quantiser (one scale per row) and the product for a few tokens, which streams
// the weights.  Products of many tokens run on the tile kernel (tcgen05.mma.kind::i8, osdp_gemm.cuh).
#include "../../include/osdp.h"

#include "osdp_i8.h"
#include "osdp_internal.h"
#include "osdp_vec.cuh"

namespace osdp {
namespace {

// One row per team of warps: the row's largest magnitude, then its codes.  The row is read twice by its own threads;
// the second read comes from L1 / L2.
__global__ void __launch_bounds__(256) quantize_rows_kernel(const __nv_bfloat16 *__restrict__ x, long long M, int K, int8_t *__restrict__ q,
                                                            float *__restrict__ scale, int warps) {
  __shared__ float red[8];
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int team = warp / warps, first_warp = team * warps;
  const int tl = (warp - first_warp) * 32 + lane, TL = warps * 32;
  const long long row = (long long)blockIdx.x * ((blockDim.x >> 5) / warps) + team;
  pdl_wait();
  if (row >= M) return;
  const __nv_bfloat16 *xr = x + row * K;
  uint32_t bits = 0u;
  for (int c = tl * 8; c < K; c += TL * 8) {
    float f[8];
    widen8(__ldg(reinterpret_cast<const uint4 *>(xr + c)), f);
#pragma unroll
    for (int k = 0; k < 8; ++k) bits = max(bits, __float_as_uint(f[k]) & 0x7FFFFFFFu);
  }
  float top = warp_max_abs(__uint_as_float(bits));
  if (warps > 1) {
    if (lane == 0) red[warp] = top;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(TL) : "memory");
    for (int k = 0; k < warps; ++k) top = __uint_as_float(max(__float_as_uint(top), __float_as_uint(red[first_warp + k])));
  }
  const float inv = int8_inverse(top);
  for (int c = tl * 8; c < K; c += TL * 8) {
    float f[8];
    widen8(__ldg(reinterpret_cast<const uint4 *>(xr + c)), f);
    *reinterpret_cast<uint2 *>(q + row * K + c) = to_int8x8(f, inv);
  }
  if (tl == 0) scale[row] = int8_scale(top);
}

// ---- Few tokens.  D[16 weight rows x 8 tokens] += W[16 x 32] X[8 x 32]^T by mma.sync (int8, exact int32 sums): at this
// many tokens the product is bound by reading W once, and the legacy path keeps W in registers on its way from memory.
// A block owns 16 weight rows; its warps take 64-byte steps of K in turn and their sums are added in shared memory.
// A lane reads 16 consecutive bytes of a row; the four words are used as the operands of two mma whose k order is a
// permutation of the real one, the same for W and X, which a sum over k does not notice.
__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

constexpr int FEW_WARPS = 8;

template <int MT>   // tokens in groups of eight
__global__ void __launch_bounds__(32 * FEW_WARPS) few_tokens_kernel(const int8_t *__restrict__ x, const float *__restrict__ x_scale,
                                                                    const int8_t *__restrict__ w, const float *__restrict__ w_scale,
                                                                    const float *__restrict__ bias, int M, int N, int K, int act,
                                                                    __nv_bfloat16 *__restrict__ out) {
  __shared__ int part[FEW_WARPS][16 * 8 * MT];
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, kq = (lane & 3) * 16;
  const int n0 = blockIdx.x * 16;
  // rows past the end read the last row: in bounds, and their sums are not stored
  const int8_t *w0 = w + (long long)min(n0 + g, N - 1) * K, *w1 = w + (long long)min(n0 + g + 8, N - 1) * K;
  // The weights are not written by the kernel before this one in a serving loop, but nothing says so: only a prefetch
  // into L2, which holds whatever is written there later, may run ahead of the wait.
  if (threadIdx.x < 16) {
    const int8_t *row = w + (long long)min(n0 + (int)threadIdx.x, N - 1) * K;
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(row), "r"(K) : "memory");
  }
  pdl_wait();
  int acc[MT][4];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[t][j] = 0;
  // The loop is the warp's: mma.sync needs every lane, those whose 16 bytes lie past K bring zeros (K is a multiple of 16,
  // so a lane's 16 bytes are whole or absent).
#pragma unroll 4
  for (int k0 = warp * 64; k0 < K; k0 += FEW_WARPS * 64) {
    const int k = k0 + kq;
    const bool in = k < K;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    const uint4 a = in ? load16(w0 + k) : zero, b = in ? load16(w1 + k) : zero;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const uint4 c = (in && t * 8 + g < M) ? __ldg(reinterpret_cast<const uint4 *>(x + (long long)(t * 8 + g) * K + k)) : zero;
      mma_s8(acc[t], a.x, b.x, a.y, b.y, c.x, c.y);
      mma_s8(acc[t], a.z, b.z, a.w, b.w, c.z, c.w);
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j)   // row g (+ 8), token 2 (lane & 3) + (0, 1) of the group
      part[warp][(t * 8 + 2 * (lane & 3) + (j & 1)) * 16 + g + 8 * (j >> 1)] = acc[t][j];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * 8 * MT; i += 32 * FEW_WARPS) {
    const int m = i >> 4, n = n0 + (i & 15);
    if (m >= M || n >= N) continue;
    int s = 0;
#pragma unroll
    for (int q = 0; q < FEW_WARPS; ++q) s += part[q][i];
    float f = (float)s * x_scale[m] * w_scale[n];
    if (bias) f += bias[n];
    out[(long long)m * N + n] = __float2bfloat16_rn(gelu1(f, act));
  }
}

}  // namespace

int launch_i8_few_tokens(const void *x8, const float *x_scale, const void *w8, const float *w_scale, const float *bias, int64_t M, int64_t N,
                         int64_t K, int act, void *out, cudaStream_t stream) {
  const dim3 grid((unsigned)cdiv(N, 16)), block(32 * FEW_WARPS);
  auto go = [&](auto kernel) {
    return launch_overlapped(kernel, grid, block, 0, 1, stream, (const int8_t *)x8, x_scale, (const int8_t *)w8, w_scale, bias, (int)M, (int)N,
                             (int)K, act, (__nv_bfloat16 *)out);
  };
  if (M <= 8) return go(few_tokens_kernel<1>);
  if (M <= 16) return go(few_tokens_kernel<2>);
  return go(few_tokens_kernel<4>);
}

}  // namespace osdp

using namespace osdp;

extern "C" int osdp_quantize_rows_i8(const void *x, int64_t M, int64_t K, void *q, float *scale, void *stream) {
  if (M < 0 || K <= 0 || M > ((int64_t)1 << 30) || K > OSDP_I8_MAX_K) return OSDP_ERR_BAD_SHAPE;
  if (K & 7) return OSDP_ERR_ALIGNMENT;
  if (M == 0) return OSDP_OK;
  if (!x || !q || !scale) return OSDP_ERR_NULL_POINTER;
  if (!aligned_to(x, 16) || !aligned_to(q, 8) || !aligned_to(scale, 4)) return OSDP_ERR_ALIGNMENT;
  int warps = (int)cdiv(K, 1024);
  if (warps > 8 || M <= 148) warps = 8;
  const int teams = 8 / warps;
  return launch_overlapped(quantize_rows_kernel, dim3((unsigned)cdiv(M, teams)), dim3(teams * warps * 32), 0, 1, static_cast<cudaStream_t>(stream),
                           (const __nv_bfloat16 *)x, (long long)M, (int)K, (int8_t *)q, scale, warps);
}

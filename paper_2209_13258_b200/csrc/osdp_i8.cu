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

// ---- Few tokens.  Y^T[weight rows x tokens] by mma.sync (int8, exact int32 sums): at this many tokens the product is
// bound by reading W once, and mma.sync takes W from the registers that it is loaded into.
// A block owns 8 NT weight rows; its warps take 64-byte steps of K in turn and their sums are added in shared memory.
// A lane reads 16 consecutive bytes of a row; the four words are used as the operands of two mma whose k order is a
// permutation of the real one, the same for W and X, which a sum over k does not notice.
__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct FewArgs {
  const void *x;              // int8 [M,K], or bf16 [M,K] that the block quantises itself (QUANT)
  const float *x_scale;
  const int8_t *w;
  const float *w_scale, *bias;
  __nv_bfloat16 *out;
  int M, N, K, act;
};
constexpr int FEW_MAX_WARPS = 8;
constexpr int FUSED_MAX_M = 4, FUSED_MAX_BYTES = 16384;   // int8 rows that a block quantises for itself

// MT: 16-token tiles, NT: groups of eight weight rows per block.
template <int MT, int NT, bool QUANT>
__global__ void __launch_bounds__(32 * FEW_MAX_WARPS) few_tokens_kernel(const __grid_constant__ FewArgs a) {
  constexpr int U = 8 / NT;            // steps of K whose loads are issued together: eight 16-byte loads per lane
  __shared__ int part[FEW_MAX_WARPS][16 * MT * 8 * NT];
  __shared__ float scales[16 * MT];
  __shared__ uint32_t top[FUSED_MAX_M];
  extern __shared__ __align__(16) int8_t xq[];
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int g = lane >> 2, kq = (lane & 3) * 16;
  const int n0 = blockIdx.x * (8 * NT);
  const int K = a.K, M = a.M, N = a.N;
  // Nothing says that the weights were not written by the kernel before this one: only a prefetch into L2, where
  // whatever is written later lands as well, may run ahead of the wait.
  if (threadIdx.x < 8 * NT && n0 + (int)threadIdx.x < N)
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.w + (long long)(n0 + threadIdx.x) * K), "r"(K) : "memory");
  if (QUANT && threadIdx.x < FUSED_MAX_M) top[threadIdx.x] = 0u;
  pdl_wait();
  if (QUANT) {
    __syncthreads();
    const __nv_bfloat16 *x = static_cast<const __nv_bfloat16 *>(a.x);
    for (int m = 0; m < M; ++m) {
      uint32_t bits = 0u;
      for (int c = threadIdx.x * 8; c < K; c += blockDim.x * 8) {
        float f[8];
        widen8(__ldg(reinterpret_cast<const uint4 *>(x + (long long)m * K + c)), f);
#pragma unroll
        for (int k = 0; k < 8; ++k) bits = max(bits, __float_as_uint(f[k]) & 0x7FFFFFFFu);
      }
      bits = __reduce_max_sync(0xFFFFFFFFu, bits);
      if (lane == 0) atomicMax(&top[m], bits);
    }
    __syncthreads();
    for (int m = 0; m < M; ++m) {
      const float t = __uint_as_float(top[m]), inv = int8_inverse(t);
      for (int c = threadIdx.x * 8; c < K; c += blockDim.x * 8) {
        float f[8];
        widen8(__ldg(reinterpret_cast<const uint4 *>(x + (long long)m * K + c)), f);
        *reinterpret_cast<uint2 *>(xq + m * K + c) = to_int8x8(f, inv);
      }
      if (threadIdx.x == 0) scales[m] = int8_scale(t);
    }
    __syncthreads();
  } else if (threadIdx.x < 16 * MT) {
    scales[threadIdx.x] = (int)threadIdx.x < M ? a.x_scale[threadIdx.x] : 0.f;
  }
  // rows past the end read the last row: in bounds, and their sums are not stored
  const int8_t *w[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) w[n] = a.w + (long long)min(n0 + n * 8 + g, N - 1) * K;
  const int8_t *x8 = QUANT ? xq : static_cast<const int8_t *>(a.x);
  int acc[MT][NT][4];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[t][n][j] = 0;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  // The loop is the warp's: mma.sync needs every lane, those whose 16 bytes lie past K bring zeros (K is a multiple of
  // 16, so a lane's 16 bytes are whole or absent).
  for (int k0 = warp * 64; k0 < K; k0 += warps * 64 * U) {
    uint4 b[U][NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * warps * 64 + kq;
#pragma unroll
      for (int n = 0; n < NT; ++n) b[u][n] = k < K ? load16(w[n] + k) : zero;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * warps * 64 + kq;
      if (k0 + u * warps * 64 >= K) break;
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const int m = t * 16 + g;
        const uint4 lo = (k < K && m < M) ? *reinterpret_cast<const uint4 *>(x8 + (long long)m * K + k) : zero;
        const uint4 hi = (k < K && m + 8 < M) ? *reinterpret_cast<const uint4 *>(x8 + (long long)(m + 8) * K + k) : zero;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_s8(acc[t][n], lo.x, hi.x, lo.y, hi.y, b[u][n].x, b[u][n].y);
          mma_s8(acc[t][n], lo.z, hi.z, lo.w, hi.w, b[u][n].z, b[u][n].w);
        }
      }
    }
  }
  constexpr int ROWS = 8 * NT;
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j)   // token g (+ 8) of the tile, weight row 2 (lane & 3) + (0, 1) of the group
        part[warp][(t * 16 + g + 8 * (j >> 1)) * ROWS + n * 8 + 2 * (lane & 3) + (j & 1)] = acc[t][n][j];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * MT * ROWS; i += blockDim.x) {
    const int m = i / ROWS, n = n0 + i % ROWS;
    if (m >= M || n >= N) continue;
    int s = 0;
    for (int q = 0; q < warps; ++q) s += part[q][i];
    float f = (float)s * scales[m] * a.w_scale[n];
    if (a.bias) f += a.bias[n];
    a.out[(long long)m * N + n] = __float2bfloat16_rn(gelu1(f, a.act));
  }
}

template <int MT, int NT, bool QUANT>
int launch_few(const FewArgs &a, cudaStream_t stream) {
  const int64_t blocks = cdiv(a.N, 8 * NT);
  const int warps = blocks < 148 * 4 ? 8 : 4;     // few blocks: more warps each, to have as many loads in flight
  return launch_overlapped(few_tokens_kernel<MT, NT, QUANT>, dim3((unsigned)blocks), dim3(32 * warps), QUANT ? (size_t)a.M * a.K : 0, 1, stream, a);
}

int launch_quantize(const void *x, int64_t M, int64_t K, void *q, float *scale, cudaStream_t stream) {
  int warps = (int)cdiv(K, 1024);
  if (warps > 8 || M <= 148) warps = 8;
  const int teams = 8 / warps;
  return launch_overlapped(quantize_rows_kernel, dim3((unsigned)cdiv(M, teams)), dim3(teams * warps * 32), 0, 1, stream,
                           (const __nv_bfloat16 *)x, (long long)M, (int)K, (int8_t *)q, scale, warps);
}

}  // namespace

int launch_i8_quantize(const void *x, int64_t M, int64_t K, void *q, float *scale, cudaStream_t stream) {
  return launch_quantize(x, M, K, q, scale, stream);
}

bool i8_quantises_itself(int64_t M, int64_t K) { return M <= FUSED_MAX_M && M * K <= FUSED_MAX_BYTES; }

int launch_i8_few_tokens(const void *x, const float *x_scale, const void *w8, const float *w_scale, const float *bias, int64_t M, int64_t N,
                         int64_t K, int act, void *out, cudaStream_t stream) {
  const FewArgs a{x, x_scale, static_cast<const int8_t *>(w8), w_scale, bias, static_cast<__nv_bfloat16 *>(out), (int)M, (int)N, (int)K, act};
  if (!x_scale) return launch_few<1, 1, true>(a, stream);
  // more weight rows to a block as the tokens grow: every block reads all of x
  if (M <= 8) return launch_few<1, 1, false>(a, stream);
  if (M <= 16) return launch_few<1, 2, false>(a, stream);
  return launch_few<2, 4, false>(a, stream);
}

}  // namespace osdp

using namespace osdp;

extern "C" int osdp_quantize_rows_i8(const void *x, int64_t M, int64_t K, void *q, float *scale, void *stream) {
  if (M < 0 || K <= 0 || M > ((int64_t)1 << 30) || K > OSDP_I8_MAX_K) return OSDP_ERR_BAD_SHAPE;
  if (K & 7) return OSDP_ERR_ALIGNMENT;
  if (M == 0) return OSDP_OK;
  if (!x || !q || !scale) return OSDP_ERR_NULL_POINTER;
  if (!aligned_to(x, 16) || !aligned_to(q, 8) || !aligned_to(scale, 4)) return OSDP_ERR_ALIGNMENT;
  return launch_i8_quantize(x, M, K, q, scale, static_cast<cudaStream_t>(stream));
}

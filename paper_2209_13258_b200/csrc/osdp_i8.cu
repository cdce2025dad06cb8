// int8 operands of the serving path: the quantiser (one scale per row) and the product for a few tokens, which streams
// the weights.  Products of many tokens run on the tile kernel (tcgen05.mma.kind::i8, osdp_gemm.cuh).
#include "../../include/osdp.h"

#include <atomic>
#include <mutex>

#include "osdp_i8.h"
#include "osdp_internal.h"
#include "osdp_vec.cuh"

namespace osdp {
namespace {

// One row per team of warps: the row's largest magnitude, then its codes.  The row is read twice by its own threads;
// the second read comes from L1 / L2.  One token of 8192: 2.9 us, next to nothing but the launch; 8192 x 8192 59 us of 31 that its
// bytes take: the two loops' loads wait for one another.
__global__ void __launch_bounds__(256) quantize_rows_kernel(const __nv_bfloat16 *x, long long M, int K, int8_t *q, float *scale, int warps) {
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
    widen8(*reinterpret_cast<const uint4 *>(xr + c), f);
#pragma unroll
    for (int k = 0; k < 8; ++k) bits = max(bits, __float_as_uint(f[k]) & 0x7FFFFFFFu);
  }
  float top = warp_max_abs(__uint_as_float(bits));
  if (warps > 1) {
    if (lane == 0) red[warp] = top;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(TL) : "memory");
    for (int k = 0; k < warps; ++k) top = __uint_as_float(max(__float_as_uint(top), __float_as_uint(red[first_warp + k])));
  }
  const float step = int8_scale(top), inv = int8_inverse(step);
  for (int c = tl * 8; c < K; c += TL * 8) {
    float f[8];
    widen8(*reinterpret_cast<const uint4 *>(xr + c), f);
    *reinterpret_cast<uint2 *>(q + row * K + c) = to_int8x8(f, step, inv);
  }
  if (tl == 0) scale[row] = step;
}

// ---- Few tokens: the product is bound by reading W once; mma.sync (int8, exact int32 sums) takes W straight from
// registers.  (An mma.sync of 16 x 8 x 32 keeps an SM's quarter busy for about 40 cycles here, two for every 512 bytes of
// W and 16 tokens, so the memory is the longer part up to about 16 tokens.  dp4a is no way around it: eight per token
// and 512 bytes took 12 us per token at 32768 x 8192.)
//
// One block per SM.  Its 16 warps form groups of WK warps; a group walks units of 8 NT weight rows, each warp with a
// contiguous share of K, and the warps' sums meet in shared memory at the end of a unit.  A warp copies its pieces of W
// asynchronously into its own ring, stages ahead and on into the next unit, so that the stream from memory does not stop
// at a unit's end; a copy instruction covers whole 128-byte lines, and a lane then picks the pieces of its mma operands.  A stage is Q steps of 64 bytes per row:
// the instructions around one 64-byte step (512 bytes of W per warp) would by themselves take as long as the memory.
// The four words of a piece are used as operands of two mma whose k order is a permutation of the real one, the same
// for W and X, which a sum over k does not notice.
//
// Measured on B200 on ready-made codes (bf16 tokens: the quantiser's launch comes before), one token, 8192 x 8192 (67 MB of W):
// 15.6 us, 4300 GB/s, where the bare stream takes 13 us (a read that short does not reach the copy rate); 32768 x 8192: 45.5 us,
// 5900 GB/s; 8 tokens 54 us, 16 tokens 70 us.  With bf16 tokens 8192 x 8192 takes 20 us.
__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct FewArgs {
  const int8_t *x;
  const float *x_scale;
  const int8_t *w;
  const float *w_scale, *bias;
  __nv_bfloat16 *out;
  int M, N, K, act;
  int wk;                     // warps that share a unit (a power of two)
};
constexpr int FEW_WARPS = 16;
constexpr int X_SMEM = 66 * 1024;                                         // shared memory for the tokens where they fit

// T8: groups of eight tokens, NT: groups of eight weight rows per unit.
template <int T8, int NT>
struct FewShape {
  static constexpr int MT = (T8 + 1) / 2;                                 // 16-token tiles
  static constexpr int Q = 4 / NT;                                        // 64-byte steps of a stage
  static constexpr int STAGE = 8 * NT * 64 * Q;                           // 2 KB of W per warp
  static constexpr int STAGES = 4;
  static constexpr int OUT = 16 * MT * 8 * NT;                            // sums of a unit
  static constexpr int PITCH = OUT + 4;                                   // a warp's sums: the four words keep the readers below off each other's banks
  static constexpr int RING = FEW_WARPS * STAGES * STAGE;
  static constexpr int TURNS = MT * NT >= 8 ? 1 : 2;                      // buffers for the warps' sums: two units in turn where there is room
  static constexpr int PART = TURNS * FEW_WARPS * PITCH * 4;
  static constexpr int SMEM = RING + PART;                                // and the tokens, with XS
};

// XS: the tokens are copied to shared memory first (rows 64 bytes apart beyond K, so that two rows read together do not
// meet in a bank); otherwise they are read through L1.
template <int T8, int NT, bool XS>
__global__ void __launch_bounds__(32 * FEW_WARPS, 1) few_tokens_kernel(const __grid_constant__ FewArgs a) {
  using SH = FewShape<T8, NT>;
  constexpr int MT = SH::MT, Q = SH::Q, S = SH::STAGES, ROWS = 8 * NT, KSTAGE = 64 * Q;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float scales[16 * MT];
  int8_t *xs = reinterpret_cast<int8_t *>(smem + SH::SMEM);
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, kq = (lane & 3) * 16;
  const int K = a.K, M = a.M, N = a.N, WK = a.wk;
  const int group = warp / WK, wk = warp % WK, groups = FEW_WARPS / WK;
  const int units = (N + ROWS - 1) / ROWS, first = (int)blockIdx.x + group * (int)gridDim.x, stride = groups * (int)gridDim.x;
  // Nothing says that the weights were not written by the kernel before this one: only a prefetch into L2, where
  // whatever is written later lands as well, may run ahead of the wait.
  if (wk == 0) {
    for (int i = lane; i < 3 * ROWS; i += 32) {
      const long long row = (long long)(first + i / ROWS * stride) * ROWS + i % ROWS;
      if (row < N) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.w + row * K), "r"(K) : "memory");
    }
  }
  pdl_wait();

  const int all_stages = (K + KSTAGE - 1) / KSTAGE, share = (all_stages + WK - 1) / WK;
  const int k_first = wk * share * KSTAGE;                                // this warp's share of K: n_st stages from k_first
  const int n_st = min(max(all_stages - wk * share, 0), share);
  int f_unit = n_st > 0 ? first : units, f_st = 0, f_slot = 0;            // the stage that is copied next
  // A copy instruction brings COPY_ROWS rows of KSTAGE bytes.  16-byte piece c of row r lies at place c ^ 4 (r & 1) of the
  // row's 4 Q places, so that the eight lanes that read together (two rows, four pieces each) hit all banks.
  constexpr int PIECES = 4 * Q, COPY_ROWS = 32 / PIECES, COPIES = ROWS / COPY_ROWS;
  const int c_row = lane / PIECES, c_piece = lane % PIECES;
  const int8_t *f_w[COPIES];
  auto f_rows = [&]() {   // rows past the end read the last row: in bounds, and their sums are not stored
#pragma unroll
    for (int n = 0; n < COPIES; ++n) f_w[n] = a.w + (long long)min(f_unit * ROWS + n * COPY_ROWS + c_row, N - 1) * K + (k_first + c_piece * 16);
  };
  f_rows();
  uint8_t *ring = smem + warp * (S * SH::STAGE);
  const uint32_t ring_u32 = static_cast<uint32_t>(__cvta_generic_to_shared(ring)) + (uint32_t)(c_row * KSTAGE + (c_piece ^ ((c_row & 1) << 2)) * 16);
  auto fetch = [&]() {
    if (f_unit < units) {
      const uint32_t to = ring_u32 + (uint32_t)(f_slot * SH::STAGE);
      const bool there = k_first + f_st * KSTAGE + c_piece * 16 < K;   // K is a multiple of 16: a piece is whole, or zeros are written
#pragma unroll
      for (int n = 0; n < COPIES; ++n)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + (uint32_t)(n * COPY_ROWS * KSTAGE)), "l"(there ? f_w[n] : a.w), "r"(there ? 16 : 0) : "memory");
      if (++f_st == n_st) {
        f_st = 0;
        f_unit += stride;
        f_rows();
      } else {
#pragma unroll
        for (int n = 0; n < COPIES; ++n) f_w[n] += KSTAGE;
      }
    }
    if (++f_slot == S) f_slot = 0;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll 1
  for (int s = 0; s < S - 1; ++s) fetch();

  if (threadIdx.x < 16 * MT) scales[threadIdx.x] = (int)threadIdx.x < M ? a.x_scale[threadIdx.x] : 0.f;
  if (XS) {
    const int pieces = K / 16;
    for (int i = threadIdx.x; i < M * pieces; i += blockDim.x) {
      const int m = i / pieces, c = i - m * pieces;
      *reinterpret_cast<uint4 *>(xs + m * (K + 64) + c * 16) = *reinterpret_cast<const uint4 *>(a.x + (long long)m * K + c * 16);
    }
  }
  __syncthreads();
  const int8_t *x8 = (XS ? xs : a.x) + (k_first + kq);
  const int x_pitch = XS ? K + 64 : K;
  // tokens past the end read the last one: their sums are not stored
  const int8_t *x_row[T8];
#pragma unroll
  for (int t = 0; t < T8; ++t) x_row[t] = x8 + (long long)min(t * 8 + g, M - 1) * x_pitch;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  int slot = 0, turn = 0;
  // Numbers of barriers end at 15: groups of two warps or more are eight at most, a group of one warp needs none.
  auto group_sync = [&]() {
    if (WK > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(WK * 32) : "memory");
    else __syncwarp();
  };
  // The sums of a unit are added by all threads of the group: `per` adjacent lanes to an output, each a part of the warps.
  constexpr int OUTPUTS = T8 * 8 * ROWS;
  const int in_group = wk * 32 + lane;
  int per = 1;
  while (per < WK && per < 8 && 2 * per * OUTPUTS <= WK * 32) per *= 2;
  for (int unit = first; unit < units; unit += stride, turn = (turn + 1) % SH::TURNS) {
    // what the epilogue needs of this thread's first output's column, while the products run
    const int n_first = min(unit * ROWS + (in_group / per) % ROWS, N - 1);
    const float ws_first = a.w_scale[n_first], b_first = a.bias ? a.bias[n_first] : 0.f;
    int acc[MT][NT][4];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[t][n][j] = 0;
#pragma unroll 1
    for (int st = 0; st < n_st; ++st) {     // the loop is the warp's: mma.sync needs every lane
      const int off = st * KSTAGE;
      const bool whole = k_first + off + KSTAGE <= K;
      __syncwarp();      // every lane has read the slot that is filled now
      fetch();
      asm volatile("cp.async.wait_group %0;" ::"n"(S - 1) : "memory");
      __syncwarp();      // every lane's copies of this stage have landed
      const uint8_t *from = ring + slot * SH::STAGE + g * KSTAGE + kq;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const bool there = whole || k_first + off + kq + q * 64 < K;
        uint4 x[2 * MT];
#pragma unroll
        for (int t = 0; t < 2 * MT; ++t) x[t] = (t < T8 && there) ? *reinterpret_cast<const uint4 *>(x_row[t < T8 ? t : 0] + off + q * 64) : zero;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint4 b = *reinterpret_cast<const uint4 *>(from + n * 8 * KSTAGE + ((q ^ (g & 1)) * 64));
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            mma_s8(acc[t][n], x[2 * t].x, x[2 * t + 1].x, x[2 * t].y, x[2 * t + 1].y, b.x, b.y);
            mma_s8(acc[t][n], x[2 * t].z, x[2 * t + 1].z, x[2 * t].w, x[2 * t + 1].w, b.z, b.w);
          }
        }
      }
      if (++slot == S) slot = 0;
    }
    int *sums = reinterpret_cast<int *>(smem + SH::RING) + (turn * FEW_WARPS + group * WK) * SH::PITCH;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h)   // token g (+ 8) of the tile, weight rows 2 (lane & 3) + (0, 1) of the group
          if (2 * t + h < T8)
            *reinterpret_cast<int2 *>(sums + wk * SH::PITCH + (t * 16 + g + 8 * h) * ROWS + n * 8 + 2 * (lane & 3)) = make_int2(acc[t][n][2 * h], acc[t][n][2 * h + 1]);
    // with two buffers the only barrier of a unit: this buffer is written again only after the next one
    group_sync();
    for (int i = in_group / per; i < OUTPUTS; i += WK * 32 / per) {   // whole warps, or all their lanes, leave together
      int s = 0;
      for (int q = in_group % per; q < WK; q += per) s += sums[q * SH::PITCH + i];
      for (int o = per / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
      const int m = i / ROWS, n = unit * ROWS + i % ROWS;
      if (m < M && n < N && in_group % per == 0) {
        const bool f1 = i == in_group / per;
        const float f = __fadd_rn(dequantise1(s, scales[m], f1 ? ws_first : a.w_scale[n]), f1 ? b_first : a.bias ? a.bias[n] : 0.f);
        a.out[(long long)m * N + n] = __float2bfloat16_rn(gelu1(f, a.act));
      }
    }
    if (SH::TURNS == 1) group_sync();
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <int T8, int NT, bool XS>
int launch_few(const FewArgs &args, cudaStream_t stream) {
  using SH = FewShape<T8, NT>;
  int sms = 0;
  const int rc = sm_count(&sms);
  if (rc) return rc;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return report_cuda(e);
  static std::atomic<bool> ready[64];
  static std::mutex setup;
  constexpr int most = SH::SMEM + (XS ? X_SMEM : 0);
  if (!ready[dev & 63].load(std::memory_order_acquire)) {
    std::lock_guard<std::mutex> lock(setup);
    e = cudaFuncSetAttribute(few_tokens_kernel<T8, NT, XS>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e != cudaSuccess) return report_cuda(e);
    ready[dev & 63].store(true, std::memory_order_release);
  }
  FewArgs a = args;
  // as many warps to a unit as leave each two stages of it
  const int64_t stages = cdiv(a.K, 64 * SH::Q);
  a.wk = FEW_WARPS;
  while (a.wk > 1 && stages < 2 * a.wk) a.wk /= 2;
  int64_t blocks = cdiv(a.N, 8 * NT);
  if (blocks > sms) blocks = sms;
  return launch_overlapped(few_tokens_kernel<T8, NT, XS>, dim3((unsigned)blocks), dim3(32 * FEW_WARPS),
                           (size_t)SH::SMEM + (XS ? (size_t)a.M * (a.K + 64) : 0), 1, stream, a);
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

// A tile kernel's block streams 64 weight rows over all of K by itself, so its time goes with K, and with few columns most
// SMs are idle; this one's goes with N K, and from about 16 tokens on with the mma.  Measured on B200 (us, few / tile):
// 24 tokens 2048 x 8192 10 / 24, 8192 x 2048 10 / 13, 8192 x 8192 32 / 27; 48 tokens 2048 x 2048 7.9 / 11.5, 2048 x 8192
// 14 / 24, 8192 x 2048 14 / 13, 8192 x 8192 49 / 28, 32768 x 8192 156 / 68; 16 tokens 32768 x 8192 74 / 67.
bool i8_few_tokens(int64_t M, int64_t N, int64_t K) {
  if (M > 64) return false;
  return M <= 16 || N <= 4096 || (M <= 32 && N * K <= ((int64_t)1 << 25));
}

int launch_i8_few_tokens(const void *x8, const float *x_scale, const void *w8, const float *w_scale, const float *bias, int64_t M, int64_t N,
                         int64_t K, int act, void *out, cudaStream_t stream) {
  const FewArgs a{static_cast<const int8_t *>(x8), x_scale, static_cast<const int8_t *>(w8), w_scale, bias, static_cast<__nv_bfloat16 *>(out),
                  (int)M, (int)N, (int)K, act, 0};
  // more weight rows to a unit as the tokens grow: every unit reads all of x
  if (M <= 8 && M * (K + 64) <= X_SMEM) return launch_few<1, 1, true>(a, stream);   // 8 tokens, 32768 x 8192: 62 -> 53 us
  if (M <= 8) return launch_few<1, 1, false>(a, stream);
  if (M <= 16) return launch_few<2, 2, false>(a, stream);   // (no faster from shared memory: 16 tokens, 8200 x 2064 7.3 / 8.2 us)
  if (M <= 32) return launch_few<4, 2, false>(a, stream);
  if (M <= 48) return launch_few<6, 2, false>(a, stream);
  return launch_few<8, 2, false>(a, stream);
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

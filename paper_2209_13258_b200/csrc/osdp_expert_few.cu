// The experts' products for a few rows each: a stream of the weights of the experts that have any.
#include "../../include/osdp.h"

#include <atomic>
#include <mutex>

#include "osdp_experts.h"
#include "osdp_internal.h"
#include "osdp_vec.cuh"

namespace osdp {
namespace {

// Out of K weights a row uses each once, so with a handful of rows the product is bound by reading the weights once.
//
// One block per SM.  Its 16 warps form groups of WK; a group walks units of 16 weight rows of an expert that has rows, each warp
// with a contiguous share of K, and the warps' sums meet in shared memory at the end of a unit, in a fixed order.  A warp
// copies its pieces of W asynchronously into a ring of its own, STAGES ahead and on into the next unit, so that the stream does not
// stop at a unit's end.  The weights are the 16-row operand of mma.sync (bf16, fp32 sums), eight rows of X the other one: the
// tensor work is no part of the time, and a lane takes 16 bytes of a row for two mma whose k order is a permutation of the
// real one, the same for W and X, which a sum over k does not notice.  X is read through L1 one step ahead.
//
// An expert may have any number of rows: 8 T8 of them are done in one reading of its weights, and more in further ones.
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct FewArgs {
  const __nv_bfloat16 *x, *w;
  const float *bias;
  const int32_t *plan;
  __nv_bfloat16 *out, *z;
  int E, N, K, act;
  int wk;                     // warps that share a unit (a power of two)
};
constexpr int WARPS = 16, ROWS = 16, KSTAGE = 64, STAGES = 4, STAGE = ROWS * KSTAGE * 2;
constexpr int RING = WARPS * STAGES * STAGE;

template <int T8>
struct FewShape {
  static constexpr int TOKENS = 8 * T8, PITCH = ROWS * TOKENS + 4;        // a warp's sums of a unit, off the other warps' banks
  static constexpr int TURNS = 2;                                         // two units in turn: one barrier for each
  static constexpr int SMEM = RING + TURNS * WARPS * PITCH * 4;
};

template <int T8>
__global__ void __launch_bounds__(32 * WARPS, 1) expert_few_kernel(const __grid_constant__ FewArgs a) {
  using SH = FewShape<T8>;
  extern __shared__ __align__(128) uint8_t smem[];
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int K = a.K, N = a.N, WK = a.wk;
  const int group = warp / WK, wk = warp % WK, groups = WARPS / WK;
  pdl_wait();
  const int32_t *live = a.plan + plan_live(a.E), *offsets = a.plan + PLAN_OFFSETS, *counts = a.plan + plan_counts(a.E);
  const int each = (N + ROWS - 1) / ROWS;
  const int first = (int)blockIdx.x + group * (int)gridDim.x, stride = groups * (int)gridDim.x;
  // the first unit's expert and whether there is one: both looked up at once
  const int first_e = live[min(first / each, a.E - 1)], units = a.plan[plan_n_live(a.E)] * each;

  const int all_stages = (K + KSTAGE - 1) / KSTAGE, share = (all_stages + WK - 1) / WK;
  const int k_first = wk * share * KSTAGE, n_st = min(max(all_stages - wk * share, 0), share);
  // the stage that is copied next: unit, reading of it, stage
  int f_unit = n_st > 0 ? first : units, f_left = 0, f_st = 0, f_slot = 0;
  constexpr int COPIES = 4;                     // of 4 rows, 8 pieces of 16 bytes each
  const int c_row = lane >> 3, c_piece = lane & 7;
  const __nv_bfloat16 *f_w[COPIES];
  auto f_rows = [&](bool start) {       // rows past the end read the last one: in bounds, and their sums are not stored
    if (f_unit >= units) return;
    const int i = f_unit / each, e = start ? first_e : live[i], n0 = (f_unit - i * each) * ROWS;
    f_left = (counts[e] + SH::TOKENS - 1) / SH::TOKENS;
#pragma unroll
    for (int n = 0; n < COPIES; ++n) f_w[n] = a.w + ((long long)e * N + min(n0 + n * 4 + c_row, N - 1)) * K + (k_first + c_piece * 8);
  };
  f_rows(true);
  uint8_t *ring = smem + warp * (STAGES * STAGE);
  // 16-byte piece c of row r lies at place c ^ 4 (r & 1), so that the eight lanes that read together (two rows, four pieces
  // each) hit all banks
  const uint32_t ring_u32 = static_cast<uint32_t>(__cvta_generic_to_shared(ring)) + (uint32_t)(c_row * KSTAGE * 2 + (c_piece ^ ((c_row & 1) << 2)) * 16);
  auto fetch = [&]() {
    if (f_unit < units) {
      const uint32_t to = ring_u32 + (uint32_t)(f_slot * STAGE);
      const bool there = k_first + f_st * KSTAGE + c_piece * 8 < K;       // K is a multiple of 8: a piece is whole, or zeros are written
#pragma unroll
      for (int n = 0; n < COPIES; ++n)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + (uint32_t)(n * 4 * KSTAGE * 2)), "l"(there ? f_w[n] : a.w), "r"(there ? 16 : 0) : "memory");
      if (++f_st < n_st) {
#pragma unroll
        for (int n = 0; n < COPIES; ++n) f_w[n] += KSTAGE;
      } else {
        f_st = 0;
        if (--f_left > 0) {
#pragma unroll
          for (int n = 0; n < COPIES; ++n) f_w[n] -= (n_st - 1) * KSTAGE;
        } else {
          f_unit += stride;
          f_rows(false);
        }
      }
    }
    if (++f_slot == STAGES) f_slot = 0;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll 1
  for (int s = 0; s < STAGES - 1; ++s) fetch();

  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  int slot = 0, turn = 0;
  const int in_group = wk * 32 + lane, threads = WK * 32;
  // Numbers of barriers end at 15: groups of two warps or more are eight at most, a group of one warp needs none.
  auto group_sync = [&]() {
    if (WK > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(WK * 32) : "memory");
    else __syncwarp();
  };
  for (int unit = first; unit < units; unit += stride) {
    const int i = unit / each, e = live[i], n0 = (unit - i * each) * ROWS, count = counts[e];
    const long long off = offsets[e];
    const float *bias = a.bias ? a.bias + (long long)e * N : nullptr;
    for (int t0 = 0; t0 < count; t0 += SH::TOKENS, turn ^= 1) {
      const int here = min(count - t0, SH::TOKENS);
      float acc[T8][4];
      const __nv_bfloat16 *x_row[T8];
#pragma unroll
      for (int t = 0; t < T8; ++t) {
        // rows past the last one read it again: their sums are not stored
        x_row[t] = a.x + (off + t0 + min(t * 8 + g, here - 1)) * K + (k_first + q * 8);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[t][j] = 0.f;
      }
      uint4 x[2][T8];
      auto load_x = [&](int step) {     // of 32 k
#pragma unroll
        for (int t = 0; t < T8; ++t) {
          const bool there = t * 8 < here && k_first + step * 32 + q * 8 < K;
          x[step & 1][t] = there ? *reinterpret_cast<const uint4 *>(x_row[t] + step * 32) : zero;
        }
      };
      if (n_st > 0) load_x(0);
#pragma unroll 1
      for (int st = 0; st < n_st; ++st) {       // the loop is the warp's: mma.sync needs every lane
        __syncwarp();      // every lane has read the slot that is filled now
        fetch();
        load_x(2 * st + 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        __syncwarp();      // every lane's copies of this stage have landed
        const uint8_t *from = ring + slot * STAGE + g * KSTAGE * 2;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int place = ((4 * h + q) ^ ((g & 1) << 2)) * 16;
          const uint4 lo = *reinterpret_cast<const uint4 *>(from + place);
          const uint4 hi = *reinterpret_cast<const uint4 *>(from + 8 * KSTAGE * 2 + place);
#pragma unroll
          for (int t = 0; t < T8; ++t) {
            if (T8 == 1 || t * 8 < here) {
              mma_bf16(acc[t], lo.x, hi.x, lo.y, hi.y, x[h][t].x, x[h][t].y);
              mma_bf16(acc[t], lo.z, hi.z, lo.w, hi.w, x[h][t].z, x[h][t].w);
            }
          }
          if (h == 0 && st + 1 < n_st) load_x(2 * st + 2);
        }
        if (++slot == STAGES) slot = 0;
      }
      if (WK == 1) {
#pragma unroll
        for (int t = 0; t < T8; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int tok = t * 8 + 2 * q + (j & 1), n = n0 + g + (j & 2) * 4;
            if (tok < here && n < N) {
              const float s = acc[t][j] + (bias ? bias[n] : 0.f);
              const long long at = (off + t0 + tok) * N + n;
              if (a.z) a.z[at] = __float2bfloat16_rn(s);
              a.out[at] = __float2bfloat16_rn(expert_gelu1(s, a.act));
            }
          }
        continue;
      }
      float *sums = reinterpret_cast<float *>(smem + RING) + (turn * WARPS + group * WK) * SH::PITCH;
#pragma unroll
      for (int t = 0; t < T8; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)   // weight row g (+ 8), rows 2 q + (0, 1) of X
          if (t * 8 < here) sums[wk * SH::PITCH + (t * 8 + 2 * q + (j & 1)) * ROWS + g + (j & 2) * 4] = acc[t][j];
      group_sync();        // the only barrier: this buffer is written again only after the next one
      for (int o = in_group; o < here * ROWS; o += threads) {
        const int n = n0 + o % ROWS;
        float s = 0.f;
        for (int p = 0; p < WK; ++p) s += sums[p * SH::PITCH + o];
        if (n < N) {
          if (bias) s += bias[n];
          const long long at = (off + t0 + o / ROWS) * N + n;
          if (a.z) a.z[at] = __float2bfloat16_rn(s);
          a.out[at] = __float2bfloat16_rn(expert_gelu1(s, a.act));
        }
      }
    }
    // the rows up to the next expert's, 16 columns of them
    const int between = offsets[e + 1] - (int)off - count;
    for (int o = in_group; o < between * 2; o += threads) {
      const int n = n0 + (o & 1) * 8;
      if (n < N) {
        const long long at = (off + count + (o >> 1)) * N + n;
        *reinterpret_cast<uint4 *>(a.out + at) = zero;
        if (a.z) *reinterpret_cast<uint4 *>(a.z + at) = zero;
      }
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// Warps to a unit: as few as keep most of the warps busy, with at most 2048 of K for each and two stages at least.  One token, two
// experts 2048 -> 8192: 1 / 2 / 4 / 16 warps 24.4 / 17.0 / 17.4 / 21.3 us; 8192 -> 2048 (a quarter of the units): 99 / 52 / 29 / 20 us,
// with 8 19.4; eight tokens, eight experts 8192 -> 8192: 209 / 174 / 161 / 171 us.
int warps_to_unit(int64_t live, int64_t N, int64_t K, int sms) {
  int wk = 1;
  while (wk < WARPS && (live * cdiv(N, ROWS) * wk < (int64_t)sms * WARPS * 6 / 7 || K > 2048 * wk)) wk *= 2;
  while (wk > 1 && cdiv(K, KSTAGE) < 2 * wk) wk /= 2;
  return wk;
}

template <int T8>
int launch_few(FewArgs a, int64_t live, cudaStream_t stream) {
  using SH = FewShape<T8>;
  int sms = 0, dev = 0;
  const int rc = sm_count(&sms);
  if (rc) return rc;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return report_cuda(e);
  if (dev < 0 || dev >= 64) return report_cuda(cudaErrorInvalidDevice);
  static std::atomic<bool> ready[64];
  static std::mutex setup;
  if (!ready[dev].load(std::memory_order_acquire)) {
    std::lock_guard<std::mutex> lock(setup);
    e = cudaFuncSetAttribute(expert_few_kernel<T8>, cudaFuncAttributeMaxDynamicSharedMemorySize, SH::SMEM);
    if (e != cudaSuccess) return report_cuda(e);
    ready[dev].store(true, std::memory_order_release);
  }
  a.wk = warps_to_unit(live, a.N, a.K, sms);
  int64_t blocks = live * cdiv(a.N, ROWS);
  if (blocks > sms) blocks = sms;
  return launch_overlapped(expert_few_kernel<T8>, dim3((unsigned)blocks), dim3(32 * WARPS), (size_t)SH::SMEM, 1, stream, a);
}

}  // namespace

// The tile kernel streams the weights as well where it has a tile for each SM, but a k-block takes it 0.2 us, and it has some 5 us
// before its first and behind its last.  Measured on B200 (us, few / tile), T x top_k of E, K -> N.  Up to eight rows to an expert:
// 1 x 2 of 8, 2048 -> 8192 17.1 / 17.2, 8192 -> 2048 19.4 / 36.7, 1024 -> 1024 3.7 / 8.8; 4 x 4 of 64, 1024 -> 1024 10.2 / 15.8;
// 1 x 8 of 64, 2048 -> 2048 20.4 / 22.5; 8 x 2 of 8, 8192 -> 8192 159 / 160.  With more, where the tiles are few: 16 x 2 of 2,
// 8192 -> 2048 20.7 / 36.5; or the weights: 100 of 16, 512 -> 512 4.6 / 7.6; 56 x 2 of 55, 192 -> 408 5.2 / 11.4; 79 x 2 of 68, 400 -> 480
// 9.2 / 14.4; but 37 x 2 of 16, 1032 -> 2064 22.9 / 19.7, 64 x 2 of 16, 2048 -> 2048 38 / 29, 32 x 2 of 64, 1024 -> 1024 33 / 26.
//
// Only the device knows how many rows an expert has.  Should all tokens choose the same ones, these are read once for every 16
// tokens by a few warps, 0.55 us for 64 of K a warp, while the tile kernel takes no longer than otherwise.  More than 40 such steps
// in the worst case (at most twice the tile kernel's time) are not risked: 512 x 1 of 32, 8192 -> 256 takes 75 / 42 with even
// choices and 520 / 33 if all are one; 200 x 1 of 20, 1024 -> 520 10.4 / 9.3 and 38 / 8.7; but 79 x 2 of 68 21.8 / 12.1, 64 x 2 of 16, 2048 -> 128
// 5.7 / 12.0 and 10.5 / 11.7.
bool expert_few_rows(int64_t T, int top_k, int E, int64_t N, int64_t K) {
  const int64_t n = T * top_k, used = n < E ? n : E;
  if (used * cdiv(N, ROWS) >= ((int64_t)1 << 30)) return false;
  if (T <= 8) return true;
  int sms = 0;
  if (n > 16 * used || (used * cdiv(N, 128) > 64 && used * N * K >= (1 << 24)) || sm_count(&sms)) return false;
  return cdiv(T, 16) * cdiv(cdiv(K, KSTAGE), warps_to_unit(used, N, K, sms)) <= 40;
}

int launch_expert_few(const void *rows, const int32_t *plan, const void *w, const float *bias, int64_t T, int top_k, int E, int64_t N, int64_t K, int act,
                      void *out, void *z_save, cudaStream_t stream) {
  const FewArgs a{static_cast<const __nv_bfloat16 *>(rows), static_cast<const __nv_bfloat16 *>(w), bias, plan, static_cast<__nv_bfloat16 *>(out),
                  static_cast<__nv_bfloat16 *>(z_save), E, (int)N, (int)K, act, 0};
  const int64_t n = T * top_k, used = n < E ? n : E;
  // an expert has T rows at most, unless a token chose it twice
  return T <= 8 ? launch_few<1>(a, used, stream) : launch_few<2>(a, used, stream);
}

}  // namespace osdp

// Norms, gate and residual sum between two blocks, forward and backward:
//   p = N_post(y),  r = alpha x + beta gate (.) p,  u = N_pre(r).
// HBM-bound: the forward reads x, y and writes r, u once; the backward reads y, r, du, dr and writes dx, dy once, the
// sums over rows (weights' gradients) are kept in registers over all rows of a thread block.  Measured on B200 against a
// copy rate of 6547 GB/s, at full clocks: 16384 x 8192 RMS bf16 forward 161 us (6690 GB/s of what has to move), backward 261 us
// (6170); in a loop under the power cap 185 and 301.  Layer norm on an fp32 stream, 8192 x 2048, forward 48 us (4170), backward 89
// (3400): latency, 43 % of the issue slots are taken.
#include "../../include/osdp.h"

#include <atomic>
#include <cmath>
#include <mutex>

#include "osdp_internal.h"
#include "osdp_vec.cuh"

namespace osdp {
namespace {

struct RowNorm {
  int has;          // a norm at all (RMS or layer)
  int layer;        // layer norm: subtracts the mean
  float eps;
  const float *w, *b;
};

// Sum over a team of `warps` warps (all of them call it).  `red`: two buffers with a float per warp of the block, used in
// turn, so that one barrier per call is enough: a buffer is written again only after the barrier of the call in between,
// which every reader of the buffer has passed.
__device__ __forceinline__ float team_sum(float v, int warps, int first_warp, int warp, int lane, int bar_id, float *red, int &turn) {
  v = warp_sum(v);
  if (warps == 1) return v;
  float *buf = red + turn * 32;
  turn ^= 1;
  if (lane == 0) buf[warp] = v;
  asm volatile("bar.sync %0, %1;" ::"r"(bar_id), "r"(warps * 32) : "memory");
  float s = 0.f;
  for (int q = 0; q < warps; ++q) s += buf[first_warp + q];
  return s;
}

// ------------------------------------------------------------------------------------------------ forward

struct FwdArgs {
  const void *x;
  const __nv_bfloat16 *y;
  void *r;
  void *u;
  float *u_scale;
  float4 *stats;
  const float *gate;
  float alpha, beta;
  RowNorm post, pre;
  long long M;
  int D;
  int warps;       // of a row's team
};

__device__ __forceinline__ void weights8(const float *w, int col, float fill, float (&f)[8]) {
  if (w) {
    const float4 a = *reinterpret_cast<const float4 *>(w + col), b = *reinterpret_cast<const float4 *>(w + col + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = fill;
  }
}

// Few rows, and int8 u (which needs the row's largest magnitude before anything is written).  A team of `warps` warps
// owns a row; a lane holds V vectors of eight adjacent channels, vector j at channel
// (j * 32 * warps + lane of the team) * 8, so that a warp's accesses are whole lines.  The row stays in registers
// between the two norms: sums are taken over the values themselves (mean first, then squared distances from it), not
// as differences of moments.
template <typename RT, int V>
__global__ void __launch_bounds__(1024) block_norm_fwd_kernel(const __grid_constant__ FwdArgs a) {
  __shared__ float red[2 * 32];
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int team = warp / a.warps, first_warp = team * a.warps;
  const int tl = (warp - first_warp) * 32 + lane, TL = a.warps * 32;
  const int teams = (blockDim.x >> 5) / a.warps;
  const long long row = (long long)blockIdx.x * teams + team;
  if (row >= a.M) return;
  int turn = 0;
  auto sum1 = [&](float s) { return team_sum(s, a.warps, first_warp, warp, lane, 1 + team, red, turn); };
  pdl_wait();
  const float inv_d = 1.0f / (float)a.D;
  const RT *xr = static_cast<const RT *>(a.x) + row * a.D;
  float v[V][8];     // r, then u
  uint4 yv[V];
  bool act[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int col = (j * TL + tl) * 8;
    act[j] = col < a.D;
    yv[j] = make_uint4(0u, 0u, 0u, 0u);
    if (act[j]) {
      if (a.y) yv[j] = load16(a.y + row * a.D + col);
      load8(xr + col, v[j]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[j][k] = 0.f;
    }
  }
  float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
  if (a.y) {
    float mean = 0.f, rstd = 1.f;
    if (a.post.has) {
      if (a.post.layer) {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float f[8];
          widen8(yv[j], f);
#pragma unroll
          for (int k = 0; k < 8; ++k) s += f[k];
        }
        mean = sum1(s) * inv_d;
      }
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float f[8];
        widen8(yv[j], f);
        if (act[j]) {
#pragma unroll
          for (int k = 0; k < 8; ++k) s = fmaf(f[k] - mean, f[k] - mean, s);
        }
      }
      rstd = rsqrtf(fmaf(sum1(s), inv_d, a.post.eps));
      st.x = mean;
      st.y = rstd;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (!act[j]) continue;
      const int col = (j * TL + tl) * 8;
      float f[8], w[8], b[8], g[8];
      widen8(yv[j], f);
      weights8(a.post.w, col, 1.f, w);
      weights8(a.post.b, col, 0.f, b);
      weights8(a.gate, col, 1.f, g);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float p = fmaf((f[k] - mean) * rstd, w[k], b[k]);
        v[j][k] = fmaf(a.beta * g[k], p, a.alpha * v[j][k]);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) v[j][k] *= a.alpha;
  }
  if (a.r) {
    RT *rr = static_cast<RT *>(a.r) + row * a.D;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (act[j]) store8(rr + (j * TL + tl) * 8, v[j]);
  }
  if (a.pre.has) {
    float mean = 0.f;
    if (a.pre.layer) {
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) s += v[j][k];
      mean = sum1(s) * inv_d;
    }
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (act[j]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s = fmaf(v[j][k] - mean, v[j][k] - mean, s);
      }
    }
    const float rstd = rsqrtf(fmaf(sum1(s), inv_d, a.pre.eps));
    st.z = mean;
    st.w = rstd;
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (!act[j]) continue;
      const int col = (j * TL + tl) * 8;
      float w[8], b[8];
      weights8(a.pre.w, col, 1.f, w);
      weights8(a.pre.b, col, 0.f, b);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[j][k] = fmaf((v[j][k] - mean) * rstd, w[k], b[k]);
        top = __uint_as_float(max(__float_as_uint(top), __float_as_uint(v[j][k]) & 0x7FFFFFFFu));
      }
      if (!a.u_scale) store8(static_cast<__nv_bfloat16 *>(a.u) + row * a.D + col, v[j]);
    }
    if (a.u_scale) {
      top = warp_max_abs(top);
      if (a.warps > 1) {
        float *buf = red + turn * 32;
        if (lane == 0) buf[warp] = top;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(TL) : "memory");
        for (int q = 0; q < a.warps; ++q)
          top = __uint_as_float(max(__float_as_uint(top), __float_as_uint(buf[first_warp + q])));
      }
      const float scale = int8_scale(top), inv = int8_inverse(scale);
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (act[j])
          *reinterpret_cast<uint2 *>(static_cast<int8_t *>(a.u) + row * a.D + (j * TL + tl) * 8) = to_int8x8(v[j], scale, inv);
      if (tl == 0) a.u_scale[row] = scale;
    }
  }
  if (a.stats && tl == 0) a.stats[row] = st;
}

// ------------------------------------------------------------------------------------------------ teams over many rows
//
// Kernels for many rows: one block per SM, or a cluster of CL = 2 or 4 blocks that share their rows where a row does not
// fit one (registers: 8192 channels; shared memory: three rows of what a kernel reads), teams of warps that take rows in a fixed stride, a lane with the same two vectors of eight channels for all of them, so
// that weights stay in its registers.  What a lane needs of the next rows it copies itself, asynchronously, into its own
// slots of a ring in shared memory; no thread reads another's slots, so the ring needs no barrier, and several rows per
// team are in flight whatever the arithmetic does.  Rows are worked on in a software pipeline: a step does the last part
// of one row and the first part of the next, whose sums over the row are then exchanged with ONE barrier, so that its
// latency and that of the shuffles is met with independent work.

// Threads of a block: what the registers allow without spills (spilled values come back from L2, there is hardly any L1
// beside the ring: the layer norm's backward took 1.5 times as long with 512 threads of 128 registers).
constexpr int fwd_warps(bool layer, bool fp32, int cl) { return layer && fp32 && cl > 1 ? 12 : 16; }
constexpr int bwd_warps(bool layer) { return layer ? 12 : 16; }
constexpr int MAX_STAGES = 6;
constexpr int ROW_MAX_BLOCKS = 160;   // partial sums over rows that the workspace holds

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// waits until at most `left` (0 ... MAX_STAGES - 2) of this thread's groups are still in flight
__device__ __forceinline__ void cp_async_wait(int left) {
  switch (left) {
    case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
    case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
    case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
    case 3: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
    default: asm volatile("cp.async.wait_group 4;" ::: "memory"); break;
  }
}

// Sums of N values over the warp; every lane returns the sum with index `idx` (a function of the lane).  Halving the
// values at each exchange takes N - 1 + log2(32 / N) shuffles instead of 5 N.
template <int N>
__device__ __forceinline__ float warp_sum_scattered(float (&v)[N], int lane, int &idx) {
  static_assert(N == 2 || N == 4 || N == 8, "");
  idx = 0;
  int o = 16;
#pragma unroll
  for (int n = N / 2; n > 0; n >>= 1, o >>= 1) {
    const bool up = (lane & o) != 0;
#pragma unroll
    for (int k = 0; k < n; ++k) {
      const float give = up ? v[k] : v[k + n];
      v[k] = (up ? v[k + n] : v[k]) + __shfl_xor_sync(0xFFFFFFFFu, give, o);
    }
    idx += up ? n : 0;
  }
  float s = v[0];
  for (; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  return s;
}

// channels of a row that a block of a cluster holds (the last one may have fewer)
__host__ __device__ constexpr int block_channels(int D, int cl) { return (D / 8 + cl - 1) / cl * 8; }

struct TeamShape {
  int warps;    // of a team
  int teams;    // of a block
  int stages;
};

// Where a thread stands, and the exchange of a row's partial sums.
template <int CL, int NS>
struct Team {
  int warp, lane, team, first_warp, tl, TL, warps, unit, units, c_begin, c_end, turn;
  uint32_t rank;
  float *red;    // [2 turns][CL blocks][16 warps][NS]
  static constexpr int RED_FLOATS = 2 * CL * 16 * NS;

  __device__ __forceinline__ void init(const TeamShape &sh, int D, float *red_) {
    warp = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    warps = sh.warps;
    team = warp / warps;
    first_warp = team * warps;
    tl = (warp - first_warp) * 32 + lane;
    TL = warps * 32;
    rank = 0;
    if (CL > 1) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    unit = (int)blockIdx.x / CL;
    units = (int)gridDim.x / CL;
    c_begin = min((int)rank * block_channels(D, CL), D);
    c_end = min(c_begin + block_channels(D, CL), D);
    red = red_;
    turn = 0;
  }
  // channels that warp w of the team (0 ... warps - 1) of block `blk` holds
  __device__ __forceinline__ float channels(int blk, int w, int D) const {
    const int width = min(block_channels(D, CL), max(D - blk * block_channels(D, CL), 0));
    return (float)(min(max(width - w * 256, 0), 256) + min(max(width - (TL + w * 32) * 8, 0), 256));
  }
  __device__ __forceinline__ float *buffer() const { return red + turn * (RED_FLOATS / 2); }
  // Makes this warp's sums visible to the team.  A lane brings the sum with index idx; exactly the lanes with `mine`
  // set write.  Two buffers in turn: one is written again only after the barrier of the exchange in between, which
  // every reader of it has passed.
  __device__ __forceinline__ void publish(float s, int idx, bool mine) {
    float *at = buffer() + ((int)rank * 16 + warp) * NS + idx;
    if (mine) {
      *at = s;
      const uint32_t local = static_cast<uint32_t>(__cvta_generic_to_shared(at));
#pragma unroll
      for (uint32_t q = 1; q < CL; ++q)
        asm volatile("{\n\t.reg .b32 ra;\n\tmapa.shared::cluster.u32 ra, %0, %1;\n\tst.shared::cluster.f32 [ra], %2;\n\t}" ::"r"(local), "r"((rank + q) % CL), "f"(s) : "memory");
    }
  }
  // The exchange's barrier in two halves.  Across a cluster the first half comes right after publish(): as a release it
  // waits for the global stores before it to be acknowledged, so a step's own stores go between the halves.
  __device__ __forceinline__ void arrive() const {
    if (CL > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // the teams of a cluster go through it together
  }
  __device__ __forceinline__ void wait() const {
    if (CL > 1) {
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else if (warps > 1) {
      asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(TL) : "memory");
    } else {
      __syncwarp();
    }
  }
  // The exchanged sums, added over the warps that share the row (`add` is given a warp's sums and its number in count
  // order).  Up to four warps: every lane reads them all.  More: lane l takes the warps l, l + 32, ... (block by block)
  // and the lanes' totals are added by shuffles, where a loop would be a chain of up to 16 CL reads per row.
  template <int N, typename F>
  __device__ __forceinline__ void total(const float *buf, float (&t)[N], F add) const {
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] = 0.f;
    if (CL == 1 && warps <= 4) {
#pragma unroll
      for (int w = 0; w < 4; ++w)
        if (w < warps) add(t, buf + (first_warp + w) * NS, w);
      return;
    }
#pragma unroll
    for (int p = 0; p < (CL + 1) / 2; ++p) {
      const int slot = lane + 32 * p, b = slot >> 4, w = slot & 15;
      if (b < CL && w < warps) add(t, buf + (b * 16 + first_warp + w) * NS, b * 16 + w);
    }
    int idx;
    const float s = warp_sum_scattered<N>(t, lane, idx);
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] = __shfl_sync(0xFFFFFFFFu, s, lane_of<N>(k));
  }
  // a lane that warp_sum_scattered<N> leaves with sum k
  template <int N>
  static __device__ __forceinline__ constexpr int lane_of(int k) {
    return N == 2 ? (k & 1) * 16 : N == 4 ? (k >> 1) * 16 + (k & 1) * 8 : (k >> 2) * 16 + ((k >> 1) & 1) * 8 + (k & 1) * 4;
  }
};

// ------------------------------------------------------------------------------------------------ forward, many rows

// A step finishes row i (u), does row i + 1 up to its sums (r) and takes the sums of row i + 2's y.  The variance is
// taken per lane about the lane's own mean; lanes' and then warps' means and squared distances are merged, which is as
// safe as a second pass over the row and needs no second exchange.
// What bounds it: RMS on a bf16 stream the memory (97 % of the copy rate in its steady state); otherwise about 35
// instructions a channel and the latency of the exchange, both with 16 warps an SM.  Before the pipeline (a row per block,
// loads, sums and stores one after another) 16384 x 8192 took 373 us; with scalar arithmetic 187 us.
// LAYER: either norm subtracts a mean.  FULL: y, both norms, r and u are there (the form between two blocks); without
// it each may be absent, which costs branches.
template <typename RT, bool LAYER, int CL, bool FULL>
__global__ void __launch_bounds__(32 * fwd_warps(LAYER, sizeof(RT) == 4, CL), 1) block_norm_fwd_rows_kernel(const __grid_constant__ FwdArgs a, const TeamShape sh) {
  constexpr int RP = sizeof(RT) / 2;             // 16-byte pieces of a residual vector
  constexpr int PIECES = 1 + RP;                 // y, x
  constexpr int NS = LAYER ? 4 : 2;              // y's, r's: mean and squared distances, or squares alone
  constexpr bool LATE = CL > 1;                  // a step's stores go between the halves of the barrier (Team::arrive); within
                                                 // one block they are better early (16384 x 8192 RMS: 173 against 197 us)
  extern __shared__ __align__(16) uint8_t smem[];
  Team<CL, NS> tm;
  tm.init(sh, a.D, reinterpret_cast<float *>(smem));
  float *count = reinterpret_cast<float *>(smem) + Team<CL, NS>::RED_FLOATS;   // channels of each warp of a team, by block
  float4 *bias = reinterpret_cast<float4 *>(count + CL * 16);                  // layer: [warp of a team][qb, bp][4][lane]
  // ring: [warp][stage][vector][piece][lane] of 16 bytes, so that a lane's pieces are at constant distances
  constexpr int STAGE = 2 * PIECES * 512;
  uint8_t *ring = reinterpret_cast<uint8_t *>(bias + (LAYER ? 8 * 32 * sh.warps : 0)) + tm.warp * (STAGE * sh.stages) + tm.lane * 16;
  const uint32_t ring_u32 = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  const float4 *my_bias = bias + (tm.warp - tm.first_warp) * (8 * 32) + tm.lane;
  if (LAYER && threadIdx.x < CL * 16) count[threadIdx.x] = tm.channels(threadIdx.x / 16, threadIdx.x % 16, a.D);
  pdl_launch_dependents();
  pdl_wait();

  const bool has_y = FULL || a.y != nullptr, post = FULL || (has_y && a.post.has), pre = FULL || a.pre.has, has_r = FULL || a.r != nullptr;
  int col[2];
  bool act[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    col[j] = tm.c_begin + (j * tm.TL + tm.tl) * 8;
    act[j] = col[j] < tm.c_end;
  }
  const long long first = (long long)tm.unit * sh.teams + tm.team, step = (long long)tm.units * sh.teams;
  const long long n = first < a.M ? (a.M - first + step - 1) / step : 0;
  // the teams of a cluster meet at its barrier: all do as many steps as its first team, which has the most rows
  const long long n_steps = CL == 1 ? n : (a.M - (first - tm.team) + step - 1) / step;
  auto slot = [](int stage, int j, int piece) { return stage * STAGE + (j * PIECES + piece) * 512; };
  const long long row_step = step * a.D;
  long long f_at = first * a.D;                  // first channel of the row that is fetched next
  long long f_row = 0;
  auto fetch = [&](int stage) {
    if (f_row < n) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (!act[j]) continue;
        if (has_y) cp_async16(ring_u32 + slot(stage, j, 0), a.y + f_at + col[j]);
#pragma unroll
        for (int p = 0; p < RP; ++p)
          cp_async16(ring_u32 + slot(stage, j, 1 + p), reinterpret_cast<const uint8_t *>(static_cast<const RT *>(a.x) + f_at + col[j]) + 16 * p);
      }
    }
    ++f_row;
    f_at += row_step;
    cp_async_commit();
  };
  for (int s = 0; s + 1 < sh.stages; ++s) fetch(s);   // the weights come while the first rows are on their way

  f2 qw[2][4], wp[2][4];   // r = alpha x + qw h + qb, u = wp h + bp
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float q[8], b[8], w[8], c[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) q[k] = b[k] = w[k] = c[k] = 0.f;
    if (act[j]) {
      if (has_y) {
        float g[8];
        weights8(a.gate, col[j], 1.f, g);
        weights8(a.post.w, col[j], 1.f, q);
        if (LAYER) weights8(a.post.b, col[j], 0.f, b);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          q[k] *= a.beta * g[k];
          b[k] *= a.beta * g[k];
        }
      }
      if (pre) weights8(a.pre.w, col[j], 1.f, w);
      if (LAYER) weights8(a.pre.b, col[j], 0.f, c);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      qw[j][k] = pack2(q[2 * k], q[2 * k + 1]);
      wp[j][k] = pack2(w[2 * k], w[2 * k + 1]);
    }
    if (LAYER && tm.team == 0) {   // too many for the registers
      float4 *to = bias + tm.warp * (8 * 32) + tm.lane;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        to[(j * 2 + h) * 32] = make_float4(b[4 * h], b[4 * h + 1], b[4 * h + 2], b[4 * h + 3]);
        to[(4 + j * 2 + h) * 32] = make_float4(c[4 * h], c[4 * h + 1], c[4 * h + 2], c[4 * h + 3]);
      }
    }
  }
  if (LAYER) __syncthreads();
  if (CL > 1) {   // the other blocks run before anything is written to their shared memory
    tm.arrive();
    tm.wait();
  }

  const float inv_d = 1.0f / (float)a.D;
  const float my_channels = LAYER ? count[tm.rank * 16 + tm.warp - tm.first_warp] : 0.f;
  const float my_inv = my_channels > 0.f ? 1.0f / my_channels : 0.f;
  // (an RMS norm beside a layer norm: means of zero)
  const float lane_channels = (float)(8 * ((int)act[0] + (int)act[1])), lane_inv = act[0] ? 1.0f / lane_channels : 0.f;
  const float y_inv = (post && a.post.layer) ? lane_inv : 0.f, r_inv = (pre && a.pre.layer) ? lane_inv : 0.f;
  const f2 alpha = both(a.alpha), zero = both(0.f);
  f2 r[2][4];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int k = 0; k < 4; ++k) r[j][k] = zero;
  float mean_y = 0.f, rstd_y = 1.f, mean_r = 0.f, rstd_r = 0.f, shown_mean_y = 0.f, shown_rstd_y = 0.f;

  int st_a = 0, st_b = sh.stages - 1;     // ring stages of row i (its y) and of row i - 1 (then refilled)
  long long at = first * a.D - 2 * row_step;   // first channel of row i - 2
  for (long long i = 0; i < n_steps + 2; ++i, at += row_step) {
    uint4 u_out[LATE ? 2 : 1];
    float4 st_out;
    auto store_u = [&](int j, const uint4 &u) { *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.u) + at + col[j]) = u; };
    auto store_stats = [&](const float4 &st) {
      if (a.stats && tm.tl == 0 && tm.rank == 0) a.stats[first + (i - 2) * step] = st;
    };
    if (i >= 2 && i < n + 2) {
      // ---- row i - 2: u (stored below)
      if (pre) {
        const f2 shift = both(-mean_r), scale = both(rstd_r);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (!LATE && !act[j]) continue;
          f2 u[4], bp[4];
          if (LAYER) join4(my_bias[(4 + j * 2) * 32], my_bias[(5 + j * 2) * 32], bp);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const f2 h = mul2(LAYER ? add2(r[j][k], shift) : r[j][k], scale);
            u[k] = LAYER ? fma2(h, wp[j][k], bp[k]) : mul2(h, wp[j][k]);
          }
          if (LATE) u_out[LATE ? j : 0] = narrow4(u);
          else store_u(j, narrow4(u));
        }
      }
      const float4 st = make_float4(shown_mean_y, shown_rstd_y, pre ? mean_r : 0.f, pre ? rstd_r : 0.f);
      if (LATE) st_out = st;
      else store_stats(st);
    }
    f2 part_y = zero, part_r = zero;
    if (i >= 1 && i <= n) {
      // ---- row i - 1: r
      const f2 shift = both(-mean_y), scale = both(rstd_y);
      shown_mean_y = post ? mean_y : 0.f;
      shown_rstd_y = post ? rstd_y : 0.f;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (!act[j]) continue;
        f2 x[4];
        if (RP == 1)
          widen4(*reinterpret_cast<const uint4 *>(ring + slot(st_b, j, 1)), x);
        else
          join4(*reinterpret_cast<const float4 *>(ring + slot(st_b, j, 1)), *reinterpret_cast<const float4 *>(ring + slot(st_b, j, PIECES - 1)), x);
        if (has_y) {
          f2 y[4], qb[4];
          widen4(*reinterpret_cast<const uint4 *>(ring + slot(st_b, j, 0)), y);
          if (LAYER) join4(my_bias[(j * 2) * 32], my_bias[(1 + j * 2) * 32], qb);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const f2 h = mul2(LAYER ? add2(y[k], shift) : y[k], scale);
            const f2 base = LAYER ? fma2(alpha, x[k], qb[k]) : mul2(alpha, x[k]);
            r[j][k] = fma2(qw[j][k], h, base);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) r[j][k] = mul2(alpha, x[k]);
        }
        if (!LATE && has_r) store4(static_cast<RT *>(a.r) + (at + row_step) + col[j], r[j]);
#pragma unroll
        for (int k = 0; k < 4; ++k) part_r = LAYER ? add2(part_r, r[j][k]) : fma2(r[j][k], r[j][k], part_r);
      }
    }
    f2 y[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) y[j][k] = zero;
    if (i < n) {
      // ---- row i: sums of y
      cp_async_wait(sh.stages - 2);
      if (post) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (!act[j]) continue;
          widen4(*reinterpret_cast<const uint4 *>(ring + slot(st_a, j, 0)), y[j]);
#pragma unroll
          for (int k = 0; k < 4; ++k) part_y = LAYER ? add2(part_y, y[j][k]) : fma2(y[j][k], y[j][k], part_y);
        }
      }
    }
    auto refill = [&]() {
      fetch(st_b);     // row i - 1 has been read for the last time
      st_b = st_a;
      if (++st_a == sh.stages) st_a = 0;
    };
    if (!LATE) refill();
    int idx;
    if (LAYER) {
      // A lane's own mean and squared distances from it; the warp's from the lanes', with the lanes' means taken relative to
      // lane 0's: the differences are of the size of the deviation, so nothing cancels that matters (at worst, when lane 0
      // holds all of the variance, its share of the channels: 16 of 512), and one round of shuffles does it.
      const float ly = sum2(part_y) * y_inv, lr = sum2(part_r) * r_inv;
      const f2 sy = both(-ly), sr = both(-lr);
      f2 dy = zero, dr = zero;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (!act[j]) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f2 ey = add2(y[j][k], sy), er = add2(r[j][k], sr);
          dy = fma2(ey, ey, dy);
          dr = fma2(er, er, dr);
        }
      }
      const float cy = __shfl_sync(0xFFFFFFFFu, ly, 0), cr = __shfl_sync(0xFFFFFFFFu, lr, 0);
      const float ny = lane_channels * (ly - cy), nr = lane_channels * (lr - cr);
      float four[4] = {ny, fmaf(ny, ly - cy, sum2(dy)), nr, fmaf(nr, lr - cr, sum2(dr))};
      const float s = warp_sum_scattered<4>(four, tm.lane, idx), other = __shfl_xor_sync(0xFFFFFFFFu, s, 8);
      tm.publish((idx & 1) ? fmaf(-other * my_inv, other, s) : fmaf(s, my_inv, (idx & 2) ? cr : cy), idx, (tm.lane & 7) == 0);
    } else {
      float two[2] = {sum2(part_y), sum2(part_r)};
      const float s = warp_sum_scattered<2>(two, tm.lane, idx);
      tm.publish(s, idx, (tm.lane & 15) == 0);
    }
    tm.arrive();
    // what this step writes and fetches late, while the sums are exchanged
    if (LATE && i >= 2 && i < n + 2) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (pre && act[j]) store_u(j, u_out[LATE ? j : 0]);
      store_stats(st_out);
    }
    if (LATE && has_r && i >= 1 && i <= n) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (act[j]) store4(static_cast<RT *>(a.r) + (at + row_step) + col[j], r[j]);
    }
    if (LATE) refill();
    const float *buf = tm.buffer();
    tm.turn ^= 1;
    tm.wait();
    float v[2];
    if (LAYER) {
      float m[2];
      tm.template total<2>(buf, m, [&](float (&t)[2], const float *f, int w) {
        t[0] = fmaf(count[w], f[0], t[0]);
        t[1] = fmaf(count[w], f[2], t[1]);
      });
      mean_y = m[0] * inv_d;
      mean_r = m[1] * inv_d;
      tm.template total<2>(buf, v, [&](float (&t)[2], const float *f, int w) {
        const float dy = f[0] - mean_y, dr = f[2] - mean_r;
        t[0] += fmaf(count[w] * dy, dy, f[1]);
        t[1] += fmaf(count[w] * dr, dr, f[3]);
      });
    } else {
      tm.template total<2>(buf, v, [&](float (&t)[2], const float *f, int) {
        t[0] += f[0];
        t[1] += f[1];
      });
    }
    const float vy = v[0], vr = v[1];
    rstd_y = post ? rsqrtf(fmaf(vy, inv_d, a.post.eps)) : 1.f;
    rstd_r = rsqrtf(fmaf(vr, inv_d, a.pre.eps));
  }
  cp_async_wait(0);
}

// ------------------------------------------------------------------------------------------------ backward

struct BwdArgs {
  const void *dr;
  const __nv_bfloat16 *du, *y;
  const void *r;
  const float4 *stats;
  const float *w_post, *gate, *w_pre;
  float alpha, beta;
  int post_has, post_layer, pre_has, pre_layer;
  void *dx;
  __nv_bfloat16 *dy;
  float *partial;    // [units][4][D]
  long long M;
  int D;
};

// One exchange per row.  With t = dr + rstd (a - c1 - h_pre c2), c1 = mean a, c2 = mean a h_pre, the sums that dy needs,
// sum q t and sum q t h_post, are linear in c1 and c2, so all sums over the row's data are taken at once and combined:
//   sum q t h_post = sum q h_post (dr + rstd a) - rstd (c1 sum q h_post + c2 sum q h_post h_pre).
// A step takes the sums of row i + 1 and writes the gradients of row i.  The sums over rows stay in registers.
// What bounds it: RMS the memory; layer norm the registers (the sums of t and du beside those of t h and du h leave room for
// 12 warps an SM) and 61 instructions a channel.  16384 x 8192 RMS: 583 us with a row at a time, 486 us in the pipeline, 321 us
// with packed arithmetic, 257 us with the row's statistics read a step ahead (their latency stood in every step).
//
// LAYER: either norm subtracts a mean (more sums; the weights are then in shared memory, there are too few registers).
// FULL: every input, both norms, dx and dy are there.
template <typename RT, bool LAYER, int CL, bool FULL>
__global__ void __launch_bounds__(32 * bwd_warps(LAYER), 1) block_norm_bwd_kernel(const __grid_constant__ BwdArgs a, const TeamShape sh) {
  constexpr bool WREG = !LAYER;
  constexpr int NS = LAYER ? 8 : 4;                 // sums per row
  constexpr int RP = sizeof(RT) / 2;                // 16-byte pieces of a residual vector
  constexpr int PIECES = 2 + 2 * RP;                // y, du, r, dr
  extern __shared__ __align__(16) uint8_t smem[];
  Team<CL, NS> tm;
  tm.init(sh, a.D, reinterpret_cast<float *>(smem));
  const int tl = tm.tl, TL = tm.TL;
  float4 *wsm = reinterpret_cast<float4 *>(smem + Team<CL, NS>::RED_FLOATS * 4);   // layer: [warp of a team][q, w_pre][4][lane]
  // ring: [warp][stage][vector][piece][lane] of 16 bytes, so that a lane's pieces are at constant distances
  constexpr int STAGE = 2 * PIECES * 512;
  uint8_t *ring0 = reinterpret_cast<uint8_t *>(wsm + (WREG ? 0 : 8 * TL)), *ring = ring0 + tm.warp * (STAGE * sh.stages) + tm.lane * 16;
  const uint32_t ring_u32 = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  const float4 *my_w = wsm + (tm.warp - tm.first_warp) * (8 * 32) + tm.lane;

  pdl_launch_dependents();
  pdl_wait();

  const bool has_y = FULL || a.y != nullptr, has_dr = FULL || a.dr != nullptr, has_pre = FULL || a.pre_has != 0, has_post = FULL || a.post_has != 0;
  int col[2];
  bool act[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    col[j] = tm.c_begin + (j * TL + tl) * 8;
    act[j] = col[j] < tm.c_end;
  }
  const long long first = (long long)tm.unit * sh.teams + tm.team, step = (long long)tm.units * sh.teams;
  const long long n = first < a.M ? (a.M - first + step - 1) / step : 0;
  // the teams of a cluster meet at its barrier: all do as many steps as its first team, which has the most rows
  const long long n_steps = CL == 1 ? n : (a.M - (first - tm.team) + step - 1) / step;
  auto slot = [](int stage, int j, int piece) { return stage * STAGE + (j * PIECES + piece) * 512; };
  const long long row_step = step * a.D;
  long long f_at = first * a.D, f_row = 0;       // first channel and number of the row that is fetched next
  auto fetch = [&](int stage) {
    if (f_row < n) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (!act[j]) continue;
        const long long at = f_at + col[j];
        if (has_y) cp_async16(ring_u32 + slot(stage, j, 0), a.y + at);
        if (has_pre) {
          cp_async16(ring_u32 + slot(stage, j, 1), a.du + at);
#pragma unroll
          for (int p = 0; p < RP; ++p)
            cp_async16(ring_u32 + slot(stage, j, 2 + p), reinterpret_cast<const uint8_t *>(static_cast<const RT *>(a.r) + at) + 16 * p);
        }
        if (has_dr) {
#pragma unroll
          for (int p = 0; p < RP; ++p)
            cp_async16(ring_u32 + slot(stage, j, 2 + RP + p), reinterpret_cast<const uint8_t *>(static_cast<const RT *>(a.dr) + at) + 16 * p);
        }
      }
    }
    ++f_row;
    f_at += row_step;
    cp_async_commit();
  };
  for (int s = 0; s + 1 < sh.stages; ++s) fetch(s);   // the weights come while the first rows are on their way

  f2 qreg[WREG ? 2 : 1][4], wreg[WREG ? 2 : 1][4];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float q[8], w[8], g[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) q[k] = w[k] = 0.f;
    if (act[j]) {
      if (has_y) {
        weights8(a.w_post, col[j], 1.f, q);
        weights8(a.gate, col[j], 1.f, g);
#pragma unroll
        for (int k = 0; k < 8; ++k) q[k] *= a.beta * g[k];
      }
      if (has_pre) weights8(a.w_pre, col[j], 1.f, w);
    }
    if (WREG) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        qreg[j][k] = pack2(q[2 * k], q[2 * k + 1]);
        wreg[j][k] = pack2(w[2 * k], w[2 * k + 1]);
      }
    } else if (tm.team == 0) {
      float4 *to = wsm + tm.warp * (8 * 32) + tm.lane;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        to[(j * 2 + h) * 32] = make_float4(q[4 * h], q[4 * h + 1], q[4 * h + 2], q[4 * h + 3]);
        to[(4 + j * 2 + h) * 32] = make_float4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]);
      }
    }
  }
  if (!WREG) __syncthreads();
  if (CL > 1) {   // the other blocks run before anything is written to their shared memory
    tm.arrive();
    tm.wait();
  }
  auto weights = [&](int j, f2 (&q)[4], f2 (&w)[4]) {
    if (WREG) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        q[k] = qreg[j][k];
        w[k] = wreg[j][k];
      }
    } else {
      join4(my_w[(j * 2) * 32], my_w[(1 + j * 2) * 32], q);
      join4(my_w[(4 + j * 2) * 32], my_w[(5 + j * 2) * 32], w);
    }
  };

  const f2 zero = both(0.f);
  auto read = [&](int stage, int j, int piece, bool there, bool resid, f2 (&f)[4]) {   // one vector of eight channels
    if (!there) {
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k] = zero;
    } else if (resid && RP == 2) {
      join4(*reinterpret_cast<const float4 *>(ring + slot(stage, j, piece)), *reinterpret_cast<const float4 *>(ring + slot(stage, j, piece + 1)), f);
    } else {
      widen4(*reinterpret_cast<const uint4 *>(ring + slot(stage, j, piece)), f);
    }
  };

  f2 sumA[2][4], sumC[2][4], sumB[LAYER ? 2 : 1][4], sumE[LAYER ? 2 : 1][4];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      sumA[j][k] = sumC[j][k] = zero;
      if (LAYER) sumB[j][k] = sumE[j][k] = zero;
    }
  const float inv_d = 1.0f / (float)a.D;
  // h_post = (y - mp) ip, h_pre = (r - mr) ir of the rows in work (0: row i, 1: row i - 1); the mean is subtracted first:
  // folded into the product it would leave its rounding error, which is large where the mean is
  float ip[2] = {1.f, 1.f}, mp[2] = {0.f, 0.f}, ir[2] = {0.f, 0.f}, mr[2] = {0.f, 0.f};
  float c1 = 0.f, c2 = 0.f, m1 = 0.f, m2 = 0.f;    // of row i - 1
  const f2 alpha = both(a.alpha);
  // a row's statistics are read a step before they are used
  const bool has_stats = FULL || a.stats;
  float4 next_st = (has_stats && n > 0) ? a.stats[first] : make_float4(0.f, 0.f, 0.f, 0.f);
  int st_a = 0, st_b = sh.stages - 1;     // ring stages of row i and of row i - 1 (then refilled)
  long long at = first * a.D - row_step;  // first channel of row i - 1
  for (long long i = 0; i <= n_steps; ++i, at += row_step) {
    if (i < n) {
      const float4 st = next_st;
      if (has_stats && i + 1 < n) next_st = a.stats[first + (i + 1) * step];
      if (has_post) {
        ip[0] = st.y;
        mp[0] = st.x;
      }
      if (has_pre) {
        ir[0] = st.w;
        mr[0] = st.z;
      }
      cp_async_wait(sh.stages - 2);
      f2 s2[NS];
#pragma unroll
      for (int k = 0; k < NS; ++k) s2[k] = zero;
      const f2 ir2 = both(ir[0]), ip2 = both(ip[0]), nmr = both(-mr[0]), nmp = both(-mp[0]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (!act[j]) continue;
        f2 q[4], w[4], y[4], du[4], r[4], dr[4];
        weights(j, q, w);
        read(st_a, j, 0, has_y, false, y);
        read(st_a, j, 1, has_pre, false, du);
        read(st_a, j, 2, has_pre, true, r);
        read(st_a, j, 2 + RP, has_dr, true, dr);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f2 av = mul2(du[k], w[k]), z = fma2(ir2, av, dr[k]);
          if (LAYER) {
            const f2 hp = mul2(add2(y[k], nmp), ip2), hr = mul2(add2(r[k], nmr), ir2), qh = mul2(q[k], hp);
            s2[0] = fma2(av, hr, s2[0]);
            s2[1] = fma2(z, qh, s2[1]);
            s2[2] = fma2(qh, hr, s2[2]);
            s2[3] = add2(s2[3], av);
            s2[4] = fma2(q[k], z, s2[4]);
            s2[5] = fma2(q[k], hr, s2[5]);
            s2[6] = add2(s2[6], q[k]);
            s2[7] = add2(s2[7], qh);
          } else {   // without the factors ip and ir, which are the row's
            const f2 qy = mul2(q[k], y[k]);
            s2[0] = fma2(av, r[k], s2[0]);
            s2[1] = fma2(z, qy, s2[1]);
            s2[2] = fma2(qy, r[k], s2[2]);
          }
        }
      }
      float s[NS];
#pragma unroll
      for (int k = 0; k < NS; ++k) s[k] = sum2(s2[k]);
      int idx;
      const float mine = warp_sum_scattered<NS>(s, tm.lane, idx);
      tm.publish(mine, idx, (tm.lane & (32 / NS - 1)) == 0);
    }
    if (i < n_steps) tm.arrive();
    if (i > 0 && i <= n) {
      const f2 ir2 = both(ir[1]), ip2 = both(ip[1]), nmr = both(-mr[1]), nmp = both(-mp[1]);
      const f2 k1 = both(-ir[1] * c1), k2 = both(-ir[1] * c2), g2 = both(-ip[1] * m2), g1 = both(-ip[1] * m1);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (!act[j]) continue;
        f2 q[4], w[4], y[4], du[4], r[4], dr[4], dy[4];
        weights(j, q, w);
        read(st_b, j, 0, has_y, false, y);
        read(st_b, j, 1, has_pre, false, du);
        read(st_b, j, 2, has_pre, true, r);
        read(st_b, j, 2 + RP, has_dr, true, dr);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f2 hp = mul2(LAYER ? add2(y[k], nmp) : y[k], ip2), hr = mul2(LAYER ? add2(r[k], nmr) : r[k], ir2);
          f2 t = fma2(ir2, mul2(du[k], w[k]), LAYER ? add2(dr[k], k1) : dr[k]);
          t = fma2(hr, k2, t);
          sumA[j][k] = fma2(t, hp, sumA[j][k]);
          sumC[j][k] = fma2(du[k], hr, sumC[j][k]);
          if (LAYER) {
            sumB[j][k] = add2(sumB[j][k], t);
            sumE[j][k] = add2(sumE[j][k], du[k]);
          }
          dr[k] = mul2(alpha, t);
          dy[k] = fma2(hp, g2, LAYER ? fma2(mul2(q[k], t), ip2, g1) : mul2(mul2(q[k], t), ip2));
        }
        if (FULL || a.dx) store4(static_cast<RT *>(a.dx) + at + col[j], dr);
        if (FULL || a.dy) store4(a.dy + at + col[j], dy);
      }
    }
    fetch(st_b);     // row i - 1 has been read for the last time
    st_b = st_a;
    if (++st_a == sh.stages) st_a = 0;
    if (i == n_steps) break;
    const float *buf = tm.buffer();
    tm.turn ^= 1;
    tm.wait();
    float s[NS];
    tm.template total<NS>(buf, s, [&](float (&t)[NS], const float *f, int) {
#pragma unroll
      for (int k4 = 0; k4 < NS / 4; ++k4) {
        const float4 v = *reinterpret_cast<const float4 *>(f + 4 * k4);
        t[4 * k4] += v.x; t[4 * k4 + 1] += v.y; t[4 * k4 + 2] += v.z; t[4 * k4 + 3] += v.w;
      }
    });
    ip[1] = ip[0]; mp[1] = mp[0]; ir[1] = ir[0]; mr[1] = mr[0];
    if (LAYER) {
      c1 = a.pre_layer ? s[3] * inv_d : 0.f;
      c2 = s[0] * inv_d;
      m1 = a.post_layer ? (s[4] - ir[1] * (c1 * s[6] + c2 * s[5])) * inv_d : 0.f;
      m2 = (s[1] - ir[1] * (c1 * s[7] + c2 * s[2])) * inv_d;
    } else {
      c2 = s[0] * ir[1] * inv_d;
      m2 = ip[1] * (s[1] - ir[1] * ir[1] * c2 * s[2]) * inv_d;
    }
    if (!has_post) m2 = 0.f;
  }
  cp_async_wait(0);

  // Channel sums of the block: teams added in ascending order.
  __syncthreads();
  float4 *acc = reinterpret_cast<float4 *>(ring0);   // [team][vector][half][TL], one sum at a time
  constexpr int NACC = LAYER ? 4 : 2;
#pragma unroll
  for (int q = 0; q < NACC; ++q) {
    float4 *mine = acc + tm.team * (4 * TL);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f2 *p = q == 0 ? &sumA[j][2 * h] : q == 1 ? &sumC[j][2 * h] : q == 2 ? &sumB[LAYER ? j : 0][2 * h] : &sumE[LAYER ? j : 0][2 * h];
        const float2 lo = split2(p[0]), hi = split2(p[1]);
        mine[(j * 2 + h) * TL + tl] = make_float4(lo.x, lo.y, hi.x, hi.y);
      }
    __syncthreads();
    if (tm.team == 0) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (!act[j]) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float4 v = acc[(j * 2 + h) * TL + tl];
          for (int t = 1; t < sh.teams; ++t) {
            const float4 o = acc[(t * 4 + j * 2 + h) * TL + tl];
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
          }
          *reinterpret_cast<float4 *>(a.partial + ((long long)tm.unit * 4 + q) * a.D + col[j] + 4 * h) = v;
        }
      }
    }
    __syncthreads();
  }
}

struct FinalArgs {
  const float *partial;
  int units, D, layer;
  const float *w_post, *b_post, *gate;
  float beta;
  int post_has;
  float *dw_post, *db_post, *dgate, *dw_pre, *db_pre;
};

// Adds the blocks' channel sums and forms the vectors' gradients.  32 channels per block; each of the 32 warps takes every
// 32nd partial sum (ROW_MAX_BLOCKS / 32 of them, all loads issued together: the kernel is one memory latency long), the
// warps' sums are added in ascending order.
__global__ void __launch_bounds__(1024) block_norm_final_kernel(const __grid_constant__ FinalArgs a) {
  __shared__ float red[4][32][33];
  pdl_launch_dependents();
  pdl_wait();
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + c;
  constexpr int PER = ROW_MAX_BLOCKS / 32;
  float v[4][PER];
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int u = g + 32 * p;
    const bool there = col < a.D && u < a.units;
    const float *from = a.partial + (long long)u * 4 * a.D + col;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k][p] = (there && (k < 2 || a.layer)) ? from[(long long)k * a.D] : 0.f;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float s = v[k][0];
#pragma unroll
    for (int p = 1; p < PER; ++p) s += v[k][p];
    red[k][g][c] = s;
  }
  __syncthreads();
  if (g >= 4) return;
  // warp k adds sum k over the 32 warps, then every sum is in red[k][0]
  float s = red[g][0][c];
#pragma unroll
  for (int q = 1; q < 32; ++q) s += red[g][q][c];
  red[g][0][c] = s;
  asm volatile("bar.sync 1, 128;" ::: "memory");
  if (g != 0 || col >= a.D) return;
  const float sum_th = red[0][0][c], sum_dh = red[1][0][c], sum_t = red[2][0][c], sum_d = red[3][0][c];
  const float gate = a.gate ? a.gate[col] : 1.f, w = (a.post_has && a.w_post) ? a.w_post[col] : 1.f;
  const float b = a.b_post ? a.b_post[col] : 0.f;
  if (a.dw_post) a.dw_post[col] = a.beta * gate * sum_th;
  if (a.db_post) a.db_post[col] = a.beta * gate * sum_t;
  if (a.dgate) a.dgate[col] = a.beta * fmaf(w, sum_th, b * sum_t);
  if (a.dw_pre) a.dw_pre[col] = sum_dh;
  if (a.db_pre) a.db_pre[col] = sum_d;
}

// ------------------------------------------------------------------------------------------------ host

constexpr int SMEM_MAX = 227 * 1024;

template <typename RT, int V>
int launch_fwd(const FwdArgs &args, int warps, cudaStream_t stream) {
  FwdArgs a = args;
  a.warps = warps;
  const int teams = warps >= 8 ? 1 : 8 / warps;
  return launch_overlapped(block_norm_fwd_kernel<RT, V>, dim3((unsigned)cdiv(a.M, teams)), dim3(teams * warps * 32), 0, 1, stream, a);
}

// Shape and launch of a kernel that walks many rows on clusters of CL blocks.  `pieces`: 16-byte pieces of a vector in
// the ring, `red_bytes` and `w_bytes_per_thread`: what else it keeps in shared memory.  As many teams to a block as leave
// room for three rows each (one being finished, one begun, one on its way); OSDP_ERR_UNSUPPORTED if not even one does.
template <int CL, auto KERNEL, typename Args>
int launch_rows(const Args &a, int max_warps, int pieces, int red_bytes, int w_bytes_per_thread, int sms, int *units, cudaStream_t stream) {
  TeamShape sh;
  sh.warps = (int)cdiv(block_channels(a.D, CL), 512);
  if (sh.warps > max_warps) return OSDP_ERR_UNSUPPORTED;
  const int fixed = red_bytes + w_bytes_per_thread * sh.warps * 32;
  int stage = 0;
  for (sh.teams = max_warps / sh.warps; sh.teams > 0; --sh.teams) {
    stage = 2 * pieces * sh.teams * sh.warps * 32 * 16;
    sh.stages = (SMEM_MAX - fixed) / stage;
    if (sh.stages >= 3) break;
  }
  if (sh.teams == 0) return OSDP_ERR_UNSUPPORTED;
  if (sh.stages > MAX_STAGES) sh.stages = MAX_STAGES;
  const int threads = sh.warps * sh.teams * 32, smem = fixed + sh.stages * stage;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return report_cuda(e);
  static std::atomic<int> most[64];      // clusters that run at the same time (blocks, without clusters); 0: not known yet
  static std::mutex setup;
  int cap = most[dev & 63].load(std::memory_order_acquire);
  if (cap == 0) {
    std::lock_guard<std::mutex> lock(setup);
    e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MAX);
    if (e != cudaSuccess) return report_cuda(e);
    cap = sms;
    if (CL > 1) {   // fewer than sms / CL: a cluster does not cross the chip's groups of SMs
      cudaLaunchConfig_t q = {};
      q.gridDim = dim3((unsigned)(sms / CL * CL));
      q.blockDim = dim3(32 * max_warps);
      q.dynamicSmemBytes = SMEM_MAX;
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = CL;
      attr[0].val.clusterDim.y = 1;
      attr[0].val.clusterDim.z = 1;
      q.attrs = attr;
      q.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&cap, KERNEL, &q);
      if (e != cudaSuccess) return report_cuda(e);
      if (cap < 1) return report_cuda(cudaErrorLaunchOutOfResources);
    }
    most[dev & 63].store(cap, std::memory_order_release);
  }
  int64_t n = cdiv(a.M, sh.teams);
  if (n > cap) n = cap;
  if (n > ROW_MAX_BLOCKS) n = ROW_MAX_BLOCKS;
  if (n < 1) n = 1;    // no rows: the backward writes zeros
  if (units) *units = (int)n;
  return launch_overlapped(KERNEL, dim3((unsigned)(CL * n)), dim3(threads), smem, CL, stream, a, sh);
}

// The smallest cluster that the rows fit.
template <typename RT, bool LAYER, int CL = 1>
int launch_fwd_rows(const FwdArgs &a, int sms, cudaStream_t stream) {
  const int pieces = 1 + (int)sizeof(RT) / 2, red = (Team<CL, LAYER ? 4 : 2>::RED_FLOATS + CL * 16) * 4, w = LAYER ? 128 : 0;
  const bool full = a.y && a.r && a.post.has && a.pre.has;
  const int rc = full ? launch_rows<CL, block_norm_fwd_rows_kernel<RT, LAYER, CL, true>>(a, fwd_warps(LAYER, sizeof(RT) == 4, CL), pieces, red, w, sms, nullptr, stream)
                      : launch_rows<CL, block_norm_fwd_rows_kernel<RT, LAYER, CL, false>>(a, fwd_warps(LAYER, sizeof(RT) == 4, CL), pieces, red, w, sms, nullptr, stream);
  if constexpr (CL < 4) {
    if (rc == OSDP_ERR_UNSUPPORTED) return launch_fwd_rows<RT, LAYER, 2 * CL>(a, sms, stream);
  }
  return rc;
}
template <typename RT, bool LAYER, int CL = 1>
int launch_bwd(const BwdArgs &a, int sms, int *units, cudaStream_t stream) {
  const int pieces = 2 + (int)sizeof(RT), red = Team<CL, LAYER ? 8 : 4>::RED_FLOATS * 4, w = LAYER ? 128 : 0;
  const bool full = a.y && a.dr && a.post_has && a.pre_has && a.dx && a.dy;
  const int rc = full ? launch_rows<CL, block_norm_bwd_kernel<RT, LAYER, CL, true>>(a, bwd_warps(LAYER), pieces, red, w, sms, units, stream)
                      : launch_rows<CL, block_norm_bwd_kernel<RT, LAYER, CL, false>>(a, bwd_warps(LAYER), pieces, red, w, sms, units, stream);
  if constexpr (CL < 4) {
    if (rc == OSDP_ERR_UNSUPPORTED) return launch_bwd<RT, LAYER, 2 * CL>(a, sms, units, stream);
  }
  return rc;
}

bool norm_kind(int k) { return k == OSDP_NORM_NONE || k == OSDP_NORM_RMS || k == OSDP_NORM_LAYER; }

int check_shape(int64_t M, int64_t D, int resid_dtype, int post, int pre) {
  if (M < 0 || D <= 0 || M > ((int64_t)1 << 31) - 1) return OSDP_ERR_BAD_SHAPE;
  if (D & 7) return OSDP_ERR_ALIGNMENT;
  if (D > OSDP_BLOCK_NORM_MAX_D) return OSDP_ERR_UNSUPPORTED;
  if (resid_dtype != OSDP_DTYPE_BF16 && resid_dtype != OSDP_DTYPE_FP32) return OSDP_ERR_UNSUPPORTED;
  if (!norm_kind(post) || !norm_kind(pre)) return OSDP_ERR_UNSUPPORTED;
  return OSDP_OK;
}

}  // namespace
}  // namespace osdp

using namespace osdp;

extern "C" {

int osdp_block_norm_fwd(const void *x, const void *y, int64_t M, int64_t D, int resid_dtype, int post, const float *w_post,
                        const float *b_post, double eps_post, const float *gate, double alpha, double beta, int pre,
                        const float *w_pre, const float *b_pre, double eps_pre, void *r, void *u, float *u_scale,
                        float *stats, void *stream) {
  const int rc = check_shape(M, D, resid_dtype, post, pre);
  if (rc) return rc;
  if (!std::isfinite(alpha) || !std::isfinite(beta)) return OSDP_ERR_UNSUPPORTED;
  if ((post && !(eps_post >= 0.0 && std::isfinite(eps_post))) || (pre && !(eps_pre >= 0.0 && std::isfinite(eps_pre)))) return OSDP_ERR_UNSUPPORTED;
  if ((b_post && post != OSDP_NORM_LAYER) || (b_pre && pre != OSDP_NORM_LAYER)) return OSDP_ERR_UNSUPPORTED;
  if (M == 0) return OSDP_OK;
  if (!x || (pre && !u) || (!r && !pre)) return OSDP_ERR_NULL_POINTER;
  const uintptr_t ra = resid_dtype == OSDP_DTYPE_FP32 ? 32 : 16;
  if (!aligned_to(x, ra) || !aligned_to(r, ra) || !aligned_to(y, 16) || !aligned_to(u, u_scale ? 8 : 16) || !aligned_to(u_scale, 4) ||
      !aligned_to(stats, 16) || !aligned_to(w_post, 16) || !aligned_to(b_post, 16) || !aligned_to(gate, 16) || !aligned_to(w_pre, 16) ||
      !aligned_to(b_pre, 16))
    return OSDP_ERR_ALIGNMENT;
  FwdArgs a;
  a.x = x;
  a.y = static_cast<const __nv_bfloat16 *>(y);
  a.r = r;
  a.u = u;
  a.u_scale = u_scale;
  a.stats = reinterpret_cast<float4 *>(stats);
  a.gate = gate;
  a.alpha = (float)alpha;
  a.beta = (float)beta;
  a.post = RowNorm{post != OSDP_NORM_NONE, post == OSDP_NORM_LAYER, (float)eps_post, post ? w_post : nullptr, b_post};
  a.pre = RowNorm{pre != OSDP_NORM_NONE, pre == OSDP_NORM_LAYER, (float)eps_pre, w_pre, b_pre};
  a.M = M;
  a.D = (int)D;
  a.warps = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int sms = 0;
  const int src = sm_count(&sms);
  if (src) return src;
  // Few rows: one vector per lane, as many warps to a row as it has vectors, for the shortest chain of instructions, as long
  // as all rows are at work at the same time (32 warps of this kernel fit an SM).  Measured on B200 (us, this way / rows in
  // a pipeline): 1024 x 1024 RMS bf16 3.7 / 4.7, layer fp32 5.1 / 8.0; 256 x 4096 4.1 / 5.0 and 6.0 / 8.6; 512 x 4096 7.8 / 6.4
  // and 11.3 / 12.0; 256 x 8192 9.8 / 6.4 and 15.1 / 12.2.
  const bool few = D <= 8192 && M * cdiv(D, 256) <= (int64_t)sms * 32;
  if (!few && !u_scale) {
    const bool layer = a.post.layer || a.pre.layer;
#define OSDP_FWD(RT, LAYER) launch_fwd_rows<RT, LAYER>(a, sms, s)
    if (resid_dtype == OSDP_DTYPE_FP32) return layer ? OSDP_FWD(float, true) : OSDP_FWD(float, false);
    return layer ? OSDP_FWD(__nv_bfloat16, true) : OSDP_FWD(__nv_bfloat16, false);
#undef OSDP_FWD
  }
  if (few) return resid_dtype == OSDP_DTYPE_FP32 ? launch_fwd<float, 1>(a, (int)cdiv(D, 256), s) : launch_fwd<__nv_bfloat16, 1>(a, (int)cdiv(D, 256), s);
  // int8 u for many rows.  Two vectors per lane: 8192 x 2048 RMS 43 us (8192 x 8192: 177); one and four took 1.4 and 1.3
  // (1.9 and 1.2) times as long.
  return resid_dtype == OSDP_DTYPE_FP32 ? launch_fwd<float, 2>(a, (int)cdiv(D, 512), s) : launch_fwd<__nv_bfloat16, 2>(a, (int)cdiv(D, 512), s);
}

int osdp_block_norm_workspace_bytes(int64_t M, int64_t D, size_t *bytes) {
  if (!bytes) return OSDP_ERR_NULL_POINTER;
  const int rc = check_shape(M, D, OSDP_DTYPE_BF16, 0, 0);
  if (rc) return rc;
  *bytes = 256 + (size_t)ROW_MAX_BLOCKS * 4 * (size_t)D * sizeof(float);
  return OSDP_OK;
}

int osdp_block_norm_bwd(const void *dr, const void *du, const void *y, const void *r, const float *stats, int64_t M, int64_t D,
                        int resid_dtype, int post, const float *w_post, const float *b_post, const float *gate, double alpha,
                        double beta, int pre, const float *w_pre, void *dx, void *dy, float *dw_post, float *db_post,
                        float *dgate, float *dw_pre, float *db_pre, void *ws, size_t ws_bytes, void *stream) {
  int rc = check_shape(M, D, resid_dtype, post, pre);
  if (rc) return rc;
  if (!std::isfinite(alpha) || !std::isfinite(beta)) return OSDP_ERR_UNSUPPORTED;
  if (((b_post || db_post) && post != OSDP_NORM_LAYER) || (db_pre && pre != OSDP_NORM_LAYER)) return OSDP_ERR_UNSUPPORTED;
  if ((dw_post && !post) || (dw_pre && !pre)) return OSDP_ERR_UNSUPPORTED;
  if (!ws || (M > 0 && ((pre && (!du || !r)) || ((pre || (y && post)) && !stats) || (!y && (dy || dw_post || db_post || dgate)) || (!pre && !dr))))
    return OSDP_ERR_NULL_POINTER;
  const uintptr_t ra = resid_dtype == OSDP_DTYPE_FP32 ? 32 : 16;
  if (!aligned_to(dr, ra) || !aligned_to(r, ra) || !aligned_to(dx, ra) || !aligned_to(du, 16) || !aligned_to(y, 16) || !aligned_to(dy, 16) ||
      !aligned_to(stats, 16) || !aligned_to(w_post, 16) || !aligned_to(b_post, 16) || !aligned_to(gate, 16) || !aligned_to(w_pre, 16) ||
      !aligned_to(dw_post, 4) || !aligned_to(db_post, 4) || !aligned_to(dgate, 4) || !aligned_to(dw_pre, 4) || !aligned_to(db_pre, 4) ||
      !aligned_to(ws, 256))
    return OSDP_ERR_ALIGNMENT;
  size_t need = 0;
  rc = osdp_block_norm_workspace_bytes(M, D, &need);
  if (rc) return rc;
  if (ws_bytes < need) return OSDP_ERR_WORKSPACE_TOO_SMALL;
  int sms = 0;
  rc = sm_count(&sms);
  if (rc) return rc;
  BwdArgs a;
  a.dr = dr;
  a.du = static_cast<const __nv_bfloat16 *>(du);
  a.y = static_cast<const __nv_bfloat16 *>(y);
  a.r = r;
  a.stats = reinterpret_cast<const float4 *>(stats);
  a.w_post = post ? w_post : nullptr;
  a.gate = gate;
  a.w_pre = w_pre;
  a.alpha = (float)alpha;
  a.beta = (float)beta;
  a.post_has = post != OSDP_NORM_NONE;
  a.post_layer = post == OSDP_NORM_LAYER;
  a.pre_has = pre != OSDP_NORM_NONE;
  a.pre_layer = pre == OSDP_NORM_LAYER;
  a.dx = dx;
  a.dy = static_cast<__nv_bfloat16 *>(dy);
  a.partial = reinterpret_cast<float *>(static_cast<char *>(ws) + 256);
  a.M = M;
  a.D = (int)D;
  const bool layer = a.post_layer || a.pre_layer || db_post || db_pre;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int units = 0;
#define OSDP_BWD(RT, LAYER) launch_bwd<RT, LAYER>(a, sms, &units, s)
  if (resid_dtype == OSDP_DTYPE_FP32) rc = layer ? OSDP_BWD(float, true) : OSDP_BWD(float, false);
  else rc = layer ? OSDP_BWD(__nv_bfloat16, true) : OSDP_BWD(__nv_bfloat16, false);
#undef OSDP_BWD
  if (rc) return rc;
  if (!dw_post && !db_post && !dgate && !dw_pre && !db_pre) return OSDP_OK;
  FinalArgs f;
  f.partial = a.partial;
  f.units = units;
  f.D = (int)D;
  f.layer = layer;
  f.w_post = a.w_post;
  f.b_post = b_post;
  f.gate = gate;
  f.beta = a.beta;
  f.post_has = a.post_has;
  f.dw_post = dw_post;
  f.db_post = db_post;
  f.dgate = dgate;
  f.dw_pre = dw_pre;
  f.db_pre = db_pre;
  return launch_overlapped(block_norm_final_kernel, dim3((unsigned)cdiv(D, 32)), dim3(1024), 0, 1, s, f);
}

}  // extern "C"

// The experts' products of a mixture of experts: Y[r] = act(X[r] W_e(r)^T + b_e(r)) over rows sorted by expert, and its
// gradients.  The products run on the tile kernel of osdp_gemm.cuh, whose tile list is taken from the plan on the device: no
// count is read back to the host.
#include "../../include/osdp.h"

#include <atomic>
#include <cstring>
#include <mutex>

#include "osdp_experts.h"
#include "osdp_gemm.cuh"
#include "osdp_internal.h"

namespace osdp {
namespace {

// ------------------------------------------------------------------------------------------------
// G = dY (.) act'(Z) and the sums of G's columns for each expert, in one pass (bound by memory).  A block takes 256 columns
// of 64 rows, which are one expert's; the blocks' sums are added in a fixed order by a second kernel.  The sums are of the unrounded G.
// Rows between two experts become zero, whatever dY and Z hold there.
// G itself is rounded to bf16, as the operand that both products take: dX and dW are then off by 0.0023 in the norm where their own
// rounding leaves 0.0017 (without an activation G is dY, which is bf16 as it comes).
struct GradArgs {
  const __nv_bfloat16 *dy, *z;
  __nv_bfloat16 *g;             // null: column sums of dY alone
  const int32_t *plan;
  float *partial;               // [parts of 64 rows][N], or null
  int E, N, act;
};
constexpr int GRAD_ROWS = OSDP_EXPERT_ROWS, GRAD_COLS = 256;

// act'(x) of the tanh form: 0.5 (1 + tanh u) = h = 1 / (1 + exp(-2 u)), and act' = h + 2 x h (1 - h) u'.  The special-function unit's 2^-22
// (tanh.approx has 2^-11, too coarse for sums that are kept in fp32); two elements in an instruction.
__device__ __forceinline__ f2 gelu_tanh_grad2(f2 x) {
  constexpr float a = 0.7978845608028654f, k = -2.0f * 1.4426950408889634f * a;
  const f2 one = both(1.0f), x2 = mul2(x, x);
  const float2 arg = split2(mul2(x, fma2(x2, both(k * 0.044715f), both(k))));
  float e0, e1, h0, h1;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(arg.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(arg.y));
  const float2 d = split2(add2(pack2(e0, e1), one));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(h0) : "f"(d.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(h1) : "f"(d.y));
  const f2 h = pack2(h0, h1), rest = fma2(h, both(-1.0f), one), du = fma2(x2, both(2.0f * a * 0.134145f), both(2.0f * a));
  return fma2(mul2(mul2(x, h), rest), du, h);
}
__device__ __forceinline__ float gelu_erf_grad(float x) {
  return fmaf(x, 0.3989422804014327f * __expf(-0.5f * x * x), 0.5f * erfcf(-0.7071067811865476f * x));
}

__global__ void __launch_bounds__(256, 4) expert_grad_kernel(const __grid_constant__ GradArgs a) {
  __shared__ float red[8][GRAD_COLS];
  pdl_launch_dependents();
  const int cols = (a.N + GRAD_COLS - 1) / GRAD_COLS, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int part = (int)(blockIdx.x / cols), c0 = (int)(blockIdx.x % cols) * GRAD_COLS, col = c0 + lane * 8;
  pdl_wait();
  // Rows warp, warp + 8, ... of the block's 64.  They are there whoever's they are, so that the plan is looked up while they
  // are on their way.
  constexpr int EACH = GRAD_ROWS / 8;
  const long long at = ((long long)part * GRAD_ROWS + warp) * a.N + col;
  constexpr int HALF = EACH / 2;         // at a time: twice the blocks on an SM
  uint4 d[HALF], z[HALF];
  auto load = [&](int h) {
#pragma unroll
    for (int q = 0; q < HALF; ++q) {
      d[q] = load16(a.dy + at + (long long)(h * HALF + q) * 8 * a.N);
      if (a.g) z[q] = load16(a.z + at + (long long)(h * HALF + q) * 8 * a.N);
    }
  };
  if (col < a.N) load(0);
  // the expert whose rows these are: offsets[e] <= row < offsets[e + 1]
  const int32_t *offsets = a.plan + PLAN_OFFSETS;
  int e = -1;
  for (int i = lane; i - lane < a.E; i += 32) e += __popc(__ballot_sync(0xFFFFFFFFu, i < a.E && offsets[i] <= part * GRAD_ROWS));
  if (part * GRAD_ROWS >= offsets[a.E]) return;
  const int count = a.plan[plan_counts(a.E) + e] - (part * GRAD_ROWS - offsets[e]) - warp;
  f2 acc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = both(0.f);
  if (col < a.N) {
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
      if (q > 0 && q % HALF == 0) load(q / HALF);
      f2 f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = both(0.f);
      if (8 * q < count) {
        widen4(d[q % HALF], f);
        if (a.g) {
          f2 x[4];
          widen4(z[q % HALF], x);
          if (a.act == ACT_GELU_TANH) {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = mul2(f[j], gelu_tanh_grad2(x[j]));
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 v = split2(x[j]);
              f[j] = mul2(f[j], pack2(gelu_erf_grad(v.x), gelu_erf_grad(v.y)));
            }
          }
        }
      }
      if (a.g) *reinterpret_cast<uint4 *>(a.g + at + (long long)q * 8 * a.N) = narrow4(f);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = add2(acc[j], f[j]);
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int j = 0; j < 4; ++j) *reinterpret_cast<float2 *>(&red[warp][lane * 8 + 2 * j]) = split2(acc[j]);
  __syncthreads();
  const int c = c0 + threadIdx.x;
  if (c < a.N) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += red[w][threadIdx.x];
    a.partial[(long long)part * a.N + c] = s;
  }
}

// db[e, c]: the parts' sums of expert e in order.
__global__ void __launch_bounds__(128) expert_bias_kernel(const float *partial, const int32_t *plan, int E, int N, float *db) {
  pdl_launch_dependents();
  const int e = (int)blockIdx.y, c = (int)(blockIdx.x * blockDim.x + threadIdx.x);
  pdl_wait();
  if (c >= N) return;
  const int first = plan[PLAN_OFFSETS + e] / GRAD_ROWS, last = plan[PLAN_OFFSETS + e + 1] / GRAD_ROWS;
  float s = 0.f;
#pragma unroll 8
  for (int t = first; t < last; ++t) s += partial[(long long)t * N + c];
  db[(long long)e * N + c] = s;
}

// ------------------------------------------------------------------------------------------------
// Launch of the tile kernel

struct ExpertGemm {
  const void *a, *b;            // GRP_ROWS: rows [R, len], W [E, N, K]; GRP_RED: dY [R, N], X [R, K]
  const float *bias;
  void *out, *z_save;
  const int32_t *plan;
  int *status;
  int64_t T, R, N, K;
  int top_k, E, act, grp, b_mn, out_fp32, accumulate;
};

struct PreparedGemm {
  bool valid = false;
  int device = 0;
  ExpertGemm key;
  GemmParams p;
  int bn;
  bool pair;
  int64_t items;
};
// Prepared launches (encoded tensor maps, tile choice) of this thread, as for the other products: they hold addresses and
// sizes only.
constexpr int PREPARED = 32;
thread_local PreparedGemm g_prepared[PREPARED];

template <int BN, bool A_MN, bool B_MN, bool CTA2, bool HEAVY, int GRP>
int launch_tiles(const GemmParams &p, int64_t items, int sms, cudaStream_t stream) {
  static std::atomic<int> most[64];
  static std::mutex setup;
  using SL = SmemLayout<BN, CTA2, HEAVY>;
  auto kernel = gemm_kernel<BN, A_MN, B_MN, CTA2, HEAVY, 2, false, GRP>;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return report_cuda(e);
  if (dev < 0 || dev >= 64) return report_cuda(cudaErrorInvalidDevice);
  int units = most[dev].load(std::memory_order_acquire);
  if (units == 0) {
    std::lock_guard<std::mutex> lock(setup);
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SL::TOTAL);
    if (e != cudaSuccess) return report_cuda(e);
    units = sms;
    if (CTA2) {
      cudaLaunchConfig_t q = {};
      q.gridDim = dim3(2 * sms, 1, 1);
      q.blockDim = dim3(SL::THREADS, 1, 1);
      q.dynamicSmemBytes = SL::TOTAL;
      cudaLaunchAttribute qa[1];
      qa[0].id = cudaLaunchAttributeClusterDimension;
      qa[0].val.clusterDim.x = 2; qa[0].val.clusterDim.y = 1; qa[0].val.clusterDim.z = 1;
      q.attrs = qa; q.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&units, kernel, &q);
      if (e != cudaSuccess) return report_cuda(e);
      if (units < 1) return report_cuda(cudaErrorLaunchOutOfResources);
    }
    most[dev].store(units, std::memory_order_release);
  }
  const int n = (int)(items < units ? items : units);
  return launch_overlapped(kernel, dim3((unsigned)(CTA2 ? 2 * n : n)), dim3(SL::THREADS), SL::TOTAL, CTA2 ? 2 : 1, stream, p);
}

// Eight epilogue warps everywhere (four but for the widest tile elsewhere): tiles are short, and what is drained from one has to
// be out before the next one is done.
int launch_prepared(const PreparedGemm &s, int sms, cudaStream_t stream) {
  const GemmParams &p = s.p;
  if (s.key.grp == GRP_RED) {
    if (s.pair && s.bn == 512) return launch_tiles<512, true, true, true, false, GRP_RED>(p, s.items, sms, stream);
    if (s.pair) return launch_tiles<256, true, true, true, true, GRP_RED>(p, s.items, sms, stream);
    if (s.bn == 256) return launch_tiles<256, true, true, false, true, GRP_RED>(p, s.items, sms, stream);
    return launch_tiles<128, true, true, false, true, GRP_RED>(p, s.items, sms, stream);
  }
  if (s.key.b_mn) {
    if (s.pair && s.bn == 512) return launch_tiles<512, false, true, true, false, GRP_ROWS>(p, s.items, sms, stream);
    if (s.pair) return launch_tiles<256, false, true, true, true, GRP_ROWS>(p, s.items, sms, stream);
    if (s.bn == 256) return launch_tiles<256, false, true, false, true, GRP_ROWS>(p, s.items, sms, stream);
    return launch_tiles<128, false, true, false, true, GRP_ROWS>(p, s.items, sms, stream);
  }
  if (s.pair && s.bn == 512) return launch_tiles<512, false, false, true, false, GRP_ROWS>(p, s.items, sms, stream);
  if (s.pair) return launch_tiles<256, false, false, true, true, GRP_ROWS>(p, s.items, sms, stream);
  if (s.bn == 256) return launch_tiles<256, false, false, false, true, GRP_ROWS>(p, s.items, sms, stream);
  return launch_tiles<128, false, false, false, true, GRP_ROWS>(p, s.items, sms, stream);
}

int map3(CUtensorMap *m, const void *base, int eb, int64_t inner, int64_t rows, int64_t deep, int box_inner, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)deep};
  const cuuint64_t str[2] = {(cuuint64_t)(inner * eb), (cuuint64_t)(inner * rows * eb)};
  const cuuint32_t box[3] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows, 1};
  return encode_map3d(m, eb == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, base, dims, str, box, true);
}

int launch_expert_gemm(const ExpertGemm &c, cudaStream_t stream) {
  int sms = 0, dev = 0;
  int rc = sm_count(&sms);
  if (rc) return rc;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return report_cuda(e);
  // (ExpertGemm is compared as bytes: callers clear it first)
  uint64_t h = 1469598103934665603ull;
  const unsigned char *bytes = reinterpret_cast<const unsigned char *>(&c);
  for (size_t i = 0; i < sizeof(c); i += 8) {
    uint64_t w = 0;
    memcpy(&w, bytes + i, sizeof(c) - i < 8 ? sizeof(c) - i : 8);
    h = (h ^ w) * 1099511628211ull;
    h ^= h >> 29;
  }
  PreparedGemm &slot = g_prepared[h % PREPARED];
  if (slot.valid && slot.device == dev && memcmp(&slot.key, &c, sizeof(c)) == 0) return launch_prepared(slot, sms, stream);
  slot.valid = false;
  slot.device = dev;
  memcpy(&slot.key, &c, sizeof(c));
  GemmParams &p = slot.p;
  memset(&p, 0, sizeof(p));
  const int64_t n = c.T * c.top_k, used = n < c.E ? n : c.E;
  const bool red = c.grp == GRP_RED;
  p.P = (int)(red ? c.N : c.R);
  p.Q = (int)(red ? c.K : (c.b_mn ? c.K : c.N));
  p.R = (int)(red ? c.R : (c.b_mn ? c.N : c.K));
  // Tiles, were the choices spread evenly (only the device knows): one for each expert that has rows, or half a tile more than the
  // rows fill.
  auto tiles = [&](int tm, int bn) {
    const int64_t full = n / tm + cdiv(used, 2), m = red ? cdiv(c.N, tm) * c.E : (full > used ? full : used);
    return m * cdiv(p.Q, bn);
  };
  // CTA pairs on 256 rows where the experts fill most of such a tile (a weight gradient: its matrix), and there are tiles for a third
  // of the SMs; outputs of at most 128 columns take single CTAs, which waste half as much of a tile.  256 columns where there are
  // tiles for most SMs.  Measured (us; single 128, single 256, pair 256, pair 512; * is the choice), T x top_k of E, K -> N:
  //   forward  300 x 2 of 8, 1024 -> 2048    13.6* 14.6  15.8  19.2    input   600 x 2 of 4, 2048 -> 1024   14.2* 13.6  12.8  21.9
  //   forward  2000 x 2 of 8, 2048 -> 512    14.9* 19.0  25.6  29.0    input   2000 x 2 of 8, 2048 -> 512   17.2  15.3  17.9* 22.8
  //   forward  4096 x 2 of 64, 2048 -> 1024  66.7  64.6* 67.3  66.2    input   4096 x 2 of 64, 2048 -> 1024 68.7  62.6* 68.1  67.7
  //   forward  8192 x 2 of 8, 2048 -> 1024   78.6  64.4  55.6* 57.5    input   8192 x 2 of 8, 2048 -> 8192  525   456   398   385*
  //   forward  8192 x 2 of 8, 2048 -> 8192   504   416   380*  393     weights 100 x 2 of 4, 1024 -> 1024    5.2   5.4   6.6*  8.0
  //   forward  2000 x 2 of 8, 1024 -> 1024   16.9  14.0  24.1  21.7*   weights 600 x 2 of 4, 2048 -> 1024   11.9  11.1  10.2  11.7*
  //   weights  64 x 2 of 16, 2048 -> 8192    132   103   101*  123     weights 8192 x 2 of 8, 512 -> 2048   50.1  44.3  37.6  39.4*
  // (The rule is off where a few hundred rows of an expert make one short wave of wide tiles: the sixth line.)
  const bool narrow = p.Q <= 128;
  const bool pair = !narrow && tiles(256, 256) >= sms / 3 && (red ? c.N > 128 : n >= 160 * used);
  int bn = 128;
  if (pair || (!narrow && tiles(128, 256) >= (int64_t)sms * 4 / 5)) bn = 256;
  const double len = red ? (double)n / (double)used : (double)p.R;
  if (pair && c.act == ACT_NONE) {
    // The wider tile (its epilogue does not overlap the next tile): waves times us for a unit of the reduction, and 5 us for what
    // does not overlap, once in the run or once a tile; rates and epilogue as measured for the other products.
    const double t_n = (double)cdiv(tiles(256, 256), sms / 2) * (6.5e-3 * len) + 5.0;
    const double t_w = (double)cdiv(tiles(256, 512), sms / 2) * (11.5e-3 * len + 5.0);
    if (t_w < 0.97 * t_n) bn = 512;
  }
  const int b_rows = pair ? 128 : bn;
  if (red) {
    rc = map3(&p.a_main, c.a, 2, c.N, c.R, 1, 64, 64);
    if (!rc) rc = map3(&p.b_main, c.b, 2, c.K, c.R, 1, 64, 64);
    if (!rc) rc = map3(&p.out_main, c.out, c.out_fp32 ? 4 : 2, c.K, c.N, c.E, c.out_fp32 ? 32 : 64, 32);
  } else {
    rc = map3(&p.a_main, c.a, 2, p.R, c.R, 1, 64, 128);
    if (!rc) rc = map3(&p.b_main, c.b, 2, c.K, c.N, c.E, 64, c.b_mn ? 64 : b_rows);
    if (!rc) rc = map3(&p.out_main, c.out, 2, p.Q, c.R, 1, 64, 32);
    if (!rc && c.z_save) rc = map3(&p.z_main, c.z_save, 2, p.Q, c.R, 1, 64, 32);
  }
  if (rc) return rc;
  p.a_tail = p.a_main;
  p.b_tail = p.b_main; p.out_tail = p.out_main; p.z_tail = p.z_main; p.carry_map = p.out_main;
  p.mode = MODE_NONE;
  p.L = 0; p.k_total = 1; p.s_begin = 0; p.s_end = 1;
  p.red_group = 1;
  p.round_kblocks = 2;
  p.tma_epilogue = 1;
  p.bk = 64;
  p.a_rows = BM;
  p.epi.out = c.out;
  p.epi.ld_out = p.Q;
  p.epi.out_fp32 = c.out_fp32;
  p.epi.accumulate = c.accumulate;
  p.epi.bias = c.bias;
  p.epi.z_save = static_cast<__nv_bfloat16 *>(c.z_save);
  p.epi.ld_z = p.Q;
  p.epi.act = c.act;
  p.epi.scale = 1.0f;
  p.status = c.status;
  p.seg_offsets = c.plan + PLAN_OFFSETS;
  p.seg_counts = c.plan + plan_counts(c.E);
  p.seg_tiles = c.plan + (pair ? plan_tiles256(c.E) : plan_tiles128(c.E));
  p.experts = c.E;
  slot.pair = pair;
  slot.bn = bn;
  // at most: every expert that can have rows leaves one tile partly filled
  const int tm = pair ? 256 : 128;
  slot.items = red ? tiles(tm, bn) : (n / tm + used) * cdiv(p.Q, bn);
  if (slot.items >= (1 << 24)) return OSDP_ERR_BAD_SHAPE;      // what the kernel's tile arithmetic is exact for
  slot.valid = true;
  return launch_prepared(slot, sms, stream);
}

// ------------------------------------------------------------------------------------------------

struct ExpertWs {
  size_t partial, g, total;
};
int expert_workspace(int64_t T, int top_k, int E, int64_t N, int64_t K, int act, int op, ExpertWs *w) {
  const int rc = expert_check(T, top_k, E);
  if (rc) return rc;
  if (N <= 0 || K <= 0 || N > ((int64_t)1 << 24) || K > ((int64_t)1 << 24)) return OSDP_ERR_BAD_SHAPE;
  if ((N & 7) || (K & 7)) return OSDP_ERR_ALIGNMENT;
  if (act != OSDP_ACT_NONE && act != OSDP_ACT_GELU_TANH && act != OSDP_ACT_GELU_ERF) return OSDP_ERR_UNSUPPORTED;
  const int64_t R = expert_rows(T, top_k, E);
  if (R >= ((int64_t)1 << 31) - 256) return OSDP_ERR_BAD_SHAPE;
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  w->partial = w->g = w->total = 256;
  if (op == OSDP_OP_LINEAR_FWD) return OSDP_OK;
  if (op != OSDP_OP_LINEAR_BWD) return OSDP_ERR_UNSUPPORTED;
  const int64_t blocks = (R / GRAD_ROWS) * cdiv(N, GRAD_COLS);
  if (blocks >= ((int64_t)1 << 31)) return OSDP_ERR_BAD_SHAPE;
  w->g = w->partial + up((size_t)(R / GRAD_ROWS) * N * 4);
  w->total = w->g + (act == OSDP_ACT_NONE ? 0 : up((size_t)R * N * 2));
  return OSDP_OK;
}
int check_workspace(const void *ws, size_t bytes, const ExpertWs &w) {
  if (!ws) return OSDP_ERR_NULL_POINTER;
  if (!aligned_to(ws, 256)) return OSDP_ERR_ALIGNMENT;
  return bytes < w.total ? OSDP_ERR_WORKSPACE_TOO_SMALL : OSDP_OK;
}

}  // namespace
}  // namespace osdp

using namespace osdp;

extern "C" int osdp_expert_linear_workspace_bytes(int64_t T, int top_k, int E, int64_t N, int64_t K, int act, int op, size_t *bytes) {
  if (!bytes) return OSDP_ERR_NULL_POINTER;
  ExpertWs w;
  const int rc = expert_workspace(T, top_k, E, N, K, act, op, &w);
  if (rc) return rc;
  *bytes = w.total;
  return OSDP_OK;
}

extern "C" int osdp_expert_linear_fwd(const void *rows, const int32_t *plan, const void *w_flat, int64_t w_offset, const float *bias, int64_t T,
                                      int top_k, int E, int64_t N, int64_t K, int act, void *out, void *z_save, void *ws, size_t ws_bytes,
                                      void *stream) {
  ExpertWs w;
  int rc = expert_workspace(T, top_k, E, N, K, act, OSDP_OP_LINEAR_FWD, &w);
  if (rc) return rc;
  if (T == 0) return OSDP_OK;
  if (!rows || !plan || !w_flat || !out) return OSDP_ERR_NULL_POINTER;
  if (w_offset < 0 || (w_offset & 7) || !aligned_to(rows, 16) || !aligned_to(plan, 16) || !aligned_to(w_flat, 16) || !aligned_to(bias, 16) ||
      !aligned_to(out, 16) || !aligned_to(z_save, 16))
    return OSDP_ERR_ALIGNMENT;
  rc = check_workspace(ws, ws_bytes, w);
  if (rc) return rc;
  if (expert_few_rows(T, top_k, E, N, K))
    return launch_expert_few(rows, plan, static_cast<const __nv_bfloat16 *>(w_flat) + w_offset, bias, T, top_k, E, N, K, act, out, z_save,
                             static_cast<cudaStream_t>(stream));
  ExpertGemm c;
  memset(&c, 0, sizeof(c));
  c.a = rows;
  c.b = static_cast<const __nv_bfloat16 *>(w_flat) + w_offset;
  c.bias = bias;
  c.out = out;
  c.z_save = z_save;
  c.plan = plan;
  c.status = static_cast<int *>(ws);
  c.T = T; c.R = expert_rows(T, top_k, E); c.N = N; c.K = K;
  c.top_k = top_k; c.E = E; c.act = act; c.grp = GRP_ROWS;
  return launch_expert_gemm(c, static_cast<cudaStream_t>(stream));
}

extern "C" int osdp_expert_linear_bwd(const void *dy, const void *rows, const int32_t *plan, const void *w_flat, int64_t w_offset,
                                      const void *z_saved, int64_t T, int top_k, int E, int64_t N, int64_t K, int act, void *dx, void *dw_flat,
                                      int64_t dw_offset, int dw_dtype, int flags, float *dbias, void *ws, size_t ws_bytes, void *stream_) {
  ExpertWs w;
  int rc = expert_workspace(T, top_k, E, N, K, act, OSDP_OP_LINEAR_BWD, &w);
  if (rc) return rc;
  if ((flags & ~OSDP_FLAG_ACCUMULATE_DW) || (dw_dtype != OSDP_DTYPE_BF16 && dw_dtype != OSDP_DTYPE_FP32)) return OSDP_ERR_UNSUPPORTED;
  if (!plan || (T > 0 && (!dy || (dx && !w_flat) || (dw_flat && !rows) || (act != OSDP_ACT_NONE && !z_saved)))) return OSDP_ERR_NULL_POINTER;
  if (w_offset < 0 || (w_offset & 7) || dw_offset < 0 || (dw_offset & 7) || !aligned_to(dy, 16) || !aligned_to(rows, 16) || !aligned_to(plan, 16) ||
      !aligned_to(w_flat, 16) || !aligned_to(z_saved, 16) || !aligned_to(dx, 16) || !aligned_to(dw_flat, 16) || !aligned_to(dbias, 16))
    return OSDP_ERR_ALIGNMENT;
  rc = check_workspace(ws, ws_bytes, w);
  if (rc) return rc;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  const int64_t R = expert_rows(T, top_k, E);
  void *dw = nullptr;
  const size_t dw_bytes = (size_t)E * N * K * (dw_dtype == OSDP_DTYPE_FP32 ? 4 : 2);
  if (dw_flat) dw = static_cast<char *>(dw_flat) + dw_offset * (dw_dtype == OSDP_DTYPE_FP32 ? 4 : 2);
  if (T == 0) {   // no rows: the weights' gradients are zero
    cudaError_t e = cudaSuccess;
    if (dw && !(flags & OSDP_FLAG_ACCUMULATE_DW)) e = cudaMemsetAsync(dw, 0, dw_bytes, stream);
    if (e == cudaSuccess && dbias) e = cudaMemsetAsync(dbias, 0, (size_t)E * N * 4, stream);
    return report_cuda(e);
  }
  char *wsb = static_cast<char *>(ws);
  float *partial = reinterpret_cast<float *>(wsb + w.partial);
  const void *g = dy;
  if (act != OSDP_ACT_NONE || dbias) {
    __nv_bfloat16 *stage = act != OSDP_ACT_NONE ? reinterpret_cast<__nv_bfloat16 *>(wsb + w.g) : nullptr;
    const GradArgs a{static_cast<const __nv_bfloat16 *>(dy), static_cast<const __nv_bfloat16 *>(z_saved), stage, plan, dbias ? partial : nullptr, E,
                     (int)N, act};
    rc = launch_overlapped(expert_grad_kernel, dim3((unsigned)((R / GRAD_ROWS) * cdiv(N, GRAD_COLS))), dim3(256), 0, 1, stream, a);
    if (rc) return rc;
    if (stage) g = stage;
  }
  if (dbias) {
    rc = launch_overlapped(expert_bias_kernel, dim3((unsigned)cdiv(N, 128), (unsigned)E), dim3(128), 0, 1, stream, partial, plan, E, (int)N, dbias);
    if (rc) return rc;
  }
  ExpertGemm c;
  memset(&c, 0, sizeof(c));
  c.plan = plan;
  c.status = static_cast<int *>(ws);
  c.T = T; c.R = R; c.N = N; c.K = K;
  c.top_k = top_k; c.E = E; c.act = OSDP_ACT_NONE;
  if (dx) {
    c.a = g;
    c.b = static_cast<const __nv_bfloat16 *>(w_flat) + w_offset;
    c.out = dx;
    c.grp = GRP_ROWS;
    c.b_mn = 1;
    rc = launch_expert_gemm(c, stream);
    if (rc) return rc;
  }
  if (dw) {
    c.a = g;
    c.b = rows;
    c.out = dw;
    c.grp = GRP_RED;
    c.b_mn = 0;
    c.out_fp32 = dw_dtype == OSDP_DTYPE_FP32;
    c.accumulate = (flags & OSDP_FLAG_ACCUMULATE_DW) ? 1 : 0;
    rc = launch_expert_gemm(c, stream);
    if (rc) return rc;
  }
  return OSDP_OK;
}

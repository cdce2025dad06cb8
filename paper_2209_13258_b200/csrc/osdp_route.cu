// Mixture of experts around the split linear layers: which experts a token goes to (forward and backward), where its rows
// lie among the experts' rows, and the way there (dispatch) and back (combine).  The experts' products: osdp_experts.cu.
#include "../../include/osdp.h"

#include <cmath>

#include "osdp_experts.h"
#include "osdp_internal.h"
#include "osdp_vec.cuh"

namespace osdp {
namespace {

constexpr uint32_t ALL = 0xFFFFFFFFu;

// ------------------------------------------------------------------------------------------------
// Routing.  One warp per token; lane l holds experts l, l + 32, ... in registers.
//
// The choice has to be the one of exact arithmetic: another expert is another result.  Without a bias the scores are a
// monotone function of the logits, so the experts are chosen by the logits themselves.  With a bias (and for the sums of the
// groups) scores are formed in fp32, and where two of those that decide are closer than their rounding the row is done again
// in fp64: some rows in a thousand, so that the price of a batch in fp64 is not paid.

struct RouteArgs {
  const void *logits;
  long long ld, T;
  const float *bias;
  int E, k, score, groups, top_groups, take, renorm;
  float scale;
  int32_t *idx;
  float *weights;
};

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }

// Order-preserving keys; 0 is below every key.  NaN counts as minus infinity, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0x007FFFFFu;
  return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ unsigned long long key_of(double x) {
  const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);
  if ((u & 0x7FFFFFFFFFFFFFFFull) > 0x7FF0000000000000ull) return 0x000FFFFFFFFFFFFFull;
  return (u >> 63) ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ uint32_t warp_top(uint32_t k) { return __reduce_max_sync(ALL, k); }
__device__ __forceinline__ unsigned long long warp_top(unsigned long long k) {
  const uint32_t hi = __reduce_max_sync(ALL, (uint32_t)(k >> 32));
  const uint32_t lo = __reduce_max_sync(ALL, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
  return ((unsigned long long)hi << 32) | lo;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float((key >> 31) ? key & 0x7FFFFFFFu : ~key); }

__device__ __forceinline__ float exp_of(float x) { return expf(x); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }
template <typename R>
__device__ __forceinline__ R sum_of(R v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(ALL, v, o);
  return v;
}

// Chooses the row's experts: lane j < k leaves with the j-th in `mine`.  Returns false where R is too short to say.
// `room` [E] of R: this warp's shared memory.
template <typename R, int V, typename L>
__device__ __noinline__ bool choose(const RouteArgs &a, const L *row, const float (&l)[V], R *room, int lane, int &mine) {
  using Key = decltype(key_of(R(0)));
  const R low = -(R)INFINITY;
  const bool grouped = a.top_groups < a.groups;
  Key key[V];
  R c[V];
  float far = 0.f;                    // largest |bias|: what a score's rounding is relative to, beside the score
  if (a.bias || grouped) {
    if (a.score == OSDP_SCORE_SOFTMAX) {
      uint32_t top = 0;
#pragma unroll
      for (int v = 0; v < V; ++v) top = max(top, v * 32 + lane < a.E ? key_of(l[v]) : 0u);
      const R high = (R)value_of(__reduce_max_sync(ALL, top));
      R total = 0;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        c[v] = v * 32 + lane < a.E && l[v] != -INFINITY ? exp_of((R)l[v] - high) : (R)0;
        total += c[v];
      }
      total = sum_of(total);
      const R inv = total > (R)0 ? (R)1 / total : total;   // (a row of minus infinities: all scores are zero)
#pragma unroll
      for (int v = 0; v < V; ++v) c[v] *= inv;
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) c[v] = (R)1 / ((R)1 + exp_of(-(R)l[v]));
    }
    if (a.bias) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float b = v * 32 + lane < a.E ? a.bias[v * 32 + lane] : 0.f;
        c[v] += (R)b;
        far = fmaxf(far, fabsf(b));
      }
      if (sizeof(R) == 4) far = __uint_as_float(__reduce_max_sync(ALL, __float_as_uint(far)));
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) key[v] = v * 32 + lane < a.E ? (a.bias ? key_of(c[v]) : (Key)key_of((R)l[v])) : (Key)0;
  // How far the fp32 scores may be off, relative to themselves and the bias: the sigmoid's exponential (two units in the last
  // place), sum, quotient and the bias are 7 roundings of 2^-24; a softmax has up to 37 in its total, and its exponent's
  // rounding counts |l - max| times (beyond 80 nothing is left of a score).
  const float off = (a.score == OSDP_SCORE_SIGMOID ? 8.0f : 128.0f) * 5.9604645e-8f;
  bool sure = true;
  if (grouped) {
    const int size = a.E / a.groups;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v * 32 + lane < a.E) room[v * 32 + lane] = c[v] == c[v] ? c[v] : low;
    __syncwarp();
    // `per` lanes for each group
    int per = 32;
    while (per * a.groups > 32) per >>= 1;
    const int g = lane / per;
    R first = low, second = low;
    if (g < a.groups) {
      for (int e = lane % per; e < size; e += per) {
        const R x = room[g * size + e];
        second = x > first ? first : (x > second ? x : second);
        first = x > first ? x : first;
      }
    }
    for (int o = 1; o < per; o <<= 1) {
      const R f = __shfl_xor_sync(ALL, first, o), s = __shfl_xor_sync(ALL, second, o);
      const R less = f > first ? first : f;
      second = s > second ? s : second;
      second = less > second ? less : second;
      first = f > first ? f : first;
    }
    R sum = a.take > 1 && size > 1 ? first + second : first;
    if (sum != sum) sum = low;
    int rank = 0;
    for (int h = 0; h < a.groups; ++h) {
      const R other = __shfl_sync(ALL, sum, h * per);
      rank += other > sum || (other == sum && h < g) ? 1 : 0;
    }
    const bool in = g < a.groups && rank < a.top_groups;
    const uint32_t taken = __ballot_sync(ALL, in && lane % per == 0);
    if (sizeof(R) == 4) {
      // the last group that is taken against the first that is not
      const float last = value_of(~__reduce_max_sync(ALL, in ? ~key_of((float)sum) : 0u));
      const float next = value_of(__reduce_max_sync(ALL, g < a.groups && !in ? key_of((float)sum) : 0x007FFFFFu));
      if (last - next <= 2.0f * off * (fabsf(last) + 2.0f * far)) sure = false;
    }
    const uint32_t magic = (1048576u + size - 1) / size;      // e / size for e < 1024
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const uint32_t mine_g = (uint32_t)(v * 32 + lane) * magic >> 20;
      if (v * 32 + lane < a.E && !((taken >> (mine_g * per)) & 1u)) key[v] = 0;
    }
    __syncwarp();
  }
  // one more than are wanted, to see how far away it is
  float value = 0.f;
  for (int j = 0; j <= a.k; ++j) {
    Key best = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) best = key[v] > best ? key[v] : best;
    best = warp_top(best);
    if (best == 0) break;             // (only behind the last one wanted: the groups have enough experts)
    int e = 1 << 20;
#pragma unroll
    for (int v = V - 1; v >= 0; --v) e = key[v] == best ? v * 32 + lane : e;
    e = __reduce_min_sync(ALL, e);
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = v * 32 + lane == e ? (Key)0 : key[v];
    if (lane == j) {
      mine = e;
      if (sizeof(R) == 4) value = value_of((uint32_t)best);
    }
    if (!a.bias && j + 1 == a.k) break;
  }
  if (sizeof(R) == 4 && a.bias) {
    const int after = __shfl_down_sync(ALL, mine, 1);
    const float less = __shfl_down_sync(ALL, value, 1);
    // as close as that: the same in exact arithmetic only if it is the same logit and the same bias
    if (lane < a.k && after >= 0 && value - less <= off * (fabsf(value) + fabsf(less) + 2.0f * far) &&
        (widen(row[mine]) != widen(row[after]) || a.bias[mine] != a.bias[after]))
      sure = false;
  }
  return __all_sync(ALL, sure);
}

// The weights' parts of the chosen experts, lanes 0 .. k - 1 (their logits in `l`): r_j = s_j / sum s, formed from the chosen
// logits alone and relative to their largest, so that neither other logits nor a score's underflow matter.  A sum of nothing
// (all chosen logits minus infinity) gives zeros.
__device__ __forceinline__ float share_of(const RouteArgs &a, float l, bool on, int lane) {
  const float top = value_of(__reduce_max_sync(ALL, on ? key_of(l) : 0x007FFFFFu));
  float s;
  if (a.score == OSDP_SCORE_SIGMOID && top > -60.0f) s = 1.0f / (1.0f + expf(-l));
  else s = l == -INFINITY ? 0.f : expf(l - top);               // (a sigmoid this small is its exponential)
  const float total = warp_sum(on ? s : 0.f);
  return total == 0.f ? 0.f : s / total;
}

template <typename L, int V>
__global__ void __launch_bounds__(256) route_fwd_kernel(const __grid_constant__ RouteArgs a) {
  extern __shared__ double rooms[];
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long t = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  pdl_wait();
  if (t >= a.T) return;
  double *room = rooms + (threadIdx.x >> 5) * a.E;
  const L *row = static_cast<const L *>(a.logits) + t * a.ld;
  float l[V];
#pragma unroll
  for (int v = 0; v < V; ++v) l[v] = v * 32 + lane < a.E ? widen(row[v * 32 + lane]) : -INFINITY;
  int mine = -1;
  if (!choose<float, V, L>(a, row, l, reinterpret_cast<float *>(room), lane, mine)) {
    __syncwarp();
    choose<double, V, L>(a, row, l, room, lane, mine);
  }
  const bool on = lane < a.k;
  const float lj = on ? widen(row[mine]) : -INFINITY;
  float w;
  if (a.renorm) {
    w = share_of(a, lj, on, lane);
  } else if (a.score == OSDP_SCORE_SIGMOID) {
    w = 1.0f / (1.0f + expf(-lj));
  } else {
    uint32_t top = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) top = max(top, key_of(l[v]));
    const float high = value_of(__reduce_max_sync(ALL, top));
    float total = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) total += l[v] == -INFINITY ? 0.f : expf(l[v] - high);
    total = warp_sum(total);
    w = lj == -INFINITY && total == total ? 0.f : expf(lj - high) / total;
  }
  if (on) {
    a.idx[t * a.k + lane] = mine;
    a.weights[t * a.k + lane] = w * a.scale;
  }
}

// ------------------------------------------------------------------------------------------------
// Backward of the routing.  Renormalised, with r_j = s_j / sum of the chosen s and g_j = scale dw_j:
//   softmax: dl_j = r_j (g_j - sum_i g_i r_i);  sigmoid: the same times (1 - s_j);  other logits have no gradient.
// Not renormalised: sigmoid dl_j = g_j s_j (1 - s_j);  softmax dl_e = s_e (g_e - sum_i g_i s_i) for every e (g_e = 0 where
// the expert was not chosen), the one case that reads all logits.
struct RouteBackArgs {
  RouteArgs r;
  const float *dweights;
  void *dlogits;
  long long ld_out;
  int dense;                    // ld_out == E and a 16-byte aligned dlogits: rows are cleared in 16-byte pieces
};

__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

constexpr int ROUTE_WARPS = 8;

template <typename L>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) route_bwd_kernel(const __grid_constant__ RouteBackArgs b) {
  pdl_launch_dependents();
  const RouteArgs &a = b.r;
  const int lane = threadIdx.x & 31;
  const long long t0 = (long long)blockIdx.x * ROUTE_WARPS, t = t0 + (threadIdx.x >> 5);
  L *out = static_cast<L *>(b.dlogits);
  pdl_wait();
  const bool all = a.score == OSDP_SCORE_SOFTMAX && !a.renorm;
  const bool on = lane < a.k && t < a.T;
  int e = on ? a.idx[t * a.k + lane] : -1;
  if (e < 0 || e >= a.E) e = -1;           // a choice that is none has no gradient
  const float g = on && e >= 0 ? b.dweights[t * a.k + lane] * a.scale : 0.f;
  const L *row = static_cast<const L *>(a.logits) + (t < a.T ? t : 0) * a.ld;
  const float l = e >= 0 ? widen(row[e]) : -INFINITY;
  if (!all) {
    // eight whole rows are a multiple of 16 bytes
    if (b.dense) {
      const int rows = (int)min((long long)ROUTE_WARPS, a.T - t0);
      const int bytes = rows * a.E * (int)sizeof(L);
      char *base = reinterpret_cast<char *>(out + t0 * a.E);
      for (int i = threadIdx.x * 16; i + 16 <= bytes; i += blockDim.x * 16) *reinterpret_cast<uint4 *>(base + i) = make_uint4(0u, 0u, 0u, 0u);
      const int rest = bytes & ~15;
      if (rest + (int)threadIdx.x * (int)sizeof(L) < bytes) put(reinterpret_cast<L *>(base + rest) + threadIdx.x, 0.f);
    } else if (t < a.T) {
      for (int i = lane; i < a.E; i += 32) put(out + t * b.ld_out + i, 0.f);
    }
    float d;
    const float s = a.score == OSDP_SCORE_SIGMOID ? 1.0f / (1.0f + expf(-l)) : 0.f;
    if (a.renorm) {
      const float r = share_of(a, l, e >= 0, lane);
      d = r * (g - warp_sum(e >= 0 ? g * r : 0.f)) * (1.0f - s);
    } else {
      d = g * s * (1.0f - s);
    }
    // a token that was given the same expert twice: one gradient, the sum
    const uint32_t same = __match_any_sync(ALL, e);
    float sum = 0.f;
    for (int j = 0; j < a.k; ++j) {
      const float dj = __shfl_sync(ALL, d, j);
      sum += (same >> j) & 1u ? dj : 0.f;
    }
    __syncthreads();                       // the rows are clear
    if (e >= 0 && lane == __ffs(same) - 1) put(out + t * b.ld_out + e, sum);
    return;
  }
  if (t >= a.T) return;
  float high = -INFINITY, total = 0.f;
  {
    uint32_t top = 0;
    for (int i = lane; i < a.E; i += 32) top = max(top, key_of(widen(row[i])));
    high = value_of(__reduce_max_sync(ALL, top));
    for (int i = lane; i < a.E; i += 32) {
      const float x = widen(row[i]);
      total += x == -INFINITY ? 0.f : expf(x - high);
    }
    total = warp_sum(total);
  }
  const float inv = total == 0.f ? 0.f : 1.0f / total;
  const float mean = warp_sum(e >= 0 && l != -INFINITY ? g * (expf(l - high) * inv) : 0.f);
  for (int i0 = 0; i0 < a.E; i0 += 32) {
    const int i = i0 + lane;
    float ge = 0.f;
    for (int j = 0; j < a.k; ++j) {
      const int ej = __shfl_sync(ALL, e, j);
      const float gj = __shfl_sync(ALL, g, j);
      ge += ej == i ? gj : 0.f;
    }
    if (i < a.E) {
      const float x = widen(row[i]);
      put(out + t * b.ld_out + i, (x == -INFINITY ? 0.f : expf(x - high) * inv) * (ge - mean));
    }
  }
}

// ------------------------------------------------------------------------------------------------
// The plan: a stable counting sort of the T k choices by expert.  One launch of a cluster: a warp counts a contiguous part
// of the choices into its own table, the tables' prefix sums over warps and (through distributed shared memory) over the
// cluster's blocks say where each warp's rows of each expert start, and a second pass hands them out in order.  No
// atomics between warps: the same choices give the same plan.
struct PlanArgs {
  const int32_t *idx;
  long long n;
  int E;
  int32_t *plan, *pos;
};
constexpr int PLAN_WARPS = 32;

__device__ __forceinline__ uint32_t cta_rank_in_cluster() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t ctas_in_cluster() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ int peer_int(const int *p, uint32_t cta) {
  uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(p)), v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(at), "r"(cta));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return (int)v;
}
// Inclusive sums over the block's 1024 threads.
__device__ __forceinline__ int block_scan(int v, int *warps) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(ALL, v, o);
    if (lane >= o) v += u;
  }
  if (lane == 31) warps[warp] = v;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < warp; ++w) before += warps[w];
  __syncthreads();
  return v + before;
}

__global__ void __launch_bounds__(32 * PLAN_WARPS, 1) expert_plan_kernel(const __grid_constant__ PlanArgs a) {
  extern __shared__ int tables[];              // [PLAN_WARPS][E], then this block's totals [E]
  __shared__ int sums[PLAN_WARPS];
  const int E = a.E, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;
  int *totals = tables + PLAN_WARPS * E;
  const uint32_t rank = cta_rank_in_cluster(), ctas = ctas_in_cluster();
  pdl_launch_dependents();
  for (int i = tid; i < PLAN_WARPS * E; i += blockDim.x) tables[i] = 0;
  __syncthreads();
  pdl_wait();
  int *mine = tables + warp * E;
  const long long parts = (long long)ctas * PLAN_WARPS;
  const long long part = ((a.n + parts - 1) / parts + 31) / 32 * 32;
  const long long begin = ((long long)rank * PLAN_WARPS + warp) * part, end = min(a.n, begin + part);
  constexpr int AHEAD = 4;
  auto expert_at = [&](long long i) { return i < end ? a.idx[i] : -1; };
  for (long long i0 = begin; i0 < end; i0 += 32 * AHEAD) {
    int e[AHEAD];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) e[q] = expert_at(i0 + 32 * q + lane);
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      const uint32_t same = __match_any_sync(ALL, e[q]);
      if (e[q] >= 0 && e[q] < E && lane == __ffs(same) - 1) mine[e[q]] += __popc(same);
      __syncwarp();
    }
  }
  __syncthreads();
  if (tid < E) {
    int run = 0;
    for (int w = 0; w < PLAN_WARPS; ++w) {
      const int c = tables[w * E + tid];
      tables[w * E + tid] = run;
      run += c;
    }
    totals[tid] = run;
  }
  cluster_sync();
  int before = 0, count = 0;
  if (tid < E) {
    for (uint32_t c = 0; c < ctas; ++c) {
      const int v = peer_int(totals + tid, c);
      if (c < rank) before += v;
      count += v;
    }
  }
  const int padded = (count + OSDP_EXPERT_ROWS - 1) / OSDP_EXPERT_ROWS * OSDP_EXPERT_ROWS;
  const int offset = block_scan(padded, sums) - padded;
  if (tid < E)
    for (int w = 0; w < PLAN_WARPS; ++w) tables[w * E + tid] += offset + before;
  if (rank == 0) {
    int32_t *p = a.plan;
    const int t128 = (count + 127) / 128, t256 = (count + 255) / 256, live = count > 0 ? 1 : 0;
    const int s128 = block_scan(t128, sums), s256 = block_scan(t256, sums), at = block_scan(live, sums);
    if (tid < E) {
      p[PLAN_OFFSETS + tid] = offset;
      p[plan_counts(E) + tid] = count;
      p[plan_tiles128(E) + tid] = s128 - t128;
      p[plan_tiles256(E) + tid] = s256 - t256;
      if (live) p[plan_live(E) + at - 1] = tid;
      if (tid == E - 1) {
        p[PLAN_OFFSETS + E] = offset + padded;
        p[plan_tiles128(E) + E] = s128;
        p[plan_tiles256(E) + E] = s256;
        p[plan_n_live(E)] = at;
      }
    }
  }
  __syncthreads();
  for (long long i0 = begin; i0 < end; i0 += 32 * AHEAD) {
    int e[AHEAD];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) e[q] = expert_at(i0 + 32 * q + lane);
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      const long long i = i0 + 32 * q + lane;
      const uint32_t same = __match_any_sync(ALL, e[q]);
      const bool in = e[q] >= 0 && e[q] < E;
      const int first = in ? mine[e[q]] : 0;
      __syncwarp();
      if (in && lane == __ffs(same) - 1) mine[e[q]] = first + __popc(same);
      __syncwarp();
      if (i < end) a.pos[i] = in ? first + __popc(same & ((1u << lane) - 1u)) : -1;
    }
  }
  cluster_sync();        // nobody leaves while another block may still read its totals
}

// ------------------------------------------------------------------------------------------------
// Dispatch, combine.  A thread has eight channels of one token: it reads the token's piece once and writes it to the k rows,
// or adds the k rows' pieces in order of the choices.  Bound by memory.
struct RowsArgs {
  const __nv_bfloat16 *x;        // dispatch: [T, D]; combine: rows
  const int32_t *plan, *pos;
  const float *weights;
  const __nv_bfloat16 *y;        // dispatch as the backward of combine: the rows that were combined
  __nv_bfloat16 *out;            // dispatch: rows; combine: [T, D]
  float *dweights;
  long long T;
  int k, E, D;
  long long token_blocks;        // dispatch: the blocks behind these clear the rows between the experts
  int team;                      // dispatch with dweights: warps to a (token, choice)
};

__device__ __forceinline__ void clear_between(const RowsArgs &a, int e) {
  const long long first = a.plan[PLAN_OFFSETS + e] + a.plan[plan_counts(a.E) + e];
  const long long n = (a.plan[PLAN_OFFSETS + e + 1] - first) * (a.D >> 3);
  uint4 *p = reinterpret_cast<uint4 *>(a.out + first * a.D);
  for (long long i = threadIdx.x; i < n; i += blockDim.x) p[i] = make_uint4(0u, 0u, 0u, 0u);
}

__global__ void __launch_bounds__(256) dispatch_kernel(const __grid_constant__ RowsArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  if (blockIdx.x >= a.token_blocks) return clear_between(a, (int)(blockIdx.x - a.token_blocks));
  const int pieces = a.D >> 3;
  const long long n = a.T * pieces, stride = a.token_blocks * blockDim.x;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += stride) {
    const long long t = i / pieces;
    const int c = (int)(i - t * pieces) << 3;
    const uint4 v = load16(a.x + t * a.D + c);
    const int32_t *pos = a.pos + t * a.k;
    if (!a.weights) {
      for (int j = 0; j < a.k; ++j) {
        const long long r = pos[j];
        if (r >= 0) *reinterpret_cast<uint4 *>(a.out + r * a.D + c) = v;
      }
    } else {
      float f[8];
      widen8(v, f);
      for (int j = 0; j < a.k; ++j) {
        const long long r = pos[j];
        const float w = a.weights[t * a.k + j];
        float g[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) g[q] = f[q] * w;
        if (r >= 0) *reinterpret_cast<uint4 *>(a.out + r * a.D + c) = narrow8(g);
      }
    }
  }
}

// The backward of combine: rows = w dout, and dw = dout . y in fp32.  A team of warps per (token, choice).
__global__ void __launch_bounds__(256) dispatch_dot_kernel(const __grid_constant__ RowsArgs a) {
  __shared__ float part[8];
  pdl_launch_dependents();
  pdl_wait();
  if (blockIdx.x >= a.token_blocks) return clear_between(a, (int)(blockIdx.x - a.token_blocks));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, teams = 8 / a.team, team = warp / a.team;
  const int tl = (warp - team * a.team) * 32 + lane, TL = a.team * 32;
  const long long slot = (long long)blockIdx.x * teams + team;
  const bool there = slot < a.T * a.k;
  const long long t = there ? slot / a.k : 0;
  const long long r = there ? a.pos[slot] : -1;
  float dot = 0.f;
  if (r >= 0) {
    const float w = a.weights ? a.weights[slot] : 1.0f;
    const __nv_bfloat16 *x = a.x + t * a.D, *y = a.y + r * a.D;
    __nv_bfloat16 *out = a.out + r * a.D;
    for (int c = tl * 8; c < a.D; c += TL * 8) {
      float f[8], h[8];
      widen8(*reinterpret_cast<const uint4 *>(x + c), f);
      widen8(load16(y + c), h);
      float s = 0.f;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        s = fmaf(f[q], h[q], s);
        f[q] *= w;
      }
      dot += s;
      *reinterpret_cast<uint4 *>(out + c) = narrow8(f);
    }
  }
  dot = warp_sum(dot);
  if (a.team > 1) {
    if (lane == 0) part[warp] = dot;
    __syncthreads();
    dot = 0.f;
    for (int q = 0; q < a.team; ++q) dot += part[team * a.team + q];
  }
  if (there && tl == 0) a.dweights[slot] = dot;
}

__global__ void __launch_bounds__(256) combine_kernel(const __grid_constant__ RowsArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int pieces = a.D >> 3;
  const long long n = a.T * pieces, stride = (long long)gridDim.x * blockDim.x;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += stride) {
    const long long t = i / pieces;
    const int c = (int)(i - t * pieces) << 3;
    float sum[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) sum[q] = 0.f;
    constexpr int AHEAD = 4;
    for (int j0 = 0; j0 < a.k; j0 += AHEAD) {
      uint4 v[AHEAD];
      float w[AHEAD];
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) {
        const long long r = j0 + q < a.k ? a.pos[t * a.k + j0 + q] : -1;
        v[q] = r >= 0 ? load16(a.x + r * a.D + c) : make_uint4(0u, 0u, 0u, 0u);
        w[q] = r < 0 ? 0.f : a.weights ? a.weights[t * a.k + j0 + q] : 1.0f;
      }
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) {
        float f[8];
        widen8(v[q], f);
#pragma unroll
        for (int h = 0; h < 8; ++h) sum[h] = fmaf(w[q], f[h], sum[h]);
      }
    }
    *reinterpret_cast<uint4 *>(a.out + t * a.D + c) = narrow8(sum);
  }
}

// ------------------------------------------------------------------------------------------------

int check_choices(int64_t T, int top_k, int E) {
  if (T < 0 || top_k < 1 || E < 1 || E > OSDP_MAX_EXPERTS || top_k > OSDP_MAX_TOP_K || top_k > E) return OSDP_ERR_BAD_SHAPE;
  return T > ((int64_t)1 << 30) / top_k ? OSDP_ERR_BAD_SHAPE : OSDP_OK;
}
int check_routing(int64_t T, int E, int top_k, int64_t ld, int dtype, int score, double scale) {
  const int rc = check_choices(T, top_k, E);
  if (rc) return rc;
  if (ld < E) return OSDP_ERR_BAD_SHAPE;
  if ((dtype != OSDP_DTYPE_BF16 && dtype != OSDP_DTYPE_FP32) || (score != OSDP_SCORE_SOFTMAX && score != OSDP_SCORE_SIGMOID) ||
      !std::isfinite(scale) || std::fabs(scale) > 3e38)
    return OSDP_ERR_UNSUPPORTED;
  return OSDP_OK;
}

template <typename L>
int launch_route(const RouteArgs &a, cudaStream_t stream) {
  const dim3 grid((unsigned)cdiv(a.T, ROUTE_WARPS)), block(32 * ROUTE_WARPS);
  const size_t smem = a.groups > a.top_groups ? (size_t)ROUTE_WARPS * a.E * sizeof(double) : 0;   // at most 64 KB: below
  auto go = [&](auto kernel) -> int {
    if (smem > 48 * 1024) {
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ROUTE_WARPS * OSDP_MAX_EXPERTS * (int)sizeof(double));
      if (e != cudaSuccess) return report_cuda(e);
    }
    return launch_overlapped(kernel, grid, block, smem, 1, stream, a);
  };
  if (a.E <= 32) return go(route_fwd_kernel<L, 1>);
  if (a.E <= 64) return go(route_fwd_kernel<L, 2>);
  if (a.E <= 128) return go(route_fwd_kernel<L, 4>);
  if (a.E <= 256) return go(route_fwd_kernel<L, 8>);
  if (a.E <= 512) return go(route_fwd_kernel<L, 16>);
  return go(route_fwd_kernel<L, 32>);
}

int check_rows(int64_t T, int top_k, int E, int64_t D) {
  const int rc = check_choices(T, top_k, E);
  if (rc) return rc;
  if (D <= 0 || D > ((int64_t)1 << 24)) return OSDP_ERR_BAD_SHAPE;
  return (D & 7) ? OSDP_ERR_ALIGNMENT : OSDP_OK;
}

}  // namespace

int64_t expert_rows(int64_t T, int top_k, int E) {
  const int64_t n = T * top_k, used = n < E ? n : E;
  return (n + (OSDP_EXPERT_ROWS - 1) * used) / OSDP_EXPERT_ROWS * OSDP_EXPERT_ROWS;
}
int expert_check(int64_t T, int top_k, int E) { return check_choices(T, top_k, E); }

}  // namespace osdp

using namespace osdp;

extern "C" int osdp_route_fwd(const void *logits, int64_t ld, int logits_dtype, const float *bias, int64_t T, int E, int top_k, int score,
                              int n_groups, int top_groups, int group_take, int renorm, double scale, int32_t *idx, float *weights,
                              void *stream) {
  const int rc = check_routing(T, E, top_k, ld, logits_dtype, score, scale);
  if (rc) return rc;
  if (n_groups < 1 || n_groups > 32 || E % n_groups || top_groups < 1 || top_groups > n_groups || top_groups * (E / n_groups) < top_k)
    return OSDP_ERR_BAD_SHAPE;
  if (group_take != 1 && group_take != 2) return OSDP_ERR_UNSUPPORTED;
  if (T == 0) return OSDP_OK;
  if (!logits || !idx || !weights) return OSDP_ERR_NULL_POINTER;
  if (!aligned_to(logits, logits_dtype == OSDP_DTYPE_FP32 ? 4 : 2) || !aligned_to(bias, 4) || !aligned_to(idx, 4) || !aligned_to(weights, 4))
    return OSDP_ERR_ALIGNMENT;
  const RouteArgs a{logits, (long long)ld, (long long)T, bias, E, top_k, score, n_groups, top_groups, group_take, renorm ? 1 : 0, (float)scale,
                    idx, weights};
  return logits_dtype == OSDP_DTYPE_FP32 ? launch_route<float>(a, static_cast<cudaStream_t>(stream))
                                         : launch_route<__nv_bfloat16>(a, static_cast<cudaStream_t>(stream));
}

extern "C" int osdp_route_bwd(const float *dweights, const void *logits, int64_t ld, int logits_dtype, const int32_t *idx, int64_t T, int E,
                              int top_k, int score, int renorm, double scale, void *dlogits, int64_t ld_dlogits, void *stream) {
  const int rc = check_routing(T, E, top_k, ld, logits_dtype, score, scale);
  if (rc) return rc;
  if (ld_dlogits < E) return OSDP_ERR_BAD_SHAPE;
  if (T == 0) return OSDP_OK;
  if (!dweights || !logits || !idx || !dlogits) return OSDP_ERR_NULL_POINTER;
  const uintptr_t es = logits_dtype == OSDP_DTYPE_FP32 ? 4 : 2;
  if (!aligned_to(logits, es) || !aligned_to(dlogits, es) || !aligned_to(dweights, 4) || !aligned_to(idx, 4)) return OSDP_ERR_ALIGNMENT;
  RouteBackArgs b{};
  b.r = RouteArgs{logits, (long long)ld, (long long)T, nullptr, E, top_k, score, 1, 1, 1, renorm ? 1 : 0, (float)scale, const_cast<int32_t *>(idx),
                  nullptr};
  b.dweights = dweights;
  b.dlogits = dlogits;
  b.ld_out = (long long)ld_dlogits;
  b.dense = ld_dlogits == E && aligned_to(dlogits, 16) ? 1 : 0;
  const dim3 grid((unsigned)cdiv(T, ROUTE_WARPS)), block(32 * ROUTE_WARPS);
  if (logits_dtype == OSDP_DTYPE_FP32) return launch_overlapped(route_bwd_kernel<float>, grid, block, 0, 1, static_cast<cudaStream_t>(stream), b);
  return launch_overlapped(route_bwd_kernel<__nv_bfloat16>, grid, block, 0, 1, static_cast<cudaStream_t>(stream), b);
}

extern "C" int osdp_expert_rows(int64_t T, int top_k, int E, int64_t *rows, int64_t *plan_ints) {
  const int rc = check_choices(T, top_k, E);
  if (rc) return rc;
  if (rows) *rows = expert_rows(T, top_k, E);
  if (plan_ints) *plan_ints = plan_length(E);
  return OSDP_OK;
}

extern "C" int osdp_expert_plan(const int32_t *idx, int64_t T, int top_k, int E, int32_t *plan, int32_t *pos, void *stream) {
  const int rc = check_choices(T, top_k, E);
  if (rc) return rc;
  if (!plan || (T > 0 && (!idx || !pos))) return OSDP_ERR_NULL_POINTER;
  if (!aligned_to(idx, 4) || !aligned_to(plan, 16) || !aligned_to(pos, 4)) return OSDP_ERR_ALIGNMENT;
  const size_t smem = (size_t)(PLAN_WARPS + 1) * E * sizeof(int);
  if (smem > 40 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(expert_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (PLAN_WARPS + 1) * OSDP_MAX_EXPERTS * 4);
    if (e != cudaSuccess) return report_cuda(e);
  }
  const PlanArgs a{idx, (long long)(T * top_k), E, plan, pos};
  // one block up to a choice per thread, a cluster of eight beyond
  const int ctas = T * top_k <= 32 * PLAN_WARPS ? 1 : 8;
  return launch_overlapped(expert_plan_kernel, dim3(ctas), dim3(32 * PLAN_WARPS), smem, ctas, static_cast<cudaStream_t>(stream), a);
}

extern "C" int osdp_expert_dispatch(const void *x, const int32_t *plan, const int32_t *pos, const float *weights, const void *y_rows, int64_t T,
                                    int top_k, int E, int64_t D, void *rows, float *dweights, void *stream) {
  const int rc = check_rows(T, top_k, E, D);
  if (rc) return rc;
  if (T == 0) return OSDP_OK;
  if (!x || !plan || !pos || !rows || (dweights && !y_rows)) return OSDP_ERR_NULL_POINTER;
  if (!aligned_to(x, 16) || !aligned_to(rows, 16) || !aligned_to(y_rows, 16) || !aligned_to(plan, 16) || !aligned_to(pos, 4) ||
      !aligned_to(weights, 4) || !aligned_to(dweights, 4))
    return OSDP_ERR_ALIGNMENT;
  RowsArgs a{static_cast<const __nv_bfloat16 *>(x), plan, pos, weights, static_cast<const __nv_bfloat16 *>(y_rows), static_cast<__nv_bfloat16 *>(rows),
             dweights, (long long)T, top_k, E, (int)D, 0, 1};
  if (dweights) {
    int sms = 0;
    const int src = sm_count(&sms);
    if (src) return src;
    // as many warps to a row as it has pieces for, more where there are few rows
    a.team = 1;
    while (a.team < 8 && a.team * 256 < D && (T * top_k * a.team < (int64_t)sms * 16 || a.team * 2048 < D)) a.team *= 2;
    a.token_blocks = cdiv(T * top_k, 8 / a.team);
    return launch_overlapped(dispatch_dot_kernel, dim3((unsigned)(a.token_blocks + E)), dim3(256), 0, 1, static_cast<cudaStream_t>(stream), a);
  }
  a.token_blocks = cdiv(T * (D / 8), 256);
  return launch_overlapped(dispatch_kernel, dim3((unsigned)(a.token_blocks + E)), dim3(256), 0, 1, static_cast<cudaStream_t>(stream), a);
}

extern "C" int osdp_expert_combine(const void *rows, const int32_t *plan, const int32_t *pos, const float *weights, int64_t T, int top_k, int E,
                                   int64_t D, void *out, void *stream) {
  const int rc = check_rows(T, top_k, E, D);
  if (rc) return rc;
  if (T == 0) return OSDP_OK;
  if (!rows || !pos || !plan || !out) return OSDP_ERR_NULL_POINTER;
  if (!aligned_to(rows, 16) || !aligned_to(out, 16) || !aligned_to(plan, 16) || !aligned_to(pos, 4) || !aligned_to(weights, 4)) return OSDP_ERR_ALIGNMENT;
  const RowsArgs a{static_cast<const __nv_bfloat16 *>(rows), plan, pos, weights, nullptr, static_cast<__nv_bfloat16 *>(out), nullptr, (long long)T,
                   top_k, E, (int)D, 0, 1};
  return launch_overlapped(combine_kernel, dim3((unsigned)cdiv(T * (D / 8), 256)), dim3(256), 0, 1, static_cast<cudaStream_t>(stream), a);
}

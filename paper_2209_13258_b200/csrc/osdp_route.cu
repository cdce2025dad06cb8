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
constexpr int ROUTE_WARPS = 8;

// ------------------------------------------------------------------------------------------------
// Routing.  One warp per token; lane l holds experts l, l + 32, ... in registers.
//
// The choice has to be the one of 64 bits: another expert is another result.  It is made twice at most.  First in
// fp32 with approximate scores: a key is the score's order-preserving bits with the place in the lane's registers in the lowest
// ones, a lane sorts its keys once, and an expert is found by one maximum over the lanes' first keys.  Where two scores
// that decide are closer than all these roundings (and are not the same logit with the same bias), the scores in question are
// taken again in fp64.  That is kept short (a whole row in fp64 made the last of 16384 rows of 256 experts 10 us late), for how many
// rows it is depends on the logits: with sigmoid, 256 experts, groups and a bias of zeros 0.2 % at a spread of 1.2, 2.2 % at 0.02, 9 % at
// 0.005, and 24.1, 26 and 29 us; with a bias of 0.05 randn 0.2 % at most.  Bound by instructions, some 1100 a row: 16384 rows of 256
// experts, sigmoid, bias, 4 of 8 groups, 8 choices 24 us (17 MB of logits: 2.7 us); 128 experts, 4 choices, without a bias 9.8 us; one
// row 1.8 us.
struct RouteArgs {
  const void *logits;
  long long ld, T;
  const float *bias;
  int E, k, score, groups, top_groups, take, renorm;
  float scale;
  int32_t *idx;
  float *weights;
  // of the groups: experts of one, 2^20 / that rounded up (a quotient e / size for e < 1024), log2 of the lanes that look at one
  int size, lanes_log2;
  uint32_t magic;
};

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }

// Order-preserving keys; 0 is below every key.  NaN counts as minus infinity, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const int32_t u = __float_as_int(fmaxf(x, -INFINITY) + 0.0f);
  return (uint32_t)u ^ ((uint32_t)(u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float((key >> 31) ? key & 0x7FFFFFFFu : ~key); }

template <int V>
__device__ __forceinline__ float largest(const float (&l)[V]) {   // of the row; lanes past its end hold minus infinity
  uint32_t top = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) top = max(top, key_of(l[v]));
  return value_of(__reduce_max_sync(ALL, top));
}

// Which groups may be chosen from: bit g << lanes_log2 of the result.  score_of: an expert's score, NaN as minus infinity.
template <typename R, typename F>
__device__ __forceinline__ uint32_t choose_groups(const RouteArgs &a, F score_of, int lane, R &sum, bool &in) {
  const R low = -(R)INFINITY;
  const int per = 1 << a.lanes_log2, g = lane >> a.lanes_log2, sub = lane & (per - 1);
  R first = low, second = low;
  if (g < a.groups) {
#pragma unroll(sizeof(R) == 4 ? 4 : 1)
    for (int e = sub; e < a.size; e += per) {
      const R x = score_of(g * a.size + e);
      second = max(second, min(first, x));
      first = max(first, x);
    }
  }
  for (int o = 1; o < per; o <<= 1) {
    const R f = __shfl_xor_sync(ALL, first, o), s = __shfl_xor_sync(ALL, second, o);
    second = max(max(second, s), min(first, f));
    first = max(first, f);
  }
  sum = a.take > 1 && a.size > 1 ? first + second : first;
  if (sum != sum) sum = low;
  int rank = 0;
  for (int h = 0; h < a.groups; ++h) {
    const R other = __shfl_sync(ALL, sum, h << a.lanes_log2);
    rank += other > sum || (other == sum && h < g) ? 1 : 0;
  }
  in = g < a.groups && rank < a.top_groups;
  return __ballot_sync(ALL, in && sub == 0);
}

constexpr float HALF_ULP = 5.9604645e-8f;
__device__ __forceinline__ float fast_exp(float x) {   // 2^-22 and the rounding of the product: 1.5 |x| 2^-24
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * 1.4426950408889634f));
  return e;
}

// The row's scores in fp64, one at a time.  Compact loops: they are cold when they are needed.
template <typename L>
struct Exact {
  const RouteArgs &a;
  const L *row;
  double high, total;

  __device__ Exact(const RouteArgs &args, const L *r, int lane) : a(args), row(r), high(0.0), total(1.0) {
    if (a.score != OSDP_SCORE_SOFTMAX || !(a.bias || a.top_groups < a.groups)) return;
    uint32_t top = 0;
    for (int e = lane; e < a.E; e += 32) top = max(top, key_of(widen(row[e])));
    high = (double)value_of(__reduce_max_sync(ALL, top));
    total = 0.0;
#pragma unroll 1
    for (int e = lane; e < a.E; e += 32) {
      const double l = (double)widen(row[e]);
      total += l == -(double)INFINITY ? 0.0 : exp(l - high);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(ALL, total, o);
  }
  __device__ double score(int e) const {
    const double l = (double)widen(row[e]);
    double s;
    if (a.score == OSDP_SCORE_SOFTMAX) s = l == -(double)INFINITY && total == total ? 0.0 : exp(l - high) / total;
    else s = 1.0 / (1.0 + exp(-l));
    if (a.bias) s += (double)a.bias[e];
    return s == s ? s : -(double)INFINITY;
  }
  // what experts are chosen by
  __device__ double rank_by(int e) const {
    if (a.bias) return score(e);
    const double l = (double)widen(row[e]);
    return l == l ? l : -(double)INFINITY;
  }
  // Which of two experts with equal numbers `key` comes first.  fp64's sigmoid is 1 from a logit of 37 on and its softmax 0 from 746
  // below the largest: scores with one bias can be equal where the logits, in whose order exact ones are, still differ.  A
  // bias of 2^20 or more is a mask, behind which all are equal.
  __device__ bool first_of_equal(int e, int f, double key) const {
    if (a.bias && key > -(double)INFINITY) {
      const float x = logit_behind(e), y = logit_behind(f);
      if (x != y) return x > y;
    }
    return e < f;
  }
  __device__ float logit_behind(int e) const { return fabsf(a.bias[e]) < 1048576.0f ? widen(row[e]) : -INFINITY; }
};

template <typename L>
__device__ __noinline__ uint32_t exact_groups(const RouteArgs &a, const L *row, int lane) {
  const Exact<L> exact(a, row, lane);
  double sum;
  bool in;
  return choose_groups<double>(a, [&](int e) { return exact.score(e); }, lane, sum, in);
}

// Lanes 0 .. m hold candidates, behind which nothing can be chosen: the k best of them, in order.
template <typename L>
__device__ __noinline__ void exact_order(const RouteArgs &a, const L *row, int lane, int m, int &mine) {
  const Exact<L> exact(a, row, lane);
  const double key = lane <= m ? exact.rank_by(mine) : 0.0;
  int rank = 0, from = 0;
#pragma unroll 1
  for (int i = 0; i <= m; ++i) {
    const double other = __shfl_sync(ALL, key, i);
    const int e = __shfl_sync(ALL, mine, i);
    rank += other > key || (other == key && lane <= m && i != lane && exact.first_of_equal(e, mine, key)) ? 1 : 0;
  }
#pragma unroll 1
  for (int j = 0; j < a.k; ++j) {
    const int owner = __ffs(__ballot_sync(ALL, lane <= m && rank == j)) - 1;
    if (lane == j) from = owner;
  }
  mine = __shfl_sync(ALL, mine, from);
}

// Everything in question: the experts of the groups in `taken`, one after the other.
template <typename L>
__device__ __noinline__ void exact_all(const RouteArgs &a, const L *row, uint32_t taken, int lane, int &mine) {
  const Exact<L> exact(a, row, lane);
  double last = (double)INFINITY;
  int last_e = -1;
#pragma unroll 1
  for (int j = 0; j < a.k; ++j) {     // the best of those behind the last one
    double best = -(double)INFINITY;
    int best_e = -1;
#pragma unroll 1
    for (int e = lane; e < a.E; e += 32) {
      if (!((taken >> (((uint32_t)e * a.magic >> 20) << a.lanes_log2)) & 1u)) continue;
      const double x = exact.rank_by(e);
      const bool behind = j == 0 || x < last || (x == last && e != last_e && exact.first_of_equal(last_e, e, x));
      if (behind && (best_e < 0 || x > best || (x == best && exact.first_of_equal(e, best_e, x)))) {
        best = x;
        best_e = e;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const double x = __shfl_xor_sync(ALL, best, o);
      const int e = __shfl_xor_sync(ALL, best_e, o);
      if (e >= 0 && (best_e < 0 || x > best || (x == best && exact.first_of_equal(e, best_e, x)))) {
        best = x;
        best_e = e;
      }
    }
    last = best;
    last_e = best_e;
    if (lane == j) mine = best_e;
  }
}

// Chooses the row's experts: lane j < k leaves with the j-th in `mine`, its logit in `lj`.
// `list` [32 V]: this warp's shared memory.
template <int V, typename L>
__device__ __forceinline__ void choose(const RouteArgs &a, const L *row, const float (&l)[V], uint32_t *list, int lane, int &mine, float &lj) {
  const bool grouped = a.top_groups < a.groups, soft = a.score == OSDP_SCORE_SOFTMAX;
  uint32_t key[V], taken = ALL;
  float c[V];
  float slack = 0.f;                  // half units of 1 that a score with a bias may be off, beside those of itself
#pragma unroll
  for (int v = 0; v < V; ++v) c[v] = l[v];                 // without a bias the scores are in the order of the logits
  if (a.bias || grouped) {
    float s[V], far = 0.f, inv = 1.f;
    if (soft) {
      const float high = largest(l);
      float total = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        s[v] = l[v] == -INFINITY ? 0.f : fast_exp(l[v] - high);
        total += s[v];
      }
      total = warp_sum(total);
      inv = total > 0.f ? fast_rcp(total) : total;       // (a row of minus infinities: all scores are zero)
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] *= inv;
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = fast_rcp(1.0f + fast_exp(-l[v]));
    }
    if (a.bias) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float b = v * 32 + lane < a.E ? a.bias[v * 32 + lane] : 0.f;
        c[v] = s[v] += b;
        far = fmaxf(far, fabsf(b) < 1e30f ? fabsf(b) : 0.f);           // (beyond, a bias is a mask: nothing is close to it)
      }
      // A sigmoid is off by 4.4 half units at most: s (1 - s) (1.5 |l| + 4) for its exponential, 3 s for sum and reciprocal.  A
      // softmax by 46 of its own, of which `inv` is the largest: exponent 1.5 times its size, which e^-x more than takes back,
      // exponential and reciprocal 4 each, its total up to 37.  The sum with the bias adds one of its own.
      slack = soft ? 46.0f * inv : 5.0f;
    }
    if (grouped) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        list[v * 32 + lane] = __float_as_uint(fmaxf(s[v], -INFINITY));
      __syncwarp();
      float sum;
      bool in;
      taken = choose_groups<float>(a, [&](int e) { return __uint_as_float(list[e]); }, lane, sum, in);
      const float last = value_of(~__reduce_max_sync(ALL, in ? ~key_of(sum) : 0u));
      const float next = value_of(__reduce_max_sync(ALL, (lane >> a.lanes_log2) < a.groups && !in ? key_of(sum) : 0x007FFFFFu));
      far = __uint_as_float(__reduce_max_sync(ALL, __float_as_uint(far)));
      // Two sums of two scores.  A sigmoid is off by 4.4 half units of 1 at most, and the sums by theirs and the bias's; a softmax by
      // 128 of its own size (its exponent counts 1.5 times, and beyond 80 nothing is left of it).
      const float off = soft ? 256.0f * (fabsf(last) + 2.0f * far) : 24.0f + 4.0f * far + 2.0f * fabsf(last);
      if (last - next <= HALF_ULP * off) taken = exact_groups(a, row, lane);
      __syncwarp();
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const bool on = v * 32 + lane < a.E && (!grouped || ((taken >> (((uint32_t)(v * 32 + lane) * a.magic >> 20) << a.lanes_log2)) & 1u));
    key[v] = on ? (key_of(c[v]) & ~(uint32_t)(V - 1)) | (uint32_t)(V - 1 - v) : 0u;
  }
  // descending (a bitonic network)
#pragma unroll
  for (int n = 2; n <= V; n *= 2)
#pragma unroll
    for (int o = n / 2; o > 0; o /= 2)
#pragma unroll
      for (int v = 0; v < V; ++v)
        if ((v & o) == 0) {
          const uint32_t hi = max(key[v], key[v | o]), lo = min(key[v], key[v | o]);
          key[v] = (v & n) == 0 ? hi : lo;
          key[v | o] = (v & n) == 0 ? lo : hi;
        }
  // A lane's keys wait in shared memory but for the first.
#pragma unroll
  for (int v = 1; v < V; ++v) list[v * 32 + lane] = key[v];
  uint32_t got = 0, head = key[0];
  int next = lane + 32;
  auto take = [&](int from, int to) {        // lane j gets the j-th
    for (int j = from; j < to; ++j) {
      const uint32_t best = __reduce_max_sync(ALL, head);
      if (best == 0) break;             // (only behind the last one wanted: the groups have enough experts)
      const int owner = __ffs(__ballot_sync(ALL, head == best)) - 1;      // equal keys: the same register, the lower lane
      if (lane == j) {
        got = best;
        mine = owner + (V - 1 - (int)(best & (V - 1))) * 32;
      }
      if (lane == owner) {
        head = next < V * 32 ? list[next] : 0u;
        next += 32;
      }
    }
  };
  // Whether lane j's expert and the next lane's are too close to say: bits of lanes.  How far a score may be off is a bound for the
  // row, and grows with nothing but the score: where a gap is, it lies between all before it and all behind it, the experts
  // that were never looked at among them.  The bits that the place took are 2 V half units of the score.
  // `unequal`: those of them that are not the same anyway, for having the same logit and the same bias.
  auto close = [&](uint32_t &unequal) {
    float bj = 0.f;
    const float value = value_of(got & ~(uint32_t)(V - 1)), off = fmaf(a.bias ? 2.0f * V + 1.0f : 2.0f * V, fabsf(value), slack);
    if (mine >= 0) {
      lj = widen(row[mine]);
      if (a.bias) bj = a.bias[mine];
    }
    const int after = __shfl_down_sync(ALL, mine, 1);
    const float less = __shfl_down_sync(ALL, value, 1), less_off = __shfl_down_sync(ALL, off, 1), less_l = __shfl_down_sync(ALL, lj, 1),
                less_b = __shfl_down_sync(ALL, bj, 1);
    const bool near = lane < 31 && mine >= 0 && after >= 0 && value - less <= HALF_ULP * (off + less_off);
    unequal = __ballot_sync(ALL, near && (lj != less_l || bj != less_b));
    return __ballot_sync(ALL, near);
  };
  take(0, a.k + 1);     // one more than are wanted, to see how far away it is
  uint32_t unequal;
  if (((close(unequal) >> (a.k - 1)) & 1u) == 0 && (unequal & ((1u << a.k) - 1u)) == 0) return;
  // The candidates end at the first gap behind the last one wanted.  (Also where it has an equal behind it: what comes after
  // that one may be neither equal nor far away.)
  for (int many = a.k + 1; many < 32;) {
    const int more = min(many + 4, 32);
    take(many, more);
    many = more;
    const uint32_t there = __ballot_sync(ALL, mine >= 0);
    const uint32_t gaps = ~close(unequal) & ~((1u << (a.k - 1)) - 1u) & (there >> 1);      // (the last candidate's gap is not known yet)
    if (gaps || __popc(there) < many) {
      const int m = gaps ? __ffs(gaps) - 1 : __popc(there) - 1;
      if (unequal & ((1u << m) - 1u)) {          // (equal ones are in order)
        exact_order(a, row, lane, m, mine);
        if (lane < a.k) lj = widen(row[mine]);
      }
      return;
    }
  }
  exact_all(a, row, taken, lane, mine);
  if (lane < a.k) lj = widen(row[mine]);
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
__global__ void __launch_bounds__(256, V <= 8 ? 4 : 1) route_fwd_kernel(const __grid_constant__ RouteArgs a) {
  __shared__ uint32_t lists[ROUTE_WARPS * 32 * V];
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long t = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  pdl_wait();
  if (t >= a.T) return;
  const L *row = static_cast<const L *>(a.logits) + t * a.ld;
  float l[V];
#pragma unroll
  for (int v = 0; v < V; ++v) l[v] = v * 32 + lane < a.E ? widen(row[v * 32 + lane]) : -INFINITY;
  int mine = -1;
  float lj = -INFINITY;
  choose<V, L>(a, row, l, lists + (threadIdx.x >> 5) * 32 * V, lane, mine, lj);
  const bool on = lane < a.k;
  float w;
  if (a.renorm) {
    w = share_of(a, lj, on, lane);
  } else if (a.score == OSDP_SCORE_SIGMOID) {
    w = 1.0f / (1.0f + expf(-lj));
  } else {
    const float high = largest(l);
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
// the expert was not chosen), the one case that reads all logits: a kernel of its own.
struct RouteBackArgs {
  RouteArgs r;
  const float *dweights;
  void *dlogits;
  long long ld_out;
  int dense;                    // ld_out == E and a 16-byte aligned dlogits: rows are cleared in 16-byte pieces
};

__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// The choices of a token: lane j < k has the j-th expert (-1: none) and g_j.
template <typename L>
__device__ __forceinline__ void load_choices(const RouteBackArgs &b, long long t, bool there, int lane, int &e, float &g) {
  const RouteArgs &a = b.r;
  e = lane < a.k && there ? a.idx[t * a.k + lane] : -1;
  if (e < 0 || e >= a.E) e = -1;           // a choice that is none has no gradient
  g = e >= 0 ? b.dweights[t * a.k + lane] * a.scale : 0.f;
}
// A token that was given the same expert twice: one gradient, the sum, on the lane that `first` names.
__device__ __forceinline__ float sum_of_same(int k, int e, float d, int &first) {
  float sum = 0.f;
  first = 32;
  for (int j = k - 1; j >= 0; --j) {
    const int ej = __shfl_sync(ALL, e, j);
    const float dj = __shfl_sync(ALL, d, j);
    sum += ej == e ? dj : 0.f;
    first = ej == e ? j : first;
  }
  return sum;
}

// The gradient is zero but for the chosen.  Bound by latency: choices, their logits, stores behind the zeros (16384 x 256 fp32
// 7.1 us, floor 2.8; two tokens to a warp 8.9).
template <typename L>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) route_bwd_kernel(const __grid_constant__ RouteBackArgs b) {
  pdl_launch_dependents();
  const RouteArgs &a = b.r;
  const int lane = threadIdx.x & 31;
  const long long t0 = (long long)blockIdx.x * ROUTE_WARPS, t = t0 + (threadIdx.x >> 5);
  L *out = static_cast<L *>(b.dlogits);
  pdl_wait();
  int e, first;
  float g;
  load_choices<L>(b, t, t < a.T, lane, e, g);
  const float l = e >= 0 ? widen(static_cast<const L *>(a.logits)[t * a.ld + e]) : -INFINITY;
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
  // 1 - s by its own formula: as a difference it loses the digits of a confident expert, and all of them from a logit of 17 on
  const float rest = a.score == OSDP_SCORE_SIGMOID ? 1.0f / (1.0f + expf(l)) : 1.0f;
  float d;
  if (a.renorm) {
    const float r = share_of(a, l, e >= 0, lane);
    d = r * (g - warp_sum(e >= 0 ? g * r : 0.f)) * rest;
  } else {
    d = g * (1.0f / (1.0f + expf(-l))) * rest;
  }
  d = sum_of_same(a.k, e, d, first);
  __syncthreads();                       // the rows are clear
  if (e >= 0 && lane == first) put(out + t * b.ld_out + e, d);
}

// A softmax that is not renormalised: every logit has a gradient.  s_e (0 - mean) everywhere, then the chosen ones (16384 x 256
// fp32 9.0 us, floor 5.3).
template <typename L, int V>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) route_bwd_dense_kernel(const __grid_constant__ RouteBackArgs b) {
  pdl_launch_dependents();
  const RouteArgs &a = b.r;
  const int lane = threadIdx.x & 31;
  const long long t = (long long)blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5);
  pdl_wait();
  if (t >= a.T) return;
  const L *row = static_cast<const L *>(a.logits) + t * a.ld;
  L *out = static_cast<L *>(b.dlogits) + t * b.ld_out;
  float s[V];
#pragma unroll
  for (int v = 0; v < V; ++v) s[v] = v * 32 + lane < a.E ? widen(row[v * 32 + lane]) : -INFINITY;
  int e, first;
  float g;
  load_choices<L>(b, t, true, lane, e, g);
  const float l = e >= 0 ? widen(row[e]) : -INFINITY;
  const float high = largest(s);
  float total = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    s[v] = s[v] == -INFINITY ? 0.f : expf(s[v] - high);
    total += s[v];
  }
  total = warp_sum(total);
  const float inv = total == 0.f ? 0.f : 1.0f / total;
  const float mine = l == -INFINITY ? 0.f : expf(l - high) * inv;
  const float mean = warp_sum(e >= 0 ? g * mine : 0.f);
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (v * 32 + lane < a.E) put(out + v * 32 + lane, s[v] * inv * (0.f - mean));
  const float sum = sum_of_same(a.k, e, g, first);
  __syncwarp();
  if (e >= 0 && lane == first) put(out + e, mine * (sum - mean));
}

// ------------------------------------------------------------------------------------------------
// The plan: a stable counting sort of the T k choices by expert.  One launch of a cluster: a warp counts a contiguous part
// of the choices into its own table, the tables' prefix sums over warps and (through distributed shared memory) over the
// cluster's blocks say where each warp's rows of each expert start, and a second pass hands them out in order: the same
// choices give the same plan.
struct PlanArgs {
  const int32_t *idx;
  int n, E;
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
// Inclusive sums of N values over the block's 1024 threads.
template <int N>
__device__ __forceinline__ void block_scan(int (&v)[N], int (*warps)[PLAN_WARPS]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int w[N];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = __shfl_up_sync(ALL, v[i], o);
      if (lane >= o) v[i] += u;
    }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (lane == 31) warps[i][warp] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = lane < warp ? warps[i][lane] : 0;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] += __reduce_add_sync(ALL, w[i]);
}

__global__ void __launch_bounds__(32 * PLAN_WARPS, 1) expert_plan_kernel(const __grid_constant__ PlanArgs a) {
  extern __shared__ int tables[];              // [PLAN_WARPS][E], then this block's totals [E], then where its rows start [E]
  __shared__ int sums[4][PLAN_WARPS];
  const int E = a.E, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;
  int *totals = tables + PLAN_WARPS * E, *starts = totals + E;
  const uint32_t rank = cta_rank_in_cluster(), ctas = ctas_in_cluster();
  pdl_launch_dependents();
  for (int i = tid; i < PLAN_WARPS * E; i += blockDim.x) tables[i] = 0;
  __syncthreads();
  pdl_wait();
  int *mine = tables + warp * E;
  const int parts = (int)ctas * PLAN_WARPS, part = ((a.n + parts - 1) / parts + 31) / 32 * 32;
  const int begin = (int)min((long long)((int)rank * PLAN_WARPS + warp) * part, (long long)a.n), end = min(a.n, begin + part);
  constexpr int AHEAD = 4;
  const int bits = 32 - __clz(E - 1);          // (0 for one expert)
  auto expert_at = [&](int i) { return i < end ? a.idx[i] : -1; };
  for (int i0 = begin; i0 < end; i0 += 32 * AHEAD) {
    int e[AHEAD];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) e[q] = expert_at(i0 + 32 * q + lane);
#pragma unroll
    for (int q = 0; q < AHEAD; ++q)
      if (e[q] >= 0 && e[q] < E) atomicAdd(mine + e[q], 1);
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
  const int t128 = (count + 127) / 128, t256 = (count + 255) / 256, live = count > 0 ? 1 : 0;
  int upto[4] = {padded, t128, t256, live};
  block_scan(upto, sums);
  const int offset = upto[0] - padded;
  if (tid < E) starts[tid] = offset + before;
  if (rank == 0 && tid < E) {
    int32_t *p = a.plan;
    p[PLAN_OFFSETS + tid] = offset;
    p[plan_counts(E) + tid] = count;
    p[plan_tiles128(E) + tid] = upto[1] - t128;
    p[plan_tiles256(E) + tid] = upto[2] - t256;
    if (live) p[plan_live(E) + upto[3] - 1] = tid;
    if (tid == E - 1) {
      p[PLAN_OFFSETS + E] = upto[0];
      p[plan_tiles128(E) + E] = upto[1];
      p[plan_tiles256(E) + E] = upto[2];
      p[plan_n_live(E)] = upto[3];
    }
  }
  __syncthreads();
  for (int i0 = begin; i0 < end; i0 += 32 * AHEAD) {
    int e[AHEAD];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) e[q] = expert_at(i0 + 32 * q + lane);
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      const int i = i0 + 32 * q + lane;
      const bool in = e[q] >= 0 && e[q] < E;
      // the lanes with the same expert, bit by bit of its number (match.any takes 64 cycles of the whole SM: 131072 choices of
      // 256 experts 36 us with it, of which the two passes' 16 matches a warp were 30)
      uint32_t same = __ballot_sync(ALL, in);
      for (int b = 0; b < bits; ++b) {
        const uint32_t has = __ballot_sync(ALL, (e[q] >> b) & 1);
        same &= (e[q] >> b) & 1 ? has : ~has;
      }
      const int first = in ? mine[e[q]] : 0;
      __syncwarp();
      if (in && lane == __ffs(same) - 1) mine[e[q]] = first + __popc(same);
      __syncwarp();
      if (i < end) a.pos[i] = in ? starts[e[q]] + first + __popc(same & ((1u << lane) - 1u)) : -1;
    }
  }
  cluster_sync();        // nobody leaves while another block may still read its totals
}

// ------------------------------------------------------------------------------------------------
// Dispatch, combine.  A block takes CHUNK neighbouring pieces of eight channels; a thread has PER of them, reads a token's piece
// once and writes it to the k rows, or adds the k rows' pieces in order of the choices.  Bound by memory: the pieces of a
// thread are independent, all their loads are on the way together, and the one division is made per block.
struct RowsArgs {
  const __nv_bfloat16 *x;        // dispatch: [T, D]; combine: rows
  const int32_t *plan, *pos;
  const float *weights;
  const __nv_bfloat16 *y;        // dispatch as the backward of combine: the rows that were combined
  __nv_bfloat16 *out;            // dispatch: rows; combine: [T, D]
  float *dweights;
  long long T;
  int k, E, D;
  uint32_t magic;                // 2^32 / (D / 8), rounded up; 0 for D = 8
  int clear_experts, clear_blocks;   // dispatch: experts that have rows (at most), blocks for the rows behind one's
  int team;                      // dispatch with dweights: warps to a (token, choice)
};

// The first clear_experts * clear_blocks blocks: zeros in the rows between the experts that have any.
__device__ __forceinline__ void clear_between(const RowsArgs &a) {
  const int i_live = (int)blockIdx.x / a.clear_blocks, part = (int)blockIdx.x - i_live * a.clear_blocks;
  if (i_live >= a.plan[plan_n_live(a.E)]) return;
  const int e = a.plan[plan_live(a.E) + i_live];
  const long long first = a.plan[PLAN_OFFSETS + e] + a.plan[plan_counts(a.E) + e];
  const long long n = (a.plan[PLAN_OFFSETS + e + 1] - first) * (a.D >> 3);
  uint4 *p = reinterpret_cast<uint4 *>(a.out + first * a.D);
  for (long long i = part * 256 + threadIdx.x; i < n; i += a.clear_blocks * 256) p[i] = make_uint4(0u, 0u, 0u, 0u);
}

// Pieces of a thread.  More of them, or fewer threads on an SM, and the pieces' addresses and sums cost more than the loads gain:
// combine of two rows 16384 x 8192 135 us with 2 pieces and 5 blocks on an SM (4 and 2: 164, 1 and 8: 138; floor 123), of eight
// rows 8192 x 2048 48 us with one piece and 6 blocks (4 and 1: 53; floor 46); dispatch does not mind.
template <int K>
struct Combine {
  static constexpr int PER = K <= 2 ? 2 : 1, BLOCKS = K <= 2 ? 5 : 6, CHUNK = 256 * PER;
};
constexpr int PER = 2, CHUNK = 256 * PER;       // dispatch

// Token and first channel of piece `i` of a chunk that starts `lead` pieces into token t0.  Exact: lead + i < D / 8 + CHUNK, and that
// times D / 8 is below 2^32.
__device__ __forceinline__ void locate(const RowsArgs &a, long long t0, uint32_t at, long long &t, int &c) {
  const uint32_t pieces = (uint32_t)a.D >> 3, q = a.magic ? __umulhi(at, a.magic) : at;
  t = t0 + q;
  c = (int)((at - q * pieces) << 3);
}

template <bool WEIGHTED>
__global__ void __launch_bounds__(256) dispatch_kernel(const __grid_constant__ RowsArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const long long block = (long long)blockIdx.x - a.clear_experts * a.clear_blocks;
  if (block < 0) return clear_between(a);
  const long long start = block * CHUNK, n = a.T * (a.D >> 3) - start;
  const long long t0 = start / (a.D >> 3);
  const uint32_t lead = (uint32_t)(start - t0 * (a.D >> 3));
  uint4 v[PER];
  long long t[PER];
  int c[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = (int)threadIdx.x + u * 256;
    locate(a, t0, lead + i, t[u], c[u]);
    v[u] = i < n ? load16(a.x + t[u] * a.D + c[u]) : make_uint4(0u, 0u, 0u, 0u);
  }
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    if ((int)threadIdx.x + u * 256 >= n) break;
    for (int j = 0; j < a.k; ++j) {
      const long long r = a.pos[t[u] * a.k + j];
      uint4 w = v[u];
      if (WEIGHTED) {
        const float f = a.weights[t[u] * a.k + j];
        float g[8];
        widen8(v[u], g);
#pragma unroll
        for (int q = 0; q < 8; ++q) g[q] *= f;
        w = narrow8(g);
      }
      if (r >= 0) *reinterpret_cast<uint4 *>(a.out + r * a.D + c[u]) = w;
    }
  }
}

// The backward of combine: rows = w dout, and dw = dout . y in fp32.  A team of warps per (token, choice).
__global__ void __launch_bounds__(256) dispatch_dot_kernel(const __grid_constant__ RowsArgs a) {
  __shared__ float part[8];
  pdl_launch_dependents();
  pdl_wait();
  const long long block = (long long)blockIdx.x - a.clear_experts * a.clear_blocks;
  if (block < 0) return clear_between(a);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, teams = 8 / a.team, team = warp / a.team;
  const int tl = (warp - team * a.team) * 32 + lane, TL = a.team * 32;
  const long long slot = block * teams + team;
  const bool there = slot < a.T * a.k;
  const long long t = there ? slot / a.k : 0;
  const long long r = there ? a.pos[slot] : -1;
  float dot = 0.f;
  if (r >= 0) {
    const float w = a.weights ? a.weights[slot] : 1.0f;
    const __nv_bfloat16 *x = a.x + t * a.D, *y = a.y + r * a.D;
    __nv_bfloat16 *out = a.out + r * a.D;
    constexpr int AHEAD = 4;           // pieces of a lane on the way together
    for (int c = tl * 8; c < a.D; c += AHEAD * TL * 8) {
      uint4 xv[AHEAD], yv[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int at = c + u * TL * 8;
        xv[u] = at < a.D ? *reinterpret_cast<const uint4 *>(x + at) : make_uint4(0u, 0u, 0u, 0u);
        yv[u] = at < a.D ? load16(y + at) : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int at = c + u * TL * 8;
        float f[8], h[8];
        widen8(xv[u], f);
        widen8(yv[u], h);
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          s = fmaf(f[q], h[q], s);
          f[q] *= w;
        }
        dot += s;
        if (at < a.D) *reinterpret_cast<uint4 *>(out + at) = narrow8(f);
      }
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

// K: rows that a thread has on the way for each of its pieces (k itself up to 2).
template <int K>
__global__ void __launch_bounds__(256, Combine<K>::BLOCKS) combine_kernel(const __grid_constant__ RowsArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int AT_ONCE = Combine<K>::PER;
  const long long start = (long long)blockIdx.x * Combine<K>::CHUNK, n = a.T * (a.D >> 3) - start;
  const long long t0 = start / (a.D >> 3);
  const uint32_t lead = (uint32_t)(start - t0 * (a.D >> 3));
  long long t[AT_ONCE];
  int c[AT_ONCE];
  float sum[AT_ONCE][8];
#pragma unroll
  for (int u = 0; u < AT_ONCE; ++u) {
    locate(a, t0, lead + threadIdx.x + u * 256, t[u], c[u]);
#pragma unroll
    for (int q = 0; q < 8; ++q) sum[u][q] = 0.f;
  }
  for (int j0 = 0; j0 < a.k; j0 += K) {
    uint4 v[AT_ONCE][K];
    float w[AT_ONCE][K];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
      for (int q = 0; q < K; ++q) {
        const bool there = (int)threadIdx.x + u * 256 < n && (K <= 2 || j0 + q < a.k);
        const long long slot = t[u] * a.k + j0 + q, r = there ? a.pos[slot] : -1;
        v[u][q] = r >= 0 ? load16(a.x + r * a.D + c[u]) : make_uint4(0u, 0u, 0u, 0u);
        w[u][q] = r < 0 ? 0.f : a.weights ? a.weights[slot] : 1.0f;
      }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
      for (int q = 0; q < K; ++q) {
        float f[8];
        widen8(v[u][q], f);
#pragma unroll
        for (int h = 0; h < 8; ++h) sum[u][h] = fmaf(w[u][q], f[h], sum[u][h]);
      }
  }
#pragma unroll
  for (int u = 0; u < AT_ONCE; ++u)
    if ((int)threadIdx.x + u * 256 < n) *reinterpret_cast<uint4 *>(a.out + t[u] * a.D + c[u]) = narrow8(sum[u]);
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
  auto go = [&](auto kernel) { return launch_overlapped(kernel, grid, block, 0, 1, stream, a); };
  if (a.E <= 32) return go(route_fwd_kernel<L, 1>);
  if (a.E <= 64) return go(route_fwd_kernel<L, 2>);
  if (a.E <= 128) return go(route_fwd_kernel<L, 4>);
  if (a.E <= 256) return go(route_fwd_kernel<L, 8>);
  if (a.E <= 512) return go(route_fwd_kernel<L, 16>);
  return go(route_fwd_kernel<L, 32>);
}

template <typename L>
int launch_route_bwd(const RouteBackArgs &b, cudaStream_t stream) {
  const RouteArgs &a = b.r;
  const dim3 block(32 * ROUTE_WARPS);
  if (a.score != OSDP_SCORE_SOFTMAX || a.renorm)
    return launch_overlapped(route_bwd_kernel<L>, dim3((unsigned)cdiv(a.T, ROUTE_WARPS)), block, 0, 1, stream, b);
  const dim3 grid((unsigned)cdiv(a.T, ROUTE_WARPS));
  auto go = [&](auto kernel) { return launch_overlapped(kernel, grid, block, 0, 1, stream, b); };
  if (a.E <= 32) return go(route_bwd_dense_kernel<L, 1>);
  if (a.E <= 64) return go(route_bwd_dense_kernel<L, 2>);
  if (a.E <= 128) return go(route_bwd_dense_kernel<L, 4>);
  if (a.E <= 256) return go(route_bwd_dense_kernel<L, 8>);
  if (a.E <= 512) return go(route_bwd_dense_kernel<L, 16>);
  return go(route_bwd_dense_kernel<L, 32>);
}

int check_rows(int64_t T, int top_k, int E, int64_t D) {
  const int rc = check_choices(T, top_k, E);
  if (rc) return rc;
  if (D <= 0 || D > OSDP_EXPERT_MAX_D || T * (D / 8) > ((int64_t)1 << 40)) return OSDP_ERR_BAD_SHAPE;
  return (D & 7) ? OSDP_ERR_ALIGNMENT : OSDP_OK;
}

}  // namespace

namespace {
uint32_t piece_magic(int64_t D) { return D > 8 ? (uint32_t)((((uint64_t)1 << 32) + D / 8 - 1) / (D / 8)) : 0u; }
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
  RouteArgs a{logits, (long long)ld, (long long)T, bias, E, top_k, score, n_groups, top_groups, group_take, renorm ? 1 : 0, (float)scale,
              idx, weights, E / n_groups, 5, 0u};
  while ((n_groups << a.lanes_log2) > 32) --a.lanes_log2;
  a.magic = ((1u << 20) + a.size - 1) / a.size;
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
                  nullptr, E, 5, 0u};
  b.dweights = dweights;
  b.dlogits = dlogits;
  b.ld_out = (long long)ld_dlogits;
  b.dense = ld_dlogits == E && aligned_to(dlogits, 16) ? 1 : 0;
  return logits_dtype == OSDP_DTYPE_FP32 ? launch_route_bwd<float>(b, static_cast<cudaStream_t>(stream))
                                         : launch_route_bwd<__nv_bfloat16>(b, static_cast<cudaStream_t>(stream));
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
  const size_t smem = (size_t)(PLAN_WARPS + 2) * E * sizeof(int);
  if (smem > 40 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(expert_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (PLAN_WARPS + 2) * OSDP_MAX_EXPERTS * 4);
    if (e != cudaSuccess) return report_cuda(e);
  }
  const PlanArgs a{idx, (int)(T * top_k), E, plan, pos};
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
             dweights, (long long)T, top_k, E, (int)D, piece_magic(D), 0, 1, 1};
  int sms = 0;
  const int src = sm_count(&sms);
  if (src) return src;
  // up to 63 rows behind each expert's: eight pieces to a thread, where that does not make more blocks than the GPU has room for
  a.clear_blocks = (int)cdiv((OSDP_EXPERT_ROWS - 1) * (D / 8), 2048);
  a.clear_experts = (int)(T * top_k < E ? T * top_k : E);
  if (a.clear_blocks > 4 * sms / a.clear_experts) a.clear_blocks = 4 * sms / a.clear_experts > 0 ? 4 * sms / a.clear_experts : 1;
  const int64_t clear = (int64_t)a.clear_experts * a.clear_blocks;
  if (dweights) {
    // as many warps to a row as it has pieces for, more where there are few rows
    a.team = 1;
    while (a.team < 8 && a.team * 256 < D && (T * top_k * a.team < (int64_t)sms * 16 || a.team * 2048 < D)) a.team *= 2;
    return launch_overlapped(dispatch_dot_kernel, dim3((unsigned)(cdiv(T * top_k, 8 / a.team) + clear)), dim3(256), 0, 1, static_cast<cudaStream_t>(stream), a);
  }
  return launch_overlapped(weights ? dispatch_kernel<true> : dispatch_kernel<false>, dim3((unsigned)(cdiv(T * (D / 8), CHUNK) + clear)), dim3(256), 0, 1,
                           static_cast<cudaStream_t>(stream), a);
}

extern "C" int osdp_expert_combine(const void *rows, const int32_t *plan, const int32_t *pos, const float *weights, int64_t T, int top_k, int E,
                                   int64_t D, void *out, void *stream) {
  const int rc = check_rows(T, top_k, E, D);
  if (rc) return rc;
  if (T == 0) return OSDP_OK;
  if (!rows || !pos || !plan || !out) return OSDP_ERR_NULL_POINTER;
  if (!aligned_to(rows, 16) || !aligned_to(out, 16) || !aligned_to(plan, 16) || !aligned_to(pos, 4) || !aligned_to(weights, 4)) return OSDP_ERR_ALIGNMENT;
  const RowsArgs a{static_cast<const __nv_bfloat16 *>(rows), plan, pos, weights, nullptr, static_cast<__nv_bfloat16 *>(out), nullptr, (long long)T,
                   top_k, E, (int)D, piece_magic(D), 0, 1, 1};
  const dim3 grid((unsigned)cdiv(T * (D / 8), top_k <= 2 ? Combine<2>::CHUNK : Combine<4>::CHUNK));
  if (top_k == 1) return launch_overlapped(combine_kernel<1>, grid, dim3(256), 0, 1, static_cast<cudaStream_t>(stream), a);
  if (top_k == 2) return launch_overlapped(combine_kernel<2>, grid, dim3(256), 0, 1, static_cast<cudaStream_t>(stream), a);
  return launch_overlapped(combine_kernel<4>, grid, dim3(256), 0, 1, static_cast<cudaStream_t>(stream), a);
}

// The optimiser step of the flat parameters: global gradient norm with its clipping coefficient, and AdamW over
// many tensors in one launch, with 32-bit or 8-bit states.
//
//   g' = c g                       c: clipping coefficient (1 without)
//   m  = b1 m + (1 - b1) g'        v = b2 v + (1 - b2) g'^2
//   p  = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8-bit states: 256 consecutive elements share one fp32 scale = (largest magnitude) / 448 and are kept as e4m3 codes
// (448 is the largest e4m3 value).  The second moment is kept as its root, which halves the range that the codes have
// to cover (2^-9 ... 448 of a root is 10 decades of v), and a root above zero is never rounded to zero: that would turn
// a small second moment into a huge step.  The step itself uses the unrounded m and v.
//
// Rounding to nearest holds a moment where it is as long as a step moves it by less than half a code, 3 to 6 % of it, and
// beta close to one moves it by 1 - beta at most.  After half of a block's gradients had become five times smaller, their
// stored root was, 5 / (1 - beta2) and then 50 / (1 - beta2) steps later, too large by a factor of
//   beta2 0.95: 1.5 and 1.05,  0.97: 3.6 and 1.2,  0.98: 6.3 and 5.9,  0.99: 5.8 and 6.5    (normal gradients; 0.999 no better)
// while with a dither before the rounding, which makes it right on average, it was 1.10 and 1.02 at every one of them.
// So a moment whose beta is above DITHER_ABOVE is rounded with the dither.  Nearest is better below: a moment that is
// renewed within some dozen steps carries the noise of the gradients, which is dither enough, and the codes' own error is half.
// The dither takes 537 M parameters from 874 to 1035 us for one moment, 1175 for both (instructions).
#include "../../include/osdp.h"

#include <cmath>
#include <type_traits>

#include "osdp_internal.h"
#include "osdp_vec.cuh"

namespace osdp {
namespace {

constexpr int QB = OSDP_ADAMW_BLOCK;       // elements per 8-bit scale; one warp works on one such block
constexpr int THREADS = 256;
constexpr int CHUNK = 4096;                // elements of one tensor that a thread block works on
constexpr int STATUS_BYTES = 256;
constexpr double DITHER_ABOVE = 0.975;
constexpr float TINY = 7.888609052210118e-31f;   // 2^-100: a block whose largest magnitude is below it is stored as zeros

struct Entry {
  void *param;
  const void *grad;
  long long numel;
  long long state;     // element offset in the flat states
  float decay;         // 1 - lr * weight_decay
  float size;          // lr / (1 - b1^t)
  int first_chunk;
  int aligned;         // param and grad allow eight-element accesses
};
// Tensors of one launch.  The table travels as a kernel parameter (up to 32 KB): no copy to the device, nothing to
// keep alive, and a stream capture takes it along.  Three sizes, so that a step over fewer tensors does not pay for
// the launch of a full table.
constexpr int TABLE_SMALL = 48, TABLE_MIDDLE = 192, TABLE_LARGE = 640;
template <int MAXT>
struct Table {
  Entry e[MAXT];
  int n;
  int chunks;
};

template <int MAXT>
__device__ __forceinline__ int find_entry(const Table<MAXT> &t, int chunk) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].first_chunk <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

struct Hyper {
  float b1, one_minus_b1, b2, one_minus_b2, eps;
  float root_scale;    // 1 / sqrt(1 - b2^t)
  float one;           // 1, but not to the compiler: a * one + b is a sum that it cannot merge with the product a
  uint32_t seed;       // of the dither: the step's number
  int dither_m, dither_v;
};

enum States { F32, CODES, DITHERED };   // fp32; 8-bit codes; 8-bit codes of which m's, v's or both are dithered

// Random bits for eight consecutive elements from their number (the first one's index in the flat states / 8) and the step's:
// products with odd numbers (2^32 / the golden ratio, / sqrt 2, (sqrt 3 - 1) 2^32) and shifted sums in turn.  Element j of
// moment k (0 m, 1 v) takes the upper 20 bits of 2 (j + 8 k) + 1 times the result.
__device__ __forceinline__ uint32_t dither_bits(unsigned long long group, uint32_t seed) {
  uint32_t x = (uint32_t)group ^ (uint32_t)(group >> 32) * 0xB504F333u ^ seed * 0xBB67AE85u;
  x = (x ^ x >> 16) * 0xB504F333u;
  x = (x ^ x >> 15) * 0x9E3779B9u;
  return (x ^ x >> 16) * 0x9E3779B9u;
}
// x (|x| <= 448) to a value of e4m3, up or down with the probabilities that make it x on average.  A code has three
// mantissa bits below the leading one, 2^-9 at least: magnitudes below 2^-6 are moved up by 2^-6, where that is the step; the
// dither is added to the bits behind it and what is left of them cut off.
__device__ __forceinline__ float dither1(float x, uint32_t bits) {
  const float a = fabsf(x), up = a < 0.015625f ? 0.015625f : 0.f;
  return copysignf(__uint_as_float((__float_as_uint(a + up) + (bits >> 12)) & 0xFFF00000u) - up, x);
}

__device__ __forceinline__ bool has_zero_byte(uint32_t w) { return ((w - 0x01010101u) & ~w & 0x80808080u) != 0u; }

// Square roots to a relative 2^-22, for the update alone (of subnormal numbers too).
__device__ __forceinline__ f2 fast_root2(f2 v) {
  const float2 a = split2(v);
  return pack2(fast_sqrt(a.x), fast_sqrt(a.y));
}
// From -v the negated square root of v, for roots that are stored: q = -v / sqrt(v) to a relative 2^-22, then one of Heron's
// steps, q + (q^2 - v) / (2 sqrt(v)), whose remainder is 2^-45.  With one rounding after it that is the nearest fp32 value but for a case
// in 10^6; signs are chosen so that no operation goes into them.  Zeros stay zeros: the reciprocal root is taken of at least
// 2^-126.  The library's function took 60 us more for 537 M parameters.  Not for v below 2^-100 (root_of_small): the
// remainder q^2 - v leaves fp32's range there.
__device__ __forceinline__ f2 negated_root2(f2 minus_v) {
  const float2 a = split2(minus_v);
  constexpr float least = 1.17549435e-38f;
  const f2 y = pack2(fast_rsqrt(fmaxf(-a.x, least)), fast_rsqrt(fmaxf(-a.y, least)));
  const f2 q = mul2(minus_v, y);
  return fma2(fma2(q, q, minus_v), mul2(y, both(0.5f)), q);
}
__device__ __forceinline__ float root_of_small(float minus_v, float root) { return minus_v < 0.f && minus_v > -TINY ? -__fsqrt_rn(-minus_v) : root; }

// 256 elements -> codes and their scale.  ROOT: x holds negated roots; those of numbers above zero keep at least the smallest
// code.
// DITHER: rounded with a dither if `dither` is set; `bits` = dither_bits of the lane's elements.
template <bool ROOT, bool DITHER>
__device__ __forceinline__ void quantise_block(const f2 (&x)[4], uint8_t *codes, float *scale, int lane, bool dither, uint32_t bits) {
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 v = split2(x[j]);
    top = max_abs3(top, v.x, v.y);
  }
  top = warp_max_abs(top);
  const bool live = !(top < TINY);
  const float inv = live ? __frcp_rn(top) * 448.0f : 0.0f;
  const f2 inv2 = both(ROOT ? -inv : inv);
  f2 c[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) c[j] = ROOT ? fma2(x[j], inv2, both(0.0f)) : mul2(x[j], inv2);   // a root's zero has the code of +0
  if (DITHER && dither) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 v = split2(c[j]);
      const uint32_t n = (ROOT ? 16 : 0) + 4 * j + 1;
      c[j] = pack2(dither1(v.x, bits * n), dither1(v.y, bits * (n + 2)));
    }
  }
  uint2 q = encode_e4m3x8(c);
  if (ROOT && (has_zero_byte(q.x) || has_zero_byte(q.y))) {   // rare: an element that is zero, or very small in its block
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 v = split2(x[j]);
      float2 l = split2(c[j]);
      constexpr float least = 0.001953125f;   // 2^-9, the smallest e4m3 value
      if (live && v.x < 0.f) l.x = fmaxf(l.x, least);
      if (live && v.y < 0.f) l.y = fmaxf(l.y, least);
      c[j] = pack2(l.x, l.y);
    }
    q = encode_e4m3x8(c);
  }
  *reinterpret_cast<uint2 *>(codes + lane * 8) = q;
  if (lane == 0) *scale = live ? top * (1.0f / 448.0f) : 0.0f;
}

// What a lane reads of one block of 256 elements, as it lies in memory.
template <typename T>
struct Raw8 {
  uint32_t w[2 * sizeof(T)];
};
template <typename T>
__device__ __forceinline__ void load_raw(const T *p, Raw8<T> &r) {
  if constexpr (sizeof(T) == 2) {
    const uint4 v = load16(p);
    r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
  } else {
    load32(p, r.w);
  }
}
template <typename T>
__device__ __forceinline__ void load_raw_part(const T *p, int n, Raw8<T> &r) {   // the first n < 8 elements, then zeros; any alignment
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t lo = 2 * j < n ? reinterpret_cast<const uint16_t *>(p)[2 * j] : 0u, hi = 2 * j + 1 < n ? reinterpret_cast<const uint16_t *>(p)[2 * j + 1] : 0u;
      r.w[j] = lo | hi << 16;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.w[j] = j < n ? reinterpret_cast<const uint32_t *>(p)[j] : 0u;
  }
}
template <typename T>
__device__ __forceinline__ void widen_raw(const Raw8<T> &r, f2 (&f)[4]) {
  if constexpr (sizeof(T) == 2) {
    widen4(make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]), f);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = pack2(__uint_as_float(r.w[2 * j]), __uint_as_float(r.w[2 * j + 1]));
  }
}

template <bool E4M3>
struct RawState {
  uint32_t m[E4M3 ? 2 : 8], v[E4M3 ? 2 : 8];
  float fm, fv;
};

// Each warp takes blocks of 256 consecutive elements, eight per lane, so that every array is read and written in whole
// lines and a block's scale is a warp reduction.  All loads of BLOCKS blocks are issued before the first is used.
// What bounds it: HBM with 32-bit states (28 bytes an element: 134 M bf16 parameters with fp32 masters 6310 GB/s of a copy rate
// of 6547, the gradient norm before it included).  With 8-bit states (10 bytes an element) the instructions come near: 64 an
// element in scalar form took 1450 us for 537 M parameters, some 45 an element with pairs of fp32, approximate reciprocals
// and the rare paths set apart take 868 us at full clocks (6220 GB/s) and 1010 us in the power-capped state.
template <typename T, bool MASTER, States STATES, int MAXT>
__global__ void __launch_bounds__(THREADS) adamw_kernel(const __grid_constant__ Table<MAXT> t, const Hyper h, float *master,
                                                        void *state_m, void *state_v, float *scale_m, float *scale_v,
                                                        const float *clip) {
  constexpr bool E4M3 = STATES != F32, DITHER = STATES == DITHERED;
  constexpr int WARPS = THREADS / 32, PER_WARP = CHUNK / (WARPS * QB), BLOCKS = E4M3 ? PER_WARP : 1;
  pdl_launch_dependents();
  // After the gradient norm the last gradients that it read are still in L2: those first.
  const int chunk = clip ? (int)(gridDim.x - 1 - blockIdx.x) : (int)blockIdx.x;
  const Entry &e = t.e[find_entry(t, chunk)];
  const long long base = (long long)(chunk - e.first_chunk) * CHUNK;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  float coef = 1.0f;
  if (clip) {
    coef = clip[1];
    if (!isfinite(coef)) return;   // the gradient's norm is not a number: nothing is updated
  }
  T *param = static_cast<T *>(e.param);
  const T *grad = static_cast<const T *>(e.grad);
  using W = typename std::conditional<MASTER, float, T>::type;
  constexpr float sign = E4M3 ? -1.0f : 1.0f;   // 8-bit states: v and its root are negated, see negated_root2
  const f2 b1 = both(h.b1), n1 = both(h.one_minus_b1), b2 = both(sign * h.b2), n2 = both(sign * h.one_minus_b2), eps = both(h.eps),
           root_scale = both(sign * h.root_scale), clipped = both(coef), one = both(h.one), decay = both(e.decay), size = both(-e.size);
#pragma unroll 1
  for (int it = 0; it < PER_WARP; it += BLOCKS) {
    Raw8<T> rg[BLOCKS];
    Raw8<W> rw[BLOCKS];
    RawState<E4M3> rs[BLOCKS];
#pragma unroll
    for (int q = 0; q < BLOCKS; ++q) {
      const long long blk = base + ((it + q) * WARPS + warp) * QB;
      if (blk >= e.numel) break;
      const long long i = blk + lane * 8, si = e.state + i;   // first element in the tensor, and in the flat states (whole blocks are there)
      const bool whole = e.aligned && i + 8 <= e.numel;
      const int left = (int)min(max(e.numel - i, 0ll), 8ll);
      if (whole) load_raw(grad + i, rg[q]);
      else load_raw_part(grad + i, left, rg[q]);
      if constexpr (MASTER) {
        load_raw(master + si, rw[q]);
      } else {
        if (whole) load_raw(param + i, rw[q]);
        else load_raw_part(param + i, left, rw[q]);
      }
      if constexpr (E4M3) {
        const uint2 cm = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(state_m) + si),
                    cv = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(state_v) + si);
        rs[q].m[0] = cm.x; rs[q].m[1] = cm.y;
        rs[q].v[0] = cv.x; rs[q].v[1] = cv.y;
        rs[q].fm = scale_m[(e.state + blk) / QB];
        rs[q].fv = scale_v[(e.state + blk) / QB];
      } else {
        load32(static_cast<const float *>(state_m) + si, rs[q].m);
        load32(static_cast<const float *>(state_v) + si, rs[q].v);
      }
    }
#pragma unroll
    for (int q = 0; q < BLOCKS; ++q) {
      const long long blk = base + ((it + q) * WARPS + warp) * QB;
      if (blk >= e.numel) break;
      const long long i = blk + lane * 8, si = e.state + i;
      const bool whole = e.aligned && i + 8 <= e.numel;
      f2 w[4], g[4], m[4], v[4], root[4];
      widen_raw(rg[q], g);
      widen_raw(rw[q], w);
      if constexpr (E4M3) {
        decode_e4m3x8(make_uint2(rs[q].m[0], rs[q].m[1]), m);
        decode_e4m3x8(make_uint2(rs[q].v[0], rs[q].v[1]), v);
        const f2 fm = both(rs[q].fm), fv = both(rs[q].fv);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          m[j] = mul2(m[j], fm);
          v[j] = mul2(v[j], fv);
          v[j] = mul2(v[j], v[j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          m[j] = pack2(__uint_as_float(rs[q].m[2 * j]), __uint_as_float(rs[q].m[2 * j + 1]));
          v[j] = pack2(__uint_as_float(rs[q].v[2 * j]), __uint_as_float(rs[q].v[2 * j + 1]));
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // Each operation of the formulas rounded by itself: 8-bit codes jump at ties, so that another evaluation of the
        // formulas only gives the same codes where it gives the same bits.  (Contracted
        // sums and approximate roots moved a code in 10^6, and with it the next step's scale where that was the largest.)
        g[j] = mul2(g[j], clipped);
        m[j] = fma2(mul2(m[j], b1), one, mul2(g[j], n1));
        v[j] = fma2(mul2(v[j], b2), one, mul2(mul2(g[j], g[j]), n2));
        root[j] = E4M3 ? negated_root2(v[j]) : fast_root2(v[j]);
      }
      if constexpr (E4M3) {
        float smallest = TINY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 x = split2(v[j]);
          smallest = min_abs3(smallest, x.x, x.y);
        }
        if (smallest < TINY) {   // rare, but for zeros
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 x = split2(v[j]), r = split2(root[j]);
            root[j] = pack2(root_of_small(x.x, r.x), root_of_small(x.y, r.y));
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 d = split2(fma2(root[j], root_scale, eps));
        const f2 upd = mul2(m[j], pack2(fast_rcp(d.x), fast_rcp(d.y)));
        w[j] = fma2(upd, size, mul2(w[j], decay));
      }
      if constexpr (MASTER) store4(master + si, w);
      if (whole) {
        store4(param + i, w);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 p = split2(w[j >> 1]);
          if (i + j < e.numel) param[i + j] = from_f32<T>((j & 1) ? p.y : p.x);
        }
      }
      if constexpr (E4M3) {
        const long long sb = (e.state + blk) / QB;
        const uint32_t bits = DITHER ? dither_bits((unsigned long long)si >> 3, h.seed) : 0u;
        quantise_block<false, DITHER>(m, static_cast<uint8_t *>(state_m) + (e.state + blk), scale_m + sb, lane, h.dither_m != 0, bits);
        quantise_block<true, DITHER>(root, static_cast<uint8_t *>(state_v) + (e.state + blk), scale_v + sb, lane, h.dither_v != 0, bits);
      } else {
        store4(static_cast<float *>(state_m) + si, m);
        store4(static_cast<float *>(state_v) + si, v);
      }
    }
  }
}

// ---- gradient norm: one partial sum of squares per thread block, added in block order by the block that finishes
// last (no floating-point atomics: the same gradients give the same bits).  HBM-bound: 537 MB 85 us, 6330 GB/s; with two
// loads in flight a thread instead of eight it was 127 us.
constexpr int NORM_BLOCKS = 592;   // 4 per SM
constexpr int NORM_CHUNK = 16384;  // eight vectors per thread, all loads issued before the first is used

__device__ __forceinline__ void clip_coefficient(double squares, float max_norm, float *out) {
  const float norm = (float)sqrt(squares);
  out[0] = norm;
  // a norm that is not finite has no coefficient: the step that reads NaN changes nothing
  out[1] = !isfinite(norm) ? __int_as_float(0x7FC00000) : max_norm > 0.f ? fminf(max_norm / (norm + 1e-6f), 1.0f) : 1.0f;
}

template <typename T, int MAXT>
__global__ void __launch_bounds__(THREADS) grad_norm_kernel(const __grid_constant__ Table<MAXT> t, float *partial, int first_partial,
                                                            int total_partials, unsigned *ticket, float max_norm,
                                                            float *out, double *squares) {
  __shared__ float red[THREADS / 32];
  __shared__ bool last;
  pdl_launch_dependents();
  pdl_wait();
  f2 acc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = both(0.f);
  constexpr int VECS = NORM_CHUNK / (THREADS * 8);
  for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const Entry &e = t.e[find_entry(t, c)];
    const long long base = (long long)(c - e.first_chunk) * NORM_CHUNK;
    const T *grad = static_cast<const T *>(e.grad);
    Raw8<T> raw[VECS];
#pragma unroll
    for (int it = 0; it < VECS; ++it) {
      const long long i = base + (it * THREADS + threadIdx.x) * 8;
      if (e.aligned && i + 8 <= e.numel) load_raw(grad + i, raw[it]);
      else load_raw_part(grad + i, (int)min(max(e.numel - i, 0ll), 8ll), raw[it]);
    }
#pragma unroll
    for (int it = 0; it < VECS; ++it) {
      f2 g[4];
      widen_raw(raw[it], g);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = fma2(g[j], g[j], acc[j]);
    }
  }
  float s = sum2(add2(add2(acc[0], acc[1]), add2(acc[2], acc[3])));
  s = warp_sum(s);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = red[0];
#pragma unroll
    for (int k = 1; k < THREADS / 32; ++k) s += red[k];
    partial[first_partial + blockIdx.x] = s;
    __threadfence();
    last = atomicAdd(ticket, 1u) == (unsigned)total_partials - 1u;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double d = 0.0;
  for (int k = threadIdx.x; k < total_partials; k += THREADS) d += (double)__ldcg(partial + k);
  __shared__ double sum[THREADS];
  sum[threadIdx.x] = d;
  __syncthreads();
  for (int k = THREADS / 2; k > 0; k >>= 1) {
    if (threadIdx.x < k) sum[threadIdx.x] += sum[threadIdx.x + k];
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    if (squares) *squares = sum[0];
    else clip_coefficient(sum[0], max_norm, out);
    *ticket = 0u;
  }
}

// The coefficient of sums of squares that were taken apart (by dtype, by rank).
__global__ void __launch_bounds__(32) clip_kernel(const double *sums, int n, float max_norm, float *out) {
  pdl_launch_dependents();
  pdl_wait();
  if (threadIdx.x != 0) return;
  double s = 0.0;
  for (int k = 0; k < n; ++k) s += sums[k];
  clip_coefficient(s, max_norm, out);
}

int check_tensors(const osdp_adamw_tensor *t, int n, int dtype, bool need_param) {
  if (n < 0) return OSDP_ERR_BAD_SHAPE;
  if (n > 0 && !t) return OSDP_ERR_NULL_POINTER;
  if (dtype != OSDP_DTYPE_BF16 && dtype != OSDP_DTYPE_FP32) return OSDP_ERR_UNSUPPORTED;
  const uintptr_t es = dtype == OSDP_DTYPE_FP32 ? 4 : 2;
  int64_t total = 0;
  for (int i = 0; i < n; ++i) {
    // 2^42 elements in all: the chunks of any table are then below 2^31
    if (t[i].numel < 0 || t[i].numel > ((int64_t)1 << 42) - total) return OSDP_ERR_BAD_SHAPE;
    total += t[i].numel;
    if (t[i].numel == 0) continue;
    if (!t[i].grad || (need_param && !t[i].param)) return OSDP_ERR_NULL_POINTER;
    if (!aligned_to(t[i].grad, es) || (need_param && !aligned_to(t[i].param, es))) return OSDP_ERR_ALIGNMENT;
    if (need_param && (t[i].state_offset < 0 || t[i].state_offset % QB)) return OSDP_ERR_ALIGNMENT;
  }
  return OSDP_OK;
}

// Fills tables with the tensors that have elements and hands each to launch(table, is_first, index of its first chunk).
template <int MAXT, typename Fill, typename Launch>
int for_each_table(const osdp_adamw_tensor *t, int n, int dtype, bool with_param, int chunk, Fill fill, Launch launch) {
  const uintptr_t vec = dtype == OSDP_DTYPE_FP32 ? 32 : 16;
  Table<MAXT> tab;
  int i = 0;
  while (i < n) {
    tab.n = 0;
    int64_t chunks = 0;
    for (; i < n && tab.n < MAXT; ++i) {
      if (t[i].numel == 0) continue;
      Entry &e = tab.e[tab.n++];
      e.param = t[i].param;
      e.grad = t[i].grad;
      e.numel = t[i].numel;
      e.state = t[i].state_offset;
      e.first_chunk = (int)chunks;
      e.aligned = aligned_to(t[i].grad, vec) && (!with_param || aligned_to(t[i].param, vec));
      fill(t[i], e);
      chunks += cdiv(t[i].numel, chunk);
    }
    if (tab.n == 0) break;
    tab.chunks = (int)chunks;
    const int rc = launch(tab);
    if (rc) return rc;
  }
  return OSDP_OK;
}

template <typename T, bool MASTER, States STATES, int MAXT>
int launch_adamw(const osdp_adamw_tensor *t, int n, int dtype, const Hyper &h, double beta1_t, float *master, void *m, void *v,
                 float *sm, float *sv, const float *clip, cudaStream_t stream) {
  return for_each_table<MAXT>(
      t, n, dtype, true, CHUNK,
      [&](const osdp_adamw_tensor &a, Entry &e) {
        e.decay = (float)(1.0 - a.lr * a.weight_decay);
        e.size = (float)(a.lr / (1.0 - beta1_t));
      },
      [&](const Table<MAXT> &tab) {
        return launch_overlapped(adamw_kernel<T, MASTER, STATES, MAXT>, dim3((unsigned)tab.chunks), dim3(THREADS), 0, 1, stream, tab, h,
                                 master, m, v, sm, sv, clip);
      });
}

template <typename T, bool MASTER, States STATES>
int pick_table(const osdp_adamw_tensor *t, int n, int dtype, const Hyper &h, double b1t, float *master, void *m, void *v, float *sm,
               float *sv, const float *clip, cudaStream_t stream) {
  if (n <= TABLE_SMALL) return launch_adamw<T, MASTER, STATES, TABLE_SMALL>(t, n, dtype, h, b1t, master, m, v, sm, sv, clip, stream);
  if (n <= TABLE_MIDDLE) return launch_adamw<T, MASTER, STATES, TABLE_MIDDLE>(t, n, dtype, h, b1t, master, m, v, sm, sv, clip, stream);
  return launch_adamw<T, MASTER, STATES, TABLE_LARGE>(t, n, dtype, h, b1t, master, m, v, sm, sv, clip, stream);
}

template <typename T, int MAXT>
int launch_norm(const osdp_adamw_tensor *t, int n, int dtype, float max_norm, float *out, double *squares, float *partial, unsigned *ticket,
                cudaStream_t stream) {
  // the number of partial sums has to be known before the first launch
  int total = 0;
  auto blocks = [](int chunks) { return chunks < NORM_BLOCKS ? chunks : NORM_BLOCKS; };
  auto none = [](const osdp_adamw_tensor &, Entry &) {};
  int rc = for_each_table<MAXT>(t, n, dtype, false, NORM_CHUNK, none, [&](const Table<MAXT> &tab) { total += blocks(tab.chunks); return OSDP_OK; });
  if (rc) return rc;
  Table<MAXT> empty;
  empty.n = 0;
  empty.chunks = 0;
  if (total == 0)   // no elements at all: the norm is zero
    return launch_overlapped(grad_norm_kernel<T, MAXT>, dim3(1), dim3(THREADS), 0, 1, stream, empty, partial, 0, 1, ticket, max_norm, out, squares);
  int at = 0;
  return for_each_table<MAXT>(t, n, dtype, false, NORM_CHUNK, none, [&](const Table<MAXT> &tab) {
    const int b = blocks(tab.chunks);
    const int first = at;
    at += b;
    return launch_overlapped(grad_norm_kernel<T, MAXT>, dim3((unsigned)b), dim3(THREADS), 0, 1, stream, tab, partial, first, total, ticket,
                             max_norm, out, squares);
  });
}

size_t norm_workspace(int n) {
  const size_t tables = (size_t)cdiv(n > 0 ? n : 1, TABLE_LARGE);
  return STATUS_BYTES + tables * NORM_BLOCKS * sizeof(float);
}

// Norm and coefficient into `out`, or the sum of squares into `squares`.
int norm_of(const osdp_adamw_tensor *tensors, int n_tensors, int dtype, float max_norm, float *out, double *squares, void *ws,
            size_t ws_bytes, cudaStream_t s) {
  const int rc = check_tensors(tensors, n_tensors, dtype, false);
  if (rc) return rc;
  if ((!out && !squares) || !ws) return OSDP_ERR_NULL_POINTER;
  if (!aligned_to(ws, 256) || !aligned_to(out, 4) || !aligned_to(squares, 8)) return OSDP_ERR_ALIGNMENT;
  if (ws_bytes < norm_workspace(n_tensors)) return OSDP_ERR_WORKSPACE_TOO_SMALL;
  unsigned *ticket = reinterpret_cast<unsigned *>(static_cast<char *>(ws) + 64);
  float *partial = reinterpret_cast<float *>(static_cast<char *>(ws) + STATUS_BYTES);
#define OSDP_NORM(T) \
  (n_tensors <= TABLE_SMALL ? launch_norm<T, TABLE_SMALL>(tensors, n_tensors, dtype, max_norm, out, squares, partial, ticket, s) \
   : n_tensors <= TABLE_MIDDLE ? launch_norm<T, TABLE_MIDDLE>(tensors, n_tensors, dtype, max_norm, out, squares, partial, ticket, s) \
                               : launch_norm<T, TABLE_LARGE>(tensors, n_tensors, dtype, max_norm, out, squares, partial, ticket, s))
  return dtype == OSDP_DTYPE_FP32 ? OSDP_NORM(float) : OSDP_NORM(__nv_bfloat16);
#undef OSDP_NORM
}

}  // namespace
}  // namespace osdp

using namespace osdp;

extern "C" {

int osdp_adamw_layout(const int64_t *numel, int n, int64_t *state_offset, int64_t *state_elems) {
  if (n < 0) return OSDP_ERR_BAD_SHAPE;
  if ((n > 0 && !numel) || !state_elems) return OSDP_ERR_NULL_POINTER;
  int64_t at = 0;
  for (int i = 0; i < n; ++i) {
    if (numel[i] < 0 || numel[i] > ((int64_t)1 << 42) - at) return OSDP_ERR_BAD_SHAPE;
    if (state_offset) state_offset[i] = at;
    at += cdiv(numel[i], QB) * QB;
  }
  *state_elems = at;
  return OSDP_OK;
}

int osdp_grad_norm_workspace_bytes(int n_tensors, size_t *bytes) {
  if (!bytes) return OSDP_ERR_NULL_POINTER;
  if (n_tensors < 0) return OSDP_ERR_BAD_SHAPE;
  *bytes = norm_workspace(n_tensors);
  return OSDP_OK;
}

int osdp_grad_norm(const osdp_adamw_tensor *tensors, int n_tensors, int grad_dtype, float max_norm, float *out, void *ws,
                   size_t ws_bytes, void *stream) {
  if (std::isnan(max_norm)) return OSDP_ERR_UNSUPPORTED;
  return norm_of(tensors, n_tensors, grad_dtype, max_norm, out, nullptr, ws, ws_bytes, static_cast<cudaStream_t>(stream));
}

int osdp_grad_squares(const osdp_adamw_tensor *tensors, int n_tensors, int grad_dtype, double *sum, void *ws, size_t ws_bytes,
                      void *stream) {
  return norm_of(tensors, n_tensors, grad_dtype, 0.f, nullptr, sum, ws, ws_bytes, static_cast<cudaStream_t>(stream));
}

int osdp_clip_coefficient(const double *sums, int n_sums, float max_norm, float *out, void *stream) {
  if (n_sums < 0 || n_sums > (1 << 20)) return OSDP_ERR_BAD_SHAPE;
  if (!out || (n_sums > 0 && !sums)) return OSDP_ERR_NULL_POINTER;
  if (std::isnan(max_norm)) return OSDP_ERR_UNSUPPORTED;
  if (!aligned_to(sums, 8) || !aligned_to(out, 4)) return OSDP_ERR_ALIGNMENT;
  return launch_overlapped(clip_kernel, dim3(1), dim3(32), 0, 1, static_cast<cudaStream_t>(stream), sums, n_sums, max_norm, out);
}

int osdp_adamw_step(const osdp_adamw_tensor *tensors, int n_tensors, int param_dtype, int state_dtype, float *master,
                    void *state_m, void *state_v, float *scale_m, float *scale_v, double beta1, double beta2, double eps,
                    int64_t step, const float *clip, void *stream) {
  int rc = check_tensors(tensors, n_tensors, param_dtype, true);
  if (rc) return rc;
  if (state_dtype != OSDP_DTYPE_FP32 && state_dtype != OSDP_DTYPE_E4M3 && state_dtype != OSDP_DTYPE_E4M3_DITHERED) return OSDP_ERR_UNSUPPORTED;
  const bool e4m3 = state_dtype != OSDP_DTYPE_FP32, all = state_dtype == OSDP_DTYPE_E4M3_DITHERED;
  if (step < 1 || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite(eps))
    return OSDP_ERR_UNSUPPORTED;
  int64_t total = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (!std::isfinite(tensors[i].lr) || !std::isfinite(tensors[i].weight_decay)) return OSDP_ERR_UNSUPPORTED;
    total += tensors[i].numel;
  }
  if (total == 0) return OSDP_OK;
  if (!state_m || !state_v || (e4m3 && (!scale_m || !scale_v))) return OSDP_ERR_NULL_POINTER;
  if (!aligned_to(state_m, 32) || !aligned_to(state_v, 32) || !aligned_to(master, 32) || !aligned_to(scale_m, 4) ||
      !aligned_to(scale_v, 4) || !aligned_to(clip, 4))
    return OSDP_ERR_ALIGNMENT;
  if (master && param_dtype != OSDP_DTYPE_BF16) return OSDP_ERR_UNSUPPORTED;   // fp32 parameters are their own master
  Hyper h;
  h.b1 = (float)beta1;
  h.one_minus_b1 = (float)(1.0 - beta1);
  h.b2 = (float)beta2;
  h.one_minus_b2 = (float)(1.0 - beta2);
  h.eps = (float)eps;
  h.one = 1.0f;
  h.seed = (uint32_t)step;
  h.dither_m = all || beta1 > DITHER_ABOVE;
  h.dither_v = all || beta2 > DITHER_ABOVE;
  const States states = !e4m3 ? F32 : h.dither_m || h.dither_v ? DITHERED : CODES;
  h.root_scale = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
  const double b1t = std::pow(beta1, (double)step);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
#define OSDP_STEP(T, MASTER, STATES) \
  pick_table<T, MASTER, STATES>(tensors, n_tensors, param_dtype, h, b1t, master, state_m, state_v, scale_m, scale_v, clip, s)
#define OSDP_STEP_OF(T, MASTER) \
  (states == F32 ? OSDP_STEP(T, MASTER, F32) : states == CODES ? OSDP_STEP(T, MASTER, CODES) : OSDP_STEP(T, MASTER, DITHERED))
  if (param_dtype == OSDP_DTYPE_FP32) return OSDP_STEP_OF(float, false);
  return master ? OSDP_STEP_OF(__nv_bfloat16, true) : OSDP_STEP_OF(__nv_bfloat16, false);
#undef OSDP_STEP_OF
#undef OSDP_STEP
}

}  // extern "C"

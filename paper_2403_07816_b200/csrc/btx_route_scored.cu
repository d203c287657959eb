// Score routing: the choice of k experts from softmax or sigmoid scores of given logits, with a balance bias that
// takes part in the choice only, expert groups, renormalised and scaled weights, tokens per expert; and its
// gradient.  Stands beside the router of btx_routing.cu (Section 3.2), whose gates are softmaxes over at most 64
// experts; the lists it returns feed btx_moe_forward (BTX_ROUTE_GIVEN, up to 64 experts like that layer's own router) and
// btx_mx4_moe_forward (inference, up to 512).
//
//   s_e = softmax(z)_e or sigmoid(z_e)     c_e = s_e + b_e (without a bias: ordered by z itself)
//   group key = best c of the group, or the sum of its two best; the topk_group best groups stay
//   the k largest c of the groups that stay; ties go to the lower index
//   w_j = scale * s_j, or scale * s_j / sum_i s_i over the chosen
//
// 8 to 32 lanes share a row and keep its keys in registers; a round of the selection is one integer maximum over the
// row.  The memory traffic is the logits once, which bounds nothing here: at T = 16384, E = 256, 8 groups, k = 8 (20 us)
// DRAM is at 7 %, 39 % of the warps the multiprocessors could hold are there (70 registers), 55 % of the issue slots are
// used, and a warp waits for the round before: latency of the dependent rounds.  Batches of ordinary logits take 20.2
// to 24.4 us: in every second one a row's groups have to be ranked again in 64 bits, and its block ends later.  A batch
// whose rows are all decided in 64 bits takes 140 us (all logits and biases 0; without groups 77).
#include <math_constants.h>

#include "btx_route_dev.cuh"

namespace btx {
namespace {

using routedev::Vec;

constexpr unsigned kAll = 0xffffffffu;
constexpr int kRsWarps = 8;
constexpr int kMaxScoredExperts = 512;
constexpr int kMaxScoredK = 32;             // lane j keeps slot j
constexpr int kMaxScoredGroups = 32;

struct RouteParams {
  int T, E, k, n_group, group_size, topk_group, lanes_per_group;
  int renorm, single_block;
  float scale;
  long long stride;                         // elements from one row of logits to the next
  const float* bias;
  const uint8_t* row_valid;
  int32_t* topk_idx;
  float* gates;
  float* scores;
  int32_t* counts;
};

// fp32 to integers of the same order, never 0 (0 marks "no candidate"); -0 and +0 are one value
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
// Reductions over the L lanes that share a row (every lane gets the result).
template <int L> __device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int o = 1; o < L; o *= 2) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
// Sum over a row of EPL values per lane as one binary tree over the experts: the result does not depend on how many
// lanes share the row.
template <int L, int EPL> __device__ __forceinline__ float row_sum(float (&v)[EPL]) {
#pragma unroll
  for (int w = 1; w < EPL; w *= 2)
#pragma unroll
    for (int i = 0; i + w < EPL; i += 2 * w) v[i] += v[i + w];
  return row_sum<L>(v[0]);
}
// 16 lanes: a reduction of the whole warp per row is a shorter chain than four exchanges (E = 256, 8 groups, k = 8,
// T = 16384: 20.0 instead of 20.7 us); with 8 lanes four of them are not (E = 64, k = 2: 6.7 and 6.4 us).
template <int L> __device__ __forceinline__ uint32_t row_max(uint32_t v) {
  if constexpr (L == 32) {
    return __reduce_max_sync(kAll, v);
  } else if constexpr (L == 16) {
    const bool upper = (threadIdx.x & 16) != 0;
    const uint32_t a = __reduce_max_sync(kAll, upper ? 0u : v), b = __reduce_max_sync(kAll, upper ? v : 0u);
    return upper ? b : a;
  } else {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(kAll, v, o));
    return v;
  }
}
template <int L> __device__ __forceinline__ float row_max(float v) {
  if constexpr (L == 32) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
  } else {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
    return v;
  }
}
template <int L> __device__ __forceinline__ double row_max(double v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
template <int L> __device__ __forceinline__ bool row_any(bool v, int lane) {
  const uint32_t m = __ballot_sync(kAll, v);
  return L == 32 ? m != 0u : ((m >> (lane & ~(L - 1))) & ((1u << (L & 31)) - 1u)) != 0u;
}
__device__ __forceinline__ float sigmoid_rn(float z) { return 1.0f / (1.0f + expf(-z)); }
// exp(z - m) for z <= m, with exp(0) = 1 where both are +inf
__device__ __forceinline__ float exp_below(float z, float m) { return z == m ? 1.0f : expf(z - m); }

// The lane's EPL logits of one row shared by L lanes (all 32 lanes of the warp call it, each with its row; on = false: no
// candidate).  VEC: rows start on 16-byte boundaries and E is a multiple of a vector; other rows are read with
// neighbouring lanes on neighbouring logits and turned through `st` (EPL * L floats of the row).
template <typename T, int L, int EPL, bool VEC>
__device__ __forceinline__ void load_row(const T* __restrict__ row, int E, int sl, bool on, float* st, float (&z)[EPL]) {
  constexpr int VN = Vec<T>::N;
  const int e0 = sl * EPL;
  if constexpr (VEC && EPL >= VN) {
#pragma unroll
    for (int i = 0; i < EPL; i += VN) {
      float v[VN];
      if (on && e0 + i < E) Vec<T>::load(row + e0 + i, v);
#pragma unroll
      for (int j = 0; j < VN; ++j) z[i + j] = on && e0 + i < E ? v[j] : -CUDART_INF_F;
    }
  } else if constexpr (EPL <= 2) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) z[i] = on && e0 + i < E ? to_f32(row[e0 + i]) : -CUDART_INF_F;
  } else {
    float v[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) v[i] = on && i * L + sl < E ? to_f32(row[i * L + sl]) : -CUDART_INF_F;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < EPL; ++i) st[i * L + sl] = v[i];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < EPL; ++i) z[i] = st[e0 + i];
    __syncwarp();
  }
}

// Two-best merge: (a, b) with a >= b
template <typename F> __device__ __forceinline__ void push2(F v, F& a, F& b) {
  const F low = a < v ? a : v;
  a = a < v ? v : a;
  b = b < low ? low : b;
}
// Group key from its two best members' keys: the best, or the sum; in fp32 half of it, since two finite keys may add up
// past the largest float.  A group without a candidate has -inf, a missing second adds nothing.
template <typename F> __device__ __forceinline__ F group_value(F a, F b, int sum2) {
  const F part = sizeof(F) == 4 ? (F)0.5 : (F)1;
  return !sum2 ? a : b > (F)-CUDART_INF ? part * a + part * b : part * a;
}
// Bound of the magnitudes behind the key of a group with a candidate.
template <typename F> __device__ __forceinline__ F group_size(F a, F b, int sum2) {
  return group_value((F)fabs(a), b > (F)-CUDART_INF ? (F)fabs(b) : b, sum2);
}
// Whether this lane's group g stays: v is its key, the same in the P lanes g * P .. g * P + P - 1 of the row's L, which
// share the comparisons with the G groups; `size` bounds the magnitudes behind v.  `margin` receives the difference
// between the worst group that stays and the best that does not, `reach` the largest size (for the caller's error
// bound).
template <int L, typename F>
__device__ __forceinline__ bool rank_groups(F v, F size, int g, int G, int P, int lane, int topk_group, F& margin, F& reach) {
  const F low = (F)-CUDART_INF;
  int rank = 0;
  for (int q0 = 0; q0 < G; q0 += P) {
    const int q = q0 + (lane & (P - 1));
    const F o = __shfl_sync(kAll, v, (q * P) & (L - 1), L);
    rank += q < G && (o > v || (o == v && q < g));
  }
  for (int o = 1; o < P; o <<= 1) rank += __shfl_xor_sync(kAll, rank, o);
  const bool stays = g < G && rank < topk_group;
  const F worst = -row_max<L>(stays ? -v : low), best = row_max<L>(g < G && !stays ? v : low);
  reach = row_max<L>(g < G && v > low ? size : (F)0);
  margin = best > low ? worst - best : (F)CUDART_INF;
  return stays;
}

// The groups that stay, as a bit mask, from the row's keys in shared memory (expert e at e + (e / size) * P, so that the
// lanes of different groups read different banks); P lanes share a group.
template <int L, typename F>
__device__ __forceinline__ uint32_t choose_groups(const F* key, int G, int size, int P, int topk_group, int sum2, int lane,
                                                  F& margin, F& reach) {
  const F low = (F)-CUDART_INF;
  const int sl = lane & (L - 1), g = sl / P, p = sl - g * P;
  F a = low, b = low;
  if (g < G)
    for (int j = p; j < size; j += P) push2(key[g * (size + P) + j], a, b);
  for (int o = 1; o < P; o <<= 1) {
    const F oa = __shfl_xor_sync(kAll, a, o), ob = __shfl_xor_sync(kAll, b, o);
    push2(oa, a, b);
    push2(ob, a, b);
  }
  const F v = g < G ? group_value(a, b, sum2) : low;
  const bool stays = rank_groups<L, F>(v, group_size(a, b, sum2), g, G, P, lane, topk_group, margin, reach);
  const uint32_t lanes = __ballot_sync(kAll, stays && p == 0) >> (lane & ~(L - 1));
  uint32_t mask = 0;
  for (int q = 0; q < G; ++q) mask |= ((lanes >> (q * P)) & 1u) << q;
  return mask;
}

// f(i, group of expert i of the lane) for the lane's EPL experts, the first being member r0 of group g0.
template <int EPL, typename F> __device__ __forceinline__ void for_each_group(int g0, int r0, int size, F&& f) {
  int g = g0, r = r0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    f(i, g);
    if (++r == size) { r = 0; ++g; }
  }
}

// The choice with 64-bit scores, for the few rows whose order 32 bits do not settle, by the whole warp.  `keys`: E + 32
// doubles of the warp's shared memory, expert e at e + (e / group_size) * P.
struct RowScore {                           // exact scores of one row
  double zmax, total;
  template <bool SIGMOID> __device__ __forceinline__ double of(double z) const {
    return SIGMOID ? 1.0 / (1.0 + exp(-z)) : (z == zmax ? 1.0 : exp(z - zmax)) / total;
  }
};
template <typename T, bool SIGMOID>
__device__ __forceinline__ RowScore row_score(const T* __restrict__ row, int E, int lane) {
  const double low = -CUDART_INF;
  RowScore s = {low, 0.0};
  if (!SIGMOID) {
    for (int e = lane; e < E; e += 32) {
      const double z = (double)to_f32(row[e]);
      if (z > s.zmax) s.zmax = z;
    }
    s.zmax = row_max<32>(s.zmax);
    for (int e = lane; e < E; e += 32) {
      const double z = (double)to_f32(row[e]);
      if (z > low) s.total += z == s.zmax ? 1.0 : exp(z - s.zmax);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s.total += __shfl_xor_sync(kAll, s.total, o);
  }
  return s;
}
// lanes of the whole warp that share a group
__device__ __forceinline__ int warp_lanes_per_group(const RouteParams& p) {
  int P = 1;
  while (2 * P * p.n_group <= 32) P *= 2;
  return P;
}

// The groups that stay.
template <typename T, bool SIGMOID>
__device__ __noinline__ uint32_t groups_in_double(const T* __restrict__ row, const RouteParams& p, int sum2, double* keys, int lane) {
  const int P = warp_lanes_per_group(p);
  const double low = -CUDART_INF;
  const RowScore s = row_score<T, SIGMOID>(row, p.E, lane);
  for (int e = lane; e < p.E; e += 32) {
    const double z = (double)to_f32(row[e]);
    double c = low;
    if (z > low) c = p.bias ? s.of<SIGMOID>(z) + (double)p.bias[e] : sum2 ? s.of<SIGMOID>(z) : z;
    keys[e + e / p.group_size * P] = c > low ? c : low;
  }
  __syncwarp();
  double margin, reach;
  const uint32_t stay = choose_groups<32, double>(keys, p.n_group, p.group_size, P, p.topk_group, sum2, lane, margin, reach);
  __syncwarp();
  return stay;
}

// The expert of slot `lane` (-1: none).
template <typename T, bool SIGMOID>
__device__ __noinline__ int choose_in_double(const T* __restrict__ row, const RouteParams& p, int sum2, double* keys, int lane) {
  const double low = -CUDART_INF;
  const uint32_t stay = p.n_group > 1 ? groups_in_double<T, SIGMOID>(row, p, sum2, keys, lane) : kAll;
  const RowScore s = row_score<T, SIGMOID>(row, p.E, lane);
  for (int e = lane; e < p.E; e += 32) {
    const double z = (double)to_f32(row[e]);
    double c = low;
    if (z > low && ((stay >> (p.n_group > 1 ? e / p.group_size : 0)) & 1u)) c = p.bias ? s.of<SIGMOID>(z) + (double)p.bias[e] : z;
    keys[e] = c > low ? c : low;
  }
  __syncwarp();
  int mine = -1;
  for (int j = 0; j < p.k; ++j) {
    double bv = low;
    int bi = -1;
    for (int e = lane; e < p.E; e += 32)
      if (keys[e] > bv) { bv = keys[e]; bi = e; }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const double ov = __shfl_xor_sync(kAll, bv, o);
      const int oi = __shfl_xor_sync(kAll, bi, o);
      if (oi >= 0 && (bi < 0 || ov > bv || (ov == bv && oi < bi))) { bv = ov; bi = oi; }
    }
    if (bi < 0) break;
    if (lane == j) mine = bi;
    if (lane == 0) keys[bi] = low;
    __syncwarp();
  }
  return mine;
}

// Scores for the choice, from the approximate base-2 exponential and reciprocal of the hardware; the weights and the
// `scores` output are formed again to full accuracy.  Errors (exp(x) as 2^(x log2 e): within 2 + 1.173 |x| ulp, the
// reciprocal within 1; flushed subnormals are far below 2^-23):
//   sigmoid  s (1 - s) (2 + 1.173 |z|) 2^-23 + 4 * 2^-24 s <= 2^-22 s + 2^-23
//   softmax  each exponential carries the rounded difference x = max - z as well, (2 + 1.7 x) 2^-23; s x < 0.4, the
//            mean of x under s is below 7 for E <= 512, the sum rounds 21 times: below 2^-18 s + 2^-23
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float sigmoid_key(float z) { return rcp_fast(1.0f + exp2_fast(-kLog2e * z)); }

// L lanes share a row, EPL experts each: 32 / L rows per warp share the instructions of a round.
// Warps per block: every block adds its counts to E addresses, so few large blocks.  14 for 256 experts: with 12 the
// registers allow more per thread, but T = 16384 takes a third pass over the grid (24.8 instead of 21.4 us); 16 spill.
template <int E> struct RouteWarps { static constexpr int n = E <= 128 ? 16 : E <= 256 ? 14 : 8, per_sm = E <= 256 ? 2 : 3; };

template <typename T, int L, int EPL, bool SIGMOID, bool VEC>
__global__ void __launch_bounds__(RouteWarps<L * EPL>::n * 32, RouteWarps<L * EPL>::per_sm)
route_scored_kernel(const T* __restrict__ logits, const RouteParams p, int sum2) {
  constexpr int ROWS = 32 / L, W = RouteWarps<L * EPL>::n;
  constexpr int KEYS = EPL * L + 32;
  // per warp: 32-bit keys of its rows for the groups, or 64-bit keys of a row that is decided again (never both at once)
  __shared__ double keys_s[W][ROWS * KEYS / 2 > KEYS ? ROWS * KEYS / 2 : KEYS];
  __shared__ float bias_s[EPL * L];
  __shared__ int hist[EPL * L];
  // A packed key is the ordered key with its lowest bits replaced by the index, larger for lower experts: one maximum
  // over the row finds the next expert, its place and the lower index of a tie.
  constexpr uint32_t IDX = EPL * L - 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sl = lane & (L - 1), seg0 = lane & ~(L - 1);
  const bool grouped = p.n_group > 1, biased = p.bias != nullptr;
  const int e0 = sl * EPL;
  const float low = -CUDART_INF_F;
  for (int i = threadIdx.x; i < EPL * L; i += W * 32) hist[i] = 0;
  allow_dependents();
  grid_dependency_wait();
  if (biased)
    for (int i = threadIdx.x; i < EPL * L; i += W * 32) bias_s[i] = i < p.E ? p.bias[i] : 0.f;
  __syncthreads();
  const float err_s = SIGMOID ? 0x1p-22f : 0x1p-18f, err_0 = 0x1p-23f, err_c = 0x1p-24f;
  const bool need_total = !SIGMOID && (p.scores != nullptr || biased || (grouped && sum2) || !p.renorm);
  const bool exact_keys = !biased && sizeof(T) == 2;               // 16-bit logits keep every bit in a packed key
  // groups of whole lanes (a power of two of them) are compared in registers, others through shared memory
  const int lanes_per = p.group_size / EPL;
  const bool by_lanes = grouped && lanes_per * EPL == p.group_size && (lanes_per & (lanes_per - 1)) == 0;
  int half_k = 1;                           // reductions over the chosen: lanes 0 .. 2 * half_k - 1 cover k
  while (2 * half_k < p.k) half_k *= 2;

  for (int t0 = (blockIdx.x * W + warp) * ROWS; t0 < p.T; t0 += gridDim.x * W * ROWS) {
    const int t = t0 + lane / L;
    const bool there = t < p.T, on = there && (p.row_valid == nullptr || p.row_valid[t] != 0);
    const T* row = logits + (long long)(there ? t : t0) * p.stride;
    float* row_s = reinterpret_cast<float*>(keys_s[warp]) + lane / L * KEYS;
    float z[EPL];                                                  // a row that is off has no candidate
    load_row<T, L, EPL, VEC>(row, p.E, sl, on, row_s, z);
    float total = 1.f, zmax = 0.f;
    if (need_total) {
      float m = low;
#pragma unroll
      for (int i = 0; i < EPL; ++i) m = fmaxf(m, z[i]);            // (fmaxf passes over NaN)
      zmax = row_max<L>(m);
      float ex[EPL];
#pragma unroll
      for (int i = 0; i < EPL; ++i) ex[i] = z[i] > low ? exp_below(z[i], zmax) : 0.f;
      total = row_sum<L, EPL>(ex);
      if (!(total > 0.f)) total = 1.f;                             // nothing is on
    }
    const float inv_total = 1.0f / total;
    auto score_key = [&](float v) {                                // v > -inf
      if (SIGMOID) return sigmoid_key(v);
      return (v == zmax ? 1.0f : exp2_fast((v - zmax) * kLog2e)) * inv_total;
    };
    if (p.scores != nullptr && there) {
#pragma unroll
      for (int i = 0; i < EPL; ++i)
        if (e0 + i < p.E)
          p.scores[(size_t)t * p.E + e0 + i] = !(z[i] > low) ? 0.f : SIGMOID ? sigmoid_rn(z[i]) : exp_below(z[i], zmax) / total;
    }
    float c[EPL];                                                  // -inf: not a candidate
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      c[i] = biased ? score_key(z[i]) + bias_s[e0 + i] : z[i];
      if (!(z[i] > low && c[i] > low)) c[i] = low;
    }
    const float smax = SIGMOID ? 1.0f : inv_total;                 // no score is larger
    if (grouped) {
      float margin, reach;
      uint32_t stay = 0;
      // The groups of the rows whose choice is within its error, in 64 bits (a few rows of a batch, but one of them holds up
      // its block: deciding all of such a row in 64 bits took 12 us); other rows keep `as_is`.  Keys compared as they stand
      // (logits) are exact.  A key's error is that of one member, or half that of two: err_s, err_0 and its roundings.
      auto redo_groups = [&](float margin_, float reach_, uint32_t as_is) {
        const float error = 2.f * (err_s * smax + err_0) + 6.f * err_c * reach_;
        for (uint32_t rows = __ballot_sync(kAll, (biased || sum2) && sl == 0 && margin_ <= error); rows != 0u; rows &= rows - 1u) {
          const int src = __ffs(rows) - 1;
          __syncwarp();
          const uint32_t exact = groups_in_double<T, SIGMOID>(logits + (long long)(t0 + src / L) * p.stride, p, sum2, keys_s[warp], lane);
          if (seg0 == src) as_is = exact;
          __syncwarp();
        }
        return as_is;
      };
      if (by_lanes) {
        float a = low, b = low;
#pragma unroll
        for (int i = 0; i < EPL; ++i) push2(c[i], a, b);
        for (int o = 1; o < lanes_per; o <<= 1) {
          const float oa = __shfl_xor_sync(kAll, a, o), ob = __shfl_xor_sync(kAll, b, o);
          push2(oa, a, b);
          push2(ob, a, b);
        }
        if (!biased && sum2) {                                     // the best logits have the best scores
          a = a > low ? score_key(a) : low;
          b = b > low ? score_key(b) : low;
        }
        bool stays = rank_groups<L, float>(group_value(a, b, sum2), group_size(a, b, sum2), sl / lanes_per, p.n_group,
                                           lanes_per, lane, p.topk_group, margin, reach);
        stay = redo_groups(margin, reach, 0u);
        if (stay != 0u) stays = (stay >> (sl / lanes_per)) & 1u;
        if (!stays) {
#pragma unroll
          for (int i = 0; i < EPL; ++i) c[i] = low;
        }
      } else {
        const int P = p.lanes_per_group;
        const int g_first = e0 / p.group_size, r_first = e0 - g_first * p.group_size;
        __syncwarp();
        for_each_group<EPL>(g_first, r_first, p.group_size, [&](int i, int g) {
          if (e0 + i < p.E) row_s[e0 + i + g * P] = !biased && sum2 && c[i] > low ? score_key(z[i]) : c[i];
        });
        __syncwarp();
        stay = choose_groups<L, float>(row_s, p.n_group, p.group_size, P, p.topk_group, sum2, lane, margin, reach);
        stay = redo_groups(margin, reach, stay);
        for_each_group<EPL>(g_first, r_first, p.group_size, [&](int i, int g) {
          if (!((stay >> (g & 31)) & 1u)) c[i] = low;              // (past the last expert there is no candidate anyway)
        });
      }
    }
    // k rounds: the largest packed key of the row goes to the next slot.  A lane holds its three best (0: none) and looks
    // through its experts again when all are taken.
    uint32_t u[EPL], best0 = 0, best1 = 0, best2 = 0;
    auto push3 = [&](uint32_t v) {
      const uint32_t d0 = min(best0, v);
      best0 = max(best0, v);
      const uint32_t d1 = min(best1, d0);
      best1 = max(best1, d0);
      best2 = max(best2, d1);
    };
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      u[i] = c[i] > low ? (order_key(c[i]) & ~IDX) | (IDX - (uint32_t)(e0 + i)) : 0u;
      push3(u[i]);
    }
    uint32_t mine = 0;                                             // key of slot `sl`
    int n = 0;                                                     // slots taken (of this lane's row)
    uint32_t next = row_max<L>(best0);
    auto pick = [&](bool take) {                                   // `take`: the same in all lanes of a row
      if (take) {
        if (sl == n) mine = next;
        ++n;
        if (best0 == next) {
          best0 = best1; best1 = best2; best2 = 0;
          if (best0 == 0u) {
#pragma unroll
            for (int i = 0; i < EPL; ++i) push3(u[i] < next ? u[i] : 0u);
          }
        }
      }
      __syncwarp();
      next = row_max<L>(best0);
    };
    for (int j = 0; j < p.k; ++j) pick(next != 0u);
    bool unsure = false;                                           // not settled in registers
    if (!exact_keys) {
      // Neighbours that lie within what a packed key leaves out and the error of the keys: take what else lies as close,
      // and order all of it in 64 bits.  The bound holds for every key from the first to the one compared.
      const uint32_t first = __shfl_sync(kAll, mine, 0, L);
      const float c0 = fabsf(order_value(first & ~IDX));
      const float fixed = biased ? 2.f * (err_s * smax + err_0) : 0.f, rel = biased ? 2.f * err_c : 0.f;
      auto close = [&](uint32_t hi, uint32_t lo) {
        const float l = order_value(lo | IDX);
        return !(order_value(hi & ~IDX) - l > fixed + rel * 1.01f * fmaxf(c0, fabsf(l)));
      };
      const uint32_t after = __shfl_down_sync(kAll, mine, 1, L);
      uint32_t last = __shfl_sync(kAll, mine, n > 0 ? n - 1 : 0, L);
      const bool tail = n > 0 && next != 0u && close(last, next);
      const bool near = row_any<L>(sl + 1 < n && close(mine, after), lane);     // (a vote of the whole warp: never behind a condition of a row)
      const bool redo = near || tail;
      if (__any_sync(kAll, redo)) {
        for (;;) {
          const bool more = redo && n < L && next != 0u && close(last, next);
          if (!__any_sync(kAll, more)) break;
          if (more) last = next;
          pick(more);
        }
        if (redo && next != 0u && close(last, next)) unsure = true;
        const double top = (double)zmax;
        double sum = 1.0;
        if (!SIGMOID && biased) {
          sum = 0.0;
#pragma unroll
          for (int i = 0; i < EPL; ++i)
            if (z[i] > low) sum += z[i] == zmax ? 1.0 : exp((double)z[i] - top);
#pragma unroll
          for (int o = L / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
        }
        const int e = (int)(IDX - (mine & IDX));
        double cd = 0.0;
        if (redo && sl < n) {
          const float zf = to_f32(row[e]);
          cd = (double)zf;
          if (biased) cd = (SIGMOID ? 1.0 / (1.0 + exp(-cd)) : (zf == zmax ? 1.0 : exp(cd - top)) / sum) + (double)p.bias[e];
        }
        int rank = 0;
        const int longest = __reduce_max_sync(kAll, n);
        for (int j = 0; j < longest; ++j) {
          const double oc = __shfl_sync(kAll, cd, j, L);
          const int oe = __shfl_sync(kAll, e, j, L);
          rank += j < n && (oc > cd || (oc == cd && oe < e));
        }
        uint32_t* order = reinterpret_cast<uint32_t*>(keys_s[warp]) + seg0;
        __syncwarp();
        if (redo && sl < n) order[rank] = mine;
        __syncwarp();
        if (redo && sl < n) mine = order[sl];
        __syncwarp();
      }
    }
    int sel = sl < n && sl < p.k ? (int)(IDX - (mine & IDX)) : -1;  // lane j of a row: the expert of slot j
    for (uint32_t rows = __ballot_sync(kAll, unsure && sl == 0); rows != 0u; rows &= rows - 1u) {
      const int src = __ffs(rows) - 1;                             // the whole warp decides the row again
      __syncwarp();
      const int got = choose_in_double<T, SIGMOID>(logits + (long long)(t0 + src / L) * p.stride, p, sum2, keys_s[warp], lane);
      const int mine_now = __shfl_sync(kAll, got, sl);
      if (seg0 == src) sel = sl < p.k ? mine_now : -1;
      __syncwarp();
    }
    // Weights: lane j has slot j.  Renormalised weights are formed from exponentials shifted by the largest chosen logit
    // where their sum could underflow, so they are a number even where every score is 0.
    const bool have = sel >= 0;
    const float zs = have ? to_f32(row[sel]) : low;
    float w = 0.f;
    if (p.renorm) {
      const bool large = row_any<L>(zs > -10.f, lane);
      const bool shift = !SIGMOID || __any_sync(kAll, !large);      // the same in the whole warp
      const float m = shift ? row_max<L>(zs) : 0.f;
      if (have) w = !SIGMOID ? exp_below(zs, m) : m > -10.f ? sigmoid_rn(zs) : expf(zs - m) / (1.0f + expf(zs));
      float sum = w;
      for (int o = half_k; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
      if (have) w = w / sum * p.scale;
    } else if (have) {
      w = (SIGMOID ? sigmoid_rn(zs) : exp_below(zs, zmax) / total) * p.scale;
    }
    if (there && sl < p.k) {
      p.topk_idx[(size_t)t * p.k + sl] = sel;
      p.gates[(size_t)t * p.k + sl] = w;
      if (have && p.counts != nullptr) atomicAdd(&hist[sel], 1);
    }
  }
  if (p.counts != nullptr) {
    __syncthreads();
    for (int i = threadIdx.x; i < p.E; i += blockDim.x) {
      if (p.single_block) p.counts[i] = hist[i];
      else if (hist[i] != 0) atomicAdd(p.counts + i, hist[i]);      // integers: any order gives the same counts
    }
  }
}

// Gradient with respect to the logits.  Chosen slots: with renormalised weights w_j = scale p_j and
// t_j = dw_j - sum_i p_i dw_i, softmax dz_j = scale p_j t_j and sigmoid dz_j = scale p_j (1 - s_j) t_j; without,
// sigmoid dz_j = scale dw_j s_j (1 - s_j); all other logits zero.  Softmax without renormalisation reaches every
// logit: dz_e = s_e (scale dw_e [e chosen] - scale sum_j dw_j s_j).  T = 16384, E = 256, k = 8, fp32: 7.8 us where
// every logit has a gradient, 4.5 to 6.3 us where the chosen ones have; bound by the latency of a row's index loads, gather
// and chained reductions (57 to 62 % of the issue slots, DRAM at 15 %), with one row in flight per warp.
// A warp per row.  Neighbouring lanes hold neighbouring experts, by the vector (VEC: rows start on 16-byte boundaries and
// hold whole vectors) or one by one, so that every load and store of the warp is contiguous: 8 experts in a row per lane,
// as in the choice above, took 9.0 instead of 7.8 us for T = 16384, E = 256, k = 8 (softmax, not renormalised).
template <typename T, int EPL, bool SIGMOID, bool VEC>
__global__ void __launch_bounds__(kRsWarps * 32)
route_scored_backward_kernel(int Tn, int E, int k, int renorm, float scale, long long stride,
                             const T* __restrict__ logits, const int32_t* __restrict__ topk_idx,
                             const float* __restrict__ dgates, T* __restrict__ dlogits, long long out_stride) {
  constexpr int VN = VEC && EPL >= Vec<T>::N ? Vec<T>::N : 1;        // experts side by side in a lane
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float low = -CUDART_INF_F;
  __shared__ __align__(16) float add_s[kRsWarps][EPL * 32];
#pragma unroll
  for (int i = 0; i < EPL; ++i) add_s[warp][i * 32 + lane] = 0.f;
  __syncwarp();
  allow_dependents();
  grid_dependency_wait();
  for (int t = blockIdx.x * kRsWarps + warp; t < Tn; t += gridDim.x * kRsWarps) {
    const T* row = logits + (long long)t * stride;
    int sel = -1;
    float dw = 0.f;
    if (lane < k) {
      sel = topk_idx[(size_t)t * k + lane];
      if (sel < 0 || sel >= E) sel = -1;
      else dw = dgates[(size_t)t * k + lane];
    }
    const bool have = sel >= 0;
    const float zs = have ? to_f32(row[sel]) : low;
    float dz[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) dz[i] = 0.f;
    float v = 0.f;
    if (renorm) {
      const float m = row_max<32>(zs);
      float pj = 0.f;
      if (SIGMOID) {
        if (have) pj = zs > 0.f ? sigmoid_rn(zs) : expf(zs - fminf(m, 0.f)) / (1.0f + expf(zs));
      } else if (have) {
        pj = exp_below(zs, m);
      }
      const float sum = row_sum<32>(pj);
      if (have) pj /= sum;
      const float inner = row_sum<32>(pj * dw);
      if (have) v = scale * pj * (dw - inner);
      if (SIGMOID && have) v *= 1.0f / (1.0f + expf(zs));            // 1 - s without cancellation
    } else if (SIGMOID) {
      if (have) v = scale * dw * sigmoid_rn(zs) * (1.0f / (1.0f + expf(zs)));
    } else {
      float z[EPL], m = low;
#pragma unroll
      for (int i = 0; i < EPL; i += VN) {
        const int e = i * 32 + lane * VN;
        float q[VN];
        if constexpr (VN > 1) {
          if (e < E) Vec<T>::load(row + e, q);
        } else {
          if (e < E) q[0] = to_f32(row[e]);
        }
#pragma unroll
        for (int j = 0; j < VN; ++j) {
          z[i + j] = e < E ? fmaxf(q[j], low) : low;                 // NaN: no candidate
          m = fmaxf(m, z[i + j]);
        }
      }
      m = row_max<32>(m);
      const float shift = fabsf(m) < CUDART_INF_F ? m : 0.f;         // (-inf: nothing is on)
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        dz[i] = m < CUDART_INF_F ? expf(z[i] - shift) : z[i] == m ? 1.f : 0.f;
        sum += dz[i];
      }
      sum = row_sum<32>(sum);
      const float s = have && sum > 0.f ? exp_below(zs, m) / sum : 0.f;
      const float inner = row_sum<32>(s * dw);
      const float factor = sum > 0.f ? -scale * inner / sum : 0.f;
#pragma unroll
      for (int i = 0; i < EPL; ++i) dz[i] *= factor;
      v = scale * s * dw;
    }
    // the chosen slots' values reach the lanes that own their experts through shared memory; an expert named in
    // several slots gets their sum, in slot order
    const unsigned same = __match_any_sync(kAll, sel);
    if (__any_sync(kAll, have && __popc(same) > 1)) {
      float acc = 0.f;
      for (int j = 0; j < k; ++j) {
        const float vj = __shfl_sync(kAll, v, j);
        if ((same >> j) & 1u) acc += vj;
      }
      v = acc;
    }
    if (have) add_s[warp][sel] = v;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < EPL; ++i) dz[i] += add_s[warp][i / VN * VN * 32 + lane * VN + i % VN];
    __syncwarp();
    if (have) add_s[warp][sel] = 0.f;
    __syncwarp();
    T* out = dlogits + (long long)t * out_stride;
#pragma unroll
    for (int i = 0; i < EPL; i += VN) {
      const int e = i * 32 + lane * VN;
      if (e >= E) continue;
      if constexpr (VN > 1) {
        __align__(16) T q[VN];
#pragma unroll
        for (int j = 0; j < VN; ++j) q[j] = from_f32<T>(dz[i + j]);
        *reinterpret_cast<uint4*>(out + e) = *reinterpret_cast<const uint4*>(q);
      } else {
        out[e] = from_f32<T>(dz[i]);
      }
    }
  }
}

btx_status check_route_desc(const btx_route_desc* d) {
  if (!d) return BTX_ERR_INVALID_ARG;
  if (d->T < 0 || d->E < 1 || d->k < 1 || d->n_group < 1 || d->topk_group < 1) return BTX_ERR_INVALID_ARG;
  if (d->dtype != BTX_F32 && d->dtype != BTX_BF16) return BTX_ERR_INVALID_ARG;
  if (d->score != BTX_SCORE_SOFTMAX && d->score != BTX_SCORE_SIGMOID) return BTX_ERR_INVALID_ARG;
  if (d->group_score != BTX_GROUP_MAX && d->group_score != BTX_GROUP_SUM2) return BTX_ERR_INVALID_ARG;
  if (d->E % d->n_group != 0 || d->topk_group > d->n_group) return BTX_ERR_INVALID_ARG;
  if ((long long)d->k > (long long)(d->E / d->n_group) * d->topk_group) return BTX_ERR_INVALID_ARG;
  if (!(d->scale > 0.f && d->scale <= 3.402823466e38f)) return BTX_ERR_INVALID_ARG;
  if (d->E > kMaxScoredExperts || d->k > kMaxScoredK || d->n_group > kMaxScoredGroups) return BTX_ERR_UNSUPPORTED;
  if ((long long)d->T * d->k > (1ll << 28)) return BTX_ERR_UNSUPPORTED;
  return BTX_OK;
}

// rows that start on 16-byte boundaries and hold whole vectors
bool row_vectors(const void* base, long long stride, int E, int esize) {
  return ((uintptr_t)base & 15) == 0 && stride * esize % 16 == 0 && E * esize % 16 == 0;
}

int row_blocks(int T, int warps, int per_sm) {
  const int want = (T + warps - 1) / warps, most = per_sm * sm_count();
  return want < most ? want : most;
}

// A kernel, not a copy-engine memset: the kernel behind it can start as its dependent.
__global__ void zero_counts_kernel(int E, int32_t* __restrict__ counts) {
  allow_dependents();
  grid_dependency_wait();
  for (int i = threadIdx.x; i < E; i += blockDim.x) counts[i] = 0;
}

template <typename T, int L, int EPL>
cudaError_t launch_route_t(const btx_route_desc* d, const void* logits, RouteParams p, cudaStream_t st) {
  constexpr int W = RouteWarps<L * EPL>::n;
  int blocks = row_blocks(p.T, W * (32 / L), RouteWarps<L * EPL>::per_sm);
  // Counting: one block writes its own counts; more add theirs to zeros.  One block takes up to 16 rows on its own, which
  // costs less than a second launch to clear the counts.
  p.single_block = p.counts != nullptr && p.T <= 16;
  if (p.single_block) blocks = 1;
  else if (p.counts != nullptr) {
    cudaError_t e = launch_after_predecessor(zero_counts_kernel, dim3(1), dim3(256), 0, st, true, p.E, p.counts);
    if (e != cudaSuccess) return e;
  }
  p.lanes_per_group = 1;
  while (2 * p.lanes_per_group * p.n_group <= L) p.lanes_per_group *= 2;
  const int sum2 = d->group_score == BTX_GROUP_SUM2;
  auto kernel = route_scored_kernel<T, L, EPL, false, false>;
  const bool sigmoid = d->score == BTX_SCORE_SIGMOID;
  if (row_vectors(logits, p.stride, p.E, sizeof(T)))
    kernel = sigmoid ? route_scored_kernel<T, L, EPL, true, true> : route_scored_kernel<T, L, EPL, false, true>;
  else if (sigmoid)
    kernel = route_scored_kernel<T, L, EPL, true, false>;
  return launch_after_predecessor(kernel, dim3(blocks), dim3(W * 32), 0, st, true, (const T*)logits, p, sum2);
}

// Lanes of a row: enough for E experts at up to 16 each, for the k slots (one per lane) and for the groups.  Fewer lanes
// per row mean more rows per warp instruction and a longer way through a row, so large batches take them and others get a
// warp per row: E = 256, 8 of 8 groups, k = 8 takes 20.0 us with 16 lanes and 23.8 with 32 at T = 16384, 10.2 and 9.5 at
// T = 4096, 8.0 and 5.3 at T = 512; E = 64, k = 2, softmax, T = 16384: 6.6 us with 8 lanes, 12.4 with 32.
template <typename T>
cudaError_t launch_route(const btx_route_desc* d, const void* logits, const RouteParams& p, cudaStream_t st) {
  const int need = p.k > p.n_group ? p.k : p.n_group;
  if (p.T > 8192) {
    if (p.E <= 32 && need <= 8) return launch_route_t<T, 8, 4>(d, logits, p, st);
    if (p.E <= 64 && need <= 8) return launch_route_t<T, 8, 8>(d, logits, p, st);
    if (p.E <= 128 && need <= 16) return launch_route_t<T, 16, 8>(d, logits, p, st);
    if (p.E <= 256 && need <= 16) return launch_route_t<T, 16, 16>(d, logits, p, st);
  }
  if (p.E <= 64) return launch_route_t<T, 32, 2>(d, logits, p, st);
  if (p.E <= 256) return launch_route_t<T, 32, 8>(d, logits, p, st);
  return launch_route_t<T, 32, 16>(d, logits, p, st);
}

template <typename T, int EPL>
cudaError_t launch_backward_t(const btx_route_desc* d, const void* logits, long long stride, const int32_t* topk_idx,
                              const float* dgates, void* dlogits, long long out_stride, cudaStream_t st) {
  auto kernel = route_scored_backward_kernel<T, EPL, false, false>;
  const bool sigmoid = d->score == BTX_SCORE_SIGMOID;
  if (row_vectors(logits, stride, d->E, sizeof(T)) && row_vectors(dlogits, out_stride, d->E, sizeof(T)))
    kernel = sigmoid ? route_scored_backward_kernel<T, EPL, true, true> : route_scored_backward_kernel<T, EPL, false, true>;
  else if (sigmoid)
    kernel = route_scored_backward_kernel<T, EPL, true, false>;
  return launch_after_predecessor(kernel, dim3(row_blocks(d->T, kRsWarps, 16)), dim3(kRsWarps * 32), 0, st, true, d->T, d->E, d->k,
                                  (int)(d->renorm != 0), d->scale, stride, (const T*)logits, topk_idx, dgates, (T*)dlogits, out_stride);
}

// experts per lane: the power of two that covers E with 32 lanes
template <typename T, typename... Args>
cudaError_t launch_backward(const btx_route_desc* d, Args... args) {
  if (d->E <= 32) return launch_backward_t<T, 1>(d, args...);
  if (d->E <= 64) return launch_backward_t<T, 2>(d, args...);
  if (d->E <= 128) return launch_backward_t<T, 4>(d, args...);
  if (d->E <= 256) return launch_backward_t<T, 8>(d, args...);
  return launch_backward_t<T, 16>(d, args...);
}

}  // namespace
}  // namespace btx

using namespace btx;

extern "C" btx_status btx_route(const btx_route_desc* desc, const void* logits, int64_t logits_stride, const float* bias,
                                const uint8_t* row_valid, int32_t* topk_idx, float* gates, float* scores,
                                int32_t* counts, void* stream) {
  btx_status s = check_route_desc(desc);
  if (s != BTX_OK) return s;
  if (desc->T == 0 && counts == nullptr) return BTX_OK;
  if (desc->T > 0 && (!logits || !topk_idx || !gates)) return BTX_ERR_INVALID_ARG;
  const int esize = desc->dtype == BTX_BF16 ? 2 : 4;
  if (desc->T > 1 && logits_stride < desc->E) return BTX_ERR_INVALID_ARG;
  if (((uintptr_t)logits & (esize - 1)) || (((uintptr_t)topk_idx | (uintptr_t)gates | (uintptr_t)scores | (uintptr_t)counts |
                                             (uintptr_t)bias) & 3))
    return BTX_ERR_INVALID_ARG;
  if ((s = check_device()) != BTX_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  if (desc->T == 0)
    return cudaMemsetAsync(counts, 0, (size_t)desc->E * sizeof(int32_t), st) == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
  RouteParams p = {};
  p.T = desc->T; p.E = desc->E; p.k = desc->k; p.n_group = desc->n_group; p.group_size = desc->E / desc->n_group;
  p.topk_group = desc->topk_group; p.renorm = desc->renorm != 0; p.scale = desc->scale; p.stride = logits_stride;
  p.bias = bias; p.row_valid = row_valid; p.topk_idx = topk_idx; p.gates = gates; p.scores = scores; p.counts = counts;
  if (p.topk_group == p.n_group) p.n_group = 1;                // every group stays: nothing to choose
  const cudaError_t e = desc->dtype == BTX_BF16 ? launch_route<__nv_bfloat16>(desc, logits, p, st) : launch_route<float>(desc, logits, p, st);
  return e == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

extern "C" btx_status btx_route_backward(const btx_route_desc* desc, const void* logits, int64_t logits_stride,
                                         const int32_t* topk_idx, const float* dgates, void* dlogits,
                                         int64_t dlogits_stride, void* stream) {
  btx_status s = check_route_desc(desc);
  if (s != BTX_OK) return s;
  if (desc->T == 0) return BTX_OK;
  if (!logits || !topk_idx || !dgates || !dlogits) return BTX_ERR_INVALID_ARG;
  if (desc->T > 1 && (logits_stride < desc->E || dlogits_stride < desc->E)) return BTX_ERR_INVALID_ARG;
  const int esize = desc->dtype == BTX_BF16 ? 2 : 4;
  if ((((uintptr_t)logits | (uintptr_t)dlogits) & (esize - 1)) || (((uintptr_t)topk_idx | (uintptr_t)dgates) & 3))
    return BTX_ERR_INVALID_ARG;
  if ((s = check_device()) != BTX_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = desc->dtype == BTX_BF16
      ? launch_backward<__nv_bfloat16>(desc, logits, logits_stride, topk_idx, dgates, dlogits, dlogits_stride, st)
      : launch_backward<float>(desc, logits, logits_stride, topk_idx, dgates, dlogits, dlogits_stride, st);
  return e == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

// Score routing: the choice of k experts from softmax or sigmoid scores of given logits, with a balance bias that
// takes part in the choice only, expert groups, renormalised and scaled weights, tokens per expert; and its
// gradient.  Stands beside the router of btx_routing.cu (Section 3.2), whose gates are softmaxes over at most 64
// experts; the lists it returns feed btx_moe_forward (BTX_ROUTE_GIVEN) and btx_mx4_moe_forward.
//
//   s_e = softmax(z)_e or sigmoid(z_e)     c_e = s_e + b_e (without a bias: ordered by z itself)
//   group key = best c of the group, or the sum of its two best; the topk_group best groups stay
//   the k largest c of the groups that stay; ties go to the lower index
//   w_j = scale * s_j, or scale * s_j / sum_i s_i over the chosen
//
// A warp owns a row and keeps its keys in registers, lane l the experts l*EPL .. l*EPL+EPL-1, so that the lowest
// lane of a tie holds the lowest index and a round of the selection is one integer warp maximum, one vote and one
// shuffle.  The memory traffic is the logits once; at T = 16384, E = 256 the kernel is bound by instruction issue
// of the k rounds and by latency, not by memory (the logits stay in L2).
#include <math_constants.h>

#include <type_traits>

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
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
__device__ __forceinline__ float sigmoid_rn(float z) { return 1.0f / (1.0f + expf(-z)); }
// exp(z - m) for z <= m, with exp(0) = 1 where both are +inf
__device__ __forceinline__ float exp_below(float z, float m) { return z == m ? 1.0f : expf(z - m); }

// The lane's EPL logits of one row.  `vec`: rows start on 16-byte boundaries and E is a multiple of a vector.
template <typename T, int EPL>
__device__ __forceinline__ void load_row(const T* __restrict__ row, int E, int lane, bool vec, float (&z)[EPL]) {
  constexpr int VN = Vec<T>::N;
  const int e0 = lane * EPL;
  if constexpr (EPL >= VN) {
    if (vec) {
#pragma unroll
      for (int i = 0; i < EPL; i += VN) {
        float v[VN];
        if (e0 + i < E) Vec<T>::load(row + e0 + i, v);
#pragma unroll
        for (int j = 0; j < VN; ++j) z[i + j] = e0 + i < E ? v[j] : -CUDART_INF_F;
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) z[i] = e0 + i < E ? to_f32(row[e0 + i]) : -CUDART_INF_F;
}

// Two-best merge: (a, b) with a >= b
template <typename F> __device__ __forceinline__ void push2(F v, F& a, F& b) {
  if (v > a) { b = a; a = v; } else if (v > b) { b = v; }
}
// Group key from its two best members' keys.  A group without a candidate has -inf, a missing second adds nothing.
template <typename F> __device__ __forceinline__ F group_value(F a, F b, int sum2) {
  return sum2 && b > (F)-CUDART_INF ? a + b : a;
}

// Which groups stay, as a bit mask, from the keys in the warp's shared memory (expert e at e + (e / size) * P, so
// that the lanes of different groups read different banks).  P lanes share a group.  `margin` receives the
// difference between the worst group that stays and the best that does not, `reach` the largest
// sum of magnitudes behind a group's key (for the caller's error bound).
template <typename F>
__device__ __forceinline__ uint32_t choose_groups(const F* key, int G, int size, int P, int topk_group, int sum2,
                                                  int lane, F& margin, F& reach) {
  const F low = (F)-CUDART_INF;
  const int g = lane / P, p = lane - g * P;
  F a = low, b = low;
  if (g < G)
    for (int j = p; j < size; j += P) push2(key[g * (size + P) + j], a, b);
  for (int o = 1; o < P; o <<= 1) {
    const F oa = __shfl_xor_sync(kAll, a, o), ob = __shfl_xor_sync(kAll, b, o);
    push2(oa, a, b);
    push2(ob, a, b);
  }
  const F v = g < G ? group_value(a, b, sum2) : low;
  int rank = 0;
  for (int q = 0; q < G; ++q) {
    const F o = __shfl_sync(kAll, v, q * P);
    rank += o > v || (o == v && q < g);
  }
  const bool leader = g < G && p == 0;
  F worst = (F)CUDART_INF, best = low;
  if (leader && rank < topk_group) worst = v;
  if (leader && rank >= topk_group) best = v;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const F ow = __shfl_xor_sync(kAll, worst, o), ob = __shfl_xor_sync(kAll, best, o);
    worst = ow < worst ? ow : worst;
    best = ob > best ? ob : best;
  }
  F size_ab = (F)0;
  if (leader && v > low) size_ab = fabs(a) + (v != a ? fabs(b) : (F)0);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) size_ab = fmax(size_ab, __shfl_xor_sync(kAll, size_ab, o));
  margin = best > low ? worst - best : (F)CUDART_INF;
  reach = size_ab;
  const uint32_t lanes = __ballot_sync(kAll, leader && rank < topk_group && v > low);
  uint32_t mask = 0;
  for (int q = 0; q < G; ++q) mask |= ((lanes >> (q * P)) & 1u) << q;
  return mask;
}

// The same choice with 64-bit scores, for the few rows whose order 32 bits do not settle.  keys: E + n_group * P
// doubles of the warp's shared memory.  Returns the expert of slot `lane` (-1: none).
template <typename T, bool SIGMOID>
__device__ __noinline__ int choose_in_double(const T* __restrict__ row, const RouteParams& p, int sum2, double* keys, int lane) {
  const int P = p.n_group > 1 ? p.lanes_per_group : 0;
  const double low = -CUDART_INF;
  double zmax = low, total = 0.0;
  if (!SIGMOID) {
    for (int e = lane; e < p.E; e += 32) {
      const double z = (double)to_f32(row[e]);
      if (z > zmax) zmax = z;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) zmax = fmax(zmax, __shfl_xor_sync(kAll, zmax, o));
    for (int e = lane; e < p.E; e += 32) {
      const double z = (double)to_f32(row[e]);
      if (z > low) total += z == zmax ? 1.0 : exp(z - zmax);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(kAll, total, o);
  }
  auto score = [&](double z) {
    return SIGMOID ? 1.0 / (1.0 + exp(-z)) : (z == zmax ? 1.0 : exp(z - zmax)) / total;
  };
  // the key that orders experts; without a bias it is the logit, and only a group's sum needs scores
  auto place = [&](bool for_groups) {
    for (int e = lane; e < p.E; e += 32) {
      const double z = (double)to_f32(row[e]);
      double c = low;
      if (z > low) c = p.bias ? score(z) + (double)p.bias[e] : (for_groups && sum2 ? score(z) : z);
      keys[e + (P ? e / p.group_size * P : 0)] = c > low ? c : low;
    }
    __syncwarp();
  };
  uint32_t stay = kAll;
  place(true);
  if (p.n_group > 1) {
    double margin, reach;
    stay = choose_groups<double>(keys, p.n_group, p.group_size, P, p.topk_group, sum2, lane, margin, reach);
    __syncwarp();
    if (!p.bias && sum2) place(false);
  }
  int mine = -1;
  for (int j = 0; j < p.k; ++j) {
    double bv = low;
    int bi = -1;
    for (int e = lane; e < p.E; e += 32) {
      const int g = p.n_group > 1 ? e / p.group_size : 0;
      const double c = keys[e + g * P];
      if (((stay >> g) & 1u) && c > bv) { bv = c; bi = e; }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const double ov = __shfl_xor_sync(kAll, bv, o);
      const int oi = __shfl_xor_sync(kAll, bi, o);
      if (oi >= 0 && (bi < 0 || ov > bv || (ov == bv && oi < bi))) { bv = ov; bi = oi; }
    }
    if (bi < 0) break;
    if (lane == j) mine = bi;
    if (lane == 0) keys[bi + (P ? bi / p.group_size * P : 0)] = low;
    __syncwarp();
  }
  return mine;
}

template <typename T, int EPL, bool SIGMOID>
__global__ void __launch_bounds__(kRsWarps * 32)
route_scored_kernel(const T* __restrict__ logits, const RouteParams p, int sum2, int vec) {
  // per warp: 32-bit keys for the groups, or 64-bit keys of a row that is decided again (never both at once)
  __shared__ double keys_s[kRsWarps][EPL * 32 + 32];
  __shared__ int hist[EPL * 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool grouped = p.n_group > 1;
  const int P = p.lanes_per_group;
  const int e0 = lane * EPL;
  const float low = -CUDART_INF_F;
  if (p.counts != nullptr) {
    for (int i = threadIdx.x; i < p.E; i += blockDim.x) hist[i] = 0;
    __syncthreads();
  }
  // Error bounds of a 32-bit key, relative to its score and to itself (expf is within 1 ulp, division and sums
  // round to nearest): sigmoid 2^-22 s; softmax also carries the rounded differences z - max, |z - max| 2^-24 each,
  // and a sum of 21 roundings, together below 2^-19 (s + 0.02) for E <= 512.
  const float err_s = SIGMOID ? 0x1p-22f : 0x1p-19f, err_0 = SIGMOID ? 0.f : 0x1p-24f, err_c = 0x1p-24f;
  const bool need_scores = p.scores != nullptr || p.bias != nullptr || (grouped && sum2);
  const bool need_total = !SIGMOID && (need_scores || !p.renorm);

  for (int t = blockIdx.x * kRsWarps + warp; t < p.T; t += gridDim.x * kRsWarps) {
    const T* row = logits + (long long)t * p.stride;
    int sel = -1;                           // lane j: the expert of slot j
    float total = 1.f, zmax = 0.f;
    if (p.row_valid == nullptr || p.row_valid[t] != 0) {
      float z[EPL], c[EPL], s[EPL];
      load_row<T, EPL>(row, p.E, lane, vec != 0, z);
      if (need_total) {
        float m = low;
#pragma unroll
        for (int i = 0; i < EPL; ++i) m = fmaxf(m, z[i]);          // (fmaxf passes over NaN)
        zmax = warp_max(m);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          s[i] = z[i] > low ? exp_below(z[i], zmax) : 0.f;
          sum += s[i];
        }
        total = warp_sum(sum);
#pragma unroll
        for (int i = 0; i < EPL; ++i) s[i] = total > 0.f ? s[i] / total : 0.f;
      } else {
#pragma unroll
        for (int i = 0; i < EPL; ++i) s[i] = SIGMOID && need_scores && z[i] > low ? sigmoid_rn(z[i]) : 0.f;
      }
      if (p.scores != nullptr) {
#pragma unroll
        for (int i = 0; i < EPL; ++i)
          if (e0 + i < p.E) p.scores[(size_t)t * p.E + e0 + i] = s[i];
      }
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        c[i] = p.bias == nullptr ? z[i] : (z[i] > low && e0 + i < p.E ? s[i] + p.bias[e0 + i] : low);
        if (!(c[i] > low)) c[i] = low;
      }
      bool doubt = false;
      if (grouped) {
        float* key = reinterpret_cast<float*>(keys_s[warp]);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          const int e = e0 + i;
          if (e < p.E)
            key[e + e / p.group_size * P] = p.bias == nullptr && sum2 ? (z[i] > low ? s[i] : low) : c[i];
        }
        __syncwarp();
        float margin, reach;
        const uint32_t stay = choose_groups<float>(key, p.n_group, p.group_size, P, p.topk_group, sum2, lane, margin, reach);
        // scores are at most 1 (two at most 2); keys compared as they stand (logits) are exact
        if (p.bias != nullptr || sum2)
          doubt = margin <= 2.f * ((sum2 ? 2.f : 1.f) * (err_s + err_0) + 3.f * err_c * reach);
#pragma unroll
        for (int i = 0; i < EPL; ++i)
          if (e0 + i < p.E && !((stay >> ((e0 + i) / p.group_size)) & 1u)) c[i] = low;
      }
      // k rounds of a warp maximum, one more to see how far the last chosen is from the next
      uint32_t u[EPL];
      uint32_t lm = 0;
      int li = 0;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        u[i] = c[i] > low ? order_key(c[i]) : 0u;
        if (u[i] > lm) { lm = u[i]; li = i; }
      }
      const int rounds = p.bias != nullptr ? min(p.k + 1, 32) : p.k;
      for (int j = 0; j < rounds; ++j) {
        const uint32_t m = __reduce_max_sync(kAll, lm);
        if (m == 0u) break;
        const int w = __ffs(__ballot_sync(kAll, lm == m)) - 1;
        const int e = __shfl_sync(kAll, e0 + li, w);
        if (lane == j) sel = e;
        if (lane == w) {
          lm = 0;
          int ni = 0;
#pragma unroll
          for (int i = 0; i < EPL; ++i) {
            if (i == li) u[i] = 0u;
            if (u[i] > lm) { lm = u[i]; ni = i; }
          }
          li = ni;
        }
      }
      if (p.bias != nullptr) {
        // neighbours in the order whose distance is within the error bound, and that are not equal by their inputs
        const float zs = sel >= 0 ? to_f32(row[sel]) : low, bs = sel >= 0 ? p.bias[sel] : 0.f;
        const float ss = sel >= 0 ? (SIGMOID ? sigmoid_rn(zs) : exp_below(zs, zmax) / total) : 0.f;
        const float cs = ss + bs;
        const float zn = __shfl_down_sync(kAll, zs, 1), bn = __shfl_down_sync(kAll, bs, 1);
        const float sn = __shfl_down_sync(kAll, ss, 1), cn = __shfl_down_sync(kAll, cs, 1);
        const int en = __shfl_down_sync(kAll, sel, 1);
        if (lane < 31 && sel >= 0 && en >= 0 && !(zs == zn && bs == bn))
          doubt |= !(cs - cn > err_s * (ss + sn) + 2.f * err_0 + err_c * (fabsf(cs) + fabsf(cn)));
        // a 33rd neighbour is not compared: with k = 32 the last place is always settled in 64 bits
        doubt |= p.k == 32 && p.E > 32;
      }
      if (__any_sync(kAll, doubt)) {
        __syncwarp();
        sel = choose_in_double<T, SIGMOID>(row, p, sum2, keys_s[warp], lane);
        __syncwarp();
      }
    } else if (p.scores != nullptr) {
      for (int e = lane; e < p.E; e += 32) p.scores[(size_t)t * p.E + e] = 0.f;
    }
    // weights: lane j has slot j.  Renormalised weights are formed from exponentials shifted by the largest chosen
    // logit, so they are a number even where every score underflows.
    if (lane >= p.k) sel = -1;
    const bool have = sel >= 0;
    const float zs = have ? to_f32(row[sel]) : low;
    float w = 0.f;
    if (p.renorm) {
      const float m = warp_max(zs);
      if (SIGMOID) {
        const float shift = fminf(m, 0.f);
        if (have) w = zs > 0.f ? sigmoid_rn(zs) : expf(zs - shift) / (1.0f + expf(zs));
      } else if (have) {
        w = exp_below(zs, m);
      }
      const float sum = warp_sum(w);
      if (have) w = w / sum * p.scale;
    } else if (have) {
      w = (SIGMOID ? sigmoid_rn(zs) : exp_below(zs, zmax) / total) * p.scale;
    }
    if (lane < p.k) {
      p.topk_idx[(size_t)t * p.k + lane] = sel;
      p.gates[(size_t)t * p.k + lane] = w;
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
// logit: dz_e = s_e (scale dw_e [e chosen] - scale sum_j dw_j s_j).  Bound by the store of the row.
template <typename T, int EPL, bool SIGMOID>
__global__ void __launch_bounds__(kRsWarps * 32)
route_scored_backward_kernel(int Tn, int E, int k, int renorm, float scale, long long stride, int vec_in, int vec_out,
                             const T* __restrict__ logits, const int32_t* __restrict__ topk_idx,
                             const float* __restrict__ dgates, T* __restrict__ dlogits, long long out_stride) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int e0 = lane * EPL;
  const float low = -CUDART_INF_F;
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
      const float m = warp_max(zs);
      float pj = 0.f;
      if (SIGMOID) {
        if (have) pj = zs > 0.f ? sigmoid_rn(zs) : expf(zs - fminf(m, 0.f)) / (1.0f + expf(zs));
      } else if (have) {
        pj = exp_below(zs, m);
      }
      const float sum = warp_sum(pj);
      if (have) pj /= sum;
      const float inner = warp_sum(pj * dw);
      if (have) v = scale * pj * (dw - inner);
      if (SIGMOID && have) v *= 1.0f / (1.0f + expf(zs));            // 1 - s without cancellation
    } else if (SIGMOID) {
      if (have) v = scale * dw * sigmoid_rn(zs) * (1.0f / (1.0f + expf(zs)));
    } else {
      float z[EPL];
      load_row<T, EPL>(row, E, lane, vec_in != 0, z);
      float m = low;
#pragma unroll
      for (int i = 0; i < EPL; ++i) m = fmaxf(m, z[i]);
      m = warp_max(m);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        dz[i] = z[i] > low ? exp_below(z[i], m) : 0.f;
        sum += dz[i];
      }
      sum = warp_sum(sum);
      const float s = have && sum > 0.f ? exp_below(zs, m) / sum : 0.f;
      const float inner = scale * warp_sum(s * dw);
#pragma unroll
      for (int i = 0; i < EPL; ++i) dz[i] = sum > 0.f ? -(dz[i] / sum) * inner : 0.f;
      v = scale * s * dw;
    }
    for (int j = 0; j < k; ++j) {
      const int i0 = __shfl_sync(kAll, sel, j) - e0;
      const float vj = __shfl_sync(kAll, v, j);
#pragma unroll
      for (int i = 0; i < EPL; ++i)
        if (i == i0) dz[i] += vj;
    }
    T* out = dlogits + (long long)t * out_stride;
    constexpr int VN = Vec<T>::N;
    if (EPL >= VN && vec_out) {
#pragma unroll
      for (int i = 0; i + VN <= EPL; i += VN) {
        if (e0 + i < E) {
          __align__(16) T q[VN];
#pragma unroll
          for (int j = 0; j < VN; ++j) q[j] = from_f32<T>(dz[(i + j) % EPL]);
          *reinterpret_cast<uint4*>(out + e0 + i) = *reinterpret_cast<const uint4*>(q);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPL; ++i)
        if (e0 + i < E) out[e0 + i] = from_f32<T>(dz[i]);
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

int row_blocks(int T) {
  const int want = (T + kRsWarps - 1) / kRsWarps, most = 8 * sm_count();
  return want < most ? want : most;
}

template <typename T, int EPL>
cudaError_t launch_route_t(const btx_route_desc* d, const void* logits, RouteParams p, cudaStream_t st) {
  const int vec = row_vectors(logits, p.stride, p.E, sizeof(T)) ? 1 : 0;
  int blocks = row_blocks(p.T);
  // Counting: one block writes its own counts; more add theirs to zeros.  A block of 8 warps takes up to 16 rows
  // on its own, which costs less than a second launch to clear the counts.
  p.single_block = p.counts != nullptr && p.T <= 2 * kRsWarps;
  if (p.single_block) blocks = 1;
  else if (p.counts != nullptr) {
    cudaError_t e = cudaMemsetAsync(p.counts, 0, (size_t)p.E * sizeof(int32_t), st);
    if (e != cudaSuccess) return e;
  }
  const int sum2 = d->group_score == BTX_GROUP_SUM2;
  if (d->score == BTX_SCORE_SIGMOID)
    route_scored_kernel<T, EPL, true><<<blocks, kRsWarps * 32, 0, st>>>((const T*)logits, p, sum2, vec);
  else
    route_scored_kernel<T, EPL, false><<<blocks, kRsWarps * 32, 0, st>>>((const T*)logits, p, sum2, vec);
  return cudaGetLastError();
}

template <typename T, int EPL>
cudaError_t launch_route_backward_t(const btx_route_desc* d, const void* logits, long long stride, const int32_t* topk_idx,
                                    const float* dgates, void* dlogits, long long out_stride, cudaStream_t st) {
  const int vi = row_vectors(logits, stride, d->E, sizeof(T)), vo = row_vectors(dlogits, out_stride, d->E, sizeof(T));
  if (d->score == BTX_SCORE_SIGMOID)
    route_scored_backward_kernel<T, EPL, true><<<row_blocks(d->T), kRsWarps * 32, 0, st>>>(
        d->T, d->E, d->k, d->renorm != 0, d->scale, stride, vi, vo, (const T*)logits, topk_idx, dgates, (T*)dlogits, out_stride);
  else
    route_scored_backward_kernel<T, EPL, false><<<row_blocks(d->T), kRsWarps * 32, 0, st>>>(
        d->T, d->E, d->k, d->renorm != 0, d->scale, stride, vi, vo, (const T*)logits, topk_idx, dgates, (T*)dlogits, out_stride);
  return cudaGetLastError();
}

// experts per lane: the power of two that covers E with 32 lanes
template <typename T, typename F>
cudaError_t by_width(int E, F&& f) {
  if (E <= 32) return f(std::integral_constant<int, 1>());
  if (E <= 64) return f(std::integral_constant<int, 2>());
  if (E <= 128) return f(std::integral_constant<int, 4>());
  if (E <= 256) return f(std::integral_constant<int, 8>());
  return f(std::integral_constant<int, 16>());
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
  p.lanes_per_group = 1;
  while (2 * p.lanes_per_group * p.n_group <= 32) p.lanes_per_group *= 2;
  if (p.topk_group == p.n_group) p.n_group = 1;                // every group stays: nothing to choose
  const cudaError_t e = desc->dtype == BTX_BF16
      ? by_width<__nv_bfloat16>(p.E, [&](auto w) { return launch_route_t<__nv_bfloat16, w.value>(desc, logits, p, st); })
      : by_width<float>(p.E, [&](auto w) { return launch_route_t<float, w.value>(desc, logits, p, st); });
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
      ? by_width<__nv_bfloat16>(desc->E, [&](auto w) {
          return launch_route_backward_t<__nv_bfloat16, w.value>(desc, logits, logits_stride, topk_idx, dgates, dlogits, dlogits_stride, st); })
      : by_width<float>(desc->E, [&](auto w) {
          return launch_route_backward_t<float, w.value>(desc, logits, logits_stride, topk_idx, dgates, dlogits, dlogits_stride, st); });
  return e == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

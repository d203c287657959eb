// The expert layer on MXFP4 experts for a small batch as one cooperative kernel: dispatch and cast, W1/W3 product with
// SwiGLU and cast, W2 product, sum over the slots.  The layer reads every used expert's weights once (287 MB, 45 us at
// the copy rate, for 32 tokens, d = 4096, F = 11008, 4 experts, top-2) and does little else.  The thread that loads
// weights starts on the next pass before each grid barrier.  That batch takes 66.7 us, a launch of its own for
// each step 69.6 us on the device and 10 us more of the host's time.  Stamps show where it goes: 7.7 us until the first
// barrier is passed, 38 us for the 688 tiles of pass 1 (4.65 a CTA at 6.7 us; the slowest CTA sets the end), 18 us for
// pass 2, 3 us behind it.  Weights on the M side of the MMAs and tokens on the N side measured 73 us.
//
//   every CTA    counts the assignments (at most 1024) for itself and lists the experts' row tiles in shared memory
//   warps 2-9    cast the CTA's tokens (t = CTA, CTA + grid, ..) to the rows of their slots;  grid barrier
//   pass 1       h1, h3 = W1 x, W3 x (rows in turn), a = silu(h1) * h3, cast;  grid barrier
//   pass 2       gate * W2 a; with few tiles the contraction is split over CTAs, each part into rows of its own;  grid barrier
//   all threads  y = sum over slots and parts, in order
// Roles in the passes: warp 0 TMA of the activations, warp 10 TMA of the weights, warp 1 MMAs, warps 11-14 scales,
// warps 2-9 epilogue.  A cooperative launch: every block is resident, or the launch is refused and the separate
// kernels run.  Waits inside a pass are bounded; every thread reaches every grid barrier whatever its waits did.
#include <cooperative_groups.h>

#include <climits>

#include "btx_mx4_dev.cuh"

namespace btx {
namespace mx4 {
namespace {

namespace cg = cooperative_groups;

constexpr int L_THREADS = 96 + EPI_WARPS * 32 + 128;
constexpr int L_RING = 214 * 1024;
// Batches of more assignments, or of more than two tokens for every multiprocessor (each ranks its assignments by a walk over
// the list), take separate launches, which are as fast there on the device: 296 tokens on 3 of 16 experts (d = 2048,
// F = 1024) 34.6 us in one kernel and 33.8, 290 tokens on one of 8 (4096 x 4096) 62.0 and 59.9.  Below, one kernel
// is ahead: 32 tokens of the batch above 66.7 and 69.6, 128 of them 70.7 and 73.1, 128 tokens on 8 of 64 experts 63.7 and
// 69.3 (d = 2048, F = 1024), on 8 of 256 179 and 202.
constexpr int L_MAX_R = 1024;
// Stages of weights on their way before the first barrier: a whole ring of every CTA holds up the cast and the barrier behind
// it (68.4 us for that batch; 1 to 3 stages 66.6, 5 stages 66.8).  Before the second barrier the whole ring pays: 66.6 us,
// 69 to 70 with 2 to 8 stages.
constexpr int kFirstStages = 2;
constexpr int L_MAX_TILES = kMaxExperts4 + L_MAX_R / kTileRows;      // min(R, E) + R / 128 bounds the row tiles

struct Lists {
  int16_t idx[L_MAX_R];              // expert of an assignment, -1 without
  int16_t tile_expert[L_MAX_TILES], tile_rows[L_MAX_TILES];
  int n_tiles, most_rows;
  int cnt[kMaxExperts4], pad[kMaxExperts4], row_of[kMaxExperts4];
};
constexpr int L_SMEM = L_RING + 1024 + 320 + (int)sizeof(Lists);
static_assert(L_SMEM <= 227 * 1024 && MAX_STAGES * 24 + 48 <= 320, "shared memory");

struct LayerParams {
  int T, k, R, E, d;
  const int32_t* topk_idx;
  const void* x;
  void* y;
  uint8_t* xs_codes;
  uint8_t* xs_scales;
  int32_t* rowmap;
  int32_t* status;
  size_t part_stride;                // floats from one part's rows to the next
  Params up, down;
};

// Parts of the contraction of pass 2: as many CTAs as keep every one busy at most once, two stages each at least.  Every
// part has room for the rows of all R assignments, so a batch of mostly empty slots counts as many row tiles as R fills.
__device__ __forceinline__ int parts_of(int tiles, int ctas, int kb) {
  int s = 1;
  while (s < 8 && 2 * s * tiles <= ctas && 4 * s <= kb) s *= 2;
  return s;
}

template <typename T>
__global__ void __launch_bounds__(L_THREADS, 1)
mx4_layer_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW13,
                 const __grid_constant__ CUtensorMap tmAct, const __grid_constant__ CUtensorMap tmW2,
                 const __grid_constant__ LayerParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t ring = (raw + 1023u) & ~1023u;
  uint8_t* ctl = smem_raw + (ring - raw) + L_RING;
  const uint32_t bar_full = smem_u32(ctl), bar_empty = bar_full + MAX_STAGES * 8;
  const uint32_t bar_tfull = bar_empty + MAX_STAGES * 8, bar_tempty = bar_tfull + 16;
  const uint32_t bar_scales = bar_tempty + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctl + MAX_STAGES * 24 + 32);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctl + MAX_STAGES * 24 + 40);
  Lists& ls = *reinterpret_cast<Lists*>(ctl + 320);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr int a_box = 32;
  const int ctas = (int)gridDim.x;
  cg::grid_group grid = cg::this_grid();

  for (int e = tid; e < p.E; e += L_THREADS) ls.cnt[e] = 0;
  if (tid == 0) {
    for (int s = 0; s < MAX_STAGES; ++s) { mbar_init(bar_full + s * 8, 2); mbar_init(bar_empty + s * 8, 1); mbar_init(bar_scales + s * 8, 4); }
    for (int a = 0; a < 2; ++a) { mbar_init(bar_tfull + a * 8, 1); mbar_init(bar_tempty + a * 8, EPI_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if (blockIdx.x == 0)
      for (int i = 0; i < kStatusWords; ++i) p.status[i] = 0;
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  // ---- counts and row tiles ----
  for (int i = tid; i < p.R; i += L_THREADS) {
    int e = p.topk_idx[i];
    if ((unsigned)e >= (unsigned)p.E) e = -1;
    ls.idx[i] = (int16_t)e;
    if (e >= 0) atomicAdd(&ls.cnt[e], 1);
  }
  __syncthreads();
  if (warp == 0) {
    int before = 0, most = 1;
    for (int e0 = 0; e0 < p.E; e0 += 32) {
      const int e = e0 + lane;
      const int c = e < p.E ? ls.cnt[e] : 0, tiles = (c + kTileRows - 1) / kTileRows;
      int incl = tiles;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(kAll, incl, o);
        if (lane >= o) incl += up;
      }
      const int first = before + incl - tiles;
      if (e < p.E) ls.pad[e] = first * kTileRows;
      for (int j = 0; j < tiles; ++j) {
        ls.tile_expert[first + j] = (int16_t)e;
        ls.tile_rows[first + j] = (int16_t)min(kTileRows, c - j * kTileRows);
      }
      before += __shfl_sync(kAll, incl, 31);
      most = max(most, min(c, kTileRows));
    }
    most = __reduce_max_sync(kAll, most);
    if (lane == 0) {
      ls.n_tiles = before;
      ls.most_rows = most;
    }
  }
  __syncthreads();
  const int m_tiles = ls.n_tiles;
  // A stage holds as many rows of activations as the fullest tile: what is in flight decides the rate (6, 8, 10 stages
  // read 4.6, 5.0, 5.2 TB/s of 190 MB), so the ring is cut for this batch.
  const int a_rows = (ls.most_rows + a_box - 1) / a_box * a_box;
  const int n_stages = stage_count(a_rows, L_RING), s_bytes = stage_bytes(a_rows);
  const int tiles1 = m_tiles * p.up.n_tiles, tiles2 = m_tiles * p.down.n_tiles;
  const int kb1 = (p.up.K + SK - 1) / SK, kb2 = (p.down.K + SK - 1) / SK;
  const int parts = parts_of(max(m_tiles, (p.R + kTileRows - 1) / kTileRows) * p.down.n_tiles, ctas, kb2);

  // The work items of a pass for this CTA: item i -> tile, stages [k0, k1), rows of the part.
  struct Work { Item it; int k0, k1, part; };
  auto work = [&](bool second, int i) {
    Work w;
    const Params& q = second ? p.down : p.up;
    const int n = second ? parts : 1, kb = second ? kb2 : kb1;
    const int tile = i / n;
    w.part = i - tile * n;
    w.it = Item();
    raster(m_tiles, q.n_tiles, tile, w.it.mt, w.it.nt);
    w.it.e = ls.tile_expert[w.it.mt];
    w.k0 = (int)((long long)w.part * kb / n);
    w.k1 = (int)((long long)(w.part + 1) * kb / n);
    return w;
  };

  // Weight loads: the first `limit` stages of a pass ahead of its grid barrier, the rest inside it.
  uint32_t stage = 0, phase = 0;            // of this thread's role
  bool ok = true;
  int ahead = 0;                            // stages of the pass that are already on their way
  auto load_weights = [&](bool second, int skip, int limit) {
    const Params& q = second ? p.down : p.up;
    const CUtensorMap* map = second ? &tmW2 : &tmW13;
    const int items = second ? tiles2 * parts : tiles1;
    int n = 0;
    for (int i = blockIdx.x; i < items && ok; i += ctas) {
      const Work w = work(second, i);
      const uint8_t* sfb = q.b_scales + w.it.e * q.b_scale_batch + (size_t)w.it.nt * q.kt * kTileBytes;
      for (int kb = w.k0; kb < w.k1; ++kb, ++n) {
        if (n < skip) continue;
        if (n >= limit) return n;
        if (!(ok = mbar_wait(bar_empty + stage * 8, phase ^ 1u, abort_flag, p.status))) return n;
        const uint32_t bar = bar_full + stage * 8;
        const uint32_t sSB = ring + stage * s_bytes + a_rows * (SK / 2) + SF_BYTES, sB = sSB + SF_BYTES;
        const uint32_t sf = (uint32_t)min(2, q.kt - 2 * kb) * kTileBytes;
        mbar_expect_tx(bar, B_BYTES + sf);
        load_3d(sB, map, kb * (SK / 2), w.it.nt * BN, w.it.e, bar);
        load_bulk(sSB, sfb + (size_t)kb * 2 * kTileBytes, sf, bar);
        if (++stage == n_stages) { stage = 0; phase ^= 1u; }
      }
    }
    return n;
  };

  // ---- cast ----
  if (warp == 10) {
    if (lane == 0) ahead = load_weights(false, 0, min(n_stages, kFirstStages));
    __syncwarp();
  } else if (warp >= 2 && warp < 10) {
    for (int t = blockIdx.x; t < p.T; t += ctas) {
      for (int j = warp - 2; j < p.k; j += EPI_WARPS) {
        const int i = t * p.k + j, e = ls.idx[i];
        int rank = 0;
        if (e >= 0)
          for (int b = 0; b < i; b += 32) rank += __popc(__ballot_sync(kAll, b + lane < i && ls.idx[b + lane] == e));
        if (lane == 0) {
          const int row = e >= 0 ? ls.pad[e] + rank : -1;
          ls.row_of[j] = row;
          if (row >= 0) p.rowmap[row] = i;
        }
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
      for (int g = warp - 2; g * kCastUnroll * 256 < p.d; g += EPI_WARPS)
        cast_token_rows<T>((const T*)p.x + (size_t)t * p.d, p.d, g, lane, p.k, ls.row_of, p.xs_codes, p.xs_scales);
      asm volatile("bar.sync 1, 256;" ::: "memory");
    }
  }

  uint32_t acc = 0, acc_phase = 0;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    // what was written with ordinary stores is read behind the barrier by other blocks, by their TMA loads too
    asm volatile("fence.proxy.async.global;" ::: "memory");
    __threadfence();
    tc_fence_before();
    grid.sync();
    tc_fence_after();
    asm volatile("fence.proxy.async.global;" ::: "memory");

    const bool second = pass == 1;
    const Params& q = second ? p.down : p.up;
    const int items = second ? tiles2 * parts : tiles1;
    if (warp == 0) {
      if (lane == 0) {
        const CUtensorMap* map = second ? &tmAct : &tmX;
        for (int i = blockIdx.x; i < items && ok; i += ctas) {
          const Work w = work(second, i);
          const uint8_t* sfa = q.a_scales + (size_t)w.it.mt * q.kt * kTileBytes;
          const int boxes = ((int)ls.tile_rows[w.it.mt] + a_box - 1) / a_box;
          for (int kb = w.k0; kb < w.k1; ++kb) {
            if (!(ok = mbar_wait(bar_empty + stage * 8, phase ^ 1u, abort_flag, p.status))) break;
            const uint32_t bar = bar_full + stage * 8;
            const uint32_t sA = ring + stage * s_bytes, sSA = sA + a_rows * (SK / 2);
            const uint32_t sf = (uint32_t)min(2, q.kt - 2 * kb) * kTileBytes;
            mbar_expect_tx(bar, boxes * a_box * (SK / 2) + sf);
            for (int r = 0; r < boxes; ++r) load_3d(sA + r * a_box * (SK / 2), map, kb * (SK / 2), w.it.mt * BM + r * a_box, 0, bar);
            load_bulk(sSA, sfa + (size_t)kb * 2 * kTileBytes, sf, bar);
            if (++stage == n_stages) { stage = 0; phase ^= 1u; }
          }
        }
      }
      __syncwarp();
    } else if (warp == 10) {
      if (lane == 0) {
        load_weights(second, ahead, INT_MAX);
        if (!second && ok) ahead = load_weights(true, 0, n_stages);
      }
      __syncwarp();
    } else if (warp == 1) {
      if (lane == 0) {
        constexpr uint32_t idesc0 = (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | (1u << 23) | ((uint32_t)(BM >> 4) << 24);
        for (int i = blockIdx.x; i < items && ok; i += ctas) {
          const Work w = work(second, i);
          if (!(ok = mbar_wait(bar_tempty + acc * 8, acc_phase ^ 1u, abort_flag, p.status))) break;
          tc_fence_after();
          const uint32_t d = tmem + acc * BN;
          for (int kb = w.k0; kb < w.k1; ++kb) {
            if (!(ok = mbar_wait(bar_full + stage * 8, phase, abort_flag, p.status))) break;
            if (!(ok = mbar_wait(bar_scales + stage * 8, phase, abort_flag, p.status))) break;
            tc_fence_after();
            const uint32_t sA = ring + stage * s_bytes, sB = sA + a_rows * (SK / 2) + 2 * SF_BYTES;
            const uint32_t tA = tmem + 2 * BN + stage * SF_COLS, tB = tA + 8;
            const int k64 = min(SK / 64, (q.K - kb * SK + 63) / 64);
            const uint64_t da = smem_desc(sA, false), db = smem_desc(sB, false);
#pragma unroll
            for (int j = 0; j < SK / 64; ++j) {
              if (j < k64) {
                const uint32_t id = (uint32_t)(j & 1) * 2;
                mma_mxf4(d, da + (uint64_t)(2 * j), db + (uint64_t)(2 * j), idesc0 | (id << 4) | (id << 29), tA + (j >> 1) * 4,
                         tB + (j >> 1) * 4, (kb > w.k0 || j > 0) ? 1u : 0u);
              }
            }
            commit(bar_empty + stage * 8);
            if (++stage == n_stages) { stage = 0; phase ^= 1u; }
          }
          if (!ok) break;
          commit(bar_tfull + acc * 8);
          acc ^= 1u;
          if (acc == 0) acc_phase ^= 1u;
        }
      }
      __syncwarp();
    } else if (warp > 10) {
      for (int i = blockIdx.x; i < items && ok; i += ctas) {
        const Work w = work(second, i);
        for (int kb = w.k0; kb < w.k1; ++kb) {
          if (!(ok = warp_wait(bar_full + stage * 8, phase, abort_flag, p.status))) break;
          const uint32_t from = ring + stage * s_bytes + a_rows * (SK / 2) + lane * 16;
          const uint32_t to = tmem + 2 * BN + stage * SF_COLS + ((uint32_t)((warp & 3) * 32) << 16);
          store_scales(to, ld_shared_v4(from), ld_shared_v4(from + kTileBytes));
          store_scales(to + 8, ld_shared_v4(from + SF_BYTES), ld_shared_v4(from + SF_BYTES + kTileBytes));
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          tc_fence_before();
          if (lane == 0) arrive(bar_scales + stage * 8);
          if (++stage == n_stages) { stage = 0; phase ^= 1u; }
        }
      }
    } else {
      const int quarter = warp & 3, half = (warp - 2) >> 2;
      const int row = quarter * 32 + lane;
      for (int i = blockIdx.x; i < items && ok; i += ctas) {
        const Work w = work(second, i);
        const int m = w.it.mt * BM + row;
        int flat = row < ls.tile_rows[w.it.mt] ? 0 : -1;
        if (second && flat >= 0) flat = __ldcg(p.rowmap + m);
        const bool any = __any_sync(kAll, flat >= 0);
        if (!(ok = warp_wait(bar_tfull + acc * 8, acc_phase, abort_flag, p.status))) break;
        tc_fence_after();
        float v[64];
        if (any) load_chunk(tmem + acc * BN + half * 64 + ((uint32_t)(quarter * 32) << 16), v);
        tc_fence_before();
        if (lane == 0) arrive(bar_tempty + acc * 8);
        if (any) {
          const int n0 = w.it.nt * BN + half * 64;
          if (second) finish_chunk<DOWN>(p.down, w.it, v, n0, m, flat, w.part * p.part_stride);
          else finish_chunk<GATE_UP>(p.up, w.it, v, n0, m, flat);
        }
        acc ^= 1u;
        if (acc == 0) acc_phase ^= 1u;
      }
      __syncwarp();
    }
  }
  __threadfence();
  tc_fence_before();
  grid.sync();

  // ---- y[t] = sum over slots and parts ----
  constexpr int VN = Vec<T>::N;
  const int vecs = p.d / VN;
  for (int i = blockIdx.x * L_THREADS + tid; i < p.T * vecs; i += ctas * L_THREADS) {
    const int t = i / vecs, c = (i - t * vecs) * VN;
    float a[VN];
#pragma unroll
    for (int j = 0; j < VN; ++j) a[j] = 0.f;
    for (int s = 0; s < p.k; ++s) {
      if (ls.idx[t * p.k + s] < 0) continue;               // its row was never written
      for (int part = 0; part < parts; ++part) {
        const float* r = (const float*)p.down.y + part * p.part_stride + ((size_t)t * p.k + s) * p.d + c;
#pragma unroll
        for (int j = 0; j < VN; j += 4) {
          const float4 f = __ldcg(reinterpret_cast<const float4*>(r + j));
          a[j] += f.x; a[j + 1] += f.y; a[j + 2] += f.z; a[j + 3] += f.w;
        }
      }
    }
    __align__(16) T out[VN];
#pragma unroll
    for (int j = 0; j < VN; ++j) out[j] = from_f32<T>(a[j]);
    *reinterpret_cast<uint4*>((T*)p.y + (size_t)t * p.d + c) = *reinterpret_cast<const uint4*>(out);
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
  }
}

}  // namespace

bool layer_fits(const Dispatch& q) {
  return q.pad_tiles == 1 && q.R <= L_MAX_R && q.T <= 2 * sm_count() && q.m_tiles_max <= L_MAX_TILES &&
         (long long)q.T * q.d < (1ll << 31);                // (vectors of y are numbered in 32 bits)
}

// Rows of all parts: s > 1 parts of t tiles (s * t at most the CTAs, t at least what R rows of d fill) are at most
// s * t * 128 * 128 floats.
size_t layer_rows_floats(const Dispatch& q) {
  const size_t one = (size_t)q.R * q.d, split = (size_t)sm_count() * kTileRows * BN;
  const size_t most = one > split ? one : split;
  return 8 * one < most ? 8 * one : most;
}

btx_status launch_layer(const GemmArgs& up, const GemmArgs& down, const Dispatch& q, int dtype, const void* x, const float* gates,
                        float* rows, uint8_t* act_codes, uint8_t* act_scales, void* y, cudaStream_t st) {
  static std::atomic<uint64_t> done[2];
  LayerParams p = {};
  p.T = q.T; p.k = q.k; p.R = q.R; p.E = q.E; p.d = q.d;
  p.topk_idx = q.topk_idx; p.x = x; p.y = y; p.rowmap = q.rowmap; p.status = q.status;
  p.xs_codes = const_cast<uint8_t*>(up.a_codes); p.xs_scales = const_cast<uint8_t*>(up.a_scales);
  p.part_stride = (size_t)q.R * q.d;
  auto fill = [&](const GemmArgs& g, Params& m) {
    m.M = g.M; m.N = g.N; m.K = g.K; m.n_tiles = (g.N + BN - 1) / BN; m.kt = (int)scale_tiles_k(g.K);
    m.a_scales = g.a_scales; m.b_scales = g.b_scales;
    m.b_scale_batch = (long long)((g.N + kTileRows - 1) / kTileRows) * m.kt * kTileBytes;
  };
  fill(up, p.up);
  fill(down, p.down);
  p.up.act_codes = act_codes; p.up.act_scales = act_scales;
  p.down.gates = gates; p.down.y = rows; p.down.wide = 1;
  CUtensorMap mx, mw13, ma, mw2;
  if (!make_codes_map(&mx, up.a_codes, up.K, up.M, 1, 32) || !make_codes_map(&mw13, up.b_codes, up.K, up.N, up.experts, BN) ||
      !make_codes_map(&ma, down.a_codes, down.K, down.M, 1, 32) || !make_codes_map(&mw2, down.b_codes, down.K, down.N, down.experts, BN))
    return BTX_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(sm_count()); cfg.blockDim = dim3(L_THREADS); cfg.dynamicSmemBytes = L_SMEM; cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  const bool bf16 = dtype == BTX_BF16;
  const void* kernel = bf16 ? (const void*)mx4_layer_kernel<__nv_bfloat16> : (const void*)mx4_layer_kernel<float>;
  if (!allow_smem(kernel, L_SMEM, done[bf16])) return BTX_ERR_CUDA;
  const cudaError_t e = bf16 ? cudaLaunchKernelEx(&cfg, mx4_layer_kernel<__nv_bfloat16>, mx, mw13, ma, mw2, p)
                             : cudaLaunchKernelEx(&cfg, mx4_layer_kernel<float>, mx, mw13, ma, mw2, p);
  if (e != cudaErrorCooperativeLaunchTooLarge) return e == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
  cudaGetLastError();                                      // answered by the caller, not an error of this thread any more
  return BTX_ERR_UNSUPPORTED;
}

}  // namespace mx4
}  // namespace btx

// Products of MXFP4 matrices on the 5th-generation tensor cores (tcgen05.mma kind::mxf4.block_scale): codes straight
// from memory to shared memory by TMA, scales through shared memory and tcgen05.st into tensor memory, fp32 sums in
// tensor memory; nothing is decoded on the way.  y = A B^T with both operands K-major, per output element
//   sum over blocks of 32:  2^(sa - 127) 2^(sb - 127) sum a_i b_i.
//
// Two kernels: mx4_gemm_kernel, a CTA per 128 x 128 tile, for few rows (bound by reading B), and below it
// mx4_gemm_pair_kernel, two CTAs per 256 x 256 tile, for many (bound by the tensor cores and their power).
//
// mx4_gemm_kernel:
//   warp 0, 10  TMA producers (one lane each: an operation costs its thread about 80 ns) of A and of B with their
//               scales: ring of stages of 256 contraction elements (codes in swizzled rows of 128 bytes, two 512-byte
//               scale tiles of each).  Of A a stage holds only as many rows as a tile can have (a multiple of 32),
//               which leaves room for more stages: with 32 rows 10 instead of 6
//   warp 1      allocates tensor memory; one lane issues up to four MMAs of 64 contraction elements per stage
//   warps 11-14 scales, from shared memory into the stage's own tensor-memory columns, a warp per 32-lane quarter (the
//               columns are free: the stage is filled again only after the MMAs that read them have retired).
//               tcgen05.cp would do the same in the pipe of the MMAs, 37 ns a tile: 46 instead of 40 us for 190 MB of B
//   warps 2-9   epilogue: a row per thread, two warps per 32-lane quarter, each half of the columns
// Persistent, two accumulators; or SPLIT: a cluster of 2 to 8 CTAs shares a tile's contraction, each leaves its
// partial sums in its shared memory and then adds up a slice of the columns over the cluster, in CTA order.
// Modes:
//   STORE    y, fp32 or bf16
//   GATE_UP  B rows alternate between W1 and W3, so h1 and h3 of a hidden unit are neighbouring columns of one thread:
//            silu(h1) * h3 in fp32, cast to MXFP4 in registers (32 neighbouring units are a block)
//   DOWN     gate-scaled fp32 rows scattered to t*k+slot
// Every wait is bounded (tcx::mbar_wait); a wait that runs out leaves BTX_ERR_TIMEOUT in the status word.
#include <cmath>

#include "btx_mx4_dev.cuh"

namespace btx {
namespace mx4 {
namespace {

constexpr int THREADS = 96 + EPI_WARPS * 32 + 128;
constexpr int RING_BYTES = 220 * 1024;
constexpr int SMEM_BYTES = RING_BYTES + 1024 + 320;
constexpr int PART_PITCH = BN + 4;                       // SPLIT: floats per row of a partial tile (a quad apart: no bank conflicts)
static_assert(MAX_STAGES * 24 + 48 <= 320 && BM * PART_PITCH * 4 <= RING_BYTES, "shared memory");

// SPLIT: a quad of a CTA's partial tile.
__device__ __forceinline__ float4 ld_cluster_v4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
template <int MODE, bool SPLIT>
__global__ void __launch_bounds__(THREADS, 1)
mx4_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t ring = (raw + 1023u) & ~1023u;
  uint8_t* ctl = smem_raw + (ring - raw) + RING_BYTES;
  const uint32_t bar_full = smem_u32(ctl), bar_empty = bar_full + MAX_STAGES * 8;
  const uint32_t bar_tfull = bar_empty + MAX_STAGES * 8, bar_tempty = bar_tfull + 16;
  const uint32_t bar_scales = bar_tempty + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctl + MAX_STAGES * 24 + 32);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctl + MAX_STAGES * 24 + 40);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool turn = MODE == STORE && !SPLIT && !p.wide;   // a piece of the ring turns tiles around
  const int ring_bytes = RING_BYTES - (turn ? EPI_WARPS * TURN_BYTES : 0);
  const int n_stages = stage_count(p.a_rows, ring_bytes), s_bytes = stage_bytes(p.a_rows);

  if (threadIdx.x == 0) {
    for (int s = 0; s < n_stages; ++s) { mbar_init(bar_full + s * 8, 2); mbar_init(bar_empty + s * 8, 1); mbar_init(bar_scales + s * 8, 4); }
    for (int a = 0; a < 2; ++a) { mbar_init(bar_tfull + a * 8, 1); mbar_init(bar_tempty + a * 8, EPI_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  allow_dependents();
  grid_dependency_wait();
  // a product of its own clears its status word (a wait of another CTA cannot have run out yet)
  if (MODE == STORE && blockIdx.x == 0 && threadIdx.x < kStatusWords) p.status[threadIdx.x] = 0;
  const int m_tiles = p.grouped ? p.n_row_tiles[0] : p.m_tiles;
  const int n_total = m_tiles * p.n_tiles * p.batch;
  // SPLIT: one tile per cluster, an even share of its stages per CTA
  const int part = SPLIT ? (int)cluster_ctarank() : 0;
  const int t0 = SPLIT ? (int)blockIdx.x / p.split : (int)blockIdx.x, t_step = SPLIT ? n_total : (int)gridDim.x;
  const int kb_all = (p.K + SK - 1) / SK;
  const int kb0 = SPLIT ? (int)((long long)part * kb_all / p.split) : 0;
  const int kb1 = SPLIT ? (int)((long long)(part + 1) * kb_all / p.split) : kb_all;

  if (warp == 0 || warp == 10) {
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      bool ok = true;
      for (int t = t0; t < n_total && ok; t += t_step) {
        const Item it = get_item(p, m_tiles, t);
        const uint8_t* sfa = p.a_scales + it.b * p.a_scale_batch + (size_t)it.mt * p.kt * kTileBytes;
        const uint8_t* sfb = p.b_scales + it.e * p.b_scale_batch + (size_t)it.nt * p.kt * kTileBytes;
        const int rows = min(p.grouped ? p.tile_rows[it.mt] : p.M - it.mt * BM, p.a_rows);
        const int boxes = (rows + p.a_box - 1) / p.a_box;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!(ok = mbar_wait(bar_empty + stage * 8, phase ^ 1u, abort_flag, p.status))) break;
          const uint32_t bar = bar_full + stage * 8;
          const uint32_t sA = ring + stage * s_bytes, sSA = sA + p.a_rows * (SK / 2), sSB = sSA + SF_BYTES, sB = sSB + SF_BYTES;
          const uint32_t sf = (uint32_t)min(2, p.kt - 2 * kb) * kTileBytes;
          if (warp == 0) {
            mbar_expect_tx(bar, boxes * p.a_box * (SK / 2) + sf);
            for (int i = 0; i < boxes; ++i)
              load_3d(sA + i * p.a_box * (SK / 2), &tmA, kb * (SK / 2), it.mt * BM + i * p.a_box, it.b, bar);
            load_bulk(sSA, sfa + (size_t)kb * 2 * kTileBytes, sf, bar);
          } else {
            mbar_expect_tx(bar, B_BYTES + sf);
            load_3d(sB, &tmB, kb * (SK / 2), it.nt * BN, it.e, bar);
            load_bulk(sSB, sfb + (size_t)kb * 2 * kTileBytes, sf, bar);
          }
          if (++stage == n_stages) { stage = 0; phase ^= 1u; }
        }
      }
      for (int i = 0; i < n_stages && ok; ++i) {          // the MMAs that read the last stages have retired
        ok = mbar_wait(bar_empty + stage * 8, phase ^ 1u, abort_flag, p.status);
        if (++stage == n_stages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      // e2m1 x e2m1 (type code 1), UE8M0 scales, both operands K-major, M 128, N 128; scale selectors per MMA below.
      // The MMA reads 128 rows of A: those past the stage's A part (other bytes of the stage) give rows nobody reads.
      constexpr uint32_t idesc0 = (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | (1u << 23) | ((uint32_t)(BM >> 4) << 24);
      uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
      bool ok = true;
      for (int t = t0; t < n_total && ok; t += t_step) {
        if (!(ok = mbar_wait(bar_tempty + acc * 8, acc_phase ^ 1u, abort_flag, p.status))) break;
        tc_fence_after();
        const uint32_t d = tmem + acc * BN;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!(ok = mbar_wait(bar_full + stage * 8, phase, abort_flag, p.status))) break;
          if (!(ok = mbar_wait(bar_scales + stage * 8, phase, abort_flag, p.status))) break;
          tc_fence_after();
          const uint32_t sA = ring + stage * s_bytes, sB = sA + p.a_rows * (SK / 2) + 2 * SF_BYTES;
          const uint32_t tA = tmem + 2 * BN + stage * SF_COLS, tB = tA + 8;
          const int k64 = min(SK / 64, (p.K - kb * SK + 63) / 64);     // MMAs that hold elements
          const uint64_t da = smem_desc(sA, false), db = smem_desc(sB, false);
#pragma unroll
          for (int j = 0; j < SK / 64; ++j) {
            if (j < k64) {
              const uint32_t id = (uint32_t)(j & 1) * 2;                 // which half of the four scale bytes of a word
              mma_mxf4(d, da + (uint64_t)(2 * j), db + (uint64_t)(2 * j), idesc0 | (id << 4) | (id << 29), tA + (j >> 1) * 4,
                       tB + (j >> 1) * 4, (kb > kb0 || j > 0) ? 1u : 0u);
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
  } else if (warp > 10) {
    uint32_t stage = 0, phase = 0;
    bool ok = true;
    for (int t = t0; t < n_total && ok; t += t_step) {
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!(ok = warp_wait(bar_full + stage * 8, phase, abort_flag, p.status))) break;
        const uint32_t from = ring + stage * s_bytes + p.a_rows * (SK / 2) + lane * 16;
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
    const int q = warp & 3, half = (warp - 2) >> 2;
    const int row = q * 32 + lane;
    uint32_t acc = 0, acc_phase = 0;
    bool ok = true;
    for (int t = t0; t < n_total && ok; t += t_step) {
      const Item it = get_item(p, m_tiles, t);
      const int m = it.mt * BM + row;
      const int flat = MODE == STORE ? (m < p.M ? m : -1) : p.rowmap[m];
      const bool any = __any_sync(0xffffffffu, flat >= 0);
      if (!(ok = warp_wait(bar_tfull + acc * 8, acc_phase, abort_flag, p.status))) break;
      tc_fence_after();
      float v[64];
      if (any) load_chunk(tmem + acc * BN + half * 64 + ((uint32_t)(q * 32) << 16), v);
      tc_fence_before();
      if (lane == 0) arrive(bar_tempty + acc * 8);        // the accumulator is read: the next tile may have it
      if (SPLIT) {
        // every MMA of this CTA has retired and every copy has landed: its ring is free for the partial tile
        if (flat >= 0) {
          const uint32_t to = ring + (uint32_t)(row * PART_PITCH + half * 64) * 4;
#pragma unroll
          for (int i = 0; i < 64; i += 4)
            asm volatile("st.shared::cta.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + i * 4), "f"(v[i]), "f"(v[i + 1]), "f"(v[i + 2]),
                         "f"(v[i + 3]) : "memory");
        }
      } else if (any) {
        if (turn)
          store_turned(p, it, v, it.nt * BN + half * 64, it.mt * BM + q * 32, lane,
                       reinterpret_cast<uint32_t*>(smem_raw + (ring - raw) + ring_bytes + (warp - 2) * TURN_BYTES));
        else
          finish_chunk<MODE>(p, it, v, it.nt * BN + half * 64, m, flat);
      }
      acc ^= 1u;
      if (acc == 0) acc_phase ^= 1u;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
  }
  if constexpr (SPLIT) {
    cluster_sync_all();
    if (t0 < n_total && !*abort_flag) {
      const Item it = get_item(p, m_tiles, t0);
      const int rows = p.grouped ? p.tile_rows[it.mt] : min(BM, p.M - it.mt * BM);
      const int width = BN / p.split, c0 = part * width, n0 = it.nt * BN + c0;
      const int cols = min(width, p.N - n0);
      const int quads = (cols + 3) / 4;                   // (none where cols is negative: the slice lies past the last column)
      for (int i = threadIdx.x; i < rows * quads; i += THREADS) {
        const int r = i / quads, c = (i - r * quads) * 4;
        const uint32_t at = ring + (uint32_t)(r * PART_PITCH + c0 + c) * 4;
        float4 x[8];                                      // all CTAs' loads on their way at once
#pragma unroll
        for (int s = 0; s < 8; ++s)
          if (s < p.split) x[s] = ld_cluster_v4(map_to_cta(at, s));
        float4 a = x[0];
#pragma unroll
        for (int s = 1; s < 8; ++s)
          if (s < p.split) { a.x += x[s].x; a.y += x[s].y; a.z += x[s].z; a.w += x[s].w; }
        if (MODE == DOWN) {
          const int flat = p.rowmap[it.mt * BM + r];
          const float g = p.gates[flat];
          *reinterpret_cast<float4*>((float*)p.y + (size_t)flat * p.N + n0 + c) = make_float4(a.x * g, a.y * g, a.z * g, a.w * g);
        } else {
          const size_t o = ((size_t)it.b * p.M + it.mt * BM + r) * p.N + n0 + c;
          const float f[4] = {a.x, a.y, a.z, a.w};
          if (p.wide) {                                   // whole quads on 16-byte (bf16: 8-byte) boundaries
            if (p.out_bf16) {
              __nv_bfloat162 h[2] = {__floats2bfloat162_rn(a.x, a.y), __floats2bfloat162_rn(a.z, a.w)};
              *reinterpret_cast<uint2*>((__nv_bfloat16*)p.y + o) = *reinterpret_cast<const uint2*>(h);
            } else {
              *reinterpret_cast<float4*>((float*)p.y + o) = a;
            }
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (c + j < cols) {
                if (p.out_bf16) ((__nv_bfloat16*)p.y)[o + j] = __float2bfloat16_rn(f[j]);
                else ((float*)p.y)[o + j] = f[j];
              }
          }
        }
      }
    }
    cluster_sync_all();                                   // nobody leaves while its partial tile is being read
  }
}

// ---------------------------------------------------------------------------------------------
// Two CTAs on one 256 x 256 tile (cta_group::2)
// ---------------------------------------------------------------------------------------------
// A stage brings 128 rows of A and 128 of the 256 rows of B per CTA, half of what two CTAs with tiles of their own
// would fetch for the same products.
// Scales: tcgen05.cp runs in the pipe of the MMAs and took 37 ns a tile of 512 bytes, six of them 220 ns beside the
// 384 ns of a stage's MMAs.  Four warps store the scales instead (tcgen05.st, a warp per 32-lane quarter) from a ring
// of their own in shared memory, and keep up to five stages of scales in tensor memory.  M = 8192, N = 11008,
// K = 11008: 519 us with the copies, 415 us with the four warps reading the tiles from global memory four stages
// ahead (every warp its own copy: a third more traffic from L2), 386 us with the ring.
// Tensor memory: an accumulator takes 256 of the 512 columns, so two do not fit beside the scales whole.  They
// overlap in 128 columns: 0..255 and 128..383.  The epilogue reads the shared columns of a tile into registers first
// and hands them over, so the next tile starts before anything is computed or stored.
//   warp 0  TMA   warp 1  MMAs (one lane of the leader CTA)   warps 2-9  epilogue, two 64-column chunks each
//   warps 10-13  scales   warp 14  TMA of the scales
constexpr int P_STAGES = 6, P_RING = 8;                  // stages of codes, of scales (half of them where tiles are turned around)
constexpr int P_STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int P_SCALE_BYTES = 6 * kTileBytes;            // of a stage and CTA: two tiles of A, two of each half of B
constexpr int P_TURN_MORE = EPI_WARPS * TURN_BYTES - P_RING / 2 * P_SCALE_BYTES;       // beyond the freed half
constexpr int P_SMEM = P_STAGES * P_STAGE_BYTES + P_RING * P_SCALE_BYTES + P_TURN_MORE + 1024 + 384;
constexpr int P_THREADS = 64 + EPI_WARPS * 32 + 160;
constexpr int P_ACC1 = 128, P_SF0 = 384, P_SF_COLS = 24, P_SF_SLOTS = 5;
static_assert(P_SF0 + P_SF_SLOTS * P_SF_COLS <= 512 && P_ACC1 + 256 <= P_SF0, "tensor memory");
static_assert(P_STAGES * 16 + P_SF_SLOTS * 8 + P_RING * 16 + 40 <= 384 && P_SMEM <= 227 * 1024, "shared memory");

__device__ __forceinline__ void mma_mxf4_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                              uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accum) : "memory");
}

template <int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(P_THREADS, 1)
mx4_gemm_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                     const __grid_constant__ CUtensorMap tmSA, const __grid_constant__ CUtensorMap tmSB, const Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t ring = (raw + 1023u) & ~1023u;
  const uint32_t sf_ring = ring + P_STAGES * P_STAGE_BYTES;
  const bool turn = MODE == STORE && !p.wide;
  const uint32_t ring_slots = turn ? P_RING / 2 : P_RING;
  uint8_t* ctl = smem_raw + (sf_ring - raw) + P_RING * P_SCALE_BYTES + P_TURN_MORE;
  const uint32_t bar_full = smem_u32(ctl), bar_empty = bar_full + P_STAGES * 8;
  const uint32_t bar_scales = bar_empty + P_STAGES * 8;                 // used in the leader
  const uint32_t bar_tfull = bar_scales + P_SF_SLOTS * 8, bar_handed = bar_tfull + 16;
  const uint32_t bar_sfull = bar_handed + 8, bar_sempty = bar_sfull + P_RING * 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctl + P_STAGES * 16 + P_SF_SLOTS * 8 + 24 + P_RING * 16);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < P_STAGES; ++s) { mbar_init(bar_full + s * 8, 1); mbar_init(bar_empty + s * 8, 1); }
    for (int s = 0; s < P_SF_SLOTS; ++s) mbar_init(bar_scales + s * 8, 8);
    for (int s = 0; s < P_RING; ++s) { mbar_init(bar_sfull + s * 8, 1); mbar_init(bar_sempty + s * 8, 4); }
    for (int a = 0; a < 2; ++a) mbar_init(bar_tfull + a * 8, 1);
    mbar_init(bar_handed, 2 * EPI_WARPS);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  allow_dependents();
  grid_dependency_wait();
  if (MODE == STORE && blockIdx.x == 0 && threadIdx.x < kStatusWords) p.status[threadIdx.x] = 0;
  const int m_tiles = p.grouped ? p.n_row_tiles[0] / 2 : p.m_tiles;       // of 256 rows
  const int n_total = m_tiles * p.n_tiles * p.batch;
  const int kb_total = (p.K + SK - 1) / SK;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      bool ok = true;
      for (int t = pair; t < n_total && ok; t += n_pairs) {
        const Item it = get_item(p, m_tiles, t);
        const int row0 = it.mt * 256 + (int)rank * 128, col0 = it.nt * 256 + (int)rank * 128;
        for (int kb = 0; kb < kb_total; ++kb) {
          if (!(ok = mbar_wait(bar_empty + stage * 8, phase ^ 1u, abort_flag, p.status))) break;
          const uint32_t full_local = bar_full + stage * 8;
          const uint32_t full = map_to_cta(full_local, 0);
          const uint32_t sA = ring + stage * P_STAGE_BYTES, sB = sA + A_BYTES;
          if (rank == 0) mbar_expect_tx(full_local, 2 * P_STAGE_BYTES);
          tma_load_3d(sA, &tmA, kb * (SK / 2), row0, it.b, full);
          tma_load_3d(sB, &tmB, kb * (SK / 2), col0, it.e, full);
          if (++stage == P_STAGES) { stage = 0; phase ^= 1u; }
        }
      }
      for (int i = 0; i < P_STAGES && ok; ++i) {
        ok = mbar_wait(bar_empty + stage * 8, phase ^ 1u, abort_flag, p.status);
        if (++stage == P_STAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc0 = (1u << 7) | (1u << 10) | ((uint32_t)(256 >> 3) << 17) | (1u << 23) | ((uint32_t)(256 >> 4) << 24);
      uint32_t stage = 0, phase = 0, acc = 0, tile = 0, slot = 0, slot_phase = 0;
      bool ok = true;
      for (int t = pair; t < n_total && ok; t += n_pairs, ++tile) {
        // the tile before has handed over the shared columns
        if (tile > 0 && !(ok = mbar_wait(bar_handed, (tile - 1) & 1u, abort_flag, p.status))) break;
        tc_fence_after();
        const uint32_t d = tmem + (acc ? P_ACC1 : 0);
        for (int kb = 0; kb < kb_total; ++kb) {
          if (!(ok = mbar_wait(bar_scales + slot * 8, slot_phase, abort_flag, p.status))) break;
          if (!(ok = mbar_wait(bar_full + stage * 8, phase, abort_flag, p.status))) break;
          tc_fence_after();
          const uint32_t sA = ring + stage * P_STAGE_BYTES, sB = sA + A_BYTES;
          const uint32_t tA = tmem + P_SF0 + slot * P_SF_COLS, tB = tA + 8;
          if (++slot == P_SF_SLOTS) { slot = 0; slot_phase ^= 1u; }
          const int k64 = min(SK / 64, (p.K - kb * SK + 63) / 64);
          const uint64_t da = smem_desc(sA, false), db = smem_desc(sB, false);
#pragma unroll
          for (int j = 0; j < SK / 64; ++j) {
            if (j < k64) {
              const uint32_t id = (uint32_t)(j & 1) * 2;
              mma_mxf4_pair(d, da + (uint64_t)(2 * j), db + (uint64_t)(2 * j), idesc0 | (id << 4) | (id << 29), tA + (j >> 1) * 4,
                            tB + (j >> 1) * 8, (kb > 0 || j > 0) ? 1u : 0u);
            }
          }
          tc_commit_pair(bar_empty + stage * 8);
          if (++stage == P_STAGES) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        tc_commit_pair(bar_tfull + acc * 8);
        acc ^= 1u;
      }
    }
  } else if (warp == 14) {
    // ---- TMA of the scales; tiles past the end of either matrix arrive as zeros ----
    if (lane == 0) {
      uint32_t slot = 0, phase = 0;
      bool ok = true;
      for (int t = pair; t < n_total && ok; t += n_pairs) {
        const Item it = get_item(p, m_tiles, t);
        const int a_tile = it.b * p.a_row_tiles + it.mt * 2 + (int)rank, b_tile = it.e * p.b_row_tiles + it.nt * 2;
        for (int kb = 0; kb < kb_total; ++kb) {
          if (!(ok = mbar_wait(bar_sempty + slot * 8, phase ^ 1u, abort_flag, p.status))) break;
          const uint32_t bar = bar_sfull + slot * 8, to = sf_ring + slot * P_SCALE_BYTES;
          mbar_expect_tx(bar, P_SCALE_BYTES);
          load_3d(to, &tmSA, 0, kb * 2, a_tile, bar);
          load_3d(to + 2 * kTileBytes, &tmSB, 0, kb * 2, b_tile, bar);
          if (++slot == ring_slots) { slot = 0; phase ^= 1u; }
        }
      }
      for (uint32_t i = 0; i < ring_slots && ok; ++i) {            // every copy has landed and has been read
        ok = mbar_wait(bar_sempty + slot * 8, phase ^ 1u, abort_flag, p.status);
        if (++slot == ring_slots) { slot = 0; phase ^= 1u; }
      }
    }
  } else if (warp >= 2 + EPI_WARPS) {
    // ---- scales: word c of a lane's 16 bytes is row c * 32 + lane of a tile, and column c of tensor memory ----
    const uint32_t taddr = tmem + P_SF0 + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t ready = map_to_cta(bar_scales, 0);
    uint32_t slot = 0, steps = 0, ret_stage = 0, ret_phase = 0, in = 0, in_phase = 0;
    bool ok = true;
    for (int t = pair; t < n_total && ok; t += n_pairs) {
      for (int kb = 0; kb < kb_total; ++kb) {
        if (!(ok = warp_wait(bar_sfull + in * 8, in_phase, abort_flag, p.status))) break;
        uint4 r[6];                                       // A: two tiles along K; B: two of the first half, two of the second
#pragma unroll
        for (int i = 0; i < 6; ++i) r[i] = ld_shared_v4(sf_ring + in * P_SCALE_BYTES + i * kTileBytes + lane * 16);
        if (steps >= P_SF_SLOTS) {                        // the MMAs that read this slot's last scales have retired
          if (!(ok = warp_wait(bar_empty + ret_stage * 8, ret_phase, abort_flag, p.status))) break;
          if (++ret_stage == P_STAGES) { ret_stage = 0; ret_phase ^= 1u; }
          tc_fence_after();
        }
        ++steps;
        const uint32_t to = taddr + slot * P_SF_COLS;
        store_scales(to, r[0], r[1]);
        store_scales(to + 8, r[2], r[4]);
        store_scales(to + 16, r[3], r[5]);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        if (lane == 0) {
          mbar_arrive_cluster(ready + slot * 8);
          arrive(bar_sempty + in * 8);
        }
        if (++slot == P_SF_SLOTS) slot = 0;
        if (++in == ring_slots) { in = 0; in_phase ^= 1u; }
      }
    }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2;
    const int row = q * 32 + lane;
    const uint32_t handed = map_to_cta(bar_handed, 0);
    uint32_t acc = 0, acc_phase = 0;
    bool ok = true;
    for (int t = pair; t < n_total && ok; t += n_pairs) {
      const Item it = get_item(p, m_tiles, t);
      const int m = it.mt * 256 + (int)rank * 128 + row;
      const int flat = MODE == STORE ? (m < p.M ? m : -1) : p.rowmap[m];
      const bool any = __any_sync(0xffffffffu, flat >= 0);
      if (!(ok = warp_wait(bar_tfull + acc * 8, acc_phase, abort_flag, p.status))) break;
      tc_fence_after();
      const uint32_t taddr = tmem + (acc ? P_ACC1 : 0) + ((uint32_t)(q * 32) << 16);
      const int n0 = it.nt * 256;
      // columns 128 .. 255 of tensor memory belong to both accumulators: chunks 2, 3 of the one at 0 and 0, 1 of the other
      const int c0 = (acc ? 0 : 2) + half, c1 = (acc ? 2 : 0) + half;
      float v[64];
      if (any) load_chunk(taddr + c0 * 64, v);
      tc_fence_before();
      if (lane == 0) mbar_arrive_cluster(handed);         // (and all of the tile before has been read)
      auto finish = [&](int c) {
        if (turn)
          store_turned(p, it, v, n0 + c * 64, it.mt * 256 + (int)rank * 128 + q * 32, lane,
                       reinterpret_cast<uint32_t*>(smem_raw + (sf_ring - raw) + P_RING / 2 * P_SCALE_BYTES + (warp - 2) * TURN_BYTES));
        else
          finish_chunk<MODE>(p, it, v, n0 + c * 64, m, flat);
      };
      if (any) {
        finish(c0);
        load_chunk(taddr + c1 * 64, v);
        finish(c1);
      }
      __syncwarp();
      tc_fence_before();
      acc ^= 1u;
      if (acc == 0) acc_phase ^= 1u;
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
  }
}

// scale tiles [row tiles][kt][512 bytes] of all matrices, box of two tiles along K x box_tiles row tiles
bool make_scales_map(CUtensorMap* m, const void* base, long long kt, long long row_tiles, uint32_t box_tiles) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {kTileBytes / 4, (cuuint64_t)kt, (cuuint64_t)row_tiles};
  cuuint64_t strides[2] = {kTileBytes, (cuuint64_t)(kt * kTileBytes)};
  cuuint32_t box[3] = {kTileBytes / 4, 2, box_tiles};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_INT32, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int MODE, bool SPLIT>
btx_status launch(const GemmArgs& g, const Params& p, long long max_tiles, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  CUtensorMap a, b;
  if (!make_codes_map(&a, g.a_codes, g.K, g.M, g.batch, p.a_box) || !make_codes_map(&b, g.b_codes, g.K, g.N, g.experts, BN) ||
      !allow_smem((const void*)mx4_gemm_kernel<MODE, SPLIT>, SMEM_BYTES, done))
    return BTX_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  const long long blocks = SPLIT ? max_tiles * p.split : (max_tiles < sm_count() ? max_tiles : sm_count());
  cfg.gridDim = dim3((unsigned)blocks); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = SMEM_BYTES; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;      // a programmatic dependent of the kernel before it
  attr[n++].val.programmaticStreamSerializationAllowed = 1;
  if (SPLIT) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = p.split; attr[n].val.clusterDim.y = 1; attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr; cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, mx4_gemm_kernel<MODE, SPLIT>, a, b, p) == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

// CTAs per tile: as many as keep every multiprocessor busy at most once, with two stages each at least
int split_of(long long tiles, long long K) {
  int s = 1;
  while (s < 8 && 2 * s * tiles <= sm_count() && 4 * s <= (K + SK - 1) / SK) s *= 2;
  return s;
}

template <int MODE>
btx_status launch_pair(const GemmArgs& g, Params p, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  CUtensorMap a, b, sa, sb;
  p.m_tiles = (g.M + 255) / 256; p.n_tiles = (g.N + 255) / 256; p.tile_step = 2;
  if (!make_codes_map(&a, g.a_codes, g.K, g.M, g.batch, 128) || !make_codes_map(&b, g.b_codes, g.K, g.N, g.experts, 128) ||
      !make_scales_map(&sa, g.a_scales, p.kt, (long long)p.a_row_tiles * g.batch, 1) ||
      !make_scales_map(&sb, g.b_scales, p.kt, (long long)p.b_row_tiles * g.experts, 2) ||
      !allow_smem((const void*)mx4_gemm_pair_kernel<MODE>, P_SMEM, done))
    return BTX_ERR_CUDA;
  const long long items = (long long)p.m_tiles * p.n_tiles * p.batch;
  int pairs = sm_count() / 2;
  if (items < pairs) pairs = (int)items;
  return launch_after_predecessor(mx4_gemm_pair_kernel<MODE>, dim3(2 * pairs), dim3(P_THREADS), P_SMEM, st, true, a, b, sa,
                                  sb, p) == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

Params base_params(const GemmArgs& g) {
  Params p = {};
  p.M = g.M; p.N = g.N; p.K = g.K; p.batch = g.batch; p.status = g.status;
  p.m_tiles = (g.M + BM - 1) / BM; p.n_tiles = (g.N + BN - 1) / BN; p.split = 1;
  p.kt = (int)scale_tiles_k(g.K); p.tile_step = 1;
  p.a_row_tiles = (g.M + kTileRows - 1) / kTileRows; p.b_row_tiles = (g.N + kTileRows - 1) / kTileRows;
  p.a_scales = g.a_scales; p.b_scales = g.b_scales;
  p.a_scale_batch = (long long)p.m_tiles * p.kt * kTileBytes;
  p.b_scale_batch = (long long)((g.N + kTileRows - 1) / kTileRows) * p.kt * kTileBytes;
  return p;
}

// Which kernel a product takes: rounds of tiles over the multiprocessors times the time of a tile, in measured us: 0.38 a
// stage of a 128 x 128 tile (its contraction split over a cluster where that keeps CTAs busy) and 0.47 of a 256 x 256 tile,
// or the epilogue `epi` of the larger tile (the smaller one's takes half) where that is longer, and what a tile costs
// beside them.  E.g. N = 4096, K = 4096: 512 rows 10.1 and 11.3 us, 768 rows 16.0 and 12.0 us; N = 4096, K = 11008: 256
// rows 14.6 and 21.4, 768 rows 35.7 and 22.8; N = 11008, K = 4096: 192 rows 15.6 and 11.8, 384 rows 16.4 and 18.4.
double single_us(double tiles, long long K, double epi) {
  const double split = split_of((long long)(tiles + 0.5), K), kb = (double)((K + SK - 1) / SK);
  return ceil(tiles * split / sm_count()) * (fmax(ceil(kb / split) * 0.38, epi / 2) + 0.4);
}
double pair_us(double tiles, long long K, double epi) {
  return ceil(tiles / (sm_count() / 2)) * (fmax((double)((K + SK - 1) / SK) * 0.47, epi) + 0.85);
}
constexpr double kStoreUs = 2.0, kGateUpUs = 5.5, kDownUs = 3.5;       // epilogues of a 256 x 256 tile

}  // namespace

// The expert layer's two products, for experts with about rows / experts rows each (a tile more than they fill for
// every second).  d = 4096, F = 11008, 4 experts, top-2: 128 tokens take 73 us on single CTAs and 82 on pairs, 256 tokens
// 106 and 86, 1024 tokens 253 and 180.  d = 2048, F = 1024, 64 experts, top-8: 1024 tokens 113 and 126.
bool pairs_fit(long long rows, long long experts, long long d, long long F) {
  if (rows == 0) return false;
  const double each = (double)rows / (double)experts;
  const double t1 = experts * fmax(1.0, each / 128 + 0.5), t2 = experts * fmax(1.0, each / 256 + 0.5);
  const double n1 = (double)((2 * F + 127) / 128), m1 = (double)((d + 127) / 128);
  const double n2 = (double)((2 * F + 255) / 256), m2 = (double)((d + 255) / 256);
  return pair_us(t2 * n2, d, kGateUpUs) + pair_us(t2 * m2, F, kDownUs) <
         single_us(t1 * n1, d, kGateUpUs) + single_us(t1 * m1, F, kDownUs);
}

btx_status launch_matmul(const GemmArgs& g, int dtype, void* y, cudaStream_t st) {
  Params p = base_params(g);
  p.y = y; p.out_bf16 = dtype == BTX_BF16;
  p.wide = aligned32(y) && (size_t)g.N * (p.out_bf16 ? 2 : 4) % 32 == 0;
  const long long tiles = (long long)p.m_tiles * p.n_tiles * p.batch;
  if (pair_us((double)g.batch * ((g.M + 255) / 256) * ((g.N + 255) / 256), g.K, kStoreUs) < single_us((double)tiles, g.K, kStoreUs))
    return launch_pair<STORE>(g, p, st);
  p.a_rows = p.a_box = g.M < BM ? (g.M + 31) / 32 * 32 : BM;
  p.split = split_of(tiles, g.K);
  return p.split > 1 ? launch<STORE, true>(g, p, tiles, st) : launch<STORE, false>(g, p, tiles, st);
}

static Params grouped_params(const GemmArgs& g, const Dispatch& q) {
  Params p = base_params(g);
  p.grouped = 1; p.n_row_tiles = q.n_tiles; p.tile_expert = q.tile_expert; p.tile_rows = q.tile_rows; p.rowmap = q.rowmap;
  // a tile holds at most R rows; in small batches few of its rows are used, and only those are fetched
  p.a_rows = q.R < BM ? (q.R + 31) / 32 * 32 : BM;
  p.a_box = q.R <= 16 * BM ? 32 : BM;
  return p;
}

btx_status launch_gate_up(const GemmArgs& g, const Dispatch& q, uint8_t* act_codes, uint8_t* act_scales, cudaStream_t st) {
  Params p = grouped_params(g, q);
  p.act_codes = act_codes; p.act_scales = act_scales;
  if (q.pad_tiles == 2) return launch_pair<GATE_UP>(g, p, st);
  return launch<GATE_UP, false>(g, p, (long long)p.m_tiles * p.n_tiles, st);
}

btx_status launch_down(const GemmArgs& g, const Dispatch& q, const float* gates, float* rows, cudaStream_t st) {
  Params p = grouped_params(g, q);
  p.gates = gates; p.y = rows; p.wide = 1;                // rows of a multiple of 32 columns in a workspace region
  if (q.pad_tiles == 2) return launch_pair<DOWN>(g, p, st);
  const long long tiles = (long long)p.m_tiles * p.n_tiles;
  p.split = split_of(tiles, g.K);
  return p.split > 1 ? launch<DOWN, true>(g, p, tiles, st) : launch<DOWN, false>(g, p, tiles, st);
}

}  // namespace mx4
}  // namespace btx

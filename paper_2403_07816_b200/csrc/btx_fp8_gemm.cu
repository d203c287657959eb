// Products of FP8 matrices on the 5th-generation tensor cores (tcgen05.mma kind::mxf8f6f4.block_scale): codes straight from
// memory to shared memory by TMA, scales through shared memory into tensor memory (tcgen05.cp), fp32 sums in tensor memory.
// y = A B^T with both operands K-major, per output element
//   sum over blocks of 128:  2^(sa - 127) 2^(sb - 127) sum a_i b_i.
// An MMA covers 32 contraction elements and takes one scale per row for them; the four MMAs of a block name the same byte of
// the row's word in tensor memory, the four blocks of a scale tile the four bytes in turn.  So one 512-byte tile of 128 rows
// serves 512 contraction elements, and nothing is scaled or summed outside the tensor core.
//
// Two kernels, as for MXFP4: fp8_gemm_kernel, a CTA per tile of 128 rows and 64 or 128 columns, for few rows (bound by reading B), and
// fp8_gemm_pair_kernel, two CTAs per 256 x 256 tile, for many (bound by the tensor cores and their power).
//
// Measured on one B200 (replayed): 1 x 4096 x 11008 12.5-13.3 us (45 MB of B, 6.9 at the rate of a copy), 333 x 1001 x 2083 9.0,
// 1024 x 4096 x 4096 16.4-16.8; 8192 x 11008 x 4096 256-267 us in short runs, 2.8 PFLOP/s, and 307 under the power limit, 2.4 PFLOP/s
// (a library product with one scale for each operand 301).  At 4001 x 4096 x 11008 256 tiles on 74 pairs are four
// rounds where 3.46 would do: 163 us (143).  The tensor pipe is active 65-69 % of the time in the pair kernel; in the layer of 32
// tokens gate_up reads its 361 MB at 5.3 TB/s.
//
// fp8_gemm_kernel:
//   warp 0, 10  TMA producers (one lane each) of A and of B: ring of stages of 128 contraction elements, a block (swizzled rows
//               of 128 bytes), and in every fourth stage a scale tile of each.  Of A a stage holds only as many rows as a
//               tile can have (a multiple of 32)
//   warp 1      allocates tensor memory; copies scale tiles there (tcgen05.cp: two tiles for sixteen MMAs; warps that store them
//               cost 0.7 us a tile, which was the time of four stages) and issues up to four MMAs per stage
//   warps 2-9   epilogue: a row per thread, two warps per 32-lane quarter, each half of the columns
// Persistent, two accumulators; or SPLIT: a cluster of 2 to 8 CTAs shares a tile's contraction, each leaves its
// partial sums in its shared memory and then adds up a slice of the columns over the cluster, in CTA order.
// Modes:
//   STORE    y, fp32 or bf16, or added to the fp32 that is there
//   GATE_UP  B rows alternate between W1 and W3, so h1 and h3 of a hidden unit are neighbouring columns of one thread:
//            silu(h1) * h3 in fp32, cast to FP8.  A block of 128 hidden units is 256 columns: a cluster of two CTAs works on
//            neighbouring tiles, and every thread hands the largest of its 32 units to the other three that share its row
//   DOWN     gate-scaled fp32 rows scattered to t*k+slot
// Every wait is bounded (tcx::mbar_wait); a wait that runs out leaves BTX_ERR_TIMEOUT in the status word.
#include <cmath>

#include "btx_fp8_dev.cuh"
#include "btx_fp8_gemm.cuh"
#include "btx_mx4_dev.cuh"

namespace btx {
namespace fp8 {
namespace {

using namespace tcx;
using mx4::arrive;
using mx4::BM;
using mx4::BN;
using mx4::EPI_WARPS;
using mx4::get_item;
using mx4::Item;
using mx4::load_3d;
using mx4::load_bulk;
using mx4::load_chunk;
using mx4::TURN_BYTES;
using mx4::warp_wait;
using mx4::STORE;
using mx4::GATE_UP;
using mx4::DOWN;

constexpr int SKB = 128;                                 // contraction elements (and bytes of a row) per stage: a block
constexpr int SF_GROUP = 4;                              // stages that a scale tile serves
constexpr int A_BYTES = BM * SKB, B_BYTES = BN * SKB;

struct Params : mx4::Params {
  int accumulate;                                        // STORE: fp32 y is added to
  int width;                                             // columns of a tile: 64 or 128 (pairs of CTAs: 256)
};

// The MMAs of a stage, `n` of 32 contraction elements each, issued by the lane whose `leader` is not 0; a, b: the low words of the
// operands' descriptors.  The whole warp comes here: operands of an MMA are uniform registers, and in code for one lane
// each of them is moved there first, which took longer than the MMAs (86 stages of 4 on a tile of 128 columns: 0.36 us a
// stage, whatever the columns; 0.29 so).
constexpr uint32_t kDescHigh = (1024u >> 4) | 1u << 14 | 2u << 29;       // of tcx::smem_desc, K-major
__device__ __forceinline__ uint32_t desc_low(uint32_t addr) { return (addr & 0x3FFFFu) >> 4 | (16u >> 4) << 16; }
#define BTX_FP8_MMA(GROUP, P, A, B, F) \
  "@" P " tcgen05.mma.cta_group::" #GROUP ".kind::mxf8f6f4.block_scale.scale_vec::1X [%0], " A ", " B ", %3, [%4], [%5], " F ";\n\t"
#define BTX_FP8_MMAS(GROUP)                                                                                                  \
  if (n == 4) {                                                                                                              \
    asm volatile(                                                                                                            \
        "{\n\t.reg .pred l, f, t;\n\t.reg .b32 x;\n\t.reg .b64 a0, a1, a2, a3, b0, b1, b2, b3;\n\t"                          \
        "setp.ne.b32 l, %7, 0;\n\tsetp.ne.b32 f, %6, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"                                         \
        "mov.b64 a0, {%1, %8};\n\tmov.b64 b0, {%2, %8};\n\tadd.s32 x, %1, 2;\n\tmov.b64 a1, {x, %8};\n\t"                    \
        "add.s32 x, %2, 2;\n\tmov.b64 b1, {x, %8};\n\tadd.s32 x, %1, 4;\n\tmov.b64 a2, {x, %8};\n\t"                         \
        "add.s32 x, %2, 4;\n\tmov.b64 b2, {x, %8};\n\tadd.s32 x, %1, 6;\n\tmov.b64 a3, {x, %8};\n\t"                         \
        "add.s32 x, %2, 6;\n\tmov.b64 b3, {x, %8};\n\t"                                                                      \
        BTX_FP8_MMA(GROUP, "l", "a0", "b0", "f") BTX_FP8_MMA(GROUP, "l", "a1", "b1", "t")                                    \
        BTX_FP8_MMA(GROUP, "l", "a2", "b2", "t") BTX_FP8_MMA(GROUP, "l", "a3", "b3", "t") "}"                                \
        ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accum), "r"(leader), "r"(kDescHigh) : "memory");       \
  } else {                                                                                                                   \
    for (int j = 0; j < n; ++j)                                                                                              \
      asm volatile("{\n\t.reg .pred l, f;\n\t.reg .b64 a0, b0;\n\tsetp.ne.b32 l, %7, 0;\n\tsetp.ne.b32 f, %6, 0;\n\t"         \
                   "mov.b64 a0, {%1, %8};\n\tmov.b64 b0, {%2, %8};\n\t" BTX_FP8_MMA(GROUP, "l", "a0", "b0", "f") "}"         \
                   ::"r"(d), "r"(a + 2 * j), "r"(b + 2 * j), "r"(idesc), "r"(sfa), "r"(sfb), "r"(j > 0 ? 1u : accum),        \
                   "r"(leader), "r"(kDescHigh) : "memory");                                                                  \
  }
__device__ __forceinline__ void mma_stage(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accum,
                                          uint32_t leader, int n) {
  BTX_FP8_MMAS(1)
}
__device__ __forceinline__ void mma_stage_pair(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                               uint32_t accum, uint32_t leader, int n) {
  BTX_FP8_MMAS(2)
}
#undef BTX_FP8_MMAS
#undef BTX_FP8_MMA
__device__ __forceinline__ void commit_if(uint32_t bar, uint32_t leader) {
  asm volatile("{\n\t.reg .pred l;\n\tsetp.ne.b32 l, %1, 0;\n\t"
               "@l tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(leader) : "memory");
}
__device__ __forceinline__ void commit_pair_if(uint32_t bar, uint32_t leader) {
  asm volatile("{\n\t.reg .pred l;\n\tsetp.ne.b32 l, %1, 0;\n\t"
               "@l tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %2;\n\t}"
               ::"r"(bar), "r"(leader), "h"((uint16_t)3) : "memory");
}
// e4m3 x e4m3 (type code 0), UE8M0 scales, both operands K-major; byte `id` of the words of scales
__device__ __forceinline__ constexpr uint32_t instr(int m, int n, uint32_t id) {
  return ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 4) << 24) | (id << 4) | (id << 29);
}
// A scale tile (32 rows of 16 bytes: no swizzle, core matrices of eight rows 128 bytes apart) to four columns of tensor memory,
// repeated in every 32-lane quarter; of a pair, in both CTAs, each from its own shared memory to its own tensor memory.
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t smem, uint32_t leader) {
  asm volatile("{\n\t.reg .pred l;\n\t.reg .b64 d;\n\tsetp.ne.b32 l, %3, 0;\n\tmov.b64 d, {%1, %2};\n\t"
               "@l tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], d;\n\t}"
               ::"r"(tmem), "r"((smem & 0x3FFFFu) >> 4 | (128u >> 4) << 16), "r"((128u >> 4) | 1u << 14), "r"(leader) : "memory");
}
__device__ __forceinline__ void copy_scales_pair(uint32_t tmem, uint32_t smem, uint32_t leader) {
  asm volatile("{\n\t.reg .pred l;\n\t.reg .b64 d;\n\tsetp.ne.b32 l, %3, 0;\n\tmov.b64 d, {%1, %2};\n\t"
               "@l tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], d;\n\t}"
               ::"r"(tmem), "r"((smem & 0x3FFFFu) >> 4 | (128u >> 4) << 16), "r"((128u >> 4) | 1u << 14), "r"(leader) : "memory");
}
// A word into CTA `rank`'s shared memory at the offset of `slot`; four bytes complete on its barrier at the offset of `bar`.
__device__ __forceinline__ void send_word(uint32_t slot, uint32_t bar, uint32_t rank, uint32_t value) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];"
               ::"r"(map_to_cta(slot, rank)), "r"(value), "r"(map_to_cta(bar, rank)) : "memory");
}
__device__ __forceinline__ void st_shared_u32(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cta.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ float4 ld_cluster_v4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

// silu(h1) h3 in fp32, within 9 * 2^-24: expf counts for two units of the last place, the reciprocal for one, and there are three
// roundings (below h1 = -87, where 1 / (1 + e) is subnormal or 0, within 2^-119 |h3|).  The activations are cast to FP8, where
// whatever passes a border moves by a whole step: not the place for the fast exponential, whose error grows with |h1|.  The
// correctly rounded reciprocal has a branch that keeps the units of a thread one behind the other: T = 4096, 8 experts, d = 512,
// F = 2048, top-2 121 us with it, 84 without; 64 experts, d = 2048, F = 1024, top-8 365 and 320.
__device__ __forceinline__ float swiglu(float h1, float h3) {
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(1.0f + expf(-h1)));       // (infinity: 0)
  return h1 * r * h3;
}

// N/2 hidden units from N accumulator columns n0 .. (h1 and h3 in turn), 0 past the last unit, where the columns are those of
// scales that nobody wrote; their largest magnitude joins `amax`.
template <int N>
__device__ __forceinline__ void units(const float (&v)[N], int f0, int F, float* a, uint32_t& amax) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    a[i] = f0 + i < F ? swiglu(v[2 * i], v[2 * i + 1]) : 0.f;
    amax = max(amax, __float_as_uint(a[i]) & 0x7fffffffu);
  }
}
// 32 units f0 .. of row m of the activations (F is a multiple of 16)
__device__ __forceinline__ void store_units(const Params& p, const float* a, int f0, int F, int m, uint32_t byte, uint32_t inv_bits) {
  uint8_t* to = p.act_codes + (size_t)m * row_pitch(F) + f0;
#pragma unroll
  for (int h = 0; h < 32; h += 16) {
    if (f0 + h >= F) break;
    float v[16];
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = a[h + i];
    cast_codes(v, byte, inv_bits, q);
    *reinterpret_cast<uint4*>(to + h) = make_uint4(q[0], q[1], q[2], q[3]);
  }
}

// What becomes of 64 accumulator columns n0 .. of a row, of which those below n1 are the tile's.  flat: the row of y (STORE) or
// its assignment, -1 for a row that nobody asked for.
template <int MODE>
__device__ __forceinline__ void put_chunk(const Params& p, const Item& it, float (&v)[64], int n0, int n1, int flat) {
  if (flat < 0 || n0 >= n1) return;
  const size_t o = (MODE == STORE ? ((size_t)it.b * p.M + flat) * p.N : (size_t)flat * p.N) + n0;
  const bool whole = p.wide && n0 + 64 <= n1;
  if (MODE == DOWN) {
    const float g = p.gates[flat];
#pragma unroll
    for (int i = 0; i < 64; ++i) v[i] *= g;
  }
  if (MODE == STORE && p.out_bf16) {
    __nv_bfloat16* y = (__nv_bfloat16*)p.y + o;
    if (whole) {
#pragma unroll
      for (int i = 0; i < 64; i += 16) st32(y + i, pack8(v + i), pack8(v + i + 8), true);
    } else {
#pragma unroll
      for (int i = 0; i < 64; ++i)
        if (n0 + i < n1) y[i] = __float2bfloat16_rn(v[i]);
    }
    return;
  }
  float* y = (float*)p.y + o;
  if (whole) {
    if (MODE == STORE && p.accumulate) {
#pragma unroll
      for (int i = 0; i < 64; i += 4) {
        const float4 q = *reinterpret_cast<const float4*>(y + i);
        v[i] += q.x; v[i + 1] += q.y; v[i + 2] += q.z; v[i + 3] += q.w;
      }
    }
#pragma unroll
    for (int i = 0; i < 64; i += 8) st32(y + i, f4(v + i), f4(v + i + 4), true);
  } else {
#pragma unroll
    for (int i = 0; i < 64; ++i)
      if (n0 + i < n1) y[i] = MODE == STORE && p.accumulate ? v[i] + y[i] : v[i];
  }
}
// STORE where rows of y do not start on 32-byte boundaries: a warp turns its 32 rows through shared memory
__device__ __forceinline__ void put_turned(const Params& p, const Item& it, float (&v)[64], int n0, int n1, int m0, int lane, uint32_t* st) {
  if (n0 >= n1) return;
  const size_t o = ((size_t)it.b * p.M + m0) * p.N + n0;
  const int rows = p.M - m0, cols = n1 - n0;
  if (!p.out_bf16) {
    if (p.accumulate && lane < rows) {
      const float* y = (const float*)p.y + o + (size_t)lane * p.N;
#pragma unroll
      for (int i = 0; i < 64; ++i)
        if (i < cols) v[i] += y[i];
    }
    mx4::turn_words<uint32_t, 1>((uint32_t*)p.y + o, p.N, rows, cols, lane, st, [&](int i) { return __float_as_uint(v[i]); });
  } else if ((p.N & 1) == 0 && ((uintptr_t)p.y & 3) == 0) {
    mx4::turn_words<uint32_t, 2>((uint32_t*)((__nv_bfloat16*)p.y + o), p.N, rows, cols, lane, st, [&](int i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      return *reinterpret_cast<const uint32_t*>(&h);
    });
  } else {
    mx4::turn_words<uint16_t, 1>((uint16_t*)p.y + o, p.N, rows, cols, lane, st, [&](int i) {
      return (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v[i]));
    });
  }
}

// ---------------------------------------------------------------------------------------------
// One CTA on a tile of 128 rows and up to 128 columns
// ---------------------------------------------------------------------------------------------
constexpr int THREADS = 96 + EPI_WARPS * 32;
constexpr int MAX_STAGES = 20;
constexpr int SF_BYTES = 2 * kTileBytes;                 // of a stage: scale tiles of A and of B
constexpr int SF_COLS = 8, SF_COL0 = 2 * BN, SF_SLOTS = 8;               // tensor memory: scale tiles of the last eight copies
constexpr int XCH_BYTES = 2 * 4 * BM * 4;                // GATE_UP: two tiles' largest units, four for every row
constexpr int RING_BYTES = 219 * 1024;
constexpr int CTL_BYTES = 384;
constexpr int SMEM_BYTES = RING_BYTES + XCH_BYTES + CTL_BYTES + 1024;
constexpr int PART_PITCH = BN + 4;                       // SPLIT: floats per row of a partial tile (a quad apart: no bank conflicts)
static_assert(SMEM_BYTES <= 227 * 1024 && BM * PART_PITCH * 4 <= RING_BYTES && SF_COL0 + SF_SLOTS * SF_COLS <= 512, "memory");
static_assert(MAX_STAGES * 16 + 48 + 16 <= CTL_BYTES, "control block");

template <int MODE, bool SPLIT>
__global__ void __launch_bounds__(THREADS, 1)
fp8_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t ring = (raw + 1023u) & ~1023u;
  const uint32_t xch = ring + RING_BYTES;
  uint8_t* ctl = smem_raw + (xch + XCH_BYTES - raw);
  const uint32_t bar_full = smem_u32(ctl), bar_empty = bar_full + MAX_STAGES * 8;
  const uint32_t bar_tfull = bar_empty + MAX_STAGES * 8, bar_tempty = bar_tfull + 16, bar_xch = bar_tempty + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctl + MAX_STAGES * 16 + 48);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = __shfl_sync(kAll, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  constexpr bool TWIN = MODE == GATE_UP;                  // a cluster of two CTAs on neighbouring column tiles
  const bool turn = MODE == STORE && !SPLIT && !p.wide;   // a piece of the ring turns tiles around
  const int ring_bytes = RING_BYTES - (turn ? EPI_WARPS * TURN_BYTES : 0);
  // Codes of the stages (an MMA reads 128 rows of A, from the last one too: they come first), then their scales.
  const int s_bytes = (p.a_rows + p.width) * SKB;
  const int n_stages = min(MAX_STAGES, (ring_bytes - max(0, A_BYTES - s_bytes)) / (s_bytes + SF_BYTES));
  const uint32_t scales = ring + n_stages * s_bytes;

  if (threadIdx.x == 0) {
    for (int s = 0; s < n_stages; ++s) { mbar_init(bar_full + s * 8, 2); mbar_init(bar_empty + s * 8, 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(bar_tfull + a * 8, 1); mbar_init(bar_tempty + a * 8, EPI_WARPS); mbar_init(bar_xch + a * 8, 1); }
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
  if (TWIN) cluster_sync_all();                           // the twin's barriers exist before anyone signals them
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  allow_dependents();
  // The layer's weights, and what its dispatch wrote, do not come from the kernel before (which let this one start only after
  // the dispatch was done): they are on their way while it runs.
  if (MODE == STORE || warp != 10) grid_dependency_wait();
  // a product of its own clears its status word (a wait of another CTA cannot have run out yet)
  if (MODE == STORE && blockIdx.x == 0 && threadIdx.x < kStatusWords) p.status[threadIdx.x] = 0;
  const int m_tiles = p.grouped ? p.n_row_tiles[0] : p.m_tiles;
  const int n_total = m_tiles * p.n_tiles * p.batch;      // TWIN: n_tiles counts pairs of column tiles
  // SPLIT: one tile per cluster, an even share of its stages per CTA
  const int rank = SPLIT || TWIN ? (int)cluster_ctarank() : 0;
  const int t0 = SPLIT ? (int)blockIdx.x / p.split : TWIN ? (int)blockIdx.x >> 1 : (int)blockIdx.x;
  const int t_step = SPLIT ? n_total : TWIN ? (int)gridDim.x >> 1 : (int)gridDim.x;
  const int kb_all = (p.K + SKB - 1) / SKB;
  const int kb0 = SPLIT ? (int)((long long)rank * kb_all / p.split) : 0;
  const int kb1 = SPLIT ? (int)((long long)(rank + 1) * kb_all / p.split) : kb_all;
  auto item = [&](int t) {
    Item it = get_item(p, m_tiles, t);
    if (TWIN) it.nt = it.nt * 2 + rank;
    return it;
  };

  if (warp == 0 || warp == 10) {
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      bool ok = true;
      for (int t = t0; t < n_total && ok; t += t_step) {
        const Item it = item(t);
        const int rows = min(p.grouped ? p.tile_rows[it.mt] : p.M - it.mt * BM, p.a_rows);
        const int boxes = (rows + p.a_box - 1) / p.a_box;
        const uint8_t* sf = warp == 0 ? p.a_scales + it.b * p.a_scale_batch + (size_t)it.mt * p.kt * kTileBytes
                                      : p.b_scales + it.e * p.b_scale_batch +
                                            (size_t)min(it.nt * p.width / kTileRows, p.b_row_tiles - 1) * p.kt * kTileBytes;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!(ok = mbar_wait(bar_empty + stage * 8, phase ^ 1u, abort_flag, p.status))) break;
          const uint32_t bar = bar_full + stage * 8, sA = ring + stage * s_bytes, sS = scales + stage * SF_BYTES;
          const bool first = kb % SF_GROUP == 0 || kb == kb0;            // brings the scales of its group
          if (warp == 0) {
            mbar_expect_tx(bar, boxes * p.a_box * SKB + (first ? kTileBytes : 0));
            for (int i = 0; i < boxes; ++i) load_3d(sA + i * p.a_box * SKB, &tmA, kb * SKB, it.mt * BM + i * p.a_box, it.b, bar);
          } else {
            mbar_expect_tx(bar, p.width * SKB + (first ? kTileBytes : 0));
            load_3d(sA + p.a_rows * SKB, &tmB, kb * SKB, it.nt * p.width, it.e, bar);
          }
          if (first) load_bulk(warp == 0 ? sS : sS + kTileBytes, sf + (size_t)(kb / SF_GROUP) * kTileBytes, kTileBytes, bar);
          if (++stage == n_stages) { stage = 0; phase ^= 1u; }
        }
      }
      for (int i = 0; i < n_stages && ok; ++i) {          // the MMAs that read the last stages have retired
        ok = mbar_wait(bar_empty + stage * 8, phase ^ 1u, abort_flag, p.status);
        if (++stage == n_stages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // The MMA reads 128 rows of A: those past the stage's A part (other bytes of the ring) give rows nobody reads.
    const uint32_t leader = lane == 0;
    uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0, slot = 0;
    const uint32_t low_b = p.a_rows * SKB >> 4, idesc0 = instr(BM, p.width, 0);
    const int tail = (p.K - (kb_all - 1) * SKB + 31) / 32;               // MMAs of the last stage that hold elements
    bool ok = true;
    for (int t = t0; t < n_total && ok; t += t_step) {
      const uint32_t b_col = 4 + item(t).nt * p.width % kTileRows / 32;  // of the tile's first column among those of the scales
      if (!(ok = warp_wait(bar_tempty + acc * 8, acc_phase ^ 1u, abort_flag, p.status))) break;
      const uint32_t d = tmem + acc * BN;
      uint32_t tA = 0;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!(ok = warp_wait(bar_full + stage * 8, phase, abort_flag, p.status))) break;
        tc_fence_after();
        const uint32_t id = kb % SF_GROUP, low = desc_low(ring + stage * s_bytes);
        if (id == 0 || kb == kb0) {
          tA = tmem + SF_COL0 + slot * SF_COLS;
          slot = (slot + 1) % SF_SLOTS;
          copy_scales(tA, scales + stage * SF_BYTES, leader);
          copy_scales(tA + 4, scales + stage * SF_BYTES + kTileBytes, leader);
        }
        mma_stage(d, low, low + low_b, idesc0 | id << 4 | id << 29, tA, tA + b_col, kb > kb0, leader, kb == kb_all - 1 ? tail : SKB / 32);
        commit_if(bar_empty + stage * 8, leader);
        if (++stage == n_stages) { stage = 0; phase ^= 1u; }
      }
      if (!ok) break;
      commit_if(bar_tfull + acc * 8, leader);
      acc ^= 1u;
      if (acc == 0) acc_phase ^= 1u;
    }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2;
    const int row = q * 32 + lane;
    uint32_t acc = 0, acc_phase = 0;
    bool ok = true;
    for (int t = t0; t < n_total && ok; t += t_step) {
      const Item it = item(t);
      const int m = it.mt * BM + row;
      const int flat = MODE == STORE ? (m < p.M ? m : -1) : p.rowmap[m];
      const bool any = __any_sync(kAll, flat >= 0);
      if (!(ok = warp_wait(bar_tfull + acc * 8, acc_phase, abort_flag, p.status))) break;
      tc_fence_after();
      float v[64];
      if (any) load_chunk(tmem + acc * BN + half * 64 + ((uint32_t)(q * 32) << 16), v);
      tc_fence_before();
      if (lane == 0) arrive(bar_tempty + acc * 8);        // the accumulator is read: the next tile may have it
      const int n0 = it.nt * p.width + half * 64, n1 = min(p.N, (it.nt + 1) * p.width);
      if (MODE == GATE_UP) {
        // A tile's maxima take place acc of two: nobody writes to it again before everybody has passed the next tile's barrier.
        const int F = p.N / 2, f0 = n0 / 2;
        float a[32];
        uint32_t most = 0;
        if (flat >= 0) units(v, f0, F, a, most);
        const uint32_t bar = bar_xch + acc * 8, at = xch + (acc * 4 * BM + row) * 4;
        send_word(at + (rank * 2 + half) * BM * 4, bar, 0, most);
        send_word(at + (rank * 2 + half) * BM * 4, bar, 1, most);
        if (threadIdx.x == 64) mbar_expect_tx(bar, 4 * BM * 4);
        if (!(ok = warp_wait(bar, acc_phase, abort_flag, p.status))) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max(most, ld_shared_u32(at + i * BM * 4));
        uint32_t inv;
        const uint32_t byte = scale_byte(most, inv);
        if (flat >= 0 && f0 < F) {
          store_units(p, a, f0, F, m, byte, inv);
          if (f0 % kBlock == 0) p.act_scales[scale_offset(0, m, (int)scale_tiles_k(F), f0 / kBlock)] = (uint8_t)byte;
        }
      } else if (SPLIT) {
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
          put_turned(p, it, v, n0, n1, it.mt * BM + q * 32, lane,
                     reinterpret_cast<uint32_t*>(smem_raw + (ring - raw) + ring_bytes + (warp - 2) * TURN_BYTES));
        else
          put_chunk<MODE>(p, it, v, n0, n1, flat);
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
  if (TWIN) cluster_sync_all();                           // nobody leaves while its twin may still send
  if constexpr (SPLIT) {
    cluster_sync_all();
    if (t0 < n_total && !*abort_flag) {
      const Item it = item(t0);
      const int rows = p.grouped ? p.tile_rows[it.mt] : min(BM, p.M - it.mt * BM);
      const int slice = (p.width / p.split + 3) / 4 * 4, c0 = rank * slice, n0 = it.nt * p.width + c0;
      const int cols = min(min(slice, p.width - c0), p.N - n0);
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
          if (p.wide) {                                   // whole quads on 16-byte (bf16: 8-byte) boundaries
            if (p.out_bf16) {
              __nv_bfloat162 h[2] = {__floats2bfloat162_rn(a.x, a.y), __floats2bfloat162_rn(a.z, a.w)};
              *reinterpret_cast<uint2*>((__nv_bfloat16*)p.y + o) = *reinterpret_cast<const uint2*>(h);
            } else {
              float4* y = reinterpret_cast<float4*>((float*)p.y + o);
              if (p.accumulate) { const float4 b = *y; a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w; }
              *y = a;
            }
          } else {
            const float f[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (c + j < cols) {
                if (p.out_bf16) ((__nv_bfloat16*)p.y)[o + j] = __float2bfloat16_rn(f[j]);
                else ((float*)p.y)[o + j] = p.accumulate ? f[j] + ((float*)p.y)[o + j] : f[j];
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
// would fetch for the same products.  Tensor memory: an accumulator takes 256 of the 512 columns, so two do not fit beside
// the scales whole.  They overlap in 128 columns: 0..255 and 128..383.  The epilogue reads the shared columns of a tile
// into registers first and hands them over, so the next tile starts before anything is computed or stored.
//   warp 0  TMA   warp 1  scale copies and MMAs (the leader CTA's)   warps 2-9  epilogue, two 64-column chunks each
// GATE_UP: a tile's 256 columns are a block of 128 units; the two warps of a row hand each other the largest of theirs.
constexpr int P_STAGES = 6, P_SLOTS = 8;
constexpr int P_STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int P_SF_BYTES = 3 * kTileBytes, P_SF_COLS = 12;               // of a stage and CTA: a scale tile of A, one of each half of B
constexpr int P_ACC1 = 128, P_SF0 = 384;
constexpr int P_XCH_BYTES = 2 * 2 * BM * 4;
constexpr int P_THREADS = 64 + EPI_WARPS * 32;
constexpr int P_CTL_BYTES = 256;
constexpr int P_SMEM = P_STAGES * (P_STAGE_BYTES + P_SF_BYTES) + EPI_WARPS * TURN_BYTES + P_XCH_BYTES + P_CTL_BYTES + 1024;
static_assert(P_SF0 + P_SLOTS * P_SF_COLS <= 512 && P_ACC1 + 256 <= P_SF0, "tensor memory");
static_assert(P_STAGES * 16 + 24 + 64 + 16 <= P_CTL_BYTES && P_SMEM <= 227 * 1024, "shared memory");

template <int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(P_THREADS, 1)
fp8_gemm_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                     const __grid_constant__ CUtensorMap tmSA, const __grid_constant__ CUtensorMap tmSB, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t ring = (raw + 1023u) & ~1023u;
  const uint32_t scales = ring + P_STAGES * P_STAGE_BYTES, turned = scales + P_STAGES * P_SF_BYTES;
  const uint32_t xch = turned + EPI_WARPS * TURN_BYTES;
  const bool turn = MODE == STORE && !p.wide;
  uint8_t* ctl = smem_raw + (xch + P_XCH_BYTES - raw);
  const uint32_t bar_full = smem_u32(ctl), bar_empty = bar_full + P_STAGES * 8;
  const uint32_t bar_tfull = bar_empty + P_STAGES * 8, bar_handed = bar_tfull + 16, bar_xch = bar_handed + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctl + P_STAGES * 16 + 24 + 64);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = __shfl_sync(kAll, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < P_STAGES; ++s) { mbar_init(bar_full + s * 8, 1); mbar_init(bar_empty + s * 8, 1); }
    for (int a = 0; a < 2; ++a) mbar_init(bar_tfull + a * 8, 1);
    mbar_init(bar_handed, 2 * EPI_WARPS);
    for (int a = 0; a < 8; ++a) mbar_init(bar_xch + a * 8, 2);
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
  const int kb_total = (p.K + SKB - 1) / SKB;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      bool ok = true;
      for (int t = pair; t < n_total && ok; t += n_pairs) {
        const Item it = get_item(p, m_tiles, t);
        const int row0 = it.mt * 256 + (int)rank * 128, col0 = it.nt * 256 + (int)rank * 128;
        const int a_tile = it.b * p.a_row_tiles + it.mt * 2 + (int)rank, b_tile = it.e * p.b_row_tiles + it.nt * 2;
        for (int kb = 0; kb < kb_total; ++kb) {
          if (!(ok = mbar_wait(bar_empty + stage * 8, phase ^ 1u, abort_flag, p.status))) break;
          const uint32_t full_local = bar_full + stage * 8;
          const uint32_t full = map_to_cta(full_local, 0);
          const uint32_t sA = ring + stage * P_STAGE_BYTES, sB = sA + A_BYTES;
          const bool first = kb % SF_GROUP == 0;                         // brings the scales of its group
          if (rank == 0) mbar_expect_tx(full_local, 2 * (P_STAGE_BYTES + (first ? P_SF_BYTES : 0)));
          tma_load_3d(sA, &tmA, kb * SKB, row0, it.b, full);
          tma_load_3d(sB, &tmB, kb * SKB, col0, it.e, full);
          if (first) {                                                   // (tiles past the end of either matrix arrive as zeros)
            tma_load_3d(scales + stage * P_SF_BYTES, &tmSA, 0, kb / SF_GROUP, a_tile, full);
            tma_load_3d(scales + stage * P_SF_BYTES + kTileBytes, &tmSB, 0, kb / SF_GROUP, b_tile, full);
          }
          if (++stage == P_STAGES) { stage = 0; phase ^= 1u; }
        }
      }
      for (int i = 0; i < P_STAGES && ok; ++i) {
        ok = mbar_wait(bar_empty + stage * 8, phase ^ 1u, abort_flag, p.status);
        if (++stage == P_STAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    const uint32_t leader = lane == 0;
    uint32_t stage = 0, phase = 0, acc = 0, tile = 0, slot = 0;
    const uint32_t idesc0 = instr(256, 256, 0);
    const int tail = (p.K - (kb_total - 1) * SKB + 31) / 32;             // MMAs of the last stage that hold elements
    bool ok = rank == 0;
    for (int t = pair; t < n_total && ok; t += n_pairs, ++tile) {
      // the tile before has handed over the shared columns
      if (tile > 0 && !(ok = warp_wait(bar_handed, (tile - 1) & 1u, abort_flag, p.status))) break;
      const uint32_t d = tmem + (acc ? P_ACC1 : 0);
      uint32_t tA = 0;
      for (int kb = 0; kb < kb_total; ++kb) {
        if (!(ok = warp_wait(bar_full + stage * 8, phase, abort_flag, p.status))) break;
        tc_fence_after();
        const uint32_t id = kb % SF_GROUP, low = desc_low(ring + stage * P_STAGE_BYTES);
        if (id == 0) {
          const uint32_t from = scales + stage * P_SF_BYTES;
          tA = tmem + P_SF0 + slot * P_SF_COLS;
          slot = (slot + 1) % P_SLOTS;
          copy_scales_pair(tA, from, leader);
          copy_scales_pair(tA + 4, from + kTileBytes, leader);
          copy_scales_pair(tA + 8, from + 2 * kTileBytes, leader);
        }
        mma_stage_pair(d, low, low + (A_BYTES >> 4), idesc0 | id << 4 | id << 29, tA, tA + 4, kb > 0, leader, kb == kb_total - 1 ? tail : SKB / 32);
        commit_pair_if(bar_empty + stage * 8, leader);
        if (++stage == P_STAGES) { stage = 0; phase ^= 1u; }
      }
      if (!ok) break;
      commit_pair_if(bar_tfull + acc * 8, leader);
      acc ^= 1u;
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
      const bool any = __any_sync(kAll, flat >= 0);
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
      if constexpr (MODE == GATE_UP) {
        const int F = p.N / 2, fa = (n0 + c0 * 64) / 2, fb = (n0 + c1 * 64) / 2;
        float a[64];
        uint32_t most = 0;
        if (any) {
          units(v, fa, F, a, most);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float u[32];
            __syncwarp();
            tc_ld32(taddr + c1 * 64 + h * 32, u);
            units(u, fb + h * 16, F, a + 32 + h * 16, most);
          }
        }
        // place acc of two: the other warp has read it before it comes to the barrier of the tile in between
        const uint32_t bar = bar_xch + (acc * 4 + q) * 8, at = xch + (acc * 2 * BM + row) * 4;
        st_shared_u32(at + half * BM * 4, most);
        __syncwarp();
        if (lane == 0) arrive(bar);
        if (!(ok = warp_wait(bar, acc_phase, abort_flag, p.status))) break;
        most = max(most, ld_shared_u32(at + (half ^ 1) * BM * 4));
        uint32_t inv;
        const uint32_t byte = scale_byte(most, inv);
        if (flat >= 0) {
          if (fa < F) store_units(p, a, fa, F, m, byte, inv);
          if (fb < F) store_units(p, a + 32, fb, F, m, byte, inv);
          if (half == 0) p.act_scales[scale_offset(0, m, (int)scale_tiles_k(F), n0 / 2 / kBlock)] = (uint8_t)byte;
        }
      } else if (any) {
        auto finish = [&](int c) {
          if (turn)
            put_turned(p, it, v, n0 + c * 64, p.N, it.mt * 256 + (int)rank * 128 + q * 32, lane,
                       reinterpret_cast<uint32_t*>(smem_raw + (turned - raw) + (warp - 2) * TURN_BYTES));
          else
            put_chunk<MODE>(p, it, v, n0 + c * 64, p.N, flat);
        };
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

// codes [batch][rows][pitch], of which K bytes of a row count (those behind read as 0), box of a block x box_rows
bool make_codes_map(CUtensorMap* m, const void* base, long long K, long long rows, long long batch, uint32_t box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const long long pitch = row_pitch(K);
  cuuint64_t dims[3] = {(cuuint64_t)K, (cuuint64_t)rows, (cuuint64_t)batch};
  cuuint64_t strides[2] = {(cuuint64_t)pitch, (cuuint64_t)(pitch * rows)};
  cuuint32_t box[3] = {SKB, box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// scale tiles [row tiles][kt][512 bytes] of all matrices, box of one tile along K x box_tiles row tiles
bool make_scales_map(CUtensorMap* m, const void* base, long long kt, long long row_tiles, uint32_t box_tiles) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {kTileBytes / 4, (cuuint64_t)kt, (cuuint64_t)row_tiles};
  cuuint64_t strides[2] = {kTileBytes, (cuuint64_t)(kt * kTileBytes)};
  cuuint32_t box[3] = {kTileBytes / 4, 1, box_tiles};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_INT32, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int MODE, bool SPLIT>
btx_status launch(const GemmArgs& g, Params p, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  CUtensorMap a, b;
  if (!make_codes_map(&a, g.a_codes, g.K, g.M, g.batch, p.a_box) || !make_codes_map(&b, g.b_codes, g.K, g.N, g.experts, p.width) ||
      !allow_smem((const void*)fp8_gemm_kernel<MODE, SPLIT>, SMEM_BYTES, done))
    return BTX_ERR_CUDA;
  if (MODE == GATE_UP) p.n_tiles = (p.n_tiles + 1) / 2;   // pairs of column tiles
  const long long tiles = (long long)p.m_tiles * p.n_tiles * p.batch, per = SPLIT ? p.split : MODE == GATE_UP ? 2 : 1;
  const long long most = SPLIT ? tiles : sm_count() / per;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((tiles < most ? tiles : most) * per)); cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = SMEM_BYTES; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;      // a programmatic dependent of the kernel before it
  attr[n++].val.programmaticStreamSerializationAllowed = 1;
  if (per > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)per; attr[n].val.clusterDim.y = 1; attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr; cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, fp8_gemm_kernel<MODE, SPLIT>, a, b, p) == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

template <int MODE>
btx_status launch_pair(const GemmArgs& g, Params p, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  CUtensorMap a, b, sa, sb;
  p.m_tiles = (g.M + 255) / 256; p.n_tiles = (g.N + 255) / 256; p.tile_step = 2;
  if (!make_codes_map(&a, g.a_codes, g.K, g.M, g.batch, 128) || !make_codes_map(&b, g.b_codes, g.K, g.N, g.experts, 128) ||
      !make_scales_map(&sa, g.a_scales, p.kt, (long long)p.a_row_tiles * g.batch, 1) ||
      !make_scales_map(&sb, g.b_scales, p.kt, (long long)p.b_row_tiles * g.experts, 2) ||
      !allow_smem((const void*)fp8_gemm_pair_kernel<MODE>, P_SMEM, done))
    return BTX_ERR_CUDA;
  const long long items = (long long)p.m_tiles * p.n_tiles * p.batch;
  int pairs = sm_count() / 2;
  if (items < pairs) pairs = (int)items;
  return launch_after_predecessor(fp8_gemm_pair_kernel<MODE>, dim3(2 * pairs), dim3(P_THREADS), P_SMEM, st, true, a, b, sa,
                                  sb, p) == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

Params base_params(const GemmArgs& g) {
  Params p = {};
  p.M = g.M; p.N = g.N; p.K = g.K; p.batch = g.batch; p.status = g.status;
  p.m_tiles = (g.M + BM - 1) / BM; p.n_tiles = (g.N + BN - 1) / BN; p.split = 1; p.width = BN;
  p.kt = (int)scale_tiles_k(g.K); p.tile_step = 1;
  p.a_row_tiles = (int)row_tiles(g.M); p.b_row_tiles = (int)row_tiles(g.N);
  p.a_scales = g.a_scales; p.b_scales = g.b_scales;
  p.a_scale_batch = (long long)p.a_row_tiles * p.kt * kTileBytes;
  p.b_scale_batch = (long long)p.b_row_tiles * p.kt * kTileBytes;
  return p;
}

// How fp8_gemm_kernel goes about a product: columns of a tile, and the CTAs of a cluster that share its contraction.
struct Plan1 { int width, split; double us; };

// The cheapest of the plans by what was measured, in us: a launch 3.2; for a round of tiles 0.9, and a stage 0.27, or its bytes of B
// at 6.1 TB/s over the CTAs at work where that is longer; sharing the contraction 1.6 and up to 1.4 more for full
// tiles (their partial sums).  Clusters of 8 find room only up to about 64 CTAs.  E.g. one row: N = 4096, K = 4096: 8.0 us with
// four CTAs a tile, 9.7 with two, 12.5 with one; N = 2048, K = 2048: 6.0 with four, 11.4 with eight; 200 x 700 x 900: 5.8 with
// tiles of 64 columns, 6.5 with 128, 7.6 with four CTAs a tile.
Plan1 plan_single(double row_tiles_, long long rows, long long N, long long K) {
  Plan1 best = {BN, 1, 1e30};
  const int sms = sm_count();
  const double kb = (double)((K + SKB - 1) / SKB);
  const double a_rows = rows < BM ? (double)rows : BM;
  for (int width = 64; width <= BN; width += 64)
    for (int split = 1; split <= 8; split *= 2) {
      const double ctas = row_tiles_ * (double)((N + width - 1) / width) * split;
      if (split > 1 && (ctas > (split == 8 ? 64 : sms) || kb < 2 * split)) break;
      const double rounds = ceil(ctas / sms), at_work = ctas < sms ? ctas : sms;
      const double stage = fmax(width == BN ? 0.27 : 0.25, width * SKB * at_work / 6.1e6);
      const double us = 3.2 + rounds * (ceil(kb / split) * stage + 0.9) + (split > 1 ? 1.6 + 1.4 * a_rows / BM : 0.0);
      if (us < best.us) best = {width, split, us};
    }
  return best;
}
// The same for fp8_gemm_pair_kernel: rounds of tiles, 0.45 us a stage or the epilogue `epi` where that is longer.
double pair_us(double tiles, long long K, double epi) {
  return 3.5 + ceil(tiles / (sm_count() / 2)) * (fmax((double)((K + SKB - 1) / SKB) * 0.45, epi) + 0.85);
}
// Epilogues of a 256 x 256 tile.  (kGateUpUs: T = 4096, d = 128, F = 11008, one expert, 19 rounds of tiles of one stage in about 106 us.)
constexpr double kStoreUs = 2.0, kGateUpUs = 4.5, kDownUs = 3.5;

}  // namespace

// The expert layer's two products, for experts with about rows / experts rows each (a tile more than they fill for
// every second).  Whole layers in us with tiles of 128 rows, and with pairs: 4 experts, d = 4096, F = 11008, top-2: 128 tokens 133, 133;
// 256 192, 136; 512 300, 196; 64 experts, d = 2048, F = 1024, top-8: 128 tokens 116, 118; 512 109, 123; 1024 162, 147; 2048 243, 209;
// 8 experts, d = 1024, F = 4096, top-2: 512 tokens 56, 59; 1024 91, 67.
bool pairs_fit(long long rows, long long experts, long long d, long long F) {
  if (rows == 0) return false;
  const double each = (double)rows / (double)experts;
  const double t1 = experts * fmax(1.0, each / 128 + 0.5), t2 = experts * fmax(1.0, each / 256 + 0.5);
  const double n2 = (double)((2 * F + 255) / 256), m2 = (double)((d + 255) / 256);
  const double stages = (double)((d + SKB - 1) / SKB);
  const double up = 3.2 + ceil(t1 * n2 * 2 / sm_count()) * (fmax(stages * 0.39, kGateUpUs / 2) + 0.4);      // twins of 128 x 128 tiles
  return pair_us(t2 * n2, d, kGateUpUs) + pair_us(t2 * m2, F, kDownUs) < up + plan_single(t1, (long long)each + 1, d, F).us;
}

btx_status launch_matmul(const GemmArgs& g, int dtype, void* y, int accumulate, cudaStream_t st) {
  Params p = base_params(g);
  p.y = y; p.out_bf16 = dtype == BTX_BF16; p.accumulate = accumulate;
  p.wide = aligned32(y) && (size_t)g.N * (p.out_bf16 ? 2 : 4) % 32 == 0;
  const Plan1 plan = plan_single((double)p.m_tiles * p.batch, g.M, g.N, g.K);
  if (pair_us((double)g.batch * ((g.M + 255) / 256) * ((g.N + 255) / 256), g.K, kStoreUs) < plan.us) return launch_pair<STORE>(g, p, st);
  p.a_rows = p.a_box = g.M < BM ? (g.M + 31) / 32 * 32 : BM;
  p.split = plan.split; p.width = plan.width; p.n_tiles = (g.N + p.width - 1) / p.width;
  return p.split > 1 ? launch<STORE, true>(g, p, st) : launch<STORE, false>(g, p, st);
}

static Params grouped_params(const GemmArgs& g, const mx4::Dispatch& q) {
  Params p = base_params(g);
  p.grouped = 1; p.n_row_tiles = q.n_tiles; p.tile_expert = q.tile_expert; p.tile_rows = q.tile_rows; p.rowmap = q.rowmap;
  // a tile holds at most R rows; in small batches few of its rows are used, and only those are fetched
  p.a_rows = q.R < BM ? (q.R + 31) / 32 * 32 : BM;
  p.a_box = q.R <= 16 * BM ? 32 : BM;
  return p;
}

btx_status launch_gate_up(const GemmArgs& g, const mx4::Dispatch& q, uint8_t* act_codes, uint8_t* act_scales, cudaStream_t st) {
  Params p = grouped_params(g, q);
  p.act_codes = act_codes; p.act_scales = act_scales;
  return q.pad_tiles == 2 ? launch_pair<GATE_UP>(g, p, st) : launch<GATE_UP, false>(g, p, st);
}

btx_status launch_down(const GemmArgs& g, const mx4::Dispatch& q, const float* gates, float* rows, cudaStream_t st) {
  Params p = grouped_params(g, q);
  p.gates = gates; p.y = rows; p.wide = g.N % 8 == 0;
  if (q.pad_tiles == 2) return launch_pair<DOWN>(g, p, st);
  // (m_tiles bounds the row tiles in use, and it is all that is known here)
  const Plan1 plan = plan_single((double)p.m_tiles, q.R, g.N, g.K);
  p.split = plan.split; p.width = plan.width; p.n_tiles = (g.N + p.width - 1) / p.width;
  return p.split > 1 ? launch<DOWN, true>(g, p, st) : launch<DOWN, false>(g, p, st);
}

}  // namespace fp8
}  // namespace btx

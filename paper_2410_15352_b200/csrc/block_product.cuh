// C = A B^T of 8-bit matrices with a power-of-two scale for each 128 columns of a row:
//     C[i, j] = sum over blocks b of K of  sa[i, b] sb[j, b]  sum over k in b of  A[i, k] B[j, k].
// The tensor cores apply the scales themselves (tcgen05.mma kind::mxf8f6f4 with block scaling): one instruction multiplies 32
// columns of K, and takes for each row of either operand one E8M0 byte from TMEM.  A block of 128 columns is one k-step of
// four instructions that name the same byte; a 32-bit word of TMEM holds the bytes of four k-steps, so scales move once
// per 512 columns of K.
//
// Where the scales of an operand tile sit in TMEM: row i of a 128-row tile in lane i % 32, column i / 32 of the operand's
// four columns, the same in each of the four 32-lane quarters; a further 128 rows (of the N operand) in four more
// columns.  The layout of the scales in memory (one word per row and group of four column blocks) is chosen so that a warp
// loads 32 rows' words in one coalesced access and stores them to TMEM as they are: no shared memory, no transposition, and a
// tile may start at any row.
//
// Two kernels.
//   product_pair_kernel: long batches.  Pairs of SMs, 256 rows of A by up to 256 rows of B per tile
//     (tcgen05.mma.cta_group::2), accumulators double-buffered.  Bound by the tensor cores, and in a
//     loop by the power cap: 16384 x 11008 x 4096 585 us, 2.5 PFLOP/s at 1.13 GHz, 93 % of the tensor pipe's cycles.
//   product_split_kernel: few rows of A (decoding).  The rows of B are the M operand, so that a tile reads 128 rows of the weight
//     and the tokens are the N operand (16 to 128); a cluster of up to eight CTAs splits K, and its sums meet in
//     shared memory in a fixed order.  Bound by reading the weight: one token by 11008 x 4096 11.5 us, 6 TB/s after some 4 us of
//     start, first load and sums.
#pragma once
#include "block_common.cuh"
#include "block_launch.cuh"
#include "tc_common.cuh"

namespace compact {
namespace blk {

using namespace tc;

constexpr int PK = 128;                              // columns of K per k-step: a swizzle row of 128 bytes, one scale per row
constexpr int P_TILE_BYTES = 128 * PK;               // 16 KB: 128 rows of an operand

struct ProductOperand {
  const uint32_t* scales;    // word (g, row) at g * lds + row
  int64_t lds;
  int rows;
};

// What the waits of a launch are bounded by and report to.  `loaded`: k-steps of a tile that are loaded, all of them but in the test that
// makes the waits run out.
struct ProductWaits {
  unsigned int* status;
  uint32_t tag;              // the handle's mark: of two handles that have had a word in turn, the later has the larger one
  uint32_t limit;            // polls
  int loaded;
};
__device__ __forceinline__ bool bounded_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, const ProductWaits& w) {
  return mbar_wait_or(bar, parity, abort_flag, [&w] { atomicMax(w.status, w.tag); }, w.limit);
}

// ---- pairs of SMs -----------------------------------------------------------------------------------
constexpr int PP_NS = 6;
constexpr int PP_STAGE_BYTES = 2 * P_TILE_BYTES;     // [A: 128 rows | B: up to 128 rows]
constexpr int PP_BN_MAX = 256;
// TMEM: two accumulators 224 columns apart, then scales, two stages of 16 columns (four for A, eight for B).  Tiles of up to
// 224 columns have accumulators of their own.  Those of 256 columns share columns 224 .. 255: the epilogue empties these
// first, and the MMAs of the next tile wait for that (a few hundred clocks of the 16 thousand of a tile with K = 4096) but not for
// the rest.
constexpr int PP_SLOT_COLS = 224;
constexpr int PP_SF_STAGES = 2;
constexpr int PP_SF_COL = 480;
constexpr int PP_SF_BUF_BYTES = 4 * (128 + PP_BN_MAX);   // words of a group on their way to TMEM
constexpr int PP_EPI_WARPS = 8;
constexpr int PP_SCALE_WARP = 2 + PP_EPI_WARPS;      // first of four
constexpr int PP_THREADS = 32 * (PP_SCALE_WARP + 4);
constexpr int PP_SF_OFF = PP_NS * PP_STAGE_BYTES;
constexpr int PP_BARS_OFF = PP_SF_OFF + 6 * PP_SF_BUF_BYTES;
constexpr int PP_NUM_BARS = 2 * PP_NS + 5 + 2 * PP_SF_STAGES;
constexpr int PP_SMEM_BYTES = 1024 + PP_BARS_OFF + 8 * PP_NUM_BARS + 32;
static_assert(PP_SMEM_BYTES <= 232448, "shared memory budget");

struct alignas(64) PairParams {
  CUtensorMap tmA, tmB;
  void* C;
  int64_t ldc;
  ProductOperand a, b;
  int M, N, bn, ksteps;
  int tiles_m, tiles_n, panel_cols;       // column tiles per panel: a panel of B stays in the L2 while A streams past
  int c_f32;
  int per_barrier;                        // k-steps (stages) that share a barrier
  uint32_t idesc;                         // types and shape of the instruction, without the byte numbers of the scales
  ProductWaits waits;
};

__device__ __forceinline__ void tmem_st4(uint32_t taddr, const uint32_t (&v)[4]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// D (+)= A B with the scales at sa, sb: M x N x 32, over the pair or by one CTA
__device__ __forceinline__ void umma2_mx(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %3};\n\t"
      "mov.b64 db, {%2, %3};\n\t"
      "setp.ne.b32 p, %7, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], da, db, %4, [%5], [%6], p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(DESC_HI), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma1_mx(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %3};\n\t"
      "mov.b64 db, {%2, %3};\n\t"
      "setp.ne.b32 p, %7, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], da, db, %4, [%5], [%6], p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(DESC_HI), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
      : "memory");
}
// Instruction descriptor of block-scaled 8-bit products: operand types at bits 7 and 10 (0: e4m3, 1: e5m2), both K-major,
// N / 8 at bit 17, E8M0 scales (bit 23), M / 128 at bit 27.  The byte of the scale words goes to bits 29 (A) and 4 (B).
__host__ __device__ constexpr uint32_t mx_idesc(int a_type, int b_type, int m, int n) {
  return ((uint32_t)a_type << 7) | ((uint32_t)b_type << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 7) << 27);
}
__device__ __forceinline__ uint32_t mx_byte(int j) { return ((uint32_t)j << 29) | ((uint32_t)j << 4); }

__device__ __forceinline__ void tma2_load(uint32_t dst, const CUtensorMap* map, uint32_t leader_bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
      "l"(map), "r"(leader_bar), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void commit2_mc(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
               : "memory");
}
// Arrives on a barrier of the pair.  What it announces are accesses to TMEM, ordered by the waits and fences of tcgen05 around it;
// a release of cluster scope would make the thread wait for all its loads in flight as well.
__device__ __forceinline__ void arrive_cluster(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// After a wait has run out: lets the copies of the last uses of the ring land (bounded) before the CTA may leave.  `issued` uses of
// `stages` stages whose full barriers lie `step` bytes apart, use u on barrier u % stages with parity (u / stages) & 1.
__device__ __forceinline__ void drain_copies(uint32_t full0, uint32_t step, int stages, long long issued) {
  for (long long u = issued > stages ? issued - stages : 0; u < issued; ++u)
    for (int it = 0; it < 100000; ++it) {
      if (mbar_try_wait(full0 + step * (uint32_t)(u % stages), (uint32_t)((u / stages) & 1))) break;
      __nanosleep(100);
    }
}

// Scale words travel through shared memory, SF_AHEAD groups before their use: cp.async by four warps (each a quarter of the words),
// read back by all four, each for its quarter of TMEM.  They are asked for that early because a load queues behind the
// operand tiles that TMA has in flight, up to 200 KB per SM.  (8192 x 4096 x 4096: 164 thousand clocks; words loaded into
// registers one group ahead: 166; those, with a release of cluster scope in the arrival: 200.)
constexpr int SF_BUFS = 6;
static_assert(PP_BARS_OFF - PP_SF_OFF >= SF_BUFS * PP_SF_BUF_BYTES, "room for the scales in flight");
constexpr int SF_AHEAD = SF_BUFS - 1;
__device__ __forceinline__ void cp_async_word(uint32_t dst, const uint32_t* src, bool there) {
  // a row past the operand reads nothing and gets zeros: the scale 2^-127 of elements that are zeros themselves
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// Word of row r0 + i of group g to dst + 4 i
__device__ __forceinline__ void fetch_scale_word(const ProductOperand& o, int g, int r0, int i, uint32_t dst) {
  const int r = r0 + i;
  const bool there = r < o.rows;
  cp_async_word(dst + 4u * (uint32_t)i, o.scales + (int64_t)g * o.lds + (there ? r : 0), there);
}
__device__ __forceinline__ uint32_t lds_word(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
// 128 words from shared memory into four columns of this warp's quarter of TMEM
__device__ __forceinline__ void scale_words_to_tmem(uint32_t taddr, uint32_t src, int lane) {
  uint32_t v[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) v[c] = lds_word(src + 4u * (uint32_t)(32 * c + lane));
  tmem_st4(taddr, v);
}

// 32 sums of a row (the first `cols` of them) as columns of C, in whole 32-byte sectors; a row that starts in the middle of one
// has 16 bytes before them and after.  `policy`: evict first, for C would push the operands out of the L2 (16384 x 4096 x 1024:
// 69 us against 74; with 16-byte stores 86).
__device__ __forceinline__ void store32(uint32_t* p, const uint32_t* o, uint64_t policy) {
  asm volatile("st.global.L1::no_allocate.L2::cache_hint.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8}, %9;" ::"l"(p), "r"(o[0]), "r"(o[1]), "r"(o[2]),
               "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]), "l"(policy)
               : "memory");
}
__device__ __forceinline__ void store16(uint32_t* p, const uint32_t* o, uint64_t policy) {
  asm volatile("st.global.L1::no_allocate.L2::cache_hint.v4.b32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(p), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "l"(policy)
               : "memory");
}
template <typename T>
__device__ __forceinline__ void store_columns(T* c, const uint32_t (&v)[32], int cols, uint64_t policy) {
  constexpr int WORDS = 8 * (int)sizeof(T);            // 16 of bf16, 32 of fp32
  uint32_t o[WORDS];
#pragma unroll
  for (int j = 0; j < WORDS; ++j)
    o[j] = sizeof(T) == 4 ? v[j] : pack_bf16x2(__uint_as_float(v[(2 * j) % 32]), __uint_as_float(v[(2 * j + 1) % 32]));
  uint32_t* out = reinterpret_cast<uint32_t*>(c);
  if (cols == 32) {
    if ((reinterpret_cast<uintptr_t>(out) & 31u) == 0) {
#pragma unroll
      for (int j = 0; j < WORDS; j += 8) store32(out + j, o + j, policy);
    } else {
      store16(out, o, policy);
#pragma unroll
      for (int j = 4; j + 8 < WORDS; j += 8) store32(out + j, o + j, policy);
      store16(out + WORDS - 4, o + WORDS - 4, policy);
    }
    return;
  }
  constexpr int PER = 16 / (int)sizeof(T);             // columns of 16 bytes
#pragma unroll
  for (int j = 0; j < WORDS; j += 4) {
    const int first = j / 4 * PER;
    if (first + PER <= cols) {
      store16(out + j, o + j, policy);
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e)
        if (first + e < cols) {
          if (sizeof(T) == 4) out[first + e] = o[(j + e) % WORDS];
          else reinterpret_cast<uint16_t*>(c)[first + e] = (uint16_t)(o[(j + e / 2) % WORDS] >> (16 * (e & 1)));
        }
    }
  }
}

__device__ __forceinline__ void pair_tile(const PairParams& p, int tile, int& m0, int& n0) {
  const int per_panel = p.tiles_m * p.panel_cols;
  const int panel = tile / per_panel;
  const int local = tile - panel * per_panel;
  const int pc = min(p.panel_cols, p.tiles_n - panel * p.panel_cols);
  const int mb = local / pc;
  m0 = mb * 256;
  n0 = (panel * p.panel_cols + (local - mb * pc)) * p.bn;
}

// Roles in each CTA of the pair: warp 0 loads its 128 rows of A and half of the tile's rows of B; warp 1 owns TMEM and, in the
// leader (rank 0), issues the MMAs of both; warps 2-9 are the epilogue; warps 10-13 (one per TMEM quarter) bring the scales.
// Barriers: full[s] (leader's: bytes of both CTAs), empty[s] (own; the leader's commit arrives on both), tfull[a] (own, by
// commit), tempty[a] (leader's, 16 epilogue warps), shared (leader's: the columns that both accumulators have are empty, 8 epilogue
// warps), sfull[t] (leader's, 8 scale warps), sempty[t] (own, by commit).
__global__ void __launch_bounds__(PP_THREADS, 1) product_pair_kernel(const __grid_constant__ PairParams prm) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t bars = smem_base + PP_BARS_OFF;
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (PP_NS + s); };
  auto tfull_bar = [&](int a) { return bars + 8u * (2 * PP_NS + a); };
  auto tempty_bar = [&](int a) { return bars + 8u * (2 * PP_NS + 2 + a); };
  const uint32_t shared_bar = bars + 8u * (2 * PP_NS + 4);
  auto sfull_bar = [&](int t) { return bars + 8u * (2 * PP_NS + 5 + t); };
  auto sempty_bar = [&](int t) { return bars + 8u * (2 * PP_NS + 5 + PP_SF_STAGES + t); };
  uint8_t* tail = smem_gen + PP_BARS_OFF + 8 * PP_NUM_BARS;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(tail);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 8);

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const uint32_t crank = blockIdx.x & 1u;             // rank in the cluster of two
  const bool leader = crank == 0;
  const int pair_id = (int)(blockIdx.x >> 1);
  const int npairs = (int)(gridDim.x >> 1);
  const int total = prm.tiles_m * prm.tiles_n;

  let_successor_start();
  if (threadIdx.x == 0) {
    for (int s = 0; s < PP_NS; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(tfull_bar(a), 1);
      mbar_init(tempty_bar(a), 2 * PP_EPI_WARPS);
    }
    mbar_init(shared_bar, PP_EPI_WARPS);
    for (int t = 0; t < PP_SF_STAGES; ++t) {
      mbar_init(sfull_bar(t), 8);
      mbar_init(sempty_bar(t), 1);
    }
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  cluster_sync_all();                     // both CTAs' barriers and TMEM exist before anything crosses
  wait_for_predecessors();
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  const uint32_t leader_bars = map_to_cta(bars, 0u);
  const int half_bn = prm.bn >> 1;
  long long issued = 0;                   // uses of the ring, by the loader
  bool ok = true;

  if (warp == 0) {
    // ------------------------------ loader ---------------------------------------
    int s = 0;
    uint32_t ph = 0;
    const uint32_t bytes = 2u * (uint32_t)(P_TILE_BYTES + half_bn * PK);
    for (int tile = pair_id; tile < total && ok; tile += npairs) {
      int m0, n0;
      pair_tile(prm, tile, m0, n0);
      m0 += (int)crank * 128;
      n0 += (int)crank * half_bn;
      for (int ks = 0; ks < prm.ksteps; ks += prm.per_barrier) {
        if (!(ok = ks < prm.waits.loaded)) break;
        if (!(ok = __all_sync(0xffffffffu, bounded_wait(empty_bar(s), ph ^ 1u, abort_flag, prm.waits)))) break;
        if (elect_one()) {
          const int count = min(prm.per_barrier, prm.ksteps - ks);
          if (leader) mbar_arrive_expect_tx(full_bar(s), bytes * (uint32_t)count);
          for (int h = 0; h < count; ++h) {
            const uint32_t dst = smem_base + (uint32_t)(s + h) * PP_STAGE_BYTES;
            tma2_load(dst, &prm.tmA, leader_bars + 8u * s, (ks + h) * PK, m0);
            tma2_load(dst + P_TILE_BYTES, &prm.tmB, leader_bars + 8u * s, (ks + h) * PK, n0);
          }
        }
        __syncwarp();
        ++issued;
        if ((s += prm.per_barrier) == PP_NS) { s = 0; ph ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // ------------------------------ MMA issuer (leader CTA) ----------------------
    // One lane walks the whole loop: a vote and an election in every k-step cost it as much as the waits themselves.
    if (leader && elect_one()) {
      int s = 0, t = 0, slot = 0;
      uint32_t ph = 0, tph = 0, slot_phase = 0, shared_phase = 0;
      const uint32_t ring_lo = ((smem_base >> 4) & 0x3FFFu) | (1u << 16);
      for (int tile = pair_id; tile < total && ok; tile += npairs) {
        if (!(ok = bounded_wait(tempty_bar(slot), slot_phase ^ 1u, abort_flag, prm.waits))) break;
        if (prm.bn > PP_SLOT_COLS && tile != pair_id) {
          if (!(ok = bounded_wait(shared_bar, shared_phase, abort_flag, prm.waits))) break;
          shared_phase ^= 1u;
        }
        tc_fence_after();
        const uint32_t d = tmem_base + (uint32_t)(slot * PP_SLOT_COLS);
        for (int ks = 0; ks < prm.ksteps; ks += prm.per_barrier) {
          if ((ks & 3) == 0) {
            if (!(ok = bounded_wait(sfull_bar(t), tph, abort_flag, prm.waits))) break;
          }
          if (!(ok = bounded_wait(full_bar(s), ph, abort_flag, prm.waits))) break;
          tc_fence_after();
          const uint32_t sa = tmem_base + PP_SF_COL + 16u * t, sb = sa + 4;
          const int end = min(ks + prm.per_barrier, prm.ksteps);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (ks + h >= end) break;
            const uint32_t a = ring_lo + (((uint32_t)(s + h) * PP_STAGE_BYTES) >> 4), b = a + (P_TILE_BYTES >> 4);
            const uint32_t idesc = prm.idesc | mx_byte((ks + h) & 3);
            umma2_mx(d, a, b, idesc, sa, sb, ks + h > 0 ? 1u : 0u);
            umma2_mx(d, a + 2, b + 2, idesc, sa, sb, 1u);
            umma2_mx(d, a + 4, b + 4, idesc, sa, sb, 1u);
            umma2_mx(d, a + 6, b + 6, idesc, sa, sb, 1u);
          }
          commit2_mc(empty_bar(s));
          if ((end & 3) == 0 || end == prm.ksteps) {
            commit2_mc(sempty_bar(t));
            if (++t == PP_SF_STAGES) { t = 0; tph ^= 1u; }
          }
          if ((s += prm.per_barrier) == PP_NS) { s = 0; ph ^= 1u; }
        }
        if (!ok) break;
        commit2_mc(tfull_bar(slot));
        if (++slot == 2) { slot = 0; slot_phase ^= 1u; }
      }
    }
    __syncwarp();
  } else if (warp < PP_SCALE_WARP) {
    // ------------------------------ epilogue ------------------------------------
    // This CTA's 128 rows, TMEM -> registers -> C, the two sets of four warps taking alternate chunks of 32 columns.  A lane has a
    // row: its 32 columns leave as whole 32-byte sectors.  (Staging tiles and TMA stores took as long, and shared memory.)
    const int q = warp & 3, eset = (warp - 2) >> 2;
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    int slot = 0;
    uint32_t slot_phase = 0;
    for (int tile = pair_id; tile < total && ok; tile += npairs) {
      int m0, n0;
      pair_tile(prm, tile, m0, n0);
      if (!(ok = __all_sync(0xffffffffu, bounded_wait(tfull_bar(slot), slot_phase, abort_flag, prm.waits)))) break;
      tc_fence_after();
      const int row0 = m0 + (int)crank * 128 + q * 32;
      const uint32_t tcol = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(slot * PP_SLOT_COLS);
      // chunks in an order that begins with the shared columns: the last chunk of the first accumulator, the first of the second
      const int chunks = prm.bn >> 5;
      for (int i = eset; i < chunks; i += 2) {
        const int ci = slot == 0 ? chunks - 1 - i : i;
        const int col = n0 + ci * 32;
        const bool live = row0 < prm.M && col < prm.N;
        uint32_t v[32];
        if (live) {
          tmem_ld32(tcol + ci * 32, v);
          tmem_ld_wait();
        }
        if (i == 0 && prm.bn > PP_SLOT_COLS) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_cluster(leader_bars + 8u * (2 * PP_NS + 4));
        }
        if (!live) continue;
        if (row0 + lane < prm.M) {
          const int64_t o = (int64_t)(row0 + lane) * prm.ldc + col;
          const int cols = min(32, prm.N - col);
          if (prm.c_f32) store_columns<float>(reinterpret_cast<float*>(prm.C) + o, v, cols, policy);
          else store_columns<__nv_bfloat16>(reinterpret_cast<__nv_bfloat16*>(prm.C) + o, v, cols, policy);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_cluster(leader_bars + 8u * (2 * PP_NS + 2 + slot));
      if (++slot == 2) { slot = 0; slot_phase ^= 1u; }
    }
  } else {
    // ------------------------------ scales ---------------------------------------
    const int w = warp & 3;
    const uint32_t quarter = (uint32_t)(w * 32) << 16;
    const int groups = (prm.ksteps + 3) >> 2;
    const bool wide = prm.bn > 128;
    auto buffer = [&](int i) { return smem_base + PP_SF_OFF + (uint32_t)(i * PP_SF_BUF_BYTES); };
    int tile = pair_id, g = 0, m0 = 0, n0 = 0, fb = 0;      // of the next fetch
    auto fetch_next = [&]() {
      if (tile < total) {
        if (g == 0) {
          pair_tile(prm, tile, m0, n0);
          m0 += (int)crank * 128;                           // its own rows of A, all rows of B
        }
        const uint32_t dst = buffer(fb);
        fetch_scale_word(prm.a, g, m0, w * 32 + lane, dst);
        fetch_scale_word(prm.b, g, n0, w * 32 + lane, dst + 512);
        if (wide) fetch_scale_word(prm.b, g, n0, 128 + w * 32 + lane, dst + 512);
        if (++g == groups) {
          g = 0;
          tile += npairs;
        }
        if (++fb == SF_BUFS) fb = 0;
      }
      cp_async_commit();                                    // a group of none past the end
    };
#pragma unroll
    for (int d = 0; d < SF_AHEAD; ++d) fetch_next();
    long long left = total > pair_id ? (long long)((total - pair_id + npairs - 1) / npairs) * groups : 0;
    int t = 0, rb = 0;
    uint32_t tph = 0;
    // every warp goes through every group, after a wait has run out too: the barrier among the four has no limit of its own
    for (; left > 0; --left) {
      cp_async_wait<SF_AHEAD - 1>();
      named_barrier(1, 128);                                // all four quarters of this group have landed, and the previous one is read
      fetch_next();
      if (ok) ok = __all_sync(0xffffffffu, bounded_wait(sempty_bar(t), tph ^ 1u, abort_flag, prm.waits));
      if (ok) {
        tc_fence_after();
        const uint32_t at = tmem_base + quarter + PP_SF_COL + 16u * t, src = buffer(rb);
        scale_words_to_tmem(at, src, lane);
        scale_words_to_tmem(at + 4, src + 512, lane);
        if (wide) scale_words_to_tmem(at + 8, src + 1024, lane);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_cluster(leader_bars + 8u * (2 * PP_NS + 5 + t));
      }
      if (++t == PP_SF_STAGES) { t = 0; tph ^= 1u; }
      if (++rb == SF_BUFS) rb = 0;
    }
    cp_async_wait<0>();
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 0 && leader && *abort_flag) drain_copies(full_bar(0), 8u * prm.per_barrier, PP_NS / prm.per_barrier, issued);
  cluster_sync_all();                     // neither CTA frees TMEM, or leaves, while the pair may still use or signal it
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

// ---- clusters that split K ---------------------------------------------------------------------------
constexpr int PS_MAX_STAGES = 6;                     // of two k-steps each: half the barriers for the issuing thread
constexpr int PS_RING_BYTES = 200 * 1024;
constexpr int PS_BT_MAX = 128;                       // tokens of a tile
constexpr int PS_SF_STAGES = 4;
constexpr int PS_SF_COL = PS_BT_MAX;                 // scales after the accumulator: four columns of weights, four of tokens
constexpr int PS_TMEM_COLS = 256;
constexpr int PS_THREADS = 32 * 6;
constexpr int PS_SF_OFF = PS_RING_BYTES;                // words of scales in flight: 128 of weights, 128 of tokens per buffer
constexpr int PS_BARS_OFF = PS_SF_OFF + 6 * 1024;
constexpr int PS_NUM_BARS = 2 * PS_MAX_STAGES + 1 + 2 * PS_SF_STAGES;
constexpr int PS_SMEM_BYTES = 1024 + PS_BARS_OFF + 8 * PS_NUM_BARS + 32;
static_assert(PS_SMEM_BYTES <= 232448, "shared memory budget");
static_assert(PS_BARS_OFF - PS_SF_OFF >= SF_BUFS * 1024, "room for the scales in flight");
static_assert((PS_BT_MAX + 8) * 512 <= PS_RING_BYTES, "the sums, and the share past the last token, reuse the ring");

struct alignas(64) SplitParams {
  CUtensorMap tmW, tmX;                   // rows of B (the weight), rows of A (the tokens)
  ProductOperand w, x;
  void* C;
  int64_t ldc;
  int M, N, bt, splits, ksteps, stages, c_f32;
  uint32_t idesc;
  ProductWaits waits;
};

// k-steps of each CTA of a cluster: an even number
__host__ __device__ __forceinline__ int split_ksteps(int ksteps, int splits) { return ((ksteps + splits - 1) / splits + 1) / 2 * 2; }

// Grid: (cluster size x tiles of weight rows, tiles of bt tokens).  Warp 0 loads, warp 1 owns TMEM and issues the MMAs,
// warps 2-5 (one per TMEM quarter) bring the scales and, when the accumulator is complete, sum and store it.
__global__ void __launch_bounds__(PS_THREADS, 1) product_split_kernel(const __grid_constant__ SplitParams prm) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t bars = smem_base + PS_BARS_OFF;
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (PS_MAX_STAGES + s); };
  const uint32_t tfull = bars + 8u * (2 * PS_MAX_STAGES);
  auto sfull_bar = [&](int t) { return bars + 8u * (2 * PS_MAX_STAGES + 1 + t); };
  auto sempty_bar = [&](int t) { return bars + 8u * (2 * PS_MAX_STAGES + 1 + PS_SF_STAGES + t); };
  uint8_t* tail = smem_gen + PS_BARS_OFF + 8 * PS_NUM_BARS;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(tail);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 8);

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const uint32_t splits = (uint32_t)prm.splits;
  const uint32_t rank = blockIdx.x % splits;          // in the cluster, which lies along x
  const int n0 = (int)(blockIdx.x / splits) * 128, m0 = (int)blockIdx.y * prm.bt;
  // this CTA's share of the k-steps, in pairs (may be none when K is short); past the end of K a copy brings zeros
  const int per = split_ksteps(prm.ksteps, (int)splits);
  const int k_begin = min(prm.ksteps, (int)rank * per), k_end = min(prm.ksteps, k_begin + per);
  const uint32_t half_bytes = (uint32_t)(P_TILE_BYTES + prm.bt * PK), stage_bytes = 2 * half_bytes;

  let_successor_start();
  if (threadIdx.x == 0) {
    for (int s = 0; s < prm.stages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(tfull, 1);
    for (int t = 0; t < PS_SF_STAGES; ++t) {
      mbar_init(sfull_bar(t), 4);
      mbar_init(sempty_bar(t), 1);
    }
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32((const void*)tmem_slot), PS_TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  wait_for_predecessors();
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  long long issued = 0;                   // uses of the ring, by the loader
  bool ok = true;

  if (warp == 0) {
    int s = 0;
    uint32_t ph = 0;
    for (int ks = k_begin; ks < k_end; ks += 2) {
      if (!(ok = ks < prm.waits.loaded)) break;
      if (!(ok = __all_sync(0xffffffffu, bounded_wait(empty_bar(s), ph ^ 1u, abort_flag, prm.waits)))) break;
      if (elect_one()) {
        mbar_arrive_expect_tx(full_bar(s), stage_bytes);
        const uint32_t dst = smem_base + (uint32_t)s * stage_bytes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          tma_load_2d(dst + h * half_bytes, &prm.tmW, full_bar(s), (ks + h) * PK, n0);
          tma_load_2d(dst + h * half_bytes + P_TILE_BYTES, &prm.tmX, full_bar(s), (ks + h) * PK, m0);
        }
      }
      __syncwarp();
      ++issued;
      if (++s == prm.stages) { s = 0; ph ^= 1u; }
    }
  } else if (warp == 1) {
    if (elect_one()) {
      int s = 0, t = 0;
      uint32_t ph = 0, tph = 0;
      for (int ks = k_begin; ks < k_end; ks += 2) {
        if (ks == k_begin || (ks & 3) == 0) {
          if (!(ok = bounded_wait(sfull_bar(t), tph, abort_flag, prm.waits))) break;
        }
        if (!(ok = bounded_wait(full_bar(s), ph, abort_flag, prm.waits))) break;
        tc_fence_after();
        const uint32_t sa = tmem_base + PS_SF_COL + 8u * t, sb = sa + 4;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t a = (((smem_base + (uint32_t)s * stage_bytes + h * half_bytes) >> 4) & 0x3FFFu) | (1u << 16), b = a + (P_TILE_BYTES >> 4);
          const uint32_t idesc = prm.idesc | mx_byte((ks & 3) + h);
          if (h == 1 && ks + 1 == k_end) break;      // K ends between the two
          umma1_mx(tmem_base, a, b, idesc, sa, sb, ks + h > k_begin ? 1u : 0u);
          umma1_mx(tmem_base, a + 2, b + 2, idesc, sa, sb, 1u);
          umma1_mx(tmem_base, a + 4, b + 4, idesc, sa, sb, 1u);
          umma1_mx(tmem_base, a + 6, b + 6, idesc, sa, sb, 1u);
        }
        umma_commit(empty_bar(s));
        if ((ks & 3) == 2 || ks + 2 >= k_end) {
          umma_commit(sempty_bar(t));
          if (++t == PS_SF_STAGES) { t = 0; tph ^= 1u; }
        }
        if (ks + 2 >= k_end) umma_commit(tfull);
        if (++s == prm.stages) { s = 0; ph ^= 1u; }
      }
    }
    __syncwarp();
  } else {
    const uint32_t quarter = (uint32_t)((warp & 3) * 32) << 16;
    const int w = warp & 3;
    const int g_end = k_begin < k_end ? (k_end + 3) >> 2 : 0;
    const uint32_t sbuf = smem_base + PS_SF_OFF;
    int next = k_begin >> 2, fb = 0;
    auto fetch_next = [&]() {
      if (next < g_end) {
        const uint32_t dst = sbuf + (uint32_t)fb * 1024u;
        fetch_scale_word(prm.w, next, n0, w * 32 + lane, dst);
        if (w * 32 < prm.bt) fetch_scale_word(prm.x, next, m0, w * 32 + lane, dst + 512);
        ++next;
        if (++fb == SF_BUFS) fb = 0;
      }
      cp_async_commit();
    };
#pragma unroll
    for (int d = 0; d < SF_AHEAD; ++d) fetch_next();
    int t = 0, rb = 0;
    uint32_t tph = 0;
    for (int left = max(0, g_end - (k_begin >> 2)); left > 0; --left) {
      cp_async_wait<SF_AHEAD - 1>();
      named_barrier(1, 128);
      fetch_next();
      if (ok) ok = __all_sync(0xffffffffu, bounded_wait(sempty_bar(t), tph ^ 1u, abort_flag, prm.waits));
      if (ok) {
        tc_fence_after();
        const uint32_t at = tmem_base + quarter + PS_SF_COL + 8u * t, src = sbuf + (uint32_t)rb * 1024u;
        scale_words_to_tmem(at, src, lane);
        scale_words_to_tmem(at + 4, src + 512, lane);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sfull_bar(t));
      }
      if (++t == PS_SF_STAGES) { t = 0; tph ^= 1u; }
      if (++rb == SF_BUFS) rb = 0;
    }
    cp_async_wait<0>();
    if (ok && k_begin < k_end) ok = __all_sync(0xffffffffu, bounded_wait(tfull, 0u, abort_flag, prm.waits));
    tc_fence_after();
  }

  const int valid = min(prm.bt, prm.M - m0);
  const int rows = min(128, prm.N - n0);                         // of the weight, in this tile
  // Every CTA lays its sums out as [token][128 rows] where its ring was (its own copies and MMAs are done), then CTA r adds up its
  // share of the tokens over the cluster (of one CTA too), in rank order, four rows to a thread.
  const int share = (valid + (int)splits - 1) / (int)splits;
  if (warp >= 2) {
    const int row = (warp & 3) * 32 + lane;
    const bool none = k_begin >= k_end || !ok;
    for (int c = 0; c < valid; c += 32) {
      uint32_t v[32];
      if (!none) {
        tmem_ld32(tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)c, v);
        tmem_ld_wait();
      }
      uint32_t* out = reinterpret_cast<uint32_t*>(smem_gen) + c * 128 + row;
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (c + j < valid) out[j * 128] = none ? 0u : v[j];
    }
    tc_fence_before();
  }
  __syncwarp();
  cluster_sync_all();
  if (warp >= 2 && lane * 4 < rows) {
    // four tokens at a time: their loads from the cluster's shared memory, some 200 clocks each, overlap
    for (int at0 = warp - 2; at0 < share; at0 += 16) {
      float4 sum[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) sum[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      const uint32_t first = (uint32_t)(((int)rank * share + at0) * 512 + lane * 16);
      for (uint32_t r = 0; r < splits; ++r) {
        const uint32_t from = map_to_cta(smem_base, r) + first;
        float4 part[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (at0 + 4 * u < share)      // tokens past the last one are read (the sums have room) and not stored
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(part[u].x), "=f"(part[u].y), "=f"(part[u].z), "=f"(part[u].w)
                         : "r"(from + 2048u * u)
                         : "memory");
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (at0 + 4 * u < share) {
            sum[u].x += part[u].x; sum[u].y += part[u].y; sum[u].z += part[u].z; sum[u].w += part[u].w;
          }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int j = (int)rank * share + at0 + 4 * u;
        if (at0 + 4 * u >= share || j >= valid) continue;
        // tiles start at multiples of 128 columns of C, so whole quads are aligned
        const int64_t o = (int64_t)(m0 + j) * prm.ldc + n0 + lane * 4;
        const bool whole = lane * 4 + 4 <= rows;
        const float s4[4] = {sum[u].x, sum[u].y, sum[u].z, sum[u].w};
        if (prm.c_f32) {
          float* C = reinterpret_cast<float*>(prm.C) + o;
          if (whole) *reinterpret_cast<float4*>(C) = sum[u];
          else
            for (int e = 0; lane * 4 + e < rows; ++e) C[e] = s4[e];
        } else {
          __nv_bfloat16* C = reinterpret_cast<__nv_bfloat16*>(prm.C) + o;
          if (whole) *reinterpret_cast<uint2*>(C) = make_uint2(pack_bf16x2(s4[0], s4[1]), pack_bf16x2(s4[2], s4[3]));
          else
            for (int e = 0; lane * 4 + e < rows; ++e) C[e] = __float2bfloat16_rn(s4[e]);
        }
      }
    }
  }
  __syncwarp();
  if (warp == 0 && *abort_flag) drain_copies(full_bar(0), 8u, prm.stages, issued);
  cluster_sync_all();                     // nobody leaves while its sums are being read
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, PS_TMEM_COLS);
  }
}

// ---- host side -----------------------------------------------------------------------------------------
// 8-bit operand: rows of K bytes, tiles of 128 bytes x box_rows.
inline bool make_map_8bit(CUtensorMap* map, const void* base, int64_t k, int64_t rows, int64_t pitch, int box_rows) {
  cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)pitch};
  cuuint32_t box[2] = {(cuuint32_t)PK, (cuuint32_t)box_rows};
  return encode_cached(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
struct ProductCall {
  int M, N, K;
  int a_type, b_type;
  const void *A, *B, *a_scales, *b_scales;
  int64_t lda, ldb, lds_a, lds_b;
  int c_f32;
  void* C;
  int64_t ldc;
  ProductWaits waits;
  cudaStream_t stream;
};

// Width of a tile: the one whose rounds over the 74 pairs take the least time, a k-step of a tile being bound by what it brings
// into shared memory, 256 + bn rows per pair.
inline int pair_bn(int tiles_m, int N) {
  int best = 0;
  long long best_cost = 0;
  for (int bn = PP_BN_MAX; bn >= 32; bn -= 32) {
    const long long tiles = (long long)tiles_m * ((N + bn - 1) / bn);
    const long long cost = (tiles + NUM_SMS / 2 - 1) / (NUM_SMS / 2) * (256 + bn);
    if (!best || cost < best_cost) { best = bn; best_cost = cost; }
  }
  return best;
}

struct PairPlan {
  int bn, tiles_m, tiles_n;
  int per_barrier, panel_cols;      // as in PairParams
};
inline PairPlan pair_plan(int M, int N, int K) {
  PairPlan p;
  p.tiles_m = (M + 255) / 256;
  p.bn = pair_bn(p.tiles_m, N);
  p.tiles_n = (N + p.bn - 1) / p.bn;
  // Narrow tiles spend more time on barriers than on MMAs: two k-steps to each (256 x 4096 x 4096 9.2 us against 10.4).  Wide ones keep the
  // six stages of one, for the loads' sake (16384 x 4096 x 4096 214 us against 216).
  p.per_barrier = p.bn <= 128 ? 2 : 1;
  // B beyond 48 MB goes through the L2 in panels of column tiles (never narrower than a round of tiles is tall).  Rows of A by K -> N, with
  // panels and without: 16384 by 4096 -> 14336 802 us against 850, 8192 -> 8192 883 against 985, 4096 -> 22016 1215 against 1396, 4096 -> 28672
  // (three) 1566 against 2008; where A is short they make no difference: 4096 by 4096 -> 14336 206 against 209, 1024 57 against 56.
  p.panel_cols = p.tiles_n;
  const long long b_bytes = (long long)K * N, most = 48ll << 20;
  if (b_bytes > most) {
    const int panels = (int)((b_bytes + most - 1) / most);
    p.panel_cols = (p.tiles_n + panels - 1) / panels;
    if (p.panel_cols < 8) p.panel_cols = p.tiles_n < 8 ? p.tiles_n : 8;
  }
  return p;
}

inline compact_status_t product_pair(const ProductCall& c) {
  static std::atomic<bool> attr[64];
  if (!set_smem_once(product_pair_kernel, PP_SMEM_BYTES, attr)) return COMPACT_ERR_CUDA;
  const PairPlan plan = pair_plan(c.M, c.N, c.K);
  PairParams p;
  memset(&p, 0, sizeof(p));
  p.M = c.M; p.N = c.N;
  p.ksteps = (c.K + PK - 1) / PK;
  p.tiles_m = plan.tiles_m; p.tiles_n = plan.tiles_n; p.bn = plan.bn;
  p.per_barrier = plan.per_barrier; p.panel_cols = plan.panel_cols;
  p.C = c.C; p.ldc = c.ldc; p.c_f32 = c.c_f32;
  p.idesc = mx_idesc(c.a_type, c.b_type, 256, p.bn);
  p.a.scales = (const uint32_t*)c.a_scales; p.a.lds = c.lds_a; p.a.rows = c.M;
  p.b.scales = (const uint32_t*)c.b_scales; p.b.lds = c.lds_b; p.b.rows = c.N;
  p.waits = c.waits;
  if (!make_map_8bit(&p.tmA, c.A, c.K, c.M, c.lda, 128)) return COMPACT_ERR_CUDA;
  if (!make_map_8bit(&p.tmB, c.B, c.K, c.N, c.ldb, p.bn / 2)) return COMPACT_ERR_CUDA;
  const long long total = (long long)p.tiles_m * p.tiles_n;
  if (total > 0x3fffffff) return COMPACT_ERR_SHAPE;
  const int pairs = total < NUM_SMS / 2 ? (int)total : NUM_SMS / 2;
  return launch(product_pair_kernel, dim3(2 * pairs), PP_THREADS, PP_SMEM_BYTES, 2, c.stream, p);
}

// Clusters of `size` CTAs of the splitting kernel that the GPU holds at once (a GPC's SMs are not always a multiple of the size).
inline int resident_clusters(unsigned size) {
  static std::atomic<int> known[64][9];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { cudaGetLastError(); return NUM_SMS / (int)size; }
  int k = known[dev][size].load(std::memory_order_acquire);
  if (k == 0) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3(size * NUM_SMS, 1, 1);
    cfg.blockDim = dim3(PS_THREADS, 1, 1);
    cfg.dynamicSmemBytes = PS_SMEM_BYTES;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = size;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&k, product_split_kernel, &cfg) != cudaSuccess || k < 1) { cudaGetLastError(); k = NUM_SMS / (int)size; }
    known[dev][size].store(k, std::memory_order_release);
  }
  return k;
}

// Which kernel: the splitting one up to 128 tokens where K can be split, up to 64 where the weight has a tile for most SMs already.  Times of
// the splitting kernel and of the pairs, weights coming from memory, in us:
//     4096 -> 4096     1 token 7.1, 17.1    64 8.2, 10.3     77 8.9, 10.3    128 9.9, 10.4     200 10.7, 10.4
//     4096 -> 11008    1 token 11.5, 19.5   64 13.2, 13.2    77 14.5, 13.4   128 16.4, 13.7    200 26.8, 14.0
//     11008 -> 4096    1 token 11.3, 38.8   64 12.7, 22.4    77 13.8, 22.5   128 14.8, 22.7    200 17.5, 22.9
//     2736 -> 1024     1 token 5.3, 10.4    64 6.6, 7.2      77 7.1, 7.3     128 8.6, 7.3      200 7.6, 7.3
//     512 -> 1376      1 token 3.3, 4.4     64 4.8, 3.8      77 5.2, 3.8     128 6.6, 3.9      200 6.2, 3.7
// The rule looks at neither a short K, where the pairs would win from 32 tokens on, nor a long one, where splitting would up to 200.
inline bool prefer_split(int M, int N) { return M <= 64 || (M <= 128 && (N + 127) / 128 <= NUM_SMS / 2); }

inline compact_status_t product_split(const ProductCall& c) {
  static std::atomic<bool> attr[64];
  if (!set_smem_once(product_split_kernel, PS_SMEM_BYTES, attr)) return COMPACT_ERR_CUDA;
  SplitParams p;
  memset(&p, 0, sizeof(p));
  p.M = c.M; p.N = c.N;
  p.ksteps = (c.K + PK - 1) / PK;
  const int tiles_m = (c.M + PS_BT_MAX - 1) / PS_BT_MAX;
  if (tiles_m > 65535) return COMPACT_ERR_SHAPE;
  p.bt = ((c.M + tiles_m - 1) / tiles_m + 15) / 16 * 16;
  p.stages = PS_RING_BYTES / (2 * (P_TILE_BYTES + p.bt * PK));
  if (p.stages > PS_MAX_STAGES) p.stages = PS_MAX_STAGES;
  // As many CTAs to a tile as the GPU holds of clusters for all tiles at once.  The time goes with the k-steps of a CTA (about 0.19 us
  // each) as long as there is one round of clusters: one token by 4096 x 4096, 32 tiles: 9.3 us with one CTA each, 6.7 with two, 5.7
  // with four, 12.5 with eight (two rounds).
  const int tiles_n = (c.N + 127) / 128;
  unsigned splits = 1;
  while (splits < 8 && (long long)tiles_n * tiles_m <= resident_clusters(2 * splits) && p.ksteps > 2 * (int)splits) splits *= 2;
  p.splits = (int)splits;
  p.C = c.C; p.ldc = c.ldc; p.c_f32 = c.c_f32;
  p.idesc = mx_idesc(c.b_type, c.a_type, 128, p.bt);
  p.w.scales = (const uint32_t*)c.b_scales; p.w.lds = c.lds_b; p.w.rows = c.N;
  p.x.scales = (const uint32_t*)c.a_scales; p.x.lds = c.lds_a; p.x.rows = c.M;
  p.waits = c.waits;
  if (!make_map_8bit(&p.tmW, c.B, c.K, c.N, c.ldb, 128)) return COMPACT_ERR_CUDA;
  if (!make_map_8bit(&p.tmX, c.A, c.K, c.M, c.lda, p.bt)) return COMPACT_ERR_CUDA;
  return launch(product_split_kernel, dim3(tiles_n * splits, tiles_m), PS_THREADS, PS_SMEM_BYTES, splits, c.stream, p);
}

}  // namespace blk
}  // namespace compact

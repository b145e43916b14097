// RMS norm with the residual's addition.  Forward: h = x + res, rstd = 1 / sqrt(mean(h^2) + eps), y = h rstd w, out in the
// input's type and/or in 8 bits with a scale for each 128 columns.  Backward, with g = dy w:
// dx = rstd g - h rstd^3 mean(g h) + dres,  dw = sum over tokens of dy h rstd.
// Both are bound by memory: a row is read once and written once.  (16384 x 4096 bf16, calls in a replayed graph: forward with
// residual and both outputs 103 us, 5.9 TB/s; y alone 44 us, 6.1; backward with residual gradient 78 us, 6.9, and 82 with the weight's and the sum
// over CTAs.  The 8-bit output alone, without residual, is bound by instruction issue: 55 us for 31 us of traffic.  fp32, forward with
// both outputs 206 us, 5.5 TB/s.)
//
// LANES threads, a group, share a row.  A thread holds U units of sixteen columns, eight neighbouring lanes a block of 128, whose
// maximum the 8-bit output needs: three shuffles for sixteen values.  A unit is two vectors of eight: of 16-bit values, columns
// 8 l .. 8 l + 7 of either half of the block; of 32-bit values, two quads in either half, so that every access of eight lanes
// covers 128 neighbouring bytes.  One CTA per SM stays for the whole call, with as many groups as its threads allow, and group g of
// CTA b takes rows b + grid (g + groups k).  A row's sum is a chain of waits (the copy, five shuffles, a barrier, the second
// pass): what hides it is several groups per SM and rows on their way in shared memory, `stages` deep per group.
// Groups never wait for each other.
#pragma once
#include "block_common.cuh"
#include "tc_common.cuh"

namespace compact {
namespace blk {

// A thread copies the columns it will read itself (cp.async, 16 bytes each, into places of its own), so that nothing but its own wait
// stands between the copy and the read.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// until at most `pending` of this thread's groups of copies are in flight
__device__ __forceinline__ void copies_wait(int pending) {
  if (pending >= 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
  else if (pending == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (pending == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}
// A vector from its first column q: eight neighbouring columns of 16-bit values; of 32-bit values two quads, at q and q + 32.
template <typename T>
__device__ __forceinline__ Vec8<T> norm_load(const T* row, int q0, int n) {
  if constexpr (sizeof(T) == 2) {
    return load8(row, q0, n);
  } else {
    Vec8<float> x;
    float f[8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int q = q0 + 32 * k;
      if (q + 4 <= n) *reinterpret_cast<float4*>(f + 4 * k) = *reinterpret_cast<const float4*>(row + q);
      else
#pragma unroll
        for (int i = 0; i < 4; ++i) f[4 * k + i] = q + i < n ? row[q + i] : 0.f;
    }
    x.set(f);
    return x;
  }
}
template <typename T>
__device__ __forceinline__ void norm_store(T* row, int q0, int n, const Vec8<T>& x) {
  if constexpr (sizeof(T) == 2) {
    store8(row, q0, n, x);
  } else {
    float f[8];
    x.get(f);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int q = q0 + 32 * k;
      if (q + 4 <= n) *reinterpret_cast<float4*>(row + q) = make_float4(f[4 * k], f[4 * k + 1], f[4 * k + 2], f[4 * k + 3]);
      else
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (q + i < n) row[q + i] = f[4 * k + i];
    }
  }
}
template <typename T>
__device__ __forceinline__ void norm_store_fp8(uint8_t* row, int q0, int n, uint2 v) {
  if constexpr (sizeof(T) == 2) {
    store8_fp8(row, q0, n, v);
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int q = q0 + 32 * k;
      const uint32_t w = k == 0 ? v.x : v.y;
      if (q + 4 <= n) *reinterpret_cast<uint32_t*>(row + q) = w;
      else
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (q + i < n) row[q + i] = (uint8_t)(w >> (8 * i));
    }
  }
}
// The same to a vector's place in shared memory, asynchronously (q0 < n); past n: zeros.  16-byte parts of a vector lie LANES parts apart.
template <typename T, int LANES>
__device__ __forceinline__ void norm_copy(uint32_t dst, const T* row, int q0, int n) {
  constexpr int ELEMS = 16 / (int)sizeof(T);
#pragma unroll
  for (int k = 0; k < (int)sizeof(Vec8<T>) / 16; ++k) {
    const int q = q0 + 32 * k;
    if (q + ELEMS <= n) copy16(dst + 16u * LANES * k, row + q, 16);
    else copy16(dst + 16u * LANES * k, q < n ? row + q : row, max(0, n - q) * (int)sizeof(T));
  }
}
template <typename T, int LANES>
__device__ __forceinline__ Vec8<T> place_load(const uint8_t* at) {
  Vec8<T> x;
#pragma unroll
  for (int k = 0; k < (int)sizeof(x) / 16; ++k) reinterpret_cast<uint4*>(&x)[k] = *reinterpret_cast<const uint4*>(at + 16 * LANES * k);
  return x;
}
template <int LANES, typename X>
__device__ __forceinline__ void place_store(uint8_t* at, const X& x) {
#pragma unroll
  for (int k = 0; k < (int)sizeof(x) / 16; ++k) *reinterpret_cast<uint4*>(at + 16 * LANES * k) = reinterpret_cast<const uint4*>(&x)[k];
}

constexpr int PIPE_MAX_STAGES = 4;
constexpr int PIPE_BYTES = 220 * 1024;
// Threads of a CTA, by the registers (80 or 128) that a thread's units of values and sums need.  Backward 16384 x 4096 with residual: 82 us
// at 768 threads; 103 at 1024, which spill; 89 at 512.
__host__ __device__ constexpr int norm_fwd_threads(int elem_bytes, int u) { return elem_bytes == 2 ? 768 : 512; }
__host__ __device__ constexpr int norm_bwd_threads(int elem_bytes, int u) { return elem_bytes == 2 && u == 1 ? 768 : 512; }

// The forward's weight: in registers, or where two units leave no room there, in shared memory.  The backward, whose shared memory is busier,
// keeps registers.  Read again from global memory for every row it lengthens the chain.  (16384 x 11008, a thread holding 24 columns:
// forward with residual and both outputs 249 us from shared memory, 276 read again; backward 198 from registers, 224, 280.)
__host__ __device__ constexpr bool weight_in_smem(int elem_bytes, int u, bool bwd) { return !bwd && elem_bytes == 2 && u >= 2; }

// Threads to a row and units to a thread
#define NORM_FWD_LAYOUTS(F) F(32, 1) F(32, 2) F(64, 2) F(192, 1) F(256, 1) F(192, 2) F(256, 2) F(384, 2) F(512, 2)
#define NORM_BWD_LAYOUTS(F) F(32, 1) F(32, 2) F(64, 2) F(192, 1) F(256, 1) F(384, 1) F(256, 2) F(384, 2) F(512, 2)
#define NORM_LAYOUT_PAIR(L, UU) {L, UU},

struct NormPlan {
  int lanes, u;                  // of the kernel
  int groups, grid, stages;
  int weight_at, smem;           // bytes
};
// `inputs`: arrays a row is read from.
inline NormPlan norm_plan(int n, int64_t tokens, int elem_bytes, int inputs, bool bwd) {
  // the layout with the fewest idle units
  static const int fwd[9][2] = {NORM_FWD_LAYOUTS(NORM_LAYOUT_PAIR)}, back[9][2] = {NORM_BWD_LAYOUTS(NORM_LAYOUT_PAIR)};
  NormPlan p = {0, 0, 1, 1, 1, 0, 0};
  for (const auto& s : bwd ? back : fwd)
    if (n <= 16 * s[0] * s[1]) {
      p.lanes = s[0];
      p.u = s[1];
      break;
    }
  const int row_bytes = inputs * p.lanes * p.u * 16 * elem_bytes;
  int most = (bwd ? norm_bwd_threads(elem_bytes, p.u) : norm_fwd_threads(elem_bytes, p.u)) / p.lanes;
  if (p.lanes > 32 && most > 15) most = 15;              // named barriers
  // Two stages each for all groups come before more groups.  (Of fp32 rows of 513 to 2048 columns the backward without a residual's gradient
  // has more groups than with one, and so another order of the sum over tokens.  Room for three inputs in either case would make that
  // order the same, for 16384 x 600 in 31 us against 26 and 8192 x 1376 in 34 against 28.)
  const int weight_bytes = weight_in_smem(elem_bytes, p.u, bwd) ? p.lanes * p.u * 16 * elem_bytes : 0, room = PIPE_BYTES - weight_bytes;
  while (most > 1 && 2 * most * row_bytes > room) --most;
  // a row to a CTA as long as there are SMs; the backward's few rows share one CTA, which then needs no sum over CTAs
  const bool together = bwd && tokens <= most;
  p.grid = tokens < 1 || together ? 1 : (int)(tokens < tc::NUM_SMS ? tokens : tc::NUM_SMS);
  const int64_t rows = (tokens + p.grid - 1) / p.grid;          // of a CTA
  p.groups = rows < 1 ? 1 : (rows < most ? (int)rows : most);
  p.stages = room / (p.groups * row_bytes);
  if (p.stages > PIPE_MAX_STAGES) p.stages = PIPE_MAX_STAGES;
  const int64_t turns = (rows + p.groups - 1) / p.groups;
  if (p.stages > turns) p.stages = turns < 1 ? 1 : (int)turns;
  p.weight_at = p.groups * p.stages * row_bytes;
  p.smem = p.weight_at + weight_bytes;
  return p;
}

// A thread's place in its group's rows
template <typename T, int LANES, int U>
struct RowPipe {
  static constexpr int V = 2 * U;
  static constexpr int VB = (int)sizeof(Vec8<T>);
  static constexpr uint32_t INPUT_BYTES = (uint32_t)(LANES * V * VB);
  int lane, group, groups;
  int64_t row, stride;           // this group's rows
  uint8_t* base;                 // first part of vector v of input k in stage s: base + s * stage_bytes + k * INPUT_BYTES + v * LANES * VB
  uint32_t addr, stage_bytes;
  __device__ __forceinline__ RowPipe(uint8_t* smem, int stages, int inputs) {
    lane = threadIdx.x % LANES;
    group = threadIdx.x / LANES;
    groups = blockDim.x / LANES;
    row = (int64_t)blockIdx.x + (int64_t)gridDim.x * group;
    stride = (int64_t)gridDim.x * groups;
    stage_bytes = INPUT_BYTES * (uint32_t)inputs;
    base = smem + (uint32_t)(group * stages) * stage_bytes + lane * 16;
    addr = (uint32_t)__cvta_generic_to_shared(base);
  }
  __device__ __forceinline__ int block(int u) const { return (u * LANES + (lane & ~7)) * 16; }       // first column of a unit's block
  __device__ __forceinline__ int column(int v) const { return block(v >> 1) + 64 * (v & 1) + (lane & 7) * (16 / (int)sizeof(T)); }
  __device__ __forceinline__ bool has(int v, int n) const { return column(v) < n; }
  __device__ __forceinline__ Vec8<T> at(int stage, int input, int v) const {
    return place_load<T, LANES>(base + (uint32_t)stage * stage_bytes + (uint32_t)input * INPUT_BYTES + v * LANES * VB);
  }
  __device__ __forceinline__ void copy(int stage, int input, const T* src, int n) const {
    const uint32_t to = addr + (uint32_t)stage * stage_bytes + (uint32_t)input * INPUT_BYTES;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (has(v, n)) norm_copy<T, LANES>(to + (uint32_t)(v * LANES * VB), src, column(v), n);
  }
};

// The weight of a thread's columns, for the whole call.
template <typename T, int LANES, int U, bool SMEM>
struct RowWeight {
  static constexpr int V = 2 * U;
  Vec8<T> kept[SMEM ? 1 : V];
  const uint8_t* shared;
  // `shared_at`: LANES * V vectors of shared memory, laid out as the rows are, filled by the first group
  __device__ __forceinline__ RowWeight(const void* weight, const RowPipe<T, LANES, U>& pipe, int n, uint8_t* shared_at) : shared(shared_at + pipe.lane * 16) {
    const T* w = reinterpret_cast<const T*>(weight);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      Vec8<T> x;
      if (pipe.has(v, n)) x = norm_load(w, pipe.column(v), n);
      else x.clear();
      if (!SMEM) kept[SMEM ? 0 : v] = x;
      else if (threadIdx.x < LANES) place_store<LANES>(shared_at + pipe.lane * 16 + v * LANES * (int)sizeof(Vec8<T>), x);
    }
    if (SMEM) __syncthreads();
  }
  __device__ __forceinline__ Vec8<T> vector(int v) const {
    return SMEM ? place_load<T, LANES>(shared + v * LANES * (int)sizeof(Vec8<T>)) : kept[SMEM ? 0 : v];
  }
};

// Sum over the LANES threads of a row; every one of them gets it.  One warp: shuffles alone.  More: one word per warp in shared
// memory, two sets used in turn, so that one barrier (of the group) per row is enough.
template <int LANES>
__device__ __forceinline__ float row_sum(float s, float* red, int group, int turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if (LANES > 32) {
    constexpr int WARPS = LANES / 32;
    float* set = red + (group * 2 + (turn & 1)) * WARPS;
    if ((threadIdx.x & 31) == 0) set[(threadIdx.x % LANES) >> 5] = s;
    tc::named_barrier(1 + group, LANES);
    s = 0.f;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) s += set[i];
  }
  return s;
}
constexpr int RED_WORDS = 2 * 32;      // two sets of one word per warp

struct NormFwdArgs {
  const void *x, *res, *w;
  void *h, *y;
  float* rstd;
  uint8_t *q, *scales;
  int64_t ldx, ldr, ldh, ldy, ldq, lds, tokens;
  int n, stages, fp8, weight_at;      // weight_at: of the weight in shared memory
  float eps;
};

// RES: with a residual (then h is stored too, unless NULL).  OUT: 1 for y, 2 for the 8-bit output, 3 for both, 0 for h alone.  Each is a kernel of its
// own: tests of NULL pointers inside the loops cost the 16384 x 4096 forward without residual 57 us against 44.
template <typename T, int LANES, int U, bool RES, int OUT>
__global__ void __launch_bounds__(norm_fwd_threads(sizeof(T), U)) rms_norm_fwd_kernel(const __grid_constant__ NormFwdArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int V = 2 * U;
  __shared__ float red[RED_WORDS];
  let_successor_start();
  wait_for_predecessors();
  const int n = a.n, stages = a.stages;
  const float inv_n = 1.f / (float)n;
  constexpr bool Y = (OUT & 1) != 0, Q = (OUT & 2) != 0;
  RowPipe<T, LANES, U> pipe(smem, stages, RES ? 2 : 1);
  auto fetch = [&](int64_t r, int s) {
    if (r < a.tokens) {
      pipe.copy(s, 0, reinterpret_cast<const T*>(a.x) + r * a.ldx, n);
      if (RES) pipe.copy(s, 1, reinterpret_cast<const T*>(a.res) + r * a.ldr, n);
    }
    copies_commit();
  };
  int64_t ahead = pipe.row;
  int slot = 0, fslot = 0, turn = 0;
  for (int s = 0; s + 1 < stages; ++s, ahead += pipe.stride) {
    fetch(ahead, fslot);
    if (++fslot == stages) fslot = 0;
  }
  const RowWeight<T, LANES, U, weight_in_smem(sizeof(T), U, false)> weight(a.w, pipe, n, smem + a.weight_at);
  for (int64_t row = pipe.row; row < a.tokens; row += pipe.stride, ++turn) {
    fetch(ahead, fslot);
    ahead += pipe.stride;
    if (++fslot == stages) fslot = 0;
    copies_wait(stages - 1);
    Vec8<T> hv[V];
    F2 ss2 = f2(0.f, 0.f);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = pipe.column(v);
      if (!pipe.has(v, n)) {
        hv[v].clear();
        continue;
      }
      hv[v] = pipe.at(slot, 0, v);
      if (RES) {
        const Vec8<T> rv = pipe.at(slot, 1, v);
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) f2_get(f2_add(hv[v].pair(i), rv.pair(i)), f[2 * i], f[2 * i + 1]);
        // rounded before it is normed: the backward reads the stored h and must see what was normed
        hv[v].set(f);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) ss2 = f2_fma(hv[v].pair(i), hv[v].pair(i), ss2);
    }
    float ss, ss_hi;
    f2_get(ss2, ss, ss_hi);
    if (++slot == stages) slot = 0;
    const float rstd = 1.f / sqrtf(row_sum<LANES>(ss + ss_hi, red, pipe.group, turn) * inv_n + a.eps);
    if (a.rstd && pipe.lane == 0) a.rstd[row] = rstd;
    const F2 rstd2 = f2(rstd, rstd);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int first = pipe.block(u);
      if (first >= n) continue;                              // the whole block lies past the row
      F2 y[2][4];
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int v = 2 * u + j;
        const Vec8<T> w = weight.vector(v);
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[j][i] = f2_mul(f2_mul(hv[v].pair(i), rstd2), w.pair(i));
          f2_get(y[j][i], f[2 * i], f[2 * i + 1]);
        }
        if (RES && a.h && pipe.has(v, n)) norm_store(reinterpret_cast<T*>(a.h) + row * a.ldh, pipe.column(v), n, hv[v]);
        if (Y && pipe.has(v, n)) {
          Vec8<T> yv;
          yv.set(f);
          norm_store(reinterpret_cast<T*>(a.y) + row * a.ldy, pipe.column(v), n, yv);
        }
        if (Q) m = max(m, magnitude8(f));                  // past the row: zeros
      }
      if (Q) {
        const uint32_t block_lanes = 0xFFu << (threadIdx.x & 24);
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(block_lanes, m, o));
        const uint32_t byte = scale_byte(m, range_exponent(a.fp8));
        const float inv = inverse_scale(byte);
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (pipe.has(2 * u + j, n)) norm_store_fp8<T>(a.q + row * a.ldq, pipe.column(2 * u + j), n, a.fp8 == 0 ? pack8_fp8<0>(y[j], inv) : pack8_fp8<1>(y[j], inv));
        if ((pipe.lane & 7) == 0) a.scales[((int64_t)(first >> 9) * a.lds + row) * 4 + ((first >> 7) & 3)] = (uint8_t)byte;
      }
    }
    // bytes of the last word past the last block
    if (Q) {
      const int blocks = (n + QB - 1) / QB;
      if (pipe.lane < ((4 - blocks) & 3)) a.scales[((int64_t)(blocks >> 2) * a.lds + row) * 4 + (blocks & 3) + pipe.lane] = (uint8_t)SCALE_ONE;
    }
  }
  copies_wait(0);
}

struct NormBwdArgs {
  const void *dy, *h, *w, *dres;
  const float* rstd;
  void* dx;
  float* partial;        // [gridDim.x][n], or dw itself for a single CTA, or NULL
  int accumulate;        // a single CTA adds to dw
  int64_t lddy, ldh, ldr, lddx, tokens;
  int n, stages;
};

// A group keeps its part of dw for its columns in registers; a CTA's groups add theirs up at the end, in order, and the CTAs' parts
// are summed, in order, by sum_partials_kernel.
template <typename T, int LANES, int U>
__global__ void __launch_bounds__(norm_bwd_threads(sizeof(T), U)) rms_norm_bwd_kernel(const __grid_constant__ NormBwdArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int V = 2 * U;
  __shared__ float red[RED_WORDS];
  let_successor_start();
  wait_for_predecessors();
  const int n = a.n, stages = a.stages;
  const float inv_n = 1.f / (float)n;
  const bool with_res = a.dres != nullptr && a.dx != nullptr;
  RowPipe<T, LANES, U> pipe(smem, stages, a.dres ? 3 : 2);
  auto fetch = [&](int64_t r, int s) {
    if (r < a.tokens) {
      pipe.copy(s, 0, reinterpret_cast<const T*>(a.dy) + r * a.lddy, n);
      pipe.copy(s, 1, reinterpret_cast<const T*>(a.h) + r * a.ldh, n);
      if (with_res) pipe.copy(s, 2, reinterpret_cast<const T*>(a.dres) + r * a.ldr, n);
    }
    copies_commit();
  };
  int64_t ahead = pipe.row;
  int slot = 0, fslot = 0, turn = 0;
  for (int s = 0; s + 1 < stages; ++s, ahead += pipe.stride) {
    fetch(ahead, fslot);
    if (++fslot == stages) fslot = 0;
  }
  const RowWeight<T, LANES, U, false> weight(a.w, pipe, n, smem);
  F2 dw[V][4];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 4; ++i) dw[v][i] = f2(0.f, 0.f);
  float rstd_next = pipe.row < a.tokens ? a.rstd[pipe.row] : 0.f;
  for (int64_t row = pipe.row; row < a.tokens; row += pipe.stride, ++turn) {
    fetch(ahead, fslot);
    ahead += pipe.stride;
    if (++fslot == stages) fslot = 0;
    const float rstd = rstd_next;
    if (row + pipe.stride < a.tokens) rstd_next = a.rstd[row + pipe.stride];
    copies_wait(stages - 1);
    const int cur = slot;
    if (++slot == stages) slot = 0;
    const F2 rstd2 = f2(rstd, rstd);
    F2 dot2 = f2(0.f, 0.f);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!pipe.has(v, n)) continue;
      const Vec8<T> g = pipe.at(cur, 0, v), h = pipe.at(cur, 1, v), w = weight.vector(v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const F2 p = f2_mul(g.pair(i), f2_mul(h.pair(i), rstd2));        // dy * xhat
        dw[v][i] = f2_add(dw[v][i], p);
        dot2 = f2_fma(p, w.pair(i), dot2);
      }
    }
    if (!a.dx) continue;
    float dot, dot_hi;
    f2_get(dot2, dot, dot_hi);
    const float k = row_sum<LANES>(dot + dot_hi, red, pipe.group, turn) * inv_n * rstd * rstd;      // dx = rstd g - h k + dres
    const F2 k2 = f2(-k, -k);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!pipe.has(v, n)) continue;
      const Vec8<T> g = pipe.at(cur, 0, v), h = pipe.at(cur, 1, v), w = weight.vector(v);
      float o[8];
      Vec8<T> r;
      if (with_res) r = pipe.at(cur, 2, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        F2 x = f2_mul(rstd2, f2_mul(g.pair(i), w.pair(i)));
        x = f2_fma(h.pair(i), k2, x);
        if (with_res) x = f2_add(x, r.pair(i));
        f2_get(x, o[2 * i], o[2 * i + 1]);
      }
      Vec8<T> ov;
      ov.set(o);
      norm_store(reinterpret_cast<T*>(a.dx) + row * a.lddx, pipe.column(v), n, ov);
    }
  }
  copies_wait(0);
  if (!a.partial) return;
  // the groups' parts, where the rows have gone through: [group][column]
  constexpr int SPAN = LANES * V * 8;
  float* part = reinterpret_cast<float*>(smem);
  __syncthreads();
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float4 x;
      f2_get(dw[v][2 * k], x.x, x.y);
      f2_get(dw[v][2 * k + 1], x.z, x.w);
      *reinterpret_cast<float4*>(part + pipe.group * SPAN + pipe.column(v) + (sizeof(T) == 2 ? 4 : 32) * k) = x;
    }
  __syncthreads();
  float* out = a.partial + (int64_t)blockIdx.x * n;
  for (int c = threadIdx.x; c < n; c += blockDim.x) {
    float s = 0.f;
    for (int g = 0; g < pipe.groups; ++g) s += part[g * SPAN + c];
    out[c] = a.accumulate ? out[c] + s : s;
  }
}

// out[c] (+)= sum over p of partial[p][c]: 32 columns to a CTA, its 32 warps taking every 32nd part, then the warps' sums in a fixed order.
__global__ void __launch_bounds__(1024) sum_partials_kernel(const float* partial, int parts, int n, float* out, int accumulate) {
  __shared__ float red[32][33];
  let_successor_start();
  wait_for_predecessors();
  const int lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane, warp = threadIdx.x >> 5;
  float s = 0.f;
  if (c < n) {
#pragma unroll 8
    for (int p = warp; p < parts; p += 32) s += partial[(int64_t)p * n + c];
  }
  red[warp][lane] = s;
  __syncthreads();
  // warp w sums column w of the 32: its lanes hold the warps' sums
  s = red[lane][warp];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  const int mine = blockIdx.x * 32 + warp;
  if (lane == 0 && mine < n) out[mine] = accumulate ? out[mine] + s : s;
}

}  // namespace blk
}  // namespace compact

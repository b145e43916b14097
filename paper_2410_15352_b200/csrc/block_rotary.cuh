// Rotary positions: pair (a, b) of a head at position p becomes (a cos - b sin, a sin + b cos) of the angle p w_i; the
// gradient is the transpose (sin negated).  Bound by memory: every element read once and written once, in 16-byte
// pieces; a CTA computes the angles of its tokens once into shared memory and all heads of both tensors use them.
#pragma once
#include "block_common.cuh"

namespace compact {
namespace blk {

constexpr int ROT_MAX_PAIRS = 256;
constexpr int ROT_THREADS = 256;
constexpr int ROT_SMEM_PAIRS = 1024;      // cos/sin pairs a CTA holds (8 KB)
constexpr int ROT_CTAS = 8;               // of 256 threads, with 32 registers each

// Speed of each pair as a fraction of a turn per position, times 2^64.  The product with the position wraps modulo one turn, exactly.
struct RotaryTurns {
  uint64_t w[ROT_MAX_PAIRS];
};

struct RotaryArgs {
  const void *q, *k;
  void *qo, *ko;
  int64_t q_token, q_head, k_token, k_head, qo_token, qo_head, ko_token, ko_head;
  const void* positions;
  int64_t first_position, tokens;
  int pos_bits, back, heads, kv_heads, pairs, head_dim;
  int tokens_per_cta, heads_per_cta;      // a CTA takes this many tokens and this many of the heads + kv_heads
  int pieces;                             // per head: turned pieces and, when they are copied, pieces of the rest
  int turned_pieces;
  uint32_t pieces_magic, heads_magic;     // ceil(2^32 / d): exact quotients for numerators below 2^32 / d (0 stands for d = 1)
  float attention_factor;
};

__device__ __forceinline__ uint32_t quotient(uint32_t i, uint32_t magic) { return magic ? __umulhi(i, magic) : i; }

// VEC consecutive elements (16 bytes, or 1 element where strides or the head's cut do not allow it)
template <typename T, int VEC>
struct Piece {
  alignas(VEC * sizeof(T)) T e[VEC];
  __device__ __forceinline__ void load(const T* p) {
    if (VEC * sizeof(T) == 16) *reinterpret_cast<uint4*>(e) = *reinterpret_cast<const uint4*>(p);
    else
#pragma unroll
      for (int i = 0; i < VEC; ++i) e[i] = p[i];
  }
  __device__ __forceinline__ void store(T* p) const {
    if (VEC * sizeof(T) == 16) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(e);
    else
#pragma unroll
      for (int i = 0; i < VEC; ++i) p[i] = e[i];
  }
};

// Place of pair p of a token in the table.  A piece reads its VEC pairs as VEC / 2 float4, and neighbouring threads take
// neighbouring pieces: float4 j of all pieces lie side by side, so that the reads of a warp have no bank conflicts.
template <int VEC>
__device__ __forceinline__ int table_index(int tok, int p, int pieces) {
  if (VEC == 1) return tok * pieces + p;
  return ((tok * (VEC / 2) + (p % VEC) / 2) * pieces + p / VEC) * 2 + (p & 1);
}

// A piece of work, interleaved: 2 VEC consecutive elements (VEC pairs).  Halves: VEC elements of the first half and the VEC that
// belong to them in the second.  Either way two loads, VEC pairs, two stores.  A piece of the rest of the head: up to 2 VEC copied.
template <typename T, int VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(ROT_THREADS, ROT_CTAS) rotary_kernel(const __grid_constant__ RotaryArgs a, const __grid_constant__ RotaryTurns turns) {
  __shared__ __align__(16) float2 cs[ROT_SMEM_PAIRS];
  let_successor_start();
  wait_for_predecessors();
  const int64_t t0 = (int64_t)blockIdx.x * a.tokens_per_cta;
  const int nt = (int)min((int64_t)a.tokens_per_cta, a.tokens - t0);
  const int h0 = (int)blockIdx.y * a.heads_per_cta;
  const int nh = min(a.heads_per_cta, a.heads + a.kv_heads - h0);
  for (int i = threadIdx.x; i < nt * a.pairs; i += ROT_THREADS) {
    const int tok = i / a.pairs, p = i - tok * a.pairs;
    int64_t pos = a.first_position + t0 + tok;
    if (a.positions)
      pos = a.pos_bits == 64 ? reinterpret_cast<const int64_t*>(a.positions)[t0 + tok] : (int64_t)reinterpret_cast<const int32_t*>(a.positions)[t0 + tok];
    // the top 32 bits of the fraction of a turn, as a number in [-1/2, 1/2)
    const int32_t frac = (int32_t)(uint32_t)(((uint64_t)pos * turns.w[p]) >> 32);
    float s, c;
    sincospif((float)frac * 4.6566128730773926e-10f, &s, &c);      // 2^-31: sincospi takes half turns
    cs[table_index<VEC>(tok, p, a.turned_pieces)] = make_float2(c * a.attention_factor, (a.back ? -s : s) * a.attention_factor);
  }
  __syncthreads();
  // One piece at a time to a thread: with 2048 threads to an SM that keeps 64 KB on their way, and leaves registers for all of them.
  // (16384 tokens of 64 heads of 128, bf16, calls in a replayed graph: 85 us, 6.3 TB/s; fp32 163, 6.6 TB/s.  Two pieces, half the threads, took a
  // fifth longer; four, a quarter, 1.6 times as long.)
  const uint32_t items = (uint32_t)(nt * nh * a.pieces);
  for (uint32_t i = threadIdx.x; i < items; i += ROT_THREADS) {
    const uint32_t th = quotient(i, a.pieces_magic);
    const int c = (int)(i - th * (uint32_t)a.pieces);
    const uint32_t tok = nh == a.heads_per_cta ? quotient(th, a.heads_magic) : th / (uint32_t)nh;
    const int h = h0 + (int)(th - tok * (uint32_t)nh);
    const int64_t t = t0 + tok;
    const bool is_q = h < a.heads;
    const T* src = is_q ? reinterpret_cast<const T*>(a.q) + t * a.q_token + h * a.q_head
                        : reinterpret_cast<const T*>(a.k) + t * a.k_token + (h - a.heads) * a.k_head;
    T* dst = is_q ? reinterpret_cast<T*>(a.qo) + t * a.qo_token + h * a.qo_head
                  : reinterpret_cast<T*>(a.ko) + t * a.ko_token + (h - a.heads) * a.ko_head;
    Piece<T, VEC> lo, hi;
    if (c >= a.turned_pieces) {                    // the rest of the head passes through
      const int e = 2 * a.pairs + (c - a.turned_pieces) * 2 * VEC;
      const bool two = a.head_dim - e > VEC;
      lo.load(src + e);
      if (two) hi.load(src + e + VEC);
      lo.store(dst + e);
      if (two) hi.store(dst + e + VEC);
      continue;
    }
    const int e = INTERLEAVED ? c * 2 * VEC : c * VEC, other = e + (INTERLEAVED ? VEC : a.pairs);
    lo.load(src + e);
    hi.load(src + other);
    const int first = table_index<VEC>((int)tok, c * VEC, a.turned_pieces);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const float2 z = cs[first + (j / 2) * 2 * a.turned_pieces + (j & 1)];
      T& x = INTERLEAVED ? (2 * j < VEC ? lo.e[(2 * j) % VEC] : hi.e[(2 * j) % VEC]) : lo.e[j];
      T& y = INTERLEAVED ? (2 * j + 1 < VEC ? lo.e[(2 * j + 1) % VEC] : hi.e[(2 * j + 1) % VEC]) : hi.e[j];
      const float fx = to_float(x), fy = to_float(y);
      x = from_float<T>(fx * z.x - fy * z.y);
      y = from_float<T>(fx * z.y + fy * z.x);
    }
    lo.store(dst + e);
    hi.store(dst + other);
  }
}

}  // namespace blk
}  // namespace compact

// What the memory-bound block operators share: 16-byte vectors of bf16 or fp32 as floats, and the 8-bit formats.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace compact {
namespace blk {

constexpr int QB = 128;            // columns that share a scale
constexpr uint32_t SCALE_ONE = 127u;
constexpr uint32_t SCALE_NAN = 255u;

// Every kernel of this family is launched behind the one before it in its stream without waiting for its end (programmatic stream
// serialization): it lets its own successor come up, prepares what needs no memory of others, and touches global memory
// only when everything before it is done.  That hides a launch's start, 2 to 3 us, in a sequence of short calls.  What it reads may
// thus be written by its predecessor while it runs already: no pointer of these kernels is __restrict__, and nothing is read through
// the read-only path (__ldg), whose loads may be moved ahead of the wait.
__device__ __forceinline__ void let_successor_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_predecessors() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Two floats to an instruction
struct F2 {
  unsigned long long v;
};
__device__ __forceinline__ F2 f2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void f2_get(F2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v)); }
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}

// Eight consecutive elements, the unit every kernel here works in: one 16-byte load of bf16, two of fp32.
template <typename T>
struct Vec8;
template <>
struct Vec8<__nv_bfloat16> {
  uint4 r;
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ F2 pair(int i) const {
    const uint32_t w = i == 0 ? r.x : i == 1 ? r.y : i == 2 ? r.z : r.w;
    return f2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    r = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void clear() { r = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { r = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void load_once(const __nv_bfloat16* p) { r = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = r; }
};
template <>
struct Vec8<float> {
  float4 a, b;
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ F2 pair(int i) const {
    return i == 0 ? f2(a.x, a.y) : i == 1 ? f2(a.z, a.w) : i == 2 ? f2(b.x, b.y) : f2(b.z, b.w);
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    a = make_float4(f[0], f[1], f[2], f[3]);
    b = make_float4(f[4], f[5], f[6], f[7]);
  }
  __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void load_once(const float* p) {
    a = __ldcs(reinterpret_cast<const float4*>(p));
    b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = a;
    reinterpret_cast<float4*>(p)[1] = b;
  }
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Columns c .. c+7 of a row of `cols`: whole vectors where they fit (rows start on 16 bytes and c is a multiple of 8),
// element by element at the ragged end, zeros past it.
template <typename T>
__device__ __forceinline__ Vec8<T> load8(const T* row, int64_t c, int64_t cols) {
  Vec8<T> v;
  if (c + 8 <= cols) {
    v.load(row + c);
  } else {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = c + i < cols ? to_float(row[c + i]) : 0.f;
    v.set(f);
  }
  return v;
}
template <typename T>
__device__ __forceinline__ void store8(T* row, int64_t c, int64_t cols, const Vec8<T>& v) {
  if (c + 8 <= cols) {
    v.store(row + c);
  } else {
    float f[8];
    v.get(f);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) row[c + i] = from_float<T>(f[i]);
  }
}

// ---- 8-bit formats -----------------------------------------------------------------------
// Both types' largest values are 1.75 * 2^k (k = 8 for e4m3, 15 for e5m2), so the least power of two that brings a
// magnitude a inside the range is read off its bits: the exponent less k, one more when the fraction exceeds 0.75.
// `bits` are those of a non-negative float; infinities and NaN give the NaN scale.
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits, int k) {
  if (bits >= 0x7F800000u) return SCALE_NAN;
  if (bits == 0u) return SCALE_ONE;
  const int e = (int)((bits + 0x1FFFFFu) >> 23) - k;
  return e > 0 ? (uint32_t)e : 0u;
}
// 2^(127 - byte), what values are multiplied by; exact in fp32 for every byte scale_byte gives (NaN blocks: 1).
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return byte == SCALE_NAN ? 1.f : __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ int range_exponent(int fp8) { return fp8 == 0 ? 8 : 15; }

template <int FP8>
__device__ __forceinline__ uint32_t pack4_fp8(float a, float b, float c, float d) {
  uint16_t lo, hi;
  if (FP8 == 0) {
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  } else {
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  }
  return (uint32_t)lo | ((uint32_t)hi << 16);
}
// Eight values times s to 8 bits: of floats, or of a vector.
template <int FP8>
__device__ __forceinline__ uint2 pack8_fp8(const F2 (&x)[4], float s) {
  float g[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) f2_get(f2_mul(x[i], f2(s, s)), g[2 * i], g[2 * i + 1]);
  return make_uint2(pack4_fp8<FP8>(g[0], g[1], g[2], g[3]), pack4_fp8<FP8>(g[4], g[5], g[6], g[7]));
}
template <int FP8, typename T>
__device__ __forceinline__ uint2 pack8_fp8(const Vec8<T>& v, float s) {
  const F2 x[4] = {v.pair(0), v.pair(1), v.pair(2), v.pair(3)};
  return pack8_fp8<FP8>(x, s);
}
__device__ __forceinline__ void store8_fp8(uint8_t* row, int64_t c, int64_t cols, uint2 v) {
  if (c + 8 <= cols) {
    *reinterpret_cast<uint2*>(row + c) = v;
  } else {
    for (int i = 0; c + i < cols; ++i) row[c + i] = (uint8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
  }
}
// The largest magnitude of eight values, as bits: ordered like the numbers, with infinities and NaN on top.
__device__ __forceinline__ float max3_abs(float a, float b, float c) {      // a NaN wins
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint32_t magnitude8(const float (&f)[8]) {
  const float a = max3_abs(f[0], f[1], f[2]), b = max3_abs(f[3], f[4], f[5]);
  return __float_as_uint(max3_abs(max3_abs(a, b, f[6]), f[7], f[7]));
}
__device__ __forceinline__ uint32_t magnitude8(const Vec8<float>& v) {
  float f[8];
  v.get(f);
  return magnitude8(f);
}
// bf16: compared as they are, two to an instruction
__device__ __forceinline__ uint32_t magnitude8(const Vec8<__nv_bfloat16>& v) {
  const auto abs2 = [](uint32_t w) {
    w &= 0x7FFF7FFFu;
    return *reinterpret_cast<const __nv_bfloat162*>(&w);
  };
  const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(abs2(v.r.x), abs2(v.r.y)), __hmax2_nan(abs2(v.r.z), abs2(v.r.w)));
  const uint32_t w = *reinterpret_cast<const uint32_t*>(&m);
  return max(w << 16, w & 0xFFFF0000u);
}
// ... of the sixteen lanes that hold a block of 128 columns
__device__ __forceinline__ uint32_t max16(uint32_t m) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  return m;
}

}  // namespace blk
}  // namespace compact

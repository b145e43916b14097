// C ABI of the operators next to the compressed layers (see include/compact_block.h): argument checks, launch shapes, dispatch.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <atomic>
#include <mutex>
#include <new>
#include <vector>

#include "../../include/compact_block.h"
#include "block_common.cuh"
#include "block_launch.cuh"
#include "block_norm.cuh"
#include "block_product.cuh"
#include "block_quant.cuh"
#include "block_rotary.cuh"

using namespace compact;
using namespace compact::blk;

struct compact_rotary {
  compact_rotary_config_t cfg;
  RotaryTurns turns;
};

struct compact_fp8_product {
  int slot;
  uint32_t tag;           // its mark in the slot's word
  uint64_t devices;       // those it has launched on, a bit each
  int next_loaded;        // k-steps that the next product loads; -1: all
};

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool pitch_ok(int64_t ld, int64_t cols, int64_t es) { return ld >= cols && (ld * es) % 16 == 0; }
inline bool dtype_ok(int d) { return d == COMPACT_F32 || d == COMPACT_BF16; }
inline int64_t elem(int d) { return d == COMPACT_BF16 ? 2 : 4; }
constexpr int64_t kMaxRows = 0x7fffffff;
// bytes any matrix here may span: element offsets are 64-bit, this keeps products of sizes inside them
constexpr int64_t kMaxPitch = (int64_t)1 << 40;

constexpr int kMaxDevices = 64;

// Compute capability 10.x, asked once per device.
compact_status_t check_device(int* device) {
  static std::atomic<int> known[kMaxDevices];     // 0: not asked, 1: ok, 2: unsupported
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return COMPACT_ERR_CUDA; }
  if (dev < 0 || dev >= kMaxDevices) return COMPACT_ERR_INVALID_ARG;
  if (device) *device = dev;
  int k = known[dev].load(std::memory_order_acquire);
  if (k == 0) {
    int major = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) { cudaGetLastError(); return COMPACT_ERR_CUDA; }
    k = major == 10 ? 1 : 2;
    known[dev].store(k, std::memory_order_release);
  }
  return k == 1 ? COMPACT_OK : COMPACT_ERR_UNSUPPORTED_ARCH;
}


// ---- status words of the products' bounded waits ---------------------------------------------------
// A word per slot and device, zero at load.  A wait that runs out writes its handle's tag there (the largest stays), and a handle asks whether
// the word holds its own.  So no launch has to clear what a slot's earlier handle left, which would also clear, captured into a graph and
// replayed or coming back from another device, what its own kernels reported; and a kernel that outlives its handle reports to nobody else.
constexpr int kProductSlots = 1024;
__device__ unsigned int g_product_status[kProductSlots];
std::mutex g_slot_mutex;
std::vector<int> g_free_slots;
int g_slots_out = 0;
uint32_t g_slot_tags[kProductSlots];      // of the slots' last handles
std::atomic<int> g_product_kernel{0};

unsigned int* product_status(int dev, int slot) {
  static std::atomic<unsigned int*> base[kMaxDevices];
  unsigned int* p = base[dev].load(std::memory_order_acquire);
  if (!p) {
    if (cudaGetSymbolAddress((void**)&p, g_product_status) != cudaSuccess || !p) { cudaGetLastError(); return nullptr; }
    base[dev].store(p, std::memory_order_release);
  }
  return p + slot;
}

// ---- norms -------------------------------------------------------------------------------------------
template <typename T, bool RES, int OUT>
compact_status_t norm_fwd(const NormPlan& p, const NormFwdArgs& a, cudaStream_t st) {
#define CASE(L, UU) \
  if (p.lanes == L && p.u == UU) { \
    static std::atomic<bool> ready[64]; \
    if (!set_smem_once(rms_norm_fwd_kernel<T, L, UU, RES, OUT>, PIPE_BYTES, ready)) return COMPACT_ERR_CUDA; \
    return launch(rms_norm_fwd_kernel<T, L, UU, RES, OUT>, p.grid, p.groups * L, p.smem, 0, st, a); \
  }
  NORM_FWD_LAYOUTS(CASE)
#undef CASE
  return COMPACT_ERR_SHAPE;
}
template <typename T>
compact_status_t norm_fwd(const NormPlan& p, const NormFwdArgs& a, cudaStream_t st) {
  if (!a.res) return a.y ? (a.q ? norm_fwd<T, false, 3>(p, a, st) : norm_fwd<T, false, 1>(p, a, st)) : norm_fwd<T, false, 2>(p, a, st);
  if (a.y) return a.q ? norm_fwd<T, true, 3>(p, a, st) : norm_fwd<T, true, 1>(p, a, st);
  return a.q ? norm_fwd<T, true, 2>(p, a, st) : norm_fwd<T, true, 0>(p, a, st);
}

template <typename T>
compact_status_t norm_bwd(const NormPlan& p, const NormBwdArgs& a, cudaStream_t st) {
#define CASE(L, UU) \
  if (p.lanes == L && p.u == UU) { \
    static std::atomic<bool> ready[64]; \
    if (!set_smem_once(rms_norm_bwd_kernel<T, L, UU>, PIPE_BYTES, ready)) return COMPACT_ERR_CUDA; \
    return launch(rms_norm_bwd_kernel<T, L, UU>, p.grid, p.groups * L, p.smem, 0, st, a); \
  }
  NORM_BWD_LAYOUTS(CASE)
#undef CASE
  return COMPACT_ERR_SHAPE;
}

template <typename T>
compact_status_t quant_rows(int fp8, int64_t rows, int64_t cols, const void* X, int64_t ldx, void* Q, int64_t ldq, void* scales, int64_t lds,
                            cudaStream_t st) {
  const int64_t groups = ceil_div(cols, 4 * QB), blocks = ceil_div(rows, QR_ROWS) * groups;
  if (blocks > kMaxRows) return COMPACT_ERR_SHAPE;
  if (fp8 == COMPACT_E4M3)
    return launch(quantize_rows_kernel<T, 0>, (unsigned)blocks, QR_THREADS, 0, 0, st, (const T*)X, ldx, rows, cols, (uint8_t*)Q, ldq, (uint32_t*)scales, lds, (int)groups);
  else
    return launch(quantize_rows_kernel<T, 1>, (unsigned)blocks, QR_THREADS, 0, 0, st, (const T*)X, ldx, rows, cols, (uint8_t*)Q, ldq, (uint32_t*)scales, lds, (int)groups);
}
template <typename T>
compact_status_t quant_blocks(int fp8, int64_t rows, int64_t cols, const void* X, int64_t ldx, void* Q, int64_t ldq, void* scales, int64_t lds,
                              void* QT, int64_t ldqt, void* scales_t, int64_t lds_t, cudaStream_t st) {
  const int64_t cb = ceil_div(cols, QB), blocks = ceil_div(rows, QB) * cb;
  if (blocks > kMaxRows) return COMPACT_ERR_SHAPE;
  if (fp8 == COMPACT_E4M3)
    return launch(quantize_blocks_kernel<T, 0>, (unsigned)blocks, QT_THREADS, 0, 0, st, (const T*)X, ldx, rows, cols, (uint8_t*)Q, ldq, (uint8_t*)scales, lds,
                                                                         (uint8_t*)QT, ldqt, (uint8_t*)scales_t, lds_t, (int)cb);
  else
    return launch(quantize_blocks_kernel<T, 1>, (unsigned)blocks, QT_THREADS, 0, 0, st, (const T*)X, ldx, rows, cols, (uint8_t*)Q, ldq, (uint8_t*)scales, lds,
                                                                         (uint8_t*)QT, ldqt, (uint8_t*)scales_t, lds_t, (int)cb);
}

inline uint32_t magic(uint32_t d) { return d == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + d - 1) / d); }

template <typename T>
compact_status_t rotary_launch(const RotaryArgs& a, const RotaryTurns& turns, int vec, bool interleaved, dim3 grid, cudaStream_t st) {
  constexpr int V16 = 16 / (int)sizeof(T);
  if (vec == V16) {
    if (interleaved) return launch(rotary_kernel<T, V16, true>, grid, ROT_THREADS, 0, 0, st, a, turns);
    else return launch(rotary_kernel<T, V16, false>, grid, ROT_THREADS, 0, 0, st, a, turns);
  } else {
    if (interleaved) return launch(rotary_kernel<T, 1, true>, grid, ROT_THREADS, 0, 0, st, a, turns);
    else return launch(rotary_kernel<T, 1, false>, grid, ROT_THREADS, 0, 0, st, a, turns);
  }
}

}  // namespace

extern "C" {

int64_t compact_fp8_scale_groups(int64_t cols) { return cols > 0 ? ceil_div(cols, 4 * QB) : 0; }

compact_status_t compact_quantize_rows(int dtype, int64_t rows, int64_t cols, const void* X, int64_t ldx, int fp8, void* Q, int64_t ldq,
                                       void* scales, int64_t lds, void* stream) {
  if (rows < 0 || cols < 1 || rows > kMaxRows || cols > kMaxRows) return COMPACT_ERR_INVALID_ARG;
  if (!dtype_ok(dtype) || (fp8 != COMPACT_E4M3 && fp8 != COMPACT_E5M2)) return COMPACT_ERR_DTYPE;
  if (rows == 0) return COMPACT_OK;
  if (!X || !Q || !scales || lds < rows) return COMPACT_ERR_INVALID_ARG;
  if (!aligned16(X) || !aligned16(Q) || !aligned4(scales) || !pitch_ok(ldx, cols, elem(dtype)) || !pitch_ok(ldq, cols, 1)) return COMPACT_ERR_ALIGNMENT;
  if (ldx > kMaxPitch || ldq > kMaxPitch) return COMPACT_ERR_SHAPE;
  const compact_status_t s = check_device(nullptr);
  if (s != COMPACT_OK) return s;
  return dtype == COMPACT_BF16 ? quant_rows<__nv_bfloat16>(fp8, rows, cols, X, ldx, Q, ldq, scales, lds, (cudaStream_t)stream)
                               : quant_rows<float>(fp8, rows, cols, X, ldx, Q, ldq, scales, lds, (cudaStream_t)stream);
}

compact_status_t compact_quantize_blocks(int dtype, int64_t rows, int64_t cols, const void* X, int64_t ldx, int fp8, void* Q, int64_t ldq,
                                         void* scales, int64_t lds, void* QT, int64_t ldqt, void* scales_t, int64_t lds_t, void* stream) {
  if (rows < 0 || cols < 1 || rows > kMaxRows || cols > kMaxRows) return COMPACT_ERR_INVALID_ARG;
  if (!dtype_ok(dtype) || (fp8 != COMPACT_E4M3 && fp8 != COMPACT_E5M2)) return COMPACT_ERR_DTYPE;
  if (rows == 0) return COMPACT_OK;
  if (!X || (!Q && !QT) || !Q != !scales || !QT != !scales_t) return COMPACT_ERR_INVALID_ARG;
  if ((Q && lds < rows) || (QT && lds_t < cols)) return COMPACT_ERR_INVALID_ARG;
  if (!aligned16(X) || !pitch_ok(ldx, cols, elem(dtype))) return COMPACT_ERR_ALIGNMENT;
  if (Q && (!aligned16(Q) || !aligned4(scales) || !pitch_ok(ldq, cols, 1))) return COMPACT_ERR_ALIGNMENT;
  if (QT && (!aligned16(QT) || !aligned4(scales_t) || !pitch_ok(ldqt, rows, 1))) return COMPACT_ERR_ALIGNMENT;
  if (ldx > kMaxPitch || ldq > kMaxPitch || ldqt > kMaxPitch) return COMPACT_ERR_SHAPE;
  const compact_status_t s = check_device(nullptr);
  if (s != COMPACT_OK) return s;
  return dtype == COMPACT_BF16
             ? quant_blocks<__nv_bfloat16>(fp8, rows, cols, X, ldx, Q, ldq, scales, lds, QT, ldqt, scales_t, lds_t, (cudaStream_t)stream)
             : quant_blocks<float>(fp8, rows, cols, X, ldx, Q, ldq, scales, lds, QT, ldqt, scales_t, lds_t, (cudaStream_t)stream);
}

compact_status_t compact_rms_norm_fwd(int dtype, int64_t tokens, int32_t n, float eps, const void* X, int64_t ldx, const void* residual, int64_t ldr,
                                      const void* weight, void* H, int64_t ldh, void* Y, int64_t ldy, float* rstd, int fp8, void* Q, int64_t ldq,
                                      void* scales, int64_t lds, void* stream) {
  if (tokens < 0 || tokens > kMaxRows || n < 1 || !(eps >= 0.f) || !isfinite(eps)) return COMPACT_ERR_INVALID_ARG;
  if (!dtype_ok(dtype) || (Q && fp8 != COMPACT_E4M3 && fp8 != COMPACT_E5M2)) return COMPACT_ERR_DTYPE;
  if (n > COMPACT_RMS_NORM_MAX_N) return COMPACT_ERR_SHAPE;
  if (tokens == 0) return COMPACT_OK;
  if (!X || !weight || (!residual && H) || (!Y && !Q && !H) || !Q != !scales || (Q && lds < tokens)) return COMPACT_ERR_INVALID_ARG;
  const int64_t es = elem(dtype);
  if (!aligned16(X) || !aligned16(weight) || !pitch_ok(ldx, n, es)) return COMPACT_ERR_ALIGNMENT;
  if (residual && (!aligned16(residual) || !pitch_ok(ldr, n, es))) return COMPACT_ERR_ALIGNMENT;
  if (H && (!aligned16(H) || !pitch_ok(ldh, n, es))) return COMPACT_ERR_ALIGNMENT;
  if (Y && (!aligned16(Y) || !pitch_ok(ldy, n, es))) return COMPACT_ERR_ALIGNMENT;
  if (Q && (!aligned16(Q) || !aligned4(scales) || !pitch_ok(ldq, n, 1))) return COMPACT_ERR_ALIGNMENT;
  if (!aligned4(rstd)) return COMPACT_ERR_ALIGNMENT;
  if (ldx > kMaxPitch || ldr > kMaxPitch || ldh > kMaxPitch || ldy > kMaxPitch || ldq > kMaxPitch) return COMPACT_ERR_SHAPE;
  const compact_status_t s = check_device(nullptr);
  if (s != COMPACT_OK) return s;
  NormFwdArgs a;
  a.x = X; a.res = residual; a.w = weight; a.h = H; a.y = Y; a.rstd = rstd; a.q = (uint8_t*)Q; a.scales = (uint8_t*)scales;
  a.ldx = ldx; a.ldr = ldr; a.ldh = ldh; a.ldy = ldy; a.ldq = ldq; a.lds = lds; a.tokens = tokens; a.n = n; a.eps = eps;
  const NormPlan plan = norm_plan(n, tokens, (int)es, residual ? 2 : 1, false);
  a.stages = plan.stages;
  a.weight_at = plan.weight_at;
  a.fp8 = fp8;
  return dtype == COMPACT_BF16 ? norm_fwd<__nv_bfloat16>(plan, a, (cudaStream_t)stream) : norm_fwd<float>(plan, a, (cudaStream_t)stream);
}

size_t compact_rms_norm_bwd_workspace_bytes(int dtype, int64_t tokens, int32_t n) {
  if (!dtype_ok(dtype) || tokens < 0 || n < 1 || n > COMPACT_RMS_NORM_MAX_N) return 0;
  return tokens ? (size_t)norm_plan(n, tokens, (int)elem(dtype), 3, true).grid * (size_t)n * sizeof(float) : 0;
}

compact_status_t compact_rms_norm_bwd(int dtype, int64_t tokens, int32_t n, const void* dY, int64_t lddy, const void* H, int64_t ldh,
                                      const void* weight, const float* rstd, const void* residual_grad, int64_t ldr, void* dX, int64_t lddx,
                                      float* dweight, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  if (tokens < 0 || tokens > kMaxRows || n < 1) return COMPACT_ERR_INVALID_ARG;
  if (!dtype_ok(dtype)) return COMPACT_ERR_DTYPE;
  if (n > COMPACT_RMS_NORM_MAX_N) return COMPACT_ERR_SHAPE;
  if (!aligned4(dweight) || !aligned4(rstd)) return COMPACT_ERR_ALIGNMENT;
  cudaStream_t st = (cudaStream_t)stream;
  if (tokens == 0) {
    if (!dweight || accumulate) return COMPACT_OK;
    const compact_status_t s = check_device(nullptr);
    if (s != COMPACT_OK) return s;
    if (cudaMemsetAsync(dweight, 0, (size_t)n * sizeof(float), st) != cudaSuccess) { cudaGetLastError(); return COMPACT_ERR_CUDA; }
    return COMPACT_OK;
  }
  // after the empty batch, whose dX has no memory
  if (!dY || !H || !weight || !rstd || (!dX && !dweight)) return COMPACT_ERR_INVALID_ARG;
  const int64_t es = elem(dtype);
  if (!aligned16(dY) || !aligned16(H) || !aligned16(weight) || !pitch_ok(lddy, n, es) || !pitch_ok(ldh, n, es)) return COMPACT_ERR_ALIGNMENT;
  if (residual_grad && (!aligned16(residual_grad) || !pitch_ok(ldr, n, es))) return COMPACT_ERR_ALIGNMENT;
  if (dX && (!aligned16(dX) || !pitch_ok(lddx, n, es))) return COMPACT_ERR_ALIGNMENT;
  if (lddy > kMaxPitch || ldh > kMaxPitch || ldr > kMaxPitch || lddx > kMaxPitch) return COMPACT_ERR_SHAPE;
  if (dweight) {
    if (!workspace || workspace_bytes < compact_rms_norm_bwd_workspace_bytes(dtype, tokens, n)) return COMPACT_ERR_WORKSPACE;
    if (!aligned16(workspace)) return COMPACT_ERR_ALIGNMENT;
  }
  compact_status_t s = check_device(nullptr);
  if (s != COMPACT_OK) return s;
  NormBwdArgs a;
  a.dy = dY; a.h = H; a.w = weight; a.dres = residual_grad; a.rstd = rstd; a.dx = dX;
  a.lddy = lddy; a.ldh = ldh; a.ldr = ldr; a.lddx = lddx; a.tokens = tokens; a.n = n;
  const NormPlan plan = norm_plan(n, tokens, (int)es, residual_grad ? 3 : 2, true);
  a.stages = plan.stages;
  const bool alone = plan.grid == 1;
  a.partial = !dweight ? nullptr : (alone ? dweight : (float*)workspace);
  a.accumulate = alone && accumulate;
  s = dtype == COMPACT_BF16 ? norm_bwd<__nv_bfloat16>(plan, a, st) : norm_bwd<float>(plan, a, st);
  if (s != COMPACT_OK || !dweight || alone) return s;
  return launch(sum_partials_kernel, (unsigned)ceil_div(n, 32), 1024, 0, 0, st, (const float*)a.partial, plan.grid, n, dweight, accumulate);
}

compact_status_t compact_rotary_create(const compact_rotary_config_t* cfg, compact_rotary_t** out) {
  if (!cfg || !out) return COMPACT_ERR_INVALID_ARG;
  *out = nullptr;
  if (cfg->rot_dim < 2 || cfg->rot_dim % 2 || cfg->rot_dim > cfg->head_dim || cfg->head_dim > 1024 || cfg->rot_dim > 2 * ROT_MAX_PAIRS)
    return COMPACT_ERR_SHAPE;
  const bool scaled = cfg->scaling != COMPACT_ROTARY_NONE;
  if (cfg->scaling < COMPACT_ROTARY_NONE || cfg->scaling > COMPACT_ROTARY_BY_PARTS) return COMPACT_ERR_INVALID_ARG;
  if (!(cfg->base >= 1.0) || !isfinite(cfg->base) || !isfinite(cfg->attention_factor)) return COMPACT_ERR_INVALID_ARG;
  if (scaled && (!(cfg->factor > 0.0) || !isfinite(cfg->factor))) return COMPACT_ERR_INVALID_ARG;
  if (cfg->scaling == COMPACT_ROTARY_BASE && cfg->rot_dim < 4) return COMPACT_ERR_SHAPE;
  if (cfg->scaling == COMPACT_ROTARY_BY_PARTS &&
      (!(cfg->high > cfg->low) || !(cfg->trained_length > 0.0) || !isfinite(cfg->low) || !isfinite(cfg->high) || !isfinite(cfg->trained_length)))
    return COMPACT_ERR_INVALID_ARG;
  RotaryTurns speeds;
  memset(&speeds, 0, sizeof(speeds));
  const double two_pi = 6.283185307179586476925286766559, d = cfg->rot_dim;
  double base = cfg->base;
  if (cfg->scaling == COMPACT_ROTARY_BASE) base *= pow(cfg->factor, d / (d - 2.0));
  if (!(base > 0.0) || !isfinite(base)) return COMPACT_ERR_INVALID_ARG;      // a factor that takes it out of range
  for (int i = 0; i < cfg->rot_dim / 2; ++i) {
    double w = pow(base, -2.0 * i / d);
    if (cfg->scaling == COMPACT_ROTARY_LINEAR) w /= cfg->factor;
    if (cfg->scaling == COMPACT_ROTARY_BY_PARTS) {
      double t = (cfg->trained_length * w / two_pi - cfg->low) / (cfg->high - cfg->low);
      t = t < 0.0 ? 0.0 : (t > 1.0 ? 1.0 : t);
      w *= t + (1.0 - t) / cfg->factor;
    }
    if (!isfinite(w)) return COMPACT_ERR_INVALID_ARG;
    // whole turns per position do not matter at whole positions
    const double turns = fmod(w / two_pi, 1.0) * 18446744073709551616.0;
    speeds.w[i] = turns >= 18446744073709551615.0 ? 0ull : (uint64_t)turns;
  }
  compact_rotary_t* r = new (std::nothrow) compact_rotary_t;
  if (!r) return COMPACT_ERR_INVALID_ARG;
  r->cfg = *cfg;
  r->turns = speeds;
  *out = r;
  return COMPACT_OK;
}

compact_status_t compact_rotary_destroy(compact_rotary_t* rot) {
  if (!rot) return COMPACT_ERR_INVALID_ARG;
  delete rot;
  return COMPACT_OK;
}

compact_status_t compact_rotary_apply(const compact_rotary_t* rot, int dtype, int64_t tokens, int32_t heads, int32_t kv_heads, const void* Q,
                                      int64_t q_token, int64_t q_head, const void* K, int64_t k_token, int64_t k_head, const void* positions,
                                      int pos_bits, int64_t first_position, int back, void* Qout, int64_t qo_token, int64_t qo_head, void* Kout,
                                      int64_t ko_token, int64_t ko_head, void* stream) {
  if (!rot || tokens < 0 || tokens > kMaxRows || heads < 1 || kv_heads < 0 || heads > 65535 || kv_heads > 65535) return COMPACT_ERR_INVALID_ARG;
  if (!dtype_ok(dtype)) return COMPACT_ERR_DTYPE;
  if (positions && pos_bits != 64 && pos_bits != 32) return COMPACT_ERR_DTYPE;
  if (tokens == 0) return COMPACT_OK;
  if (!Q || !Qout || (kv_heads > 0 && (!K || !Kout))) return COMPACT_ERR_INVALID_ARG;
  // heads written closer together than they are long, or all to one place, would run into each other
  const int64_t d = rot->cfg.head_dim;
  const auto apart = [d](int64_t stride, int64_t count) { return count <= 1 || stride >= d || stride <= -d; };
  if (!apart(qo_token, tokens) || !apart(qo_head, heads) || (kv_heads && (!apart(ko_token, tokens) || !apart(ko_head, kv_heads)))) return COMPACT_ERR_INVALID_ARG;
  const int es = (int)elem(dtype), V16 = 16 / es;
  const uintptr_t at = reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(Qout) |
                       (kv_heads ? reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(Kout) : 0);
  if (at % es || (positions && reinterpret_cast<uintptr_t>(positions) % (pos_bits / 8))) return COMPACT_ERR_ALIGNMENT;
  const compact_status_t s = check_device(nullptr);
  if (s != COMPACT_OK) return s;
  RotaryArgs a;
  memset(&a, 0, sizeof(a));
  a.q = Q; a.k = K; a.qo = Qout; a.ko = Kout;
  a.q_token = q_token; a.q_head = q_head; a.k_token = k_token; a.k_head = k_head;
  a.qo_token = qo_token; a.qo_head = qo_head; a.ko_token = ko_token; a.ko_head = ko_head;
  a.positions = positions; a.pos_bits = pos_bits; a.first_position = first_position;
  a.tokens = tokens; a.back = back != 0; a.heads = heads; a.kv_heads = kv_heads;
  a.pairs = rot->cfg.rot_dim / 2; a.head_dim = rot->cfg.head_dim; a.attention_factor = rot->cfg.attention_factor;
  // 16-byte pieces need every stride, every pointer and both cuts of the head on 16 bytes; else element by element
  const int64_t strides = q_token | q_head | qo_token | qo_head | (kv_heads ? k_token | k_head | ko_token | ko_head : 0);
  const int rest = a.head_dim - 2 * a.pairs;
  const int vec = at % 16 == 0 && strides % V16 == 0 && a.pairs % V16 == 0 && rest % V16 == 0 ? V16 : 1;
  const bool in_place = Q == Qout && q_token == qo_token && q_head == qo_head &&
                        (!kv_heads || (K == Kout && k_token == ko_token && k_head == ko_head));
  a.turned_pieces = a.pairs / vec;
  a.pieces = a.turned_pieces + (in_place ? 0 : (rest + 2 * vec - 1) / (2 * vec));
  // Long batches: several tokens per CTA, so that the angles are computed once per token for all its heads and a thread has up
  // to eight pieces.  Few tokens: the heads are dealt to CTAs too, until the SMs are filled once or a CTA has a piece per thread.
  const int all_heads = heads + kv_heads;
  int tpc = 1, hpc = all_heads;
  while (tpc < 8 && (tpc * 2) * a.pairs <= ROT_SMEM_PAIRS && tokens / (tpc * 2) >= 8 * tc::NUM_SMS &&
         (int64_t)tpc * hpc * a.pieces < 8 * ROT_THREADS)
    tpc *= 2;
  if (tpc == 1) {
    const int64_t want = ceil_div(2 * tc::NUM_SMS, tokens);                       // CTAs per token that fill the SMs twice
    const int64_t least = ceil_div(ROT_THREADS, a.pieces);                         // heads that give every thread a piece
    int64_t h = ceil_div(all_heads, want);
    if (h < least) h = least;
    hpc = (int)(h < all_heads ? h : all_heads);
  }
  // quotients by magic numbers are exact while numerator times divisor stays below 2^32
  while (hpc > 1 && ((int64_t)tpc * hpc * a.pieces > (1 << 20) || (int64_t)tpc * hpc * hpc > (1 << 30))) hpc = (hpc + 1) / 2;
  a.tokens_per_cta = tpc;
  a.heads_per_cta = hpc;
  a.pieces_magic = magic((uint32_t)a.pieces);
  a.heads_magic = magic((uint32_t)hpc);
  const dim3 grid((unsigned)ceil_div(tokens, tpc), (unsigned)ceil_div(all_heads, hpc));
  return dtype == COMPACT_BF16 ? rotary_launch<__nv_bfloat16>(a, rot->turns, vec, rot->cfg.interleaved != 0, grid, (cudaStream_t)stream)
                               : rotary_launch<float>(a, rot->turns, vec, rot->cfg.interleaved != 0, grid, (cudaStream_t)stream);
}

compact_status_t compact_fp8_product_create(compact_fp8_product_t** out) {
  if (!out) return COMPACT_ERR_INVALID_ARG;
  *out = nullptr;
  compact_fp8_product_t* p = new (std::nothrow) compact_fp8_product_t;
  if (!p) return COMPACT_ERR_INVALID_ARG;
  p->devices = 0;
  p->next_loaded = -1;
  {
    std::lock_guard<std::mutex> lock(g_slot_mutex);
    p->slot = -1;
    if (!g_free_slots.empty()) {
      p->slot = g_free_slots.back();
      g_free_slots.pop_back();
    } else if (g_slots_out < kProductSlots) {
      // room for every slot to come back, so that giving one back allocates nothing
      try {
        g_free_slots.reserve((size_t)g_slots_out + 1);
        p->slot = g_slots_out++;
      } catch (...) {
      }
    }
    if (p->slot >= 0) p->tag = ++g_slot_tags[p->slot];
  }
  if (p->slot < 0) { delete p; return COMPACT_ERR_TOO_MANY_LAYERS; }
  *out = p;
  return COMPACT_OK;
}

compact_status_t compact_fp8_product_destroy(compact_fp8_product_t* p) {
  if (!p) return COMPACT_ERR_INVALID_ARG;
  {
    std::lock_guard<std::mutex> lock(g_slot_mutex);
    g_free_slots.push_back(p->slot);
  }
  delete p;
  return COMPACT_OK;
}

compact_status_t compact_fp8_product_run(compact_fp8_product_t* p, int64_t M, int64_t N, int64_t K, int a_type, const void* A, int64_t lda,
                                         const void* a_scales, int64_t lds_a, int b_type, const void* B, int64_t ldb, const void* b_scales,
                                         int64_t lds_b, int c_dtype, void* C, int64_t ldc, void* stream) {
  if (!p || M < 0 || N < 1 || K < 1 || M > 0x7fffff00 || N > 0x7fffff00 || K > 0x7fffff00) return COMPACT_ERR_INVALID_ARG;
  if ((a_type != COMPACT_E4M3 && a_type != COMPACT_E5M2) || (b_type != COMPACT_E4M3 && b_type != COMPACT_E5M2) || !dtype_ok(c_dtype)) return COMPACT_ERR_DTYPE;
  if (M == 0) return COMPACT_OK;
  if (!A || !B || !C || !a_scales || !b_scales || lds_a < M || lds_b < N) return COMPACT_ERR_INVALID_ARG;
  if (!aligned16(A) || !aligned16(B) || !aligned16(C) || !aligned4(a_scales) || !aligned4(b_scales)) return COMPACT_ERR_ALIGNMENT;
  if (!pitch_ok(lda, K, 1) || !pitch_ok(ldb, K, 1) || !pitch_ok(ldc, N, elem(c_dtype))) return COMPACT_ERR_ALIGNMENT;
  if (lda >= kMaxPitch || ldb >= kMaxPitch || ldc * elem(c_dtype) >= kMaxPitch) return COMPACT_ERR_SHAPE;
  int dev = 0;
  compact_status_t s = check_device(&dev);
  if (s != COMPACT_OK) return s;
  ProductCall c;
  c.M = (int)M; c.N = (int)N; c.K = (int)K;
  c.a_type = a_type; c.b_type = b_type; c.A = A; c.B = B; c.a_scales = a_scales; c.b_scales = b_scales;
  c.lda = lda; c.ldb = ldb; c.lds_a = lds_a; c.lds_b = lds_b;
  c.c_f32 = c_dtype == COMPACT_F32; c.C = C; c.ldc = ldc;
  c.waits.status = product_status(dev, p->slot);
  if (!c.waits.status) return COMPACT_ERR_CUDA;
  const bool short_waits = p->next_loaded >= 0;
  c.waits.limit = short_waits ? 4096u : tc::WAIT_LIMIT;
  c.waits.loaded = short_waits ? p->next_loaded : c.K;      // no fewer than the k-steps
  p->next_loaded = -1;
  c.waits.tag = p->tag;
  c.stream = (cudaStream_t)stream;
  p->devices |= (uint64_t)1 << dev;
  const int which = g_product_kernel.load();
  const bool split = which == 2 || (which == 0 && prefer_split(c.M, c.N));
  return split ? product_split(c) : product_pair(c);
}

compact_status_t compact_fp8_product_status(compact_fp8_product_t* p) {
  if (!p) return COMPACT_ERR_INVALID_ARG;
  if (!p->devices) return COMPACT_OK;
  int current = 0;
  if (cudaGetDevice(&current) != cudaSuccess) { cudaGetLastError(); return COMPACT_ERR_CUDA; }
  compact_status_t result = COMPACT_OK;
  for (int dev = 0; dev < kMaxDevices; ++dev) {
    if (!(p->devices >> dev & 1)) continue;
    unsigned int v = 0;
    unsigned int* w = nullptr;
    if (cudaSetDevice(dev) != cudaSuccess || !(w = product_status(dev, p->slot)) || cudaDeviceSynchronize() != cudaSuccess ||
        cudaMemcpy(&v, w, sizeof(v), cudaMemcpyDeviceToHost) != cudaSuccess) {
      cudaGetLastError();
      result = COMPACT_ERR_CUDA;
      continue;
    }
    if (v != p->tag) continue;
    v = 0;
    if (cudaMemcpy(w, &v, sizeof(v), cudaMemcpyHostToDevice) != cudaSuccess) { cudaGetLastError(); result = COMPACT_ERR_CUDA; }
    if (result == COMPACT_OK) result = COMPACT_ERR_DEVICE_TIMEOUT;
  }
  if (cudaSetDevice(current) != cudaSuccess) { cudaGetLastError(); return COMPACT_ERR_CUDA; }
  return result;
}

compact_status_t compact_debug_fp8_product_withhold(compact_fp8_product_t* p, int32_t k_steps) {
  if (!p) return COMPACT_ERR_INVALID_ARG;
  p->next_loaded = k_steps < 0 ? -1 : k_steps;
  return COMPACT_OK;
}

compact_status_t compact_debug_fp8_product_plan(int64_t M, int64_t N, int64_t K, int32_t plan[5]) {
  if (!plan || M < 1 || N < 1 || K < 1 || M > 0x7fffff00 || N > 0x7fffff00 || K > 0x7fffff00) return COMPACT_ERR_INVALID_ARG;
  const PairPlan p = pair_plan((int)M, (int)N, (int)K);
  if ((int64_t)p.tiles_m * p.tiles_n > 0x3fffffff) return COMPACT_ERR_SHAPE;
  plan[0] = prefer_split((int)M, (int)N) ? 2 : 1;
  plan[1] = p.bn;
  plan[2] = p.tiles_m * p.tiles_n;
  plan[3] = p.per_barrier;
  plan[4] = (p.tiles_n + p.panel_cols - 1) / p.panel_cols;
  return COMPACT_OK;
}

int compact_fp8_product_set_kernel(int which) {
  if (which < 0 || which > 2) return g_product_kernel.load();
  return g_product_kernel.exchange(which);
}

}  // extern "C"

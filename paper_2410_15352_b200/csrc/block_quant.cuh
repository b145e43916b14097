// Quantisation to 8 bits with a power-of-two scale for each 128 values: q = round(x / s), s = the least power of two with
// max|x| / s inside the type's range.  Bound by memory: 2 bytes read and 1 (rows) or 2 (blocks, both orientations) written
// per bf16 element, everything once.
#pragma once
#include "block_common.cuh"

namespace compact {
namespace blk {

constexpr int QR_ROWS = 8;         // rows a CTA of quantize_rows takes, one per half warp
constexpr int QR_THREADS = QR_ROWS * 16;

// A half warp takes the four column blocks of one row whose scales make up one 32-bit word: its four loads are
// independent, and it writes the word whole.  Neighbouring CTAs take neighbouring groups of the same eight rows.  What is read
// once is marked so.  (16384 x 4096 bf16, calls in a replayed graph: 34.7 us, 5.8 TB/s; sixteen rows and 48 registers a thread 36.6.
// fp32 51.2, 6.6 TB/s.)
template <typename T, int FP8>
__global__ void __launch_bounds__(QR_THREADS, sizeof(T) == 2 ? 12 : 8) quantize_rows_kernel(const T* X, int64_t ldx, int64_t rows, int64_t cols, uint8_t* Q,
                                                                                                       int64_t ldq, uint32_t* scales, int64_t lds, int groups) {
  let_successor_start();
  wait_for_predecessors();
  const int64_t tile = (int64_t)blockIdx.x / groups;
  const int g = (int)((int64_t)blockIdx.x - tile * groups);
  const int lane16 = threadIdx.x & 15;
  const int64_t row = tile * QR_ROWS + (threadIdx.x >> 4);
  const bool live = row < rows;                      // all lanes stay for the shuffles
  const T* x = X + (live ? row : 0) * ldx;
  const int64_t c0 = (int64_t)g * 4 * QB + lane16 * 8;
  Vec8<T> v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t c = c0 + j * QB;
    if (!live) v[j].clear();
    else if (c + 8 <= cols) v[j].load_once(x + c);
    else v[j] = load8(x, c, cols);
  }
  uint32_t word = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    // a block past the last column is all zeros here, and gets the scale 1
    const uint32_t byte = scale_byte(max16(magnitude8(v[j])), FP8 == 0 ? 8 : 15);
    word |= byte << (8 * j);
    if (live) store8_fp8(Q + row * ldq, c0 + j * QB, cols, pack8_fp8<FP8>(v[j], inverse_scale(byte)));
  }
  if (live && lane16 == 0) scales[(int64_t)g * lds + row] = word;
}

// A CTA takes one 128 x 128 block.  Its half warps hold four neighbouring rows each, twice (rows 4 h .. 4 h + 3 and
// 64 further), so that a lane's four rows of one column make one word of the transpose; the words go through shared
// memory (pitch 33 words) and leave as 16-byte pieces of the transpose's rows.  (4096 x 11008 bf16, calls in a replayed graph: 32.6 us, 5.5 TB/s;
// with two CTAs of 112 registers a thread to an SM instead of four 42.5.  fp32, two CTAs: 48.7, 5.6 TB/s.)
constexpr int QT_THREADS = 256;
constexpr int QT_CTAS = 4;         // of bf16 blocks: 64 registers a thread
template <typename T, int FP8>
__global__ void __launch_bounds__(QT_THREADS, sizeof(T) == 2 ? QT_CTAS : 2) quantize_blocks_kernel(const T* X, int64_t ldx, int64_t rows, int64_t cols,
                                                                                                              uint8_t* Q, int64_t ldq, uint8_t* scales, int64_t lds,
                                                                                                              uint8_t* QTr, int64_t ldqt, uint8_t* scales_t,
                                                                                                              int64_t lds_t, int col_blocks) {
  __shared__ uint32_t tr[QB * 33];
  let_successor_start();
  wait_for_predecessors();
  __shared__ uint32_t peaks[QT_THREADS / 32];
  const int64_t rb = (int64_t)blockIdx.x / col_blocks;
  const int cb = (int)((int64_t)blockIdx.x - rb * col_blocks);
  const int row_blocks = (int)((rows + QB - 1) / QB);
  const int64_t r0 = rb * QB, c0 = (int64_t)cb * QB;
  const int lane16 = threadIdx.x & 15, hw = threadIdx.x >> 4;
  Vec8<T> v[8];
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int64_t r = r0 + (p >> 2) * 64 + hw * 4 + (p & 3);
    if (r < rows) v[p] = load8(X + r * ldx, c0 + lane16 * 8, cols);
    else v[p].clear();
  }
  uint32_t m = 0;
#pragma unroll
  for (int p = 0; p < 8; ++p) m = max(m, magnitude8(v[p]));
  m = max16(m);
  m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
  if ((threadIdx.x & 31) == 0) peaks[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < QT_THREADS / 32; ++w) m = max(m, peaks[w]);
  const uint32_t byte = scale_byte(m, FP8 == 0 ? 8 : 15);
  const float inv = inverse_scale(byte);
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    uint2 q[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      q[p] = pack8_fp8<FP8>(v[4 * half + p], inv);
      const int64_t r = r0 + half * 64 + hw * 4 + p;
      if (Q && r < rows) store8_fp8(Q + r * ldq, c0 + lane16 * 8, cols, q[p]);
    }
    if (QTr) {
      // 4 x 4 bytes turned twice: words of a column's four rows
      const uint32_t in[2][4] = {{q[0].x, q[1].x, q[2].x, q[3].x}, {q[0].y, q[1].y, q[2].y, q[3].y}};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t a = __byte_perm(in[h][0], in[h][1], 0x5140), b = __byte_perm(in[h][2], in[h][3], 0x5140);   // columns 0, 1
        const uint32_t c = __byte_perm(in[h][0], in[h][1], 0x7362), d = __byte_perm(in[h][2], in[h][3], 0x7362);   // columns 2, 3
        uint32_t* t = tr + (lane16 * 8 + h * 4) * 33 + half * 16 + hw;
        t[0] = __byte_perm(a, b, 0x5410);
        t[33] = __byte_perm(a, b, 0x7632);
        t[66] = __byte_perm(c, d, 0x5410);
        t[99] = __byte_perm(c, d, 0x7632);
      }
    }
  }
  // scales: a byte for every row (column, in the transpose) of the block; the last block also writes the bytes past it
  const int t = threadIdx.x;
  if (t < QB) {
    if (scales && r0 + t < rows) {
      uint8_t* s = scales + ((int64_t)(cb >> 2) * lds + r0 + t) * 4;
      s[cb & 3] = (uint8_t)byte;
      if (cb == col_blocks - 1)
        for (int j = (cb & 3) + 1; j < 4; ++j) s[j] = (uint8_t)SCALE_ONE;
    }
  } else if (scales_t && c0 + (t - QB) < cols) {
    uint8_t* s = scales_t + ((rb >> 2) * lds_t + c0 + (t - QB)) * 4;
    s[rb & 3] = (uint8_t)byte;
    if (rb == row_blocks - 1)
      for (int j = (int)(rb & 3) + 1; j < 4; ++j) s[j] = (uint8_t)SCALE_ONE;
  }
  if (QTr) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int piece = t + i * QT_THREADS;              // 128 rows of the transpose, eight pieces each
      const int c = piece >> 3, k = (piece & 7) * 16;
      if (c0 + c >= cols) continue;
      const uint32_t* w = tr + c * 33 + (k >> 2);
      uint8_t* out = QTr + (c0 + c) * ldqt + r0 + k;
      if (r0 + k + 16 <= rows) {
        *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        for (int e = 0; e < 16 && r0 + k + e < rows; ++e) out[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
      }
    }
  }
}

}  // namespace blk
}  // namespace compact

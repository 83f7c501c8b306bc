// Dropout with a counter-based mask (abs_dropout_*): y = (kept ? x scale : 0) + r.
//
// The mask of element e is a comparison of 16 bits of draw e / 4 of the simulation's counter-based generator, so it is
// recomputed wherever it is needed and costs no memory.  One draw is two 64-bit products and some shifts, about 250
// cycles of a SIMD per 64 draws; four elements share it, which keeps the kernel on the memory's side: bf16 32768 x 2048 with
// residual 71 us, 5.7 TB/s (a copy of 1 GiB: 5.1).
#include "operators.h"

#include <algorithm>

namespace abs_impl {
namespace {

constexpr uint32_t kStreamDropout = 2;

ABS_HD uint64_t dropout_key(uint64_t seed, uint64_t offset) { return mix64(stream_key(seed, kStreamDropout) ^ offset); }
// the four elements of quad q: draw(key, q) with a 64-bit counter
ABS_HD uint64_t dropout_draw(uint64_t key, uint64_t q) { return mix64(key + kGoldenGamma * (q + 1)); }

template <typename T>
struct DropArgs {
  const T* x; const T* r; T* y;
  int64_t rows, cols, ldx, ldy, ldr;
  uint64_t key;
  uint32_t drop;
  float scale;
};

__device__ __forceinline__ float dropped(float x, uint32_t part, uint32_t drop, float scale) {
  return part >= drop ? x * scale : 0.f;       // a select: what is dropped may be infinite
}

// Pieces of 16 bytes, at any alignment of the elements: rows of whole pieces, and a flat array whose last few elements the last thread takes one by one.
// A thread takes kPieces pieces a block's width apart, all loads before the first draw is needed.
constexpr int kDropPieces = 2;
template <typename T, bool RES, bool FLAT>
__global__ __launch_bounds__(256) void dropout_vector_kernel(DropArgs<T> a) {
  constexpr int V = 16 / sizeof(T);
  typedef Piece<T, V> Vec;
  const int64_t per_row = a.cols / V, pieces = per_row * a.rows;
  const int64_t p0 = (int64_t)op_block() * (256 * kDropPieces) + threadIdx.x;
  Vec vx[kDropPieces], vr[kDropPieces];
  int64_t ox[kDropPieces], oy[kDropPieces];
#pragma unroll
  for (int i = 0; i < kDropPieces; ++i) {
    const int64_t p = p0 + i * 256;
    if (p < pieces) {
      int64_t row = 0, c = p;
      if (!FLAT) {
        if (pieces <= 0xFFFFFFFFll) { row = (uint32_t)p / (uint32_t)per_row; c = (uint32_t)p - (uint32_t)row * (uint32_t)per_row; }
        else { row = p / per_row; c = p - row * per_row; }
      }
      ox[i] = row * a.ldx + c * V;
      oy[i] = row * a.ldy + c * V;
      vx[i].load(a.x + ox[i]);
      if (RES) vr[i].load(a.r + row * a.ldr + c * V);
    }
  }
#pragma unroll
  for (int i = 0; i < kDropPieces; ++i) {
    const int64_t p = p0 + i * 256;
    if (p < pieces) {
      Vec o;
      float f[V];
#pragma unroll
      for (int h = 0; h < V / 4; ++h) {
        const uint64_t w = dropout_draw(a.key, (uint64_t)p * (V / 4) + h);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = 4 * h + j;
          f[e] = dropped(vx[i].at(e), (uint32_t)(w >> (16 * j)) & 0xFFFFu, a.drop, a.scale);
          if (RES) f[e] += vr[i].at(e);
        }
      }
      o.set(f);
      o.store(a.y + oy[i]);
    }
  }
  if (FLAT && p0 == 0) {
    for (int64_t e = pieces * V; e < a.cols; ++e) {
      const uint64_t w = dropout_draw(a.key, (uint64_t)e >> 2);
      float v = dropped(op_widen(a.x[e]), (uint32_t)(w >> (16 * (e & 3))) & 0xFFFFu, a.drop, a.scale);
      if (RES) v += op_widen(a.r[e]);
      op_narrow(v, a.y[e]);
    }
  }
}

// Rows that are not whole pieces, a pitch apart: a thread takes the four elements of a draw, one by one, also across a row's end.
template <typename T, bool RES>
__global__ __launch_bounds__(256) void dropout_element_kernel(DropArgs<T> a) {
  const uint64_t total = (uint64_t)a.rows * (uint64_t)a.cols;
  const uint64_t q = op_block() * 256 + threadIdx.x;
  uint64_t e = 4 * q;
  if (e >= total) return;
  int64_t row, col;
  if (total <= 0xFFFFFFFFull) { row = (uint32_t)e / (uint32_t)a.cols; col = (uint32_t)e - (uint32_t)row * (uint32_t)a.cols; }
  else { row = (int64_t)(e / (uint64_t)a.cols); col = (int64_t)(e - (uint64_t)row * (uint64_t)a.cols); }
  const uint64_t w = dropout_draw(a.key, q);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (e + j < total) {
      float v = dropped(op_widen(a.x[row * a.ldx + col]), (uint32_t)(w >> (16 * j)) & 0xFFFFu, a.drop, a.scale);
      if (RES) v += op_widen(a.r[row * a.ldr + col]);
      op_narrow(v, a.y[row * a.ldy + col]);
      if (++col == a.cols) { col = 0; ++row; }
    }
  }
}

template <typename T>
hipError_t launch_dropout(const abs_dropout& p, const void* x, const void* r, void* y, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  DropArgs<T> a;
  a.x = (const T*)x; a.r = (const T*)r; a.y = (T*)y;
  a.rows = p.rows; a.cols = p.cols; a.ldx = p.ldx; a.ldy = p.ldy; a.ldr = r ? p.ldr : p.cols;
  a.key = dropout_key(p.seed, p.offset);
  a.drop = (uint32_t)p.drop;
  a.scale = (float)(65536.0 / (65536 - p.drop));
  const bool flat = p.rows == 1 || (p.ldx == p.cols && p.ldy == p.cols && a.ldr == p.cols);
  if (flat) { a.cols *= a.rows; a.rows = 1; }
  if (flat || a.cols % V == 0) {                       // (at any pitch and alignment)
    const int64_t pieces = a.cols / V * a.rows;
    const dim3 grid = op_grid((uint64_t)std::max<int64_t>(1, (pieces + 256 * kDropPieces - 1) / (256 * kDropPieces)));
    if (flat) {
      if (r) dropout_vector_kernel<T, true, true><<<grid, 256, 0, s>>>(a);
      else   dropout_vector_kernel<T, false, true><<<grid, 256, 0, s>>>(a);
    } else {
      if (r) dropout_vector_kernel<T, true, false><<<grid, 256, 0, s>>>(a);
      else   dropout_vector_kernel<T, false, false><<<grid, 256, 0, s>>>(a);
    }
  } else {
    const int64_t quads = (a.rows * a.cols + 3) / 4;
    const dim3 grid = op_grid((uint64_t)((quads + 255) / 256));
    if (r) dropout_element_kernel<T, true><<<grid, 256, 0, s>>>(a);
    else   dropout_element_kernel<T, false><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

const char* dropout_problem(const abs_dropout* p) {
  if (!p) return "dropout: the description is NULL";
  if (p->dtype != ABS_X_FP32 && p->dtype != ABS_X_BF16) return "dropout: dtype must be ABS_X_FP32 or ABS_X_BF16";
  if (p->drop < 0 || p->drop > 65535) return "dropout: drop must be in [0, 65535]";
  if (p->rows < 0 || p->cols < 1) return "dropout: rows must not be negative and cols positive";
  constexpr int64_t most = 1ll << 40;
  if (p->cols >= most || p->rows >= most || (p->rows && p->cols > (most - 1) / p->rows)) return "dropout: rows x cols must be below 2^40";
  return nullptr;
}

int dropout_run(const abs_dropout* p, const void* x, const void* r, void* y, void* stream) {
  if (const char* why = dropout_problem(p)) return op_fail(ABS_E_ARG, why);
  if (p->ldx < p->cols || p->ldy < p->cols || (r && p->ldr < p->cols))
    return op_fail(ABS_E_ARG, "dropout: a row pitch is below cols");
  if (p->rows == 0) return ABS_OK;
  if (!x || !y) return op_fail(ABS_E_ARG, "dropout: a device pointer is NULL");
  const size_t size = (size_t)op_size(p->dtype);
  if (!op_aligned(x, size) || !op_aligned(y, size) || (r && !op_aligned(r, size)))
    return op_fail(ABS_E_ARG, "dropout: a pointer is not aligned to its elements");
  const hipError_t e = p->dtype == ABS_X_BF16 ? launch_dropout<uint16_t>(*p, x, r, y, (hipStream_t)stream)
                                              : launch_dropout<float>(*p, x, r, y, (hipStream_t)stream);
  return op_hip("abs_dropout", e);
}

}  // namespace
}  // namespace abs_impl

using namespace abs_impl;

extern "C" {

int abs_dropout_forward(const abs_dropout* p, const void* d_x, const void* d_r, void* d_y, void* hip_stream) {
  return dropout_run(p, d_x, d_r, d_y, hip_stream);
}

int abs_dropout_backward(const abs_dropout* p, const void* d_dy, void* d_dx, void* hip_stream) {
  return dropout_run(p, d_dy, nullptr, d_dx, hip_stream);
}

int abs_dropout_kept(const abs_dropout* p, int64_t first, int64_t count, uint8_t* h_kept) {
  if (const char* why = dropout_problem(p)) return op_fail(ABS_E_ARG, why);
  if (!h_kept || first < 0 || count < 0 || first > p->rows * p->cols || count > p->rows * p->cols - first)
    return op_fail(ABS_E_ARG, "dropout: elements outside the matrix");
  const uint64_t key = dropout_key(p->seed, p->offset);
  for (int64_t i = 0; i < count; ++i) {
    const uint64_t e = (uint64_t)(first + i);
    h_kept[i] = ((dropout_draw(key, e >> 2) >> (16 * (e & 3))) & 0xFFFFu) >= (uint32_t)p->drop;
  }
  return ABS_OK;
}

}  // extern "C"

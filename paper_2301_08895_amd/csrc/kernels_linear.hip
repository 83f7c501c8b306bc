// The product of a layer with its epilogue, and its gradients (abs_linear_*):
//   forward   z = x W + b, y = act(z) + r       rows of x times columns of W (W's contraction runs down its rows)
//   backward  dz = dy act'(z);  dx = dz W^T     rows of dz times rows of W
//             dW = x^T dz                       columns of x times columns of dz, contraction over the rows
// One tile kernel serves the three: an operand whose contraction index is contiguous arrives as [row][k], the others as
// [k][row], and only the fragment reads differ (bf16: the transposing LDS read).
#include "operators.h"

#include <algorithm>
#include <cmath>

namespace abs_impl {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

template <typename T> constexpr int kPiece = 16 / (int)sizeof(T);      // elements of a 16-byte piece
template <typename T> constexpr int kStep = 128 / (int)sizeof(T);      // contraction elements of a k-step: 128 bytes of a row

// What a request reads beyond an operand's end.
__device__ uint4 g_zero_piece;

// Global -> LDS requests by hand, counted by hand (see ring_wait): the compiler would make every LDS read wait for all of them.
__device__ __forceinline__ uint32_t lds_at(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }
__device__ __forceinline__ void lds_request16(const void* gsrc, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(gsrc), "{m0}"(lds) : "memory");
}
template <int N>
__device__ __forceinline__ void ring_wait() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory"); }

// What is done with a result: y = act(acc + bias) + r, or a share of the contraction to be added up later.
template <typename T>
struct Epilogue {
  const float* bias; const T* r; T* y; T* z; float* part;
  int64_t ldr, ldy, ldz, ldpart, part_stride;
  int act;
};

template <typename T>
struct GemmArgs {
  const T* A; const T* B;
  int64_t lda, ldb;
  int64_t M, N, K;                   // result rows and columns, contraction
  int64_t mc, nc;                    // contiguous extents of operands stored [k][.]: whole pieces
  int mt, nt, nsplit, steps_per_split;
  Epilogue<T> e;
};

// V neighbouring columns of a row, V the elements of a 16-byte piece.  (Called from loops that are not unrolled: the activations are long.)
// `bias`, `res`: theirs, where the columns are whole.
template <typename T>
__device__ __forceinline__ void finish(const Epilogue<T>& e, int64_t m, int64_t n, int64_t N, float* v, const Piece<float, kPiece<T>>& bias,
                                       const Piece<T, kPiece<T>>& res) {
  constexpr int V = kPiece<T>;
  if (e.part) {
    if (n < N) {                                  // (rows of shares are padded to whole quads)
#pragma unroll
      for (int q = 0; q < V / 4; ++q)
        if (n + 4 * q < N) *(f32x4_t*)(e.part + m * e.ldpart + n + 4 * q) = f32x4_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    }
  } else if (n + V <= N) {
    Piece<T, V> o;
    if (e.bias) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] += bias.at(i);
    }
    if (e.z) { o.set(v); o.store(e.z + m * e.ldz + n); }
    op_act_all<V, kFine<T>>(v, e.act);
    if (e.r) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] += res.at(i);
    }
    o.set(v);
    o.store(e.y + m * e.ldy + n);
  } else {
#pragma unroll 1
    for (int i = 0; i < V; ++i)
      if (n + i < N) {
        float h = v[i];
        if (e.bias) h += e.bias[n + i];
        if (e.z) op_narrow(h, e.z[m * e.ldz + n + i]);
        h = op_act<kFine<T>>(h, e.act);
        if (e.r) h += op_widen(e.r[m * e.ldr + n + i]);
        op_narrow(h, e.y[m * e.ldy + n + i]);
      }
  }
}

template <typename T>
__device__ __forceinline__ void finish(const Epilogue<T>& e, int64_t m, int64_t n, int64_t N, float* v) {
  Piece<float, kPiece<T>> bias{};
  Piece<T, kPiece<T>> res{};
  if (!e.part && n + kPiece<T> <= N) {
    if (e.r) res.load(e.r + m * e.ldr + n);
    if (e.bias) bias.load(e.bias + n);
  }
  finish(e, m, n, N, v, bias, res);
}

// A wavefront's results of BLOCKS x 32 rows and 64 columns pass through LDS, 32 rows at a time (`stage`: the function that puts those there),
// so that they leave as whole 16-byte pieces of rows.  The bias and all rows of the residual are asked for at once, before the
// first row is worked on: asked for row by row, each costs a turn to memory (32768 x 2048 x 2048 with residual and z: 302 against 312 us).
constexpr int kOutPitch = 64 + 4;           // floats of a row of a wavefront's staged results
template <typename T, int BLOCKS, typename Stage>
__device__ __forceinline__ void finish_rows(const Epilogue<T>& e, int64_t m0, int64_t n0, int64_t M, int64_t N, float* out, int lane, Stage stage) {
  constexpr int V = kPiece<T>, LPR = 64 / V, kStride = 64 / LPR, kTurns = 32 / kStride;        // LPR: lanes of a row
  const int64_t m1 = m0 + lane / LPR, n = n0 + (lane % LPR) * V;
  Piece<float, V> bias{};
  Piece<T, V> res[BLOCKS][kTurns] = {};
  if (!e.part && n + V <= N) {
    if (e.bias) bias.load(e.bias + n);
    if (e.r) {
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
          const int64_t m = m1 + i * 32 + k * kStride;
          if (m < M) res[i][k].load(e.r + m * e.ldr + n);
        }
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i) {
    stage(i);
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int k = 0; k < kTurns; ++k) {
      const int64_t m = m1 + i * 32 + k * kStride;
      float v[V];
#pragma unroll
      for (int q = 0; q < V / 4; ++q) *(f32x4_t*)&v[4 * q] = *(const f32x4_t*)&out[(lane / LPR + k * kStride) * kOutPitch + (lane % LPR) * V + 4 * q];
      if (m < M) finish(e, m, n, N, v, bias, res[i][0]);
#pragma unroll
      for (int h = 1; h < kTurns; ++h) res[i][h - 1] = res[i][h];      // (the loop stays a loop: the next row's is first)
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ---------------------------------------------------------------------- the tile kernel
// 128 x 128 of the result per workgroup, 4 wavefronts of 64 x 64 (2 x 2 blocks of 32 x 32), a k-step of 128 bytes per row.
// Tiles travel global -> LDS through a ring of RING steps.  An operand [row][k]: a row of a step is 128 bytes, its
// 16-byte piece c at position c ^ ((row >> 1) & 7).  An operand [k][row]: rows of 128 elements, bf16 with the 64-byte blocks
// at b ^ (k & 3) (the four rows of a transposing read then cover all banks), fp32 with the 128-byte blocks at
// b ^ ((k >> 2) & 1) (the two halves of a wavefront read rows 4 apart).  The operands of the matrix instruction are swapped
// (columns first), so that a lane ends up with four neighbouring columns of one row.  RING 4 for one workgroup on a CU, 2 for two, which
// then cover each other's waits.  Bound: bf16 by the bytes staged per flop (1024 x 4096 x 4096 52 us, 660 TFLOP/s), fp32 by the matrix
// cores (4096 x 1024 x 1024 80 us, 107 TFLOP/s, where a library product of 4096^3 reaches 143; one wavefront on a SIMD leaves a fifth
// of a step to barrier and first fragments).
constexpr int kTile = 128;

template <typename T, bool TR>
struct TileOperand {
  static constexpr int RPR = TR ? 1024 / (kTile * (int)sizeof(T)) : 8;      // tile rows of a request (1 KB)
  const char* src[4];                                                       // a lane's piece of requests 0..3, k-step 0
  int k[4];                                                                 // its (first) contraction index there
  int64_t step;                                                             // bytes to the next k-step

  __device__ __forceinline__ void init(const T* base, int64_t ld, int64_t r0, int64_t rows, int64_t contiguous, int64_t k0, int wave, int lane) {
    step = TR ? (int64_t)kStep<T> * ld * (int64_t)sizeof(T) : 128;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (TR) {
        constexpr int per = 64 / RPR;                     // pieces of a row
        const int row = (wave * 4 + i) * RPR + lane / per, pos = lane % per;
        int c;
        if (sizeof(T) == 2) c = ((((pos >> 2) ^ (row & 3)) << 2) | (pos & 3));
        else                c = ((((pos >> 3) ^ ((row >> 2) & 1)) << 3) | (pos & 7));
        const int64_t col = min(r0 + (int64_t)c * kPiece<T>, contiguous - kPiece<T>);
        k[i] = row;
        src[i] = (const char*)(base + (k0 + row) * ld + col);
      } else {
        const int row = (wave * 4 + i) * 8 + (lane >> 3);
        const int c = (lane & 7) ^ ((row >> 1) & 7);
        k[i] = c * kPiece<T>;
        src[i] = (const char*)(base + min(r0 + row, rows - 1) * ld + k0 + k[i]);
      }
    }
  }
  // left: contraction elements from this step's first one to the end
  __device__ __forceinline__ void request(int64_t j, int64_t left, uint32_t lds) const {
    if (left >= kStep<T>) {
#pragma unroll
      for (int i = 0; i < 4; ++i) lds_request16(src[i] + j * step, lds + i * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) lds_request16(k[i] < left ? (const void*)(src[i] + j * step) : (const void*)&g_zero_piece, lds + i * 1024);
    }
  }
};

// Fragment of 32 rows (block blk of the tile's four) for the contraction's part `sub`: bf16: 16 elements, fp32: 8 elements as
// four instructions' operands (a lane's four values belong to one instruction each).
template <bool TR>
__device__ __forceinline__ bf16x8_t fragment(const uint16_t* tile, int blk, int sub, int lane) {
  const int lk = lane >> 5;
  if (TR) {
    const int t16 = lane & 15, th = (lane >> 4) & 1, row = sub * 16 + lk * 8 + (t16 >> 2);
    const uint16_t* q = tile + row * kTile + (blk ^ (row & 3)) * 32 + th * 16 + (t16 & 3) * 4;
    union { s16x4_t h[2]; bf16x8_t v; } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(q));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(q + 4 * kTile));
    return u.v;
  }
  const int row = blk * 32 + (lane & 31);
  return *(const bf16x8_t*)(tile + row * 64 + (((sub << 1) | lk) ^ ((row >> 1) & 7)) * 8);
}
template <bool TR>
__device__ __forceinline__ f32x4_t fragment(const float* tile, int blk, int sub, int lane) {
  const int lk = lane >> 5;
  if (TR) {
    const float* q = tile + (sub * 8 + lk * 4) * kTile + (blk ^ lk) * 32 + (lane & 31);
    return f32x4_t{q[0], q[kTile], q[2 * kTile], q[3 * kTile]};
  }
  const int row = blk * 32 + (lane & 31);
  return *(const f32x4_t*)(tile + row * 32 + (((sub << 1) | lk) ^ ((row >> 1) & 7)) * 4);
}
__device__ __forceinline__ f32x16_t multiply(bf16x8_t a, bf16x8_t b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16_t multiply(f32x4_t a, f32x4_t b, f32x16_t c) {
#pragma unroll
  for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[s], b[s], c, 0, 0, 0);
  return c;
}

template <typename T> constexpr int kTileOperand = kTile * kStep<T>;       // elements of an operand's step (16 KB)

// `block`: this workgroup's number among the product's
template <typename T, bool ATR, bool BTR, int RING>
__device__ __forceinline__ void tile_product(const GemmArgs<T>& g, int block, T* smem) {
  constexpr int kOperand = kTileOperand<T>;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  // workgroups go round the eight XCDs: each takes a run of neighbouring tiles, columns fastest
  const int total = g.mt * g.nt * g.nsplit, per = (total + 7) / 8;
  const int id = (block & 7) * per + (block >> 3);
  if ((block >> 3) >= per || id >= total) return;
  const int split = id / (g.mt * g.nt), tile = id - split * (g.mt * g.nt);
  const int64_t m0 = (int64_t)(tile / g.nt) * kTile, n0 = (int64_t)(tile % g.nt) * kTile;
  const int64_t k0 = (int64_t)split * g.steps_per_split * kStep<T>;
  const int64_t kend = min(g.K, k0 + (int64_t)g.steps_per_split * kStep<T>);
  const int nks = (int)((kend - k0 + kStep<T> - 1) / kStep<T>);

  TileOperand<T, ATR> oa;
  TileOperand<T, BTR> ob;
  oa.init(g.A, g.lda, m0, g.M, g.mc, k0, wave, lane);
  ob.init(g.B, g.ldb, n0, g.N, g.nc, k0, wave, lane);
  const uint32_t lds = lds_at(smem) + (uint32_t)wave * 4096u;
  auto request = [&](int j, int stage) {
    const int64_t left = g.K - k0 - (int64_t)j * kStep<T>;
    oa.request(j, left, lds + (uint32_t)stage * 32768u);
    ob.request(j, left, lds + (uint32_t)stage * 32768u + 16384u);
  };
  f32x16_t acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
#pragma unroll
  for (int j = 0; j < RING - 1; ++j)
    if (j < nks) request(j, j);
  int stage = 0;
  for (int ks = 0; ks < nks; ++ks) {
    if (RING > 2 && ks + RING - 1 <= nks) ring_wait<(RING - 2) * 8>();   // step ks is there for every wavefront, and everybody
    else                                  ring_wait<0>();                // is done with step ks - 1
    if (ks + RING - 1 < nks) request(ks + RING - 1, stage == 0 ? RING - 1 : stage - 1);
    const T* const sa = smem + stage * 2 * kOperand;
    const T* const sb = sa + kOperand;
    stage = stage + 1 == RING ? 0 : stage + 1;
#pragma unroll
    for (int sub = 0; sub < 4; ++sub) {
      const auto a0 = fragment<ATR>(sa, wm * 2, sub, lane), a1 = fragment<ATR>(sa, wm * 2 + 1, sub, lane);
      const auto b0 = fragment<BTR>(sb, wn * 2, sub, lane), b1 = fragment<BTR>(sb, wn * 2 + 1, sub, lane);
      acc[0][0] = multiply(b0, a0, acc[0][0]);
      acc[0][1] = multiply(b1, a0, acc[0][1]);
      acc[1][0] = multiply(b0, a1, acc[1][0]);
      acc[1][1] = multiply(b1, a1, acc[1][1]);
    }
  }
  // Register r of a lane: column 8 (r / 4) + 4 (lane / 32) + r % 4, row lane % 32 of its block.
  float* const out = (float*)smem + wave * (32 * kOutPitch);
  Epilogue<T> e = g.e;
  if (e.part) e.part += split * e.part_stride;
  finish_rows<T, 2>(e, m0 + wm * 64, n0 + wn * 64, g.M, g.N, out, lane, [&](int i) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(f32x4_t*)&out[(lane & 31) * kOutPitch + j * 32 + 8 * q + 4 * (lane >> 5)] =
            f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
  });
}

// ---------------------------------------------------------------------- the large-tile kernel (bf16)
// 256 x 256 of the result, 8 wavefronts (2 x 4) of 128 x 64 as 8 x 4 blocks of MFMA 16x16x32, a k-step of 64.  What bounds a bf16
// product on tiles is the bytes staged per flop: a 256 x 256 tile stages half of what a 128 x 128 one does.  A k-step is
// four turns of 16 MFMAs per wavefront (half of A times half of B); the two wavefronts of a SIMD are half a turn apart, so that
// while one multiplies the other reads fragments and requests.  A half is requested again, for the step after the next, as soon as
// both hold it in registers: a request is seven turns in flight, counted and never drained inside the loop.
// A half of A is 64 of each wavefront row's 128 rows, a half of B 32 of each wavefront column's 64 columns: 16 KB, two requests per
// wavefront.  [row][k] operands: 128 rows of 128 bytes, pieces XORed by (row >> 1) & 7; [k][row] operands: 64 rows of 128
// elements, 64-byte blocks XORed by k & 3 and their 32-byte halves by (k >> 3) & 1 (the four quarters of a wavefront read rows 8 apart).
// 32768 x 2048 x 2048: 265 us, 1.04 PFLOP/s (a library product of 8192^3 1.32), 293 with residual and z: a workgroup fills a CU, so
// a tile's epilogue and first requests (12 us of 57) lie bare.
constexpr int kBig = 256;
constexpr int kHalf = 128 * 64;                           // elements of a half of an operand's step

template <bool TR, bool IS_A>
struct BigOperand {
  const uint16_t* src[2][2];                              // a lane's piece [half][request] of k-step 0
  int k[2];                                               // its contraction index there, by request
  int64_t step;
  __device__ __forceinline__ void init(const uint16_t* base, int64_t ld, int64_t r0, int64_t rows, int64_t contiguous, int64_t k0, int wave, int lane) {
    step = TR ? 64 * ld : 64;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      if (TR) {
        const int row = wave * 8 + q * 4 + (lane >> 4), pc = lane & 15;
        const int col = (((pc >> 2) ^ (row & 3)) << 5) | (((pc & 3) ^ (((row >> 3) & 1) << 1)) << 3);
        k[q] = row;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int64_t c = r0 + (IS_A ? (col >> 6) * 128 + h * 64 + (col & 63) : (col >> 5) * 64 + h * 32 + (col & 31));
          src[h][q] = base + (k0 + row) * ld + min(c, contiguous - 8);
        }
      } else {
        const int row = wave * 16 + q * 8 + (lane >> 3);
        k[q] = ((lane & 7) ^ ((row >> 1) & 7)) * 8;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int64_t r = r0 + (IS_A ? (row >> 6) * 128 + h * 64 + (row & 63) : (row >> 5) * 64 + h * 32 + (row & 31));
          src[h][q] = base + min(r, rows - 1) * ld + k0 + k[q];
        }
      }
    }
  }
  __device__ __forceinline__ void request(int64_t j, int64_t left, int h, uint32_t lds) const {
    if (left >= 64) {
      lds_request16(src[h][0] + j * step, lds);
      lds_request16(src[h][1] + j * step, lds + 1024);
    } else {
      lds_request16(k[0] < left ? (const void*)(src[h][0] + j * step) : (const void*)&g_zero_piece, lds);
      lds_request16(k[1] < left ? (const void*)(src[h][1] + j * step) : (const void*)&g_zero_piece, lds + 1024);
    }
  }
};

// Where a lane's fragments of a half start, in elements: block i, 32-wide part s of the step.
template <bool TR, bool IS_A>
__device__ __forceinline__ bf16x8_t big_fragment(const uint16_t* half, int w, int i, int s, int lane) {
  const int lr = lane & 15, lk = lane >> 4;
  if (TR) {
    const int tr = lr >> 2, blk = IS_A ? w * 2 + (i >> 1) : w;
    const uint16_t* q = half + (s * 32 + 8 * lk + tr) * 128 + ((blk ^ tr) << 5) + (((i & 1) ^ (lk & 1)) << 4) + 4 * (lr & 3);
    union { s16x4_t h[2]; bf16x8_t v; } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(q));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(q + 4 * 128));
    return u.v;
  }
  const int row = w * (IS_A ? 64 : 32) + i * 16 + lr;
  return *(const bf16x8_t*)(half + row * 64 + ((((s << 2) | lk) ^ ((lr >> 1) & 7)) << 3));
}

// `block`: this workgroup's number among the product's
template <bool ATR, bool BTR>
__device__ __forceinline__ void big_product(const GemmArgs<uint16_t>& g, int block, uint16_t* smem) {   // [stage][A0 A1], then [stage][B0 B1]
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  const int total = g.mt * g.nt * g.nsplit, per = (total + 7) / 8;
  const int id = (block & 7) * per + (block >> 3);
  if ((block >> 3) >= per || id >= total) return;
  const int split = id / (g.mt * g.nt), tile = id - split * (g.mt * g.nt);
  const int64_t m0 = (int64_t)(tile / g.nt) * kBig, n0 = (int64_t)(tile % g.nt) * kBig;
  const int64_t k0 = (int64_t)split * g.steps_per_split * 64;
  const int64_t kend = min(g.K, k0 + (int64_t)g.steps_per_split * 64);
  const int nks = (int)((kend - k0 + 63) / 64);

  BigOperand<ATR, true> oa;
  BigOperand<BTR, false> ob;
  oa.init(g.A, g.lda, m0, g.M, g.mc, k0, wave, lane);
  ob.init(g.B, g.ldb, n0, g.N, g.nc, k0, wave, lane);
  const uint32_t dma_a = lds_at(smem) + (uint32_t)wave * 2048u, dma_b = dma_a + 4 * kHalf * 2;
  auto request_a = [&](int j, int st, int h) { oa.request(j, g.K - k0 - (int64_t)j * 64, h, dma_a + (uint32_t)((st * 2 + h) * kHalf * 2)); };
  auto request_b = [&](int j, int st, int h) { ob.request(j, g.K - k0 - (int64_t)j * 64, h, dma_b + (uint32_t)((st * 2 + h) * kHalf * 2)); };

  f32x4_t acc[8][4];
#pragma unroll
  for (int a = 0; a < 8; ++a)
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[a][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  bf16x8_t fa[8], fbx[2][2], fby[2][2];
#define ABS_LOAD_A(st_, h_)                                                                                          \
  _Pragma("unroll") for (int q_ = 0; q_ < 8; ++q_)                                                                   \
    fa[q_] = big_fragment<ATR, true>(smem + ((st_) * 2 + (h_)) * kHalf, wm, q_ >> 1, q_ & 1, lane);
#define ABS_LOAD_B(dst_, st_, h_)                                                                                    \
  _Pragma("unroll") for (int s_ = 0; s_ < 2; ++s_) _Pragma("unroll") for (int j_ = 0; j_ < 2; ++j_)                  \
    dst_[j_][s_] = big_fragment<BTR, false>(smem + (4 + (st_) * 2 + (h_)) * kHalf, wn, j_, s_, lane);
#define ABS_MMA(ha_, hb_, b_)                                                                                        \
  __builtin_amdgcn_sched_barrier(0);                                                                                 \
  _Pragma("unroll") for (int s_ = 0; s_ < 2; ++s_) _Pragma("unroll") for (int i_ = 0; i_ < 4; ++i_)                  \
    _Pragma("unroll") for (int j_ = 0; j_ < 2; ++j_)                                                                 \
      acc[(ha_) * 4 + i_][(hb_) * 2 + j_] =                                                                          \
          __builtin_amdgcn_mfma_f32_16x16x32_bf16(b_[j_][s_], fa[2 * i_ + s_], acc[(ha_) * 4 + i_][(hb_) * 2 + j_], 0, 0, 0); \
  __builtin_amdgcn_sched_barrier(0);                                                                                 \
  asm volatile("s_barrier" ::: "memory");
#define ABS_TURN(i_)                                                                                                 \
  if (left >= 2)      ring_wait<12>();                                                                               \
  else if (left == 1) ring_wait<10 - 2 * (i_)>();                                                                    \
  else                ring_wait<(i_) == 0 ? 2 : 0>();
#define ABS_STEP(X_, Y_, st_)                                                                                        \
  {                                                                                                                  \
    const int left = nks - 1 - j;                                                                                    \
    ABS_LOAD_A(st_, 0);                                                                                              \
    if (left >= 2) request_b(j + 2, st_, 0);                                                                         \
    ABS_TURN(0); ABS_MMA(0, 0, X_);                                                                                  \
    ABS_LOAD_B(Y_, st_, 1);                                                                                          \
    if (left >= 2) request_a(j + 2, st_, 0);                                                                         \
    ABS_TURN(1); ABS_MMA(0, 1, Y_);                                                                                  \
    ABS_LOAD_A(st_, 1);                                                                                              \
    if (left >= 2) request_b(j + 2, st_, 1);                                                                         \
    ABS_TURN(2); ABS_MMA(1, 1, Y_);                                                                                  \
    if (left >= 1) ABS_LOAD_B(Y_, (st_) ^ 1, 0);                                                                     \
    if (left >= 2) request_a(j + 2, st_, 1);                                                                         \
    ABS_TURN(3); ABS_MMA(1, 0, X_);                                                                                  \
  }
  request_b(0, 0, 0); request_a(0, 0, 0); request_b(0, 0, 1); request_a(0, 0, 1);
  if (nks > 1) {
    request_b(1, 1, 0); request_a(1, 1, 0); request_b(1, 1, 1); request_a(1, 1, 1);
    ring_wait<12>();
  } else {
    ring_wait<4>();
  }
  ABS_LOAD_B(fbx, 0, 0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // (requested again in the first turn)
  if (wm) asm volatile("s_barrier" ::: "memory");
  for (int j = 0;;) {
    ABS_STEP(fbx, fby, 0);
    if (++j >= nks) break;
    ABS_STEP(fby, fbx, 1);
    if (++j >= nks) break;
  }
  if (!wm) asm volatile("s_barrier" ::: "memory");
#undef ABS_STEP
#undef ABS_TURN
#undef ABS_MMA
#undef ABS_LOAD_B
#undef ABS_LOAD_A
  // Register r of a lane: column 4 (lane / 16) + r, row lane % 16 of its block.
  float* const out = (float*)smem + wave * (32 * kOutPitch);
  Epilogue<uint16_t> e = g.e;
  if (e.part) e.part += split * e.part_stride;
  finish_rows<uint16_t, 4>(e, m0 + wm * 128, n0 + wn * 64, g.M, g.N, out, lane, [&](int i) {
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int b = 0; b < 4; ++b) *(f32x4_t*)&out[(a * 16 + (lane & 15)) * kOutPitch + b * 16 + 4 * (lane >> 4)] = acc[2 * i + a][b];
  });
}

constexpr int kBigLds = 8 * kHalf;
template <typename T, bool ATR, bool BTR, int RING>
__global__ __launch_bounds__(256, RING <= 2 ? 2 : 1) void linear_tile_kernel(GemmArgs<T> g) {
  __shared__ __attribute__((aligned(1024))) T smem[RING * 2 * kTileOperand<T>];
  tile_product<T, ATR, BTR, RING>(g, blockIdx.x, smem);
}
// dW and dx of one layer side by side, two workgroups of either on a CU
template <typename T>
__global__ __launch_bounds__(256, 2) void linear_tile_pair_kernel(GemmArgs<T> dw, GemmArgs<T> dx, int dw_blocks) {
  __shared__ __attribute__((aligned(1024))) T smem[2 * 2 * kTileOperand<T>];
  if ((int)blockIdx.x < dw_blocks) tile_product<T, true, true, 2>(dw, blockIdx.x, smem);
  else tile_product<T, false, false, 2>(dx, (int)blockIdx.x - dw_blocks, smem);
}
template <bool ATR, bool BTR>
__global__ __launch_bounds__(512, 1) void linear_big_kernel(GemmArgs<uint16_t> g) {
  __shared__ __attribute__((aligned(1024))) uint16_t smem[kBigLds];
  big_product<ATR, BTR>(g, blockIdx.x, smem);
}
// The same on large tiles: with the longer contraction cut so that all CUs get as many k-steps, they leave fewer shares
// and fewer CUs idle than one after the other.  The longer runs come first.  (8192 x 2048 x 2048 124 to 135 us, 1.0 to 1.1 PFLOP/s.)
__global__ __launch_bounds__(512, 1) void linear_big_pair_kernel(GemmArgs<uint16_t> dw, GemmArgs<uint16_t> dx, int dw_blocks) {
  __shared__ __attribute__((aligned(1024))) uint16_t smem[kBigLds];
  if ((int)blockIdx.x < dw_blocks) big_product<true, true>(dw, blockIdx.x, smem);
  else big_product<false, false>(dx, (int)blockIdx.x - dw_blocks, smem);
}

// ---------------------------------------------------------------------- shares of the contraction, added in their order
// db: rows of column sums, added in their order, 32 columns x 8 rows at a time
struct DbShares { const float* sums; int shares, N; float* db; };
__device__ __forceinline__ void add_db(const DbShares& d) {
  __shared__ float red[8][33];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
  for (int n0 = blockIdx.x * 32; n0 < d.N; n0 += gridDim.x * 32) {
    const int n = n0 + c;
    float v = 0.f;
    if (n < d.N)
#pragma unroll 8
      for (int k = r; k < d.shares; k += 8) v += d.sums[(int64_t)k * d.N + n];
    red[r][c] = v;
    __syncthreads();
    if (r == 0 && n < d.N) {
      for (int k = 1; k < 8; ++k) v += red[k][c];
      d.db[n] = v;
    }
    __syncthreads();
  }
}

template <typename T>
struct Join { Epilogue<T> e; int64_t M, N; int shares; };
template <typename T>
__global__ __launch_bounds__(256) void linear_join_kernel(Join<T> first, Join<T> second, DbShares d) {
  constexpr int V = kPiece<T>;
  const Join<T>& j = blockIdx.y ? second : first;
  const int shares = j.shares;
  if (d.db && blockIdx.y == 0) add_db(d);
  Epilogue<T> e = j.e;
  const float* const part = e.part;
  e.part = nullptr;
  const int64_t pieces = (j.N + V - 1) / V, total = j.M * pieces;
#pragma unroll 1
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
    const int64_t m = q / pieces, n = (q - m * pieces) * V;
    float v[V];
#pragma unroll
    for (int h = 0; h < V / 4; ++h) {
      if (n + 4 * h >= j.N) { v[4 * h] = v[4 * h + 1] = v[4 * h + 2] = v[4 * h + 3] = 0.f; continue; }
      const float* p = part + m * e.ldpart + n + 4 * h;
      f32x4_t s = *(const f32x4_t*)p;
#pragma unroll 8
      for (int k = 1; k < shares; ++k) s += *(const f32x4_t*)(p + k * e.part_stride);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * h + i] = s[i];
    }
    finish(e, m, n, j.N, v);
  }
}

// ---------------------------------------------------------------------- small products: operands straight from memory into registers
// A product that a handful of tiles covers waits for launches and memory's latency, not for arithmetic.  So a whole forward or
// backward pass is one launch (and one more where a long contraction is cut into shares): a tile is 32 x 64 of the result (dW: 64 x 64),
// a workgroup's eight wavefronts share its contraction (blocks of 16 bf16 or 8 fp32 go round them) or, with little of that, several
// tiles; every operand goes from memory into the matrix instruction's registers with no LDS in between, and the partial results
// meet in LDS once.  Reads are per element, pair or piece at any alignment; dz is computed where it is read, and db summed by the
// workgroups of dW's first row of tiles.  810 x 520 x 300 6.4 us, 1 x 2048 x 2048 7.7 (8 MB: 1.1 TB/s), fp32 640 x 400 x 120 8.8: one chain
// of loads, products and the exchange.
// [k][column] operands: a lane reads two neighbouring columns of 8 (fp32: 4) rows, so its even columns make one fragment
// and its odd ones another; [row][k] operands follow the same numbering, row 2 (lane % 32) + j in fragment j.
constexpr int kSmallWaves = 8;
template <typename T> constexpr int kBlockK = sizeof(T) == 2 ? 16 : 8;       // contraction of one wavefront's step

template <typename T> struct FragOf;
template <> struct FragOf<uint16_t> { typedef bf16x8_t type; };
template <> struct FragOf<float> { typedef f32x4_t type; };
template <typename T> using Frag = typename FragOf<T>::type;

// dz goes through the matrix instruction as the sum of two bf16 values (15 bits of it and more: a gradient's rounding is then its output's
// alone, for instructions that a product waiting for memory has to spare).  Both have dz's sign, and neither is 0 unless dz is: the first
// is the largest bf16 value below dz in size, the second the rest.  An infinite x or W thus meets no other factors than it meets in dz; of
// an infinite dz both are infinite.  shrink: 1 - 2^-23, or, for relu, whose dz is a bf16 value already, 1 (there is no second part).
template <int N>
__device__ __forceinline__ void two_parts(const float* f, float shrink, Piece<uint16_t, N>& first, Piece<uint16_t, N>& rest) {
  float r[N];
#pragma unroll
  for (int i = 0; i < N / 2; ++i)
    first.w[i] = __builtin_amdgcn_perm(__float_as_uint(f[2 * i + 1] * shrink), __float_as_uint(f[2 * i] * shrink), 0x07060302u);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float l = f[i] - first.at(i);
    r[i] = fabsf(l) < 3e38f ? l : f[i];
  }
  rest.set(r);
}
__device__ __forceinline__ float parts_shrink(int act) { return act > ABS_ACT_RELU ? 0.99999988f : 1.0f; }

// [row][k]: elements k .. k + 7 (fp32: 3) of a row, zeros from K on
template <typename T>
struct RowPart {
  uint32_t w[4];
  __device__ __forceinline__ void load(const T* p, int k, int K) {
    constexpr int N = kPiece<T>;
    if (k + N <= K) {
      const Loose<T, N> l = *(const Loose<T, N>*)(p + k);
      __builtin_memcpy(w, &l, 16);
    } else {
      T v[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const T x = p[min(k + e, K - 1)];
        v[e] = k + e < K ? x : T(0);
      }
      __builtin_memcpy(w, v, 16);
    }
  }
  __device__ __forceinline__ Frag<T> frag() const { Frag<T> f; __builtin_memcpy(&f, w, 16); return f; }
  // this = dz, from dy (this) and z, which becomes the second part of a bf16 dz
  __device__ __forceinline__ void slope(RowPart& z, int act) {
    Piece<T, kPiece<T>> d, h;
    float f[kPiece<T>], g[kPiece<T>];
#pragma unroll
    for (int i = 0; i < 4; ++i) { d.w[i] = w[i]; h.w[i] = z.w[i]; }
#pragma unroll
    for (int e = 0; e < kPiece<T>; ++e) { f[e] = d.at(e); g[e] = h.at(e); }
    op_slope_all<kPiece<T>, kFine<T>>(f, g, act);
    if constexpr (sizeof(T) == 2) two_parts<kPiece<T>>(f, parts_shrink(act), d, h);
    else d.set(f);
#pragma unroll
    for (int i = 0; i < 4; ++i) { w[i] = d.w[i]; if (sizeof(T) == 2) z.w[i] = h.w[i]; }
  }
};

// [k][column]: two neighbouring columns of rows k .. k + 7 (fp32: 3), zeros from K on.  A lane's columns are c and c + 1; beyond the last
// column it reads the last two (what it computes from them is not stored), at the last of an odd number the pair before (swap).
struct ColumnPlace { int at; bool swap; };
__device__ __forceinline__ ColumnPlace column_place(int c, int N) { return {min(c, N - 2), c == N - 1}; }
template <typename T> struct ColumnPart;
template <>
struct ColumnPart<uint16_t> {
  uint32_t w[8];                                            // a row's two columns
  __device__ __forceinline__ void load(const uint16_t* p, int64_t ld, int k, int K, ColumnPlace c, int N) {
    const uint16_t* q = p + (int64_t)min(k, K - 1) * ld + c.at;
    if (k + 8 <= K) {
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const Loose<uint16_t, 2> l = *(const Loose<uint16_t, 2>*)q;
        __builtin_memcpy(&w[r], &l, 4);
        q += ld;
      }
    } else {
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        w[r] = 0u;
        if (k + r < K) {
          const Loose<uint16_t, 2> l = *(const Loose<uint16_t, 2>*)q;
          __builtin_memcpy(&w[r], &l, 4);
          q += ld;
        }
      }
    }
    if (N & 1) {
#pragma unroll
      for (int r = 0; r < 8; ++r) w[r] = c.swap ? w[r] >> 16 : w[r];
    }
  }
  __device__ __forceinline__ bf16x8_t frag(int odd) const {
    uint32_t f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], odd ? 0x07060302u : 0x05040100u);
    bf16x8_t v;
    __builtin_memcpy(&v, f, 16);
    return v;
  }
  __device__ __forceinline__ void slope(ColumnPart& z, int act, float& s0, float& s1) {
#pragma unroll
    for (int r = 0; r < 8; r += 4) {
      float f[8], h[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[r + i] << 16); f[2 * i + 1] = __uint_as_float(w[r + i] & 0xFFFF0000u);
        h[2 * i] = __uint_as_float(z.w[r + i] << 16); h[2 * i + 1] = __uint_as_float(z.w[r + i] & 0xFFFF0000u);
      }
      op_slope_all<8, false>(f, h, act);
      Piece<uint16_t, 8> o, rest;
      two_parts<8>(f, parts_shrink(act), o, rest);
#pragma unroll
      for (int i = 0; i < 4; ++i) { s0 += f[2 * i]; s1 += f[2 * i + 1]; w[r + i] = o.w[i]; z.w[r + i] = rest.w[i]; }
    }
  }
  __device__ __forceinline__ void sum(float& s0, float& s1) const {
#pragma unroll
    for (int r = 0; r < 8; ++r) { s0 += __uint_as_float(w[r] << 16); s1 += __uint_as_float(w[r] & 0xFFFF0000u); }
  }
};
template <>
struct ColumnPart<float> {
  float w[2][4];                                            // [column][row]
  __device__ __forceinline__ void load(const float* p, int64_t ld, int k, int K, ColumnPlace c, int N) {
    const float* q = p + (int64_t)min(k, K - 1) * ld + c.at;
    if (k + 4 <= K) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const Loose<float, 2> l = *(const Loose<float, 2>*)q;
        w[0][r] = l.e[0]; w[1][r] = l.e[1];
        q += ld;
      }
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        w[0][r] = w[1][r] = 0.f;
        if (k + r < K) {
          const Loose<float, 2> l = *(const Loose<float, 2>*)q;
          w[0][r] = l.e[0]; w[1][r] = l.e[1];
          q += ld;
        }
      }
    }
    if (N & 1) {
#pragma unroll
      for (int r = 0; r < 4; ++r) w[0][r] = c.swap ? w[1][r] : w[0][r];
    }
  }
  __device__ __forceinline__ f32x4_t frag(int odd) const { return f32x4_t{w[odd][0], w[odd][1], w[odd][2], w[odd][3]}; }
  __device__ __forceinline__ void slope(ColumnPart& z, int act, float& s0, float& s1) {
    op_slope_all<8, true>(&w[0][0], &z.w[0][0], act);
    sum(s0, s1);
  }
  __device__ __forceinline__ void sum(float& s0, float& s1) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) { s0 += w[0][r]; s1 += w[1][r]; }
  }
};

template <typename T>
struct DzSource { const T* dy; const T* z; int64_t lddy, ldz; int act; };

// Tiles of one of the products, 8 / team in a workgroup (one above the other, `team` wavefronts each); its contraction in `splits`
// shares of `steps` blocks each, which leave in fp32 to be joined.  tiles: workgroups' worth.
template <typename T>
struct SmallPart { Epilogue<T> e; int nt, tiles, splits, steps, team; };
template <typename T>
struct SmallArgs {
  const T* x; const T* w;
  int64_t ldx, ldw;
  int rows, d_in, d_out;
  DzSource<T> dz;
  SmallPart<T> a, b;                   // a: the forward product, or dx; b: dW (its workgroups come behind dx's)
  float* db;                           // or its shares [splits][d_out]
  bool dw;
};

// 32 rows of the partial results of every team's wavefronts, added in their order, and what follows.  Tile `i` of the workgroup has rows
// m0 + i m_tile, ... + m_step each.
template <typename T>
__device__ __forceinline__ void small_finish(const Epilogue<T>& e, const f32x16_t& a0, const f32x16_t& a1, float* red, int team, int waves,
                                             int64_t m0, int m_tile, int m_step, int64_t M, int64_t n0, int64_t N) {
  constexpr int kPitch = 64 + 4, V = kPiece<T>, LPR = 64 / V;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  if ((wave & (team - 1)) < waves) {
    float* q = red + (wave * 32 + (lane & 31)) * kPitch + 8 * (lane >> 5);
#pragma unroll
    for (int b = 0; b < 4; ++b) {       // registers 4 b .. of a0 / a1: even / odd columns 2 (8 b + 4 (lane / 32) + r)
      *(f32x4_t*)(q + 16 * b) = f32x4_t{a0[4 * b], a1[4 * b], a0[4 * b + 1], a1[4 * b + 1]};
      *(f32x4_t*)(q + 16 * b + 4) = f32x4_t{a0[4 * b + 2], a1[4 * b + 2], a0[4 * b + 3], a1[4 * b + 3]};
    }
  }
  __syncthreads();
  for (int j = t / LPR; j < 32 * (kSmallWaves / team); j += 512 / LPR) {
    const int i = j >> 5, r = j & 31;
    float v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = 0.f;
    const float* q = red + (i * team * 32 + r) * kPitch + (t % LPR) * V;
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int h = 0; h < V / 4; ++h) {
        const f32x4_t s = *(const f32x4_t*)(q + w * 32 * kPitch + 4 * h);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[4 * h + k] += s[k];
      }
    const int64_t m = m0 + (int64_t)i * m_tile + (int64_t)r * m_step;
    if (m < M) finish(e, m, n0 + (t % LPR) * V, N, v);
  }
}

// A wavefront's blocks first, first + team, ... of the contraction, U at a time: all their loads stand before the first use.
template <int U, typename Step, typename Load, typename Use>
__device__ __forceinline__ void in_steps(int first, int team, int blocks, Load load, Use use) {
  int kb = first;
  for (; kb + (U - 1) * team < blocks; kb += U * team) {
    Step s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) load(kb + u * team, s[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) use(s[u]);
  }
  for (; kb < blocks; kb += team) {
    Step s;
    load(kb, s);
    use(s);
  }
}

// TEAM: 8, which spares address arithmetic (1 x 2048 x 2048 7.4 us against 8.5), or 0, whatever the parts say.
template <typename T, bool BACKWARD, int TEAM>
__global__ __launch_bounds__(512, 2) void linear_small_kernel(SmallArgs<T> g) {
  constexpr int R = kPiece<T>;
  __shared__ __attribute__((aligned(16))) float red[kSmallWaves * 32 * 68];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), l32 = lane & 31, lk = lane >> 5;
  f32x16_t acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  // this workgroup's tile, share of the contraction and blocks of it
  int n0, tm, first, blocks, waves, split, team = TEAM, at, mate;             // at: this wavefront's tile of the workgroup's, mate: its number there
  auto place = [&](const SmallPart<T>& part, int id, int K) {
    split = part.splits > 1 ? id / part.tiles : 0;
    const int tile = id - split * part.tiles;
    tm = tile / part.nt;
    n0 = (tile - tm * part.nt) * 64;
    first = split * part.steps;
    blocks = min((K + kBlockK<T> - 1) / kBlockK<T>, first + part.steps);
    if (TEAM == 0) team = part.team;
    waves = min(team, blocks - first);
    at = wave / team;
    mate = wave & (team - 1);
  };
  auto epilogue = [&](const SmallPart<T>& part) {
    Epilogue<T> e = part.e;
    if (e.part) e.part += split * e.part_stride;
    return e;
  };
  if constexpr (!BACKWARD) {
    const int K = g.d_in;
    place(g.a, blockIdx.x, K);
    const int m0 = tm * (32 * kSmallWaves / team);
    const T* const xr = g.x + (int64_t)min(m0 + at * 32 + l32, g.rows - 1) * g.ldx;
    struct Step { RowPart<T> a; ColumnPart<T> b; };
    const ColumnPlace c = column_place(n0 + 2 * l32, g.d_out);
    in_steps<4, Step>(first + mate, team, blocks,
        [&](int kb, Step& s) {
          const int k = kb * kBlockK<T> + lk * R;
          s.a.load(xr, k, K);
          s.b.load(g.w, g.ldw, k, K, c, g.d_out);
        },
        [&](Step& s) {
          acc[0][0] = multiply(s.b.frag(0), s.a.frag(), acc[0][0]);
          acc[0][1] = multiply(s.b.frag(1), s.a.frag(), acc[0][1]);
        });
    small_finish<T>(epilogue(g.a), acc[0][0], acc[0][1], red, team, waves, m0, 32, 1, g.rows, n0, g.d_out);
    return;
  }
  const int dx_blocks = g.a.tiles * g.a.splits;
  if ((int)blockIdx.x < dx_blocks) {                        // dx = dz W^T
    const int K = g.d_out;
    place(g.a, blockIdx.x, K);
    const int m0 = tm * (32 * kSmallWaves / team);
    const int64_t row = min(m0 + at * 32 + l32, g.rows - 1);
    const T* const dr = g.dz.dy + row * g.dz.lddy;
    const T* const zr = g.dz.z + row * g.dz.ldz;
    const T* const w0 = g.w + (int64_t)min(n0 + 2 * l32, g.d_in - 1) * g.ldw;
    const T* const w1 = g.w + (int64_t)min(n0 + 2 * l32 + 1, g.d_in - 1) * g.ldw;
    struct Step { RowPart<T> a, z, b0, b1; };
    in_steps<4, Step>(first + mate, team, blocks,
        [&](int kb, Step& s) {
          const int k = kb * kBlockK<T> + lk * R;
          s.a.load(dr, k, K);
          if (g.dz.act != ABS_ACT_NONE) s.z.load(zr, k, K);
          s.b0.load(w0, k, K);
          s.b1.load(w1, k, K);
        },
        [&](Step& s) {
          if (g.dz.act != ABS_ACT_NONE) s.a.slope(s.z, g.dz.act);
          acc[0][0] = multiply(s.b0.frag(), s.a.frag(), acc[0][0]);
          acc[0][1] = multiply(s.b1.frag(), s.a.frag(), acc[0][1]);
          if (sizeof(T) == 2 && g.dz.act > ABS_ACT_RELU) {          // (relu's dz is dy or 0)
            acc[0][0] = multiply(s.b0.frag(), s.z.frag(), acc[0][0]);
            acc[0][1] = multiply(s.b1.frag(), s.z.frag(), acc[0][1]);
          }
        });
    small_finish<T>(epilogue(g.a), acc[0][0], acc[0][1], red, team, waves, m0, 32, 1, g.rows, n0, g.d_in);
    return;
  }
  // dW = x^T dz, and db in the first row of tiles
  const int K = g.rows;
  place(g.b, (int)blockIdx.x - dx_blocks, K);
  const int m0 = tm * (64 * kSmallWaves / team);
  float s0 = 0.f, s1 = 0.f;
  const ColumnPlace cb = column_place(n0 + 2 * l32, g.d_out);
  if (g.dw) {
    struct Step { ColumnPart<T> a, b, z; };
    const ColumnPlace ca = column_place(m0 + at * 64 + 2 * l32, g.d_in);
    in_steps<2, Step>(first + mate, team, blocks,
        [&](int kb, Step& s) {
          const int k = kb * kBlockK<T> + lk * R;
          s.a.load(g.x, g.ldx, k, K, ca, g.d_in);
          s.b.load(g.dz.dy, g.dz.lddy, k, K, cb, g.d_out);
          if (g.dz.act != ABS_ACT_NONE) s.z.load(g.dz.z, g.dz.ldz, k, K, cb, g.d_out);
        },
        [&](Step& s) {
          if (g.dz.act != ABS_ACT_NONE) s.b.slope(s.z, g.dz.act, s0, s1);
          else if (g.db && m0 == 0) s.b.sum(s0, s1);
          const Frag<T> fa0 = s.a.frag(0), fa1 = s.a.frag(1), fb0 = s.b.frag(0), fb1 = s.b.frag(1);
          acc[0][0] = multiply(fb0, fa0, acc[0][0]);
          acc[0][1] = multiply(fb1, fa0, acc[0][1]);
          acc[1][0] = multiply(fb0, fa1, acc[1][0]);
          acc[1][1] = multiply(fb1, fa1, acc[1][1]);
          if (sizeof(T) == 2 && g.dz.act > ABS_ACT_RELU) {          // (relu's dz is dy or 0)
            const Frag<T> fz0 = s.z.frag(0), fz1 = s.z.frag(1);
            acc[0][0] = multiply(fz0, fa0, acc[0][0]);
            acc[0][1] = multiply(fz1, fa0, acc[0][1]);
            acc[1][0] = multiply(fz0, fa1, acc[1][0]);
            acc[1][1] = multiply(fz1, fa1, acc[1][1]);
          }
        });
  } else {                                                          // db alone: x, which may be missing, is not read
    struct Step { ColumnPart<T> b, z; };
    in_steps<2, Step>(first + mate, team, blocks,
        [&](int kb, Step& s) {
          const int k = kb * kBlockK<T> + lk * R;
          s.b.load(g.dz.dy, g.dz.lddy, k, K, cb, g.d_out);
          if (g.dz.act != ABS_ACT_NONE) s.z.load(g.dz.z, g.dz.ldz, k, K, cb, g.d_out);
        },
        [&](Step& s) {
          if (g.dz.act != ABS_ACT_NONE) s.b.slope(s.z, g.dz.act, s0, s1);
          else s.b.sum(s0, s1);
        });
  }
  if (g.db && m0 == 0) {
    s0 += __shfl_xor(s0, 32);
    s1 += __shfl_xor(s1, 32);
    if (lane < 32) { red[wave * 64 + 2 * l32] = s0; red[wave * 64 + 2 * l32 + 1] = s1; }
    __syncthreads();
    if (t < 64 && n0 + t < g.d_out) {
      float s = 0.f;
      for (int w = 0; w < waves; ++w) s += red[w * 64 + t];
      g.db[(int64_t)split * g.d_out + n0 + t] = s;
    }
    __syncthreads();
  }
  if (!g.dw) return;
  const Epilogue<T> e = epilogue(g.b);
#pragma unroll
  for (int i = 0; i < 2; ++i) {                             // rows m0 + i, m0 + i + 2, ...
    if (i) __syncthreads();
    small_finish<T>(e, acc[i][0], acc[i][1], red, team, waves, m0 + i, 64, 2, g.d_in, n0, g.d_out);
  }
}

// ---------------------------------------------------------------------- dz = dy act'(z), and its column sums
// 256 threads: 32 pieces of columns, 8 rows at a time; a workgroup's shares of the column sums leave in `sums` [gridDim.y][N].  Rows of dz
// are whole pieces (lddz), zeros from N on.  Bound by memory: 8192 x 2048 bf16 18 us, 5.6 TB/s, a large copy's rate and more (WHOLE: N is whole
// pieces; with the ends' branch 23).  bf16: silu's and gelu's dz is rounded once here, for products whose operands go from memory to LDS
// as they are.  dx and dW are then off by 2.3e-3 in the norm, their own rounding alone by 1.65e-3 (which is what two_parts leaves small products).  Two values here
// would make both contractions twice as long: 8192 x 2048 x 2048, dx 61 -> 104 us and dW 92 -> 143, where the whole pass takes 165.
// relu's dz, and dy itself, are bf16 values already.
template <bool WHOLE, typename T>
__device__ __forceinline__ void load_columns(Piece<T, kPiece<T>>& v, const T* p, int count) {
  constexpr int V = kPiece<T>;
  if (WHOLE || count >= V) { v.load(p); return; }
  T e[V];
#pragma unroll
  for (int i = 0; i < V; ++i) e[i] = p[min(i, count - 1)];
#pragma unroll
  for (int i = 0; i < V; ++i) e[i] = i < count ? e[i] : T(0);
  __builtin_memcpy(v.w, e, 16);
}
template <typename T, bool WHOLE>
__global__ __launch_bounds__(256) void linear_dz_kernel(const T* dy, int64_t lddy, const T* z, int64_t ldz, T* dz, int64_t lddz, int64_t rows,
                                                        int N, int act, float* sums) {
  constexpr int V = kPiece<T>;
  __shared__ float red[8][32 * V + 1];
  const int t = threadIdx.x, c = t & 31, rl = t >> 5;
  const int n = ((int)blockIdx.x * 32 + c) * V;
  float s[V];
#pragma unroll
  for (int e = 0; e < V; ++e) s[e] = 0.f;
  if (n < N) {
#pragma unroll 2
    for (int64_t m = (int64_t)blockIdx.y * 8 + rl; m < rows; m += (int64_t)gridDim.y * 8) {
      Piece<T, V> d, h, o;
      load_columns<WHOLE>(d, dy + m * lddy + n, N - n);
      if (act != ABS_ACT_NONE) load_columns<WHOLE>(h, z + m * ldz + n, N - n);
      float f[V], g[V];
#pragma unroll
      for (int e = 0; e < V; ++e) { f[e] = d.at(e); g[e] = act != ABS_ACT_NONE ? h.at(e) : 0.f; }
      op_slope_all<V, kFine<T>>(f, g, act);
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] += f[e];
      o.set(f);
      if (dz) o.store(dz + m * lddz + n);
    }
  }
  if (!sums) return;
#pragma unroll
  for (int e = 0; e < V; ++e) red[rl][c * V + e] = s[e];
  __syncthreads();
  for (int j = t; j < 32 * V; j += 256) {
    const int col = (int)blockIdx.x * 32 * V + j;
    if (col < N) {
      float v = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) v += red[k][j];
      sums[(int64_t)blockIdx.y * N + col] = v;
    }
  }
}

__global__ __launch_bounds__(256) void linear_db_kernel(DbShares d) { add_db(d); }

// ---------------------------------------------------------------------- an operand whose rows are not whole 16-byte pieces: a copy that is
// (columns beyond the end are zero: they meet zeros or leave through columns that are not stored)
template <typename T>
struct Pack { const T* src; int64_t ld, rows, cols; T* dst; int64_t ldd; };
template <typename T>
__global__ __launch_bounds__(256) void linear_pack_kernel(Pack<T> first, Pack<T> second) {
  constexpr int V = kPiece<T>;
  const Pack<T>& p = blockIdx.y ? second : first;
  const int64_t pieces = p.ldd / V, total = p.rows * pieces;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
    const int64_t m = total < 1ll << 32 ? (int64_t)((uint32_t)q / (uint32_t)pieces) : q / pieces, c = (q - m * pieces) * V;
    Loose<T, V> o;
    if (c + V <= p.cols) o = *(const Loose<T, V>*)(p.src + m * p.ld + c);
    else {
#pragma unroll
      for (int e = 0; e < V; ++e) o.e[e] = c + e < p.cols ? p.src[m * p.ld + c + e] : T(0);
    }
    *(Loose<T, V>*)(p.dst + m * p.ldd + c) = o;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void linear_zero_kernel(T* p, int64_t ld, int64_t rows, int64_t cols) {
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < rows * cols; q += (int64_t)gridDim.x * 256) p[q / cols * ld + q % cols] = T(0);
}

unsigned few_blocks(int64_t threads) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((threads + 255) / 256, 1 << 16)); }

// ---------------------------------------------------------------------- the plan
struct Product {                              // one product on a tile kernel
  bool big;
  int mt, nt, nsplit, steps_per_split;
  size_t part_bytes;
};
// A product's plan is the cheapest by a model of what was measured (us; bf16, fp32 in brackets).  A k-step of 64 (32) takes a CU 1.4
// on one large tile, 0.78 (2.2) on one 128 x 128 tile and 1.04 (4.1) on two of those at a time; a workgroup's start and end cost 12,
// 5 (8) and 7 (8); shares cost a launch of 3 and their bytes, written and read, at 6 TB/s.  Model / measured: 8192 x 2048 x
// 2048 57 / 62 large, 81 / 81 small tiles; 4096 x 2048 x 2048 57 / 54 and 40 / 41; 2048^3 30 / 30 in one run, 38 / 36 in two shares;
// 256 x 4096 x 4096 26 / 25 in four; fp32 4096 x 1024 x 1024 78 / 78.
struct TileCost { double start, step, start2, step2, big_start, big_step; };
TileCost tile_cost(int dtype) { return dtype == ABS_X_BF16 ? TileCost{5, 0.78, 7, 1.04, 12, 1.4} : TileCost{8, 2.2, 8, 4.1, 0, 0}; }
double join_cost(int64_t split, int64_t M, int64_t N) { return split > 1 ? 3 + (double)split * M * N * 8 / 6e6 : 0; }

size_t shares_bytes(int shares, int64_t M, int64_t N) { return (size_t)shares * M * op_round_up(N, 4) * 4; }
Product cut_product(int64_t M, int64_t N, int64_t K, int dtype, bool big, int64_t split) {
  Product q{};
  const int tile = big ? kBig : kTile, step = dtype == ABS_X_BF16 ? 64 : 32;
  q.big = big;
  q.mt = (int)((M + tile - 1) / tile);
  q.nt = (int)((N + tile - 1) / tile);
  const int64_t steps = (K + step - 1) / step;
  q.steps_per_split = (int)((steps + split - 1) / split);
  q.nsplit = (int)((steps + q.steps_per_split - 1) / q.steps_per_split);
  if (q.nsplit > 1) q.part_bytes = shares_bytes(q.nsplit, M, N);
  return q;
}
constexpr int kCuts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
bool cut_counts(const Product& q, int split) { return q.nsplit == split && (split == 1 || (q.steps_per_split >= 4 && (int64_t)q.mt * q.nt * split <= 2048)); }

Product plan_product(int64_t M, int64_t N, int64_t K, int dtype, double* cost_out) {
  const TileCost c = tile_cost(dtype);
  Product best{};
  double least = 1e30;
  for (int big = dtype == ABS_X_BF16 ? 1 : 0; big >= 0; --big)
    for (int split : kCuts) {
      const Product q = cut_product(M, N, K, dtype, big != 0, split);
      if (!cut_counts(q, split)) continue;
      const double units = (double)q.mt * q.nt * q.nsplit, steps = q.steps_per_split;
      const double us = (big ? std::ceil(units / 256) * (c.big_start + c.big_step * steps)
                             : units <= 256 ? c.start + c.step * steps : std::ceil(units / 512) * (c.start2 + c.step2 * steps)) +
                        join_cost(q.nsplit, M, N);
      if (us < least) { least = us; best = q; }
    }
  if (cost_out) *cost_out = least;
  return best;
}

// When the last of `nb` runs of tb us and then `na` of ta us ends, each taking the first of `slots` places that is free.
double last_end(int64_t nb, double tb, int64_t na, double ta, int64_t slots) {
  const int64_t each = nb / slots, more = nb % slots;             // `more` places take one more of the first kind
  const double early = each * tb, late = early + (more ? tb : 0);
  double end = late;
  int64_t fit_early = 0, fit_late = 0;                            // runs of the second kind that places of either sort have taken
  while (fit_early * (slots - more) + fit_late * more < na) {
    const double e = early + (fit_early + 1) * ta, l = late + (fit_late + 1) * ta;
    if (e <= l) ++fit_early; else ++fit_late;
    end = std::max(end, std::min(e, l));
  }
  return end;
}

// dx and dW in one launch, or, where that is cheaper, one after the other (false).  Workgroups of both kinds share the CUs, dW's first,
// a step costing 1.15 of what it does alone on large tiles.  Model / measured, bf16: 8192 x 2048 x 2048 127 / 128 (apart 139 / 160).
bool plan_pair(const abs_linear& p, double apart, Product& dx, Product& dw) {
  const TileCost c = tile_cost(p.dtype);
  double least = apart + 3;                                       // (their two launches' gap)
  bool found = false;
  for (int big = p.dtype == ABS_X_BF16 ? 1 : 0; big >= 0; --big)
    for (int sa : kCuts) {
      const Product a = cut_product(p.rows, p.d_in, p.d_out, p.dtype, big != 0, sa);
      if (!cut_counts(a, sa)) continue;
      for (int sb : kCuts) {
        const Product b = cut_product(p.d_in, p.d_out, p.rows, p.dtype, big != 0, sb);
        if (!cut_counts(b, sb)) continue;
        const double start = big ? c.big_start : c.start2, step = big ? 1.15 * c.big_step : c.step2, join = std::max(join_cost(sa, p.rows, p.d_in), join_cost(sb, p.d_in, p.d_out));
        const double ta = start + step * a.steps_per_split, tb = start + step * b.steps_per_split;
        const int64_t na = (int64_t)a.mt * a.nt * sa, nb = (int64_t)b.mt * b.nt * sb, slots = big ? 256 : 512;
        if (join + std::max(std::max(ta, tb), (na * ta + nb * tb) / slots) >= least) continue;
        const double us = join + last_end(nb, tb, na, ta, slots);
        if (us < least) { least = us; dx = a; dw = b; found = true; }
      }
    }
  return found;
}

// Which products linear_small_kernel takes (us, it / the tile kernels with their copies, dz and joins; bf16 unless said).  Forward
// 810 x 520 x 300 6.4 / 24, 1024^3 10 / 21, 2048 x 2048 x 512 20 / 23, 4096 x 256 x 1024 12.5 / 10.9; fp32 2048 x 512 x 512 22 / 28,
// 410 x 1736 x 1088 37 / 36, 1024^3 39 / 36.  Backward 512^3 11 / 17, 13556 x 176 x 94 35 / 36, 1024 x 512 x 512 24 / 19, 64 x 2048 x
// 2048 21 / 20, 4096 x 512 x 512 52 / 30; fp32 1024 x 512 x 512 30 / 34, 2048 x 512 x 512 53 / 42.  Layers so narrow that dW is a tile
// or two stay longer: 100000 x 64 x 64 53 / 65, fp32 73 / 175, 20000 x 64 x 512 71 / 111 (8192 x 256 x 256 55 / 45).  A dW of many tiles with
// few rows each is not for it: 8 x 4096 x 4096 80 / 35.
bool small_product(const abs_linear& p, bool backward) {
  const bool half = p.dtype == ABS_X_BF16;
  const double macs = (double)p.rows * p.d_in * p.d_out;
  if (p.d_in < 2 || p.d_out < 2) return false;                       // (columns are read in pairs)
  if (!backward) return macs <= (half ? 2.2e9 : 7.5e8);
  const double width = (double)p.d_in * p.d_out;
  return width <= 4.3e6 && macs <= (width <= (half ? 8192 : 40000) ? (half ? 8e8 : 1e9) : 3e8);
}

struct SmallProduct { int nt, tiles, splits, steps, team; size_t part_bytes; };

struct LinearPlan {
  bool small, pair, pack_x, pack_w, dz;
  int sum_rows;
  SmallProduct sa, sb;                        // the forward product or dx; dW
  Product fwd, dx, dw, pair_dx, pair_dw;
  int64_t in8, out8;                          // d_in, d_out in whole pieces
  size_t off_x, off_w, off_dz, off_sums, off_part, off_part2, bytes;
};

// x_ok, w_ok, dy_ok: the pointers are aligned to pieces.  shares: the forward product, or dW, stays in shares, also where there is one.
LinearPlan linear_plan(const abs_linear& p, bool backward, bool x_ok, bool w_ok, bool dy_ok, bool shares = false) {
  LinearPlan q{};
  const int size = op_size(p.dtype), piece = 16 / size;
  q.in8 = (int64_t)op_round_up(p.d_in, piece);
  q.out8 = (int64_t)op_round_up(p.d_out, piece);
  const bool x_whole = x_ok && p.d_in % piece == 0 && p.ldx % piece == 0;
  const bool w_whole = w_ok && p.d_out % piece == 0 && p.ldw % piece == 0;
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = op_round_up(o + bytes, 256); return at; };
  q.small = small_product(p, backward);
  if (q.small) {
    const int block = p.dtype == ABS_X_BF16 ? 16 : 8;
    auto split = [&](int64_t M, int64_t N, int64_t K, int rows_of_tile, bool keep) {
      SmallProduct s{};
      s.nt = (int)((N + 63) / 64);
      s.tiles = (int)((M + rows_of_tile - 1) / rows_of_tile) * s.nt;
      // a long contraction of few tiles in shares, four blocks a wavefront at least
      const int64_t blocks = (K + block - 1) / block, each = 4 * kSmallWaves;
      const int64_t cuts = blocks <= (p.dtype == ABS_X_BF16 && rows_of_tile == 32 ? 4 : 2) * each ? 1 : std::max<int64_t>(1, std::min<int64_t>((blocks + each - 1) / each, 640 / s.tiles));
      s.steps = (int)((blocks + cuts - 1) / cuts);
      s.splits = (int)((blocks + s.steps - 1) / s.steps);
      // several tiles in a workgroup: with blocks too few for eight wavefronts as long as every CU has a workgroup, else two
      // (30000 x 300 x 20, gradients 81 -> 50 us; 2 x 645 x 23, whose few workgroups would do eight tiles' epilogues each, 8 -> 21)
      const int64_t mt = (M + rows_of_tile - 1) / rows_of_tile, mine = std::min<int64_t>(blocks, s.steps);
      s.team = kSmallWaves;
      while (s.team > 1 && mt * s.nt * s.splits * (s.team / 2) >= (s.team / 2 >= mine ? 256 : 512) * kSmallWaves) s.team /= 2;
      s.tiles = (int)((mt * s.team + kSmallWaves - 1) / kSmallWaves) * s.nt;
      s.part_bytes = s.splits > 1 || keep ? op_round_up(shares_bytes(s.splits, M, N), 256) : 0;
      return s;
    };
    q.sa = backward ? split(p.rows, p.d_in, p.d_out, 32, false) : split(p.rows, p.d_out, p.d_in, 32, shares);
    if (backward) q.sb = split(p.d_in, p.d_out, p.rows, 64, shares);
    q.off_part = take(q.sa.part_bytes);
    q.off_dz = take(q.sb.part_bytes);
    q.off_sums = take(q.sb.splits > 1 ? (size_t)q.sb.splits * p.d_out * 4 : 0);
    q.bytes = o;
    return q;
  }
  if (!backward) {
    q.pack_x = !x_whole;
    q.pack_w = !w_whole;
    if (q.pack_x) q.off_x = take((size_t)p.rows * q.in8 * size);
    if (q.pack_w) q.off_w = take((size_t)p.d_in * q.out8 * size);
    q.fwd = plan_product(p.rows, p.d_out, p.d_in, p.dtype, nullptr);
    if (shares) q.fwd.part_bytes = shares_bytes(q.fwd.nsplit, p.rows, p.d_out);
    q.off_part = take(q.fwd.part_bytes);
  } else {
    q.pack_x = !x_whole;
    q.pack_w = !w_whole;
    if (q.pack_x) q.off_x = take((size_t)p.rows * q.in8 * size);
    if (q.pack_w) q.off_w = take((size_t)p.d_in * q.out8 * size);
    q.dz = p.act != ABS_ACT_NONE || !(dy_ok && p.d_out % piece == 0 && p.lddy % piece == 0);
    if (q.dz) q.off_dz = take((size_t)p.rows * q.out8 * size);
    // eight workgroups on every CU, 16 rows each at least
    const int cols = (int)((q.out8 / piece + 31) / 32);
    q.sum_rows = (int)std::max<int64_t>(1, std::min<int64_t>((p.rows + 15) / 16, std::max(1, 2048 / cols)));
    q.off_sums = take((size_t)q.sum_rows * p.d_out * 4);
    double ca, cb;
    q.dx = plan_product(p.rows, p.d_in, p.d_out, p.dtype, &ca);
    q.dw = plan_product(p.d_in, p.d_out, p.rows, p.dtype, &cb);
    if (shares) q.dw.part_bytes = shares_bytes(q.dw.nsplit, p.d_in, p.d_out);
    q.off_part = take(std::max(q.dx.part_bytes, q.dw.part_bytes));
    q.off_part2 = q.off_part;
    Product a, b;
    if (plan_pair(p, ca + cb, a, b)) {        // (used where both are asked for)
      q.pair = true;
      if (shares) b.part_bytes = shares_bytes(b.nsplit, p.d_in, p.d_out);
      q.pair_dx = a; q.pair_dw = b;
      q.off_part2 = q.off_part + op_round_up(b.part_bytes, 256);
      o = std::max(o, op_round_up(q.off_part2 + a.part_bytes, 256));
    }
  }
  q.bytes = o;
  return q;
}

const char* linear_problem(const abs_linear* p, bool backward) {
  if (!p) return "linear: the description is NULL";
  if (p->dtype != ABS_X_FP32 && p->dtype != ABS_X_BF16) return "linear: dtype must be ABS_X_FP32 or ABS_X_BF16";
  if (p->act < ABS_ACT_NONE || p->act > ABS_ACT_GELU) return "linear: act must be 0..3";
  if (p->rows < 0 || p->rows > 0x7FFFFFFF) return "linear: rows must be in [0, 2^31)";
  if (p->d_in < 1 || p->d_out < 1 || p->d_in > 1 << 20 || p->d_out > 1 << 20) return "linear: d_in and d_out must be in [1, 2^20]";
  constexpr int64_t most = 1ll << 32;
  if (p->ldx < p->d_in || p->ldw < p->d_out || p->ldx >= most || p->ldw >= most) return "linear: a pitch is below the row's length, or 2^32 or more";
  const int64_t wide = std::max(p->d_in, p->d_out) / kTile + 1, narrow = std::min(p->d_in, p->d_out) / kTile + 1;
  if (std::max(p->rows / kTile + 1, narrow) * wide > 1 << 22) return "linear: the result has more than 2^22 tiles of 128 x 128";
  (void)backward;
  return nullptr;
}
bool bad_pitch(int64_t ld, int64_t cols) { return ld < cols || ld >= 1ll << 32; }

// The copies that a pass's operands need, side by side.
template <typename T>
hipError_t pack_operands(const abs_linear& p, const LinearPlan& q, const void* x, const void* w, bool want_x, bool want_w, char* ws, hipStream_t s) {
  const Pack<T> px{(const T*)x, p.ldx, p.rows, p.d_in, (T*)(ws + q.off_x), q.in8}, pw{(const T*)w, p.ldw, p.d_in, p.d_out, (T*)(ws + q.off_w), q.out8};
  want_x = want_x && q.pack_x;
  want_w = want_w && q.pack_w;
  if (!want_x && !want_w) return hipSuccess;
  auto threads = [](const Pack<T>& c) { return c.rows * (c.ldd / kPiece<T>); };
  const int64_t most = std::max(want_x ? threads(px) : 0, want_w ? threads(pw) : 0);
  linear_pack_kernel<T><<<dim3(few_blocks(most), want_x && want_w ? 2 : 1), 256, 0, s>>>(want_x ? px : pw, pw);
  return hipGetLastError();
}

// What is left after the products: shares to be joined (a job without them is left out) and db's.
template <typename T>
hipError_t launch_join(const Join<T>& a, const Join<T>& b, const DbShares& d, hipStream_t s) {
  if (!a.shares && !b.shares) {
    if (!d.db) return hipSuccess;
    linear_db_kernel<<<dim3((unsigned)((d.N + 31) / 32)), 256, 0, s>>>(d);
    return hipGetLastError();
  }
  const Join<T>& one = a.shares ? a : b;
  auto threads = [](const Join<T>& j) { return j.shares ? j.M * ((j.N + kPiece<T> - 1) / kPiece<T>) : 0; };
  const bool both = a.shares && b.shares;
  const int64_t most = std::max(std::max(threads(a), threads(b)), d.db ? (int64_t)d.N * 8 : 0);
  linear_join_kernel<T><<<dim3(few_blocks(most), both ? 2 : 1), 256, 0, s>>>(one, b, d);
  return hipGetLastError();
}

// shares of a product that its caller adds: nothing is joined
template <typename T>
void hand_over(Join<T>& j, OpShares* out) {
  *out = OpShares{j.e.part, j.e.ldpart, j.e.part_stride, j.shares};
  j = Join<T>{};
}

// g with the plan's tiles and, where its contraction is cut (or `keep` wants its shares), shares that go to `part` and join into what g wanted
template <typename T>
Join<T> set_product(const Product& q, GemmArgs<T>& g, float* part, OpShares* keep = nullptr) {
  g.mt = q.mt; g.nt = q.nt; g.nsplit = q.nsplit; g.steps_per_split = q.steps_per_split;
  if (q.nsplit == 1 && !keep) return Join<T>{};
  g.e.ldpart = (int64_t)op_round_up(g.N, 4);
  g.e.part_stride = g.M * g.e.ldpart;
  g.e.part = part;
  Join<T> join{g.e, g.M, g.N, q.nsplit};
  if (keep) hand_over(join, keep);
  return join;
}
int product_blocks(const Product& q) { return (q.mt * q.nt * q.nsplit + 7) / 8 * 8; }

template <typename T, bool ATR, bool BTR>
hipError_t run_product(const Product& q, GemmArgs<T> g, float* part, const DbShares& d, OpShares* keep, hipStream_t s) {
  const Join<T> join = set_product(q, g, part, keep);
  const dim3 grid((unsigned)product_blocks(q));
  if (q.big) {
    if constexpr (sizeof(T) == 2) linear_big_kernel<ATR, BTR><<<grid, 512, 0, s>>>(g);
  } else if (q.mt * q.nt * q.nsplit > 256) linear_tile_kernel<T, ATR, BTR, 2><<<grid, 256, 0, s>>>(g);
  else linear_tile_kernel<T, ATR, BTR, 4><<<grid, 256, 0, s>>>(g);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? launch_join(join, Join<T>{}, d, s) : e;
}

template <typename T>
SmallArgs<T> small_args(const abs_linear& p, const void* x, const void* w) {
  SmallArgs<T> g{};
  g.x = (const T*)x; g.w = (const T*)w; g.ldx = p.ldx; g.ldw = p.ldw;
  g.rows = (int)p.rows; g.d_in = p.d_in; g.d_out = p.d_out;
  return g;
}
// one product of linear_small_kernel, and what joins its shares (join.shares stays 0 where there is one)
template <typename T>
SmallPart<T> small_part(const SmallProduct& q, const Epilogue<T>& e, float* part, int64_t M, int64_t N, Join<T>& join, OpShares* keep = nullptr) {
  SmallPart<T> s{e, q.nt, q.tiles, q.splits, q.steps, q.team};
  if (q.splits > 1 || keep) {
    s.e.part = part;
    s.e.ldpart = (int64_t)op_round_up(N, 4);
    s.e.part_stride = M * s.e.ldpart;
    join = Join<T>{s.e, M, N, q.splits};
    if (keep) hand_over(join, keep);
  }
  return s;
}

template <typename T>
hipError_t forward_run(const abs_linear& p, const LinearPlan& q, const void* x, const void* w, const float* b, const void* r, void* y, void* z,
                       OpShares* keep, char* ws, hipStream_t s) {
  Epilogue<T> e{};
  e.bias = b; e.r = (const T*)r; e.y = (T*)y; e.z = (T*)z;
  e.ldr = p.ldr; e.ldy = p.ldy; e.ldz = p.ldz; e.act = p.act;
  if (q.small) {
    SmallArgs<T> g = small_args<T>(p, x, w);
    Join<T> join{};
    g.a = small_part(q.sa, e, (float*)(ws + q.off_part), p.rows, p.d_out, join, keep);
    const dim3 grid((unsigned)(q.sa.tiles * q.sa.splits));
    if (q.sa.team == kSmallWaves) linear_small_kernel<T, false, kSmallWaves><<<grid, 512, 0, s>>>(g);
    else                          linear_small_kernel<T, false, 0><<<grid, 512, 0, s>>>(g);
    const hipError_t err = hipGetLastError();
    return err == hipSuccess ? launch_join(join, Join<T>{}, DbShares{}, s) : err;
  }
  float* part = (float*)(ws + q.off_part);
  GemmArgs<T> g{};
  g.A = (const T*)x; g.lda = p.ldx; g.B = (const T*)w; g.ldb = p.ldw;
  hipError_t err = hipSuccess;
  if (q.pack_x) { g.A = (const T*)(ws + q.off_x); g.lda = q.in8; }
  if (q.pack_w) { g.B = (const T*)(ws + q.off_w); g.ldb = q.out8; }
  err = pack_operands<T>(p, q, x, w, true, true, ws, s);
  if (err != hipSuccess) return err;
  g.M = p.rows; g.N = p.d_out; g.K = p.d_in; g.nc = q.out8; g.mc = 0;
  g.e = e;
  return run_product<T, false, true>(q.fwd, g, part, DbShares{}, keep, s);
}

template <typename T>
hipError_t backward_run(const abs_linear& p, const LinearPlan& q, const void* x, const void* w, const void* z, const void* dy, void* dx, void* dw,
                        OpShares* keep, float* db, char* ws, hipStream_t s) {          // keep: dW's shares in place of dW
  constexpr int V = kPiece<T>;
  const bool want_dw = dw || keep;
  hipError_t err = hipSuccess;
  if (q.small) {
    SmallArgs<T> g = small_args<T>(p, x, w);
    g.dz = {(const T*)dy, (const T*)z, p.lddy, p.ldz, p.act};
    Epilogue<T> ea{}, eb{};
    ea.y = (T*)dx; ea.ldy = p.lddx;
    eb.y = (T*)dw; eb.ldy = p.lddw;
    Join<T> ja{}, jb{};
    DbShares d{};
    if (dx) g.a = small_part(q.sa, ea, (float*)(ws + q.off_part), p.rows, p.d_in, ja);
    if (want_dw || db) {
      g.b = small_part(q.sb, eb, (float*)(ws + q.off_dz), want_dw ? p.d_in : 0, p.d_out, jb, keep);
      if (!want_dw) g.b.tiles = g.b.nt;                            // (db alone: the first row of dW's tiles)
      g.dw = want_dw;
      g.db = db && q.sb.splits > 1 ? (float*)(ws + q.off_sums) : db;
      if (db && q.sb.splits > 1) d = DbShares{g.db, q.sb.splits, p.d_out, db};
    }
    const int blocks = g.a.tiles * g.a.splits + g.b.tiles * g.b.splits;
    if (blocks == 0) return hipSuccess;
    const dim3 grid((unsigned)blocks);
    if (q.sa.team == kSmallWaves && q.sb.team == kSmallWaves) linear_small_kernel<T, true, kSmallWaves><<<grid, 512, 0, s>>>(g);
    else                                                       linear_small_kernel<T, true, 0><<<grid, 512, 0, s>>>(g);
    err = hipGetLastError();
    return err == hipSuccess ? launch_join(ja, jb, d, s) : err;
  }
  const T* dz = (const T*)dy;
  int64_t lddz = p.lddy;
  const bool products = dx || want_dw;
  DbShares d{};
  float* sums = db ? (float*)(ws + q.off_sums) : nullptr;
  if ((q.dz && products) || db) {
    T* out = q.dz && products ? (T*)(ws + q.off_dz) : nullptr;
    const dim3 grid((unsigned)((p.d_out + 32 * V - 1) / (32 * V)), (unsigned)q.sum_rows);
    if (p.d_out % V == 0) linear_dz_kernel<T, true><<<grid, 256, 0, s>>>((const T*)dy, p.lddy, (const T*)z, p.ldz, out, q.out8, p.rows, p.d_out, p.act, sums);
    else                  linear_dz_kernel<T, false><<<grid, 256, 0, s>>>((const T*)dy, p.lddy, (const T*)z, p.ldz, out, q.out8, p.rows, p.d_out, p.act, sums);
    err = hipGetLastError();
    if (db) d = DbShares{sums, q.sum_rows, p.d_out, db};
    if (out) { dz = out; lddz = q.out8; }
  }
  float* part = (float*)(ws + q.off_part);
  GemmArgs<T> ga{}, gb{};
  if (err == hipSuccess && dx) {
    ga.A = dz; ga.lda = lddz; ga.B = (const T*)w; ga.ldb = p.ldw;
    if (q.pack_w) { ga.B = (const T*)(ws + q.off_w); ga.ldb = q.out8; }
    ga.M = p.rows; ga.N = p.d_in; ga.K = p.d_out;
    ga.e.y = (T*)dx; ga.e.ldy = p.lddx;
  }
  if (err == hipSuccess && want_dw) {
    gb.A = (const T*)x; gb.lda = p.ldx; gb.B = dz; gb.ldb = lddz;
    if (q.pack_x) { gb.A = (const T*)(ws + q.off_x); gb.lda = q.in8; }
    gb.M = p.d_in; gb.N = p.d_out; gb.K = p.rows; gb.mc = q.in8; gb.nc = q.out8;
    gb.e.y = (T*)dw; gb.e.ldy = p.lddw;
  }
  if (err == hipSuccess) err = pack_operands<T>(p, q, x, w, want_dw, dx != nullptr, ws, s);
  if (err != hipSuccess) return err;
  if (q.pair && dx && want_dw) {
    const Join<T> jb = set_product(q.pair_dw, gb, part, keep), ja = set_product(q.pair_dx, ga, (float*)(ws + q.off_part2));
    const int first = product_blocks(q.pair_dw);
    const dim3 grid((unsigned)(first + product_blocks(q.pair_dx)));
    if (!q.pair_dw.big) linear_tile_pair_kernel<T><<<grid, 256, 0, s>>>(gb, ga, first);
    else if constexpr (sizeof(T) == 2) linear_big_pair_kernel<<<grid, 512, 0, s>>>(gb, ga, first);
    err = hipGetLastError();
    return err == hipSuccess ? launch_join(ja, jb, d, s) : err;
  }
  if (dx) { err = run_product<T, false, false>(q.dx, ga, part, d, nullptr, s); d = DbShares{}; }
  if (err == hipSuccess && want_dw) { err = run_product<T, true, true>(q.dw, gb, part, d, keep, s); d = DbShares{}; }
  return err == hipSuccess ? launch_join(Join<T>{}, Join<T>{}, d, s) : err;
}

// Both passes behind their checks of what they write: keep: shares (OpShares) in place of y, or of dW.
int forward_call(const abs_linear* p, const void* x, const void* w, const float* b, const void* r, void* y, void* z, OpShares* keep, void* ws,
                 size_t bytes, hipStream_t s) {
  if (!x || !w || !(y || keep)) return op_fail(ABS_E_ARG, "linear: a device pointer is NULL");
  const uintptr_t all = (uintptr_t)x | (uintptr_t)w | (uintptr_t)r | (uintptr_t)y | (uintptr_t)z;
  if (all & (uintptr_t)(op_size(p->dtype) - 1) || (uintptr_t)b & 3) return op_fail(ABS_E_ARG, "linear: a pointer is not aligned to its elements");
  const LinearPlan q = linear_plan(*p, false, op_aligned(x, 16), op_aligned(w, 16), true, keep != nullptr);
  if (q.bytes && (!ws || (uintptr_t)ws & 255)) return op_fail(ABS_E_ARG, "linear: d_workspace must be 256-byte aligned");
  if (bytes < q.bytes) return op_fail(ABS_E_WORKSPACE, "linear: workspace too small");
  const hipError_t e = p->dtype == ABS_X_BF16 ? forward_run<uint16_t>(*p, q, x, w, b, r, y, z, keep, (char*)ws, s)
                                              : forward_run<float>(*p, q, x, w, b, r, y, z, keep, (char*)ws, s);
  return op_hip("abs_linear_forward", e);
}

int backward_call(const abs_linear* p, const void* x, const void* w, const void* z, const void* dy, void* dx, void* dw, OpShares* keep, float* db,
                  void* ws, size_t bytes, hipStream_t s) {
  if (!dy || ((dw || keep) && !x) || (dx && !w) || (p->act != ABS_ACT_NONE && !z)) return op_fail(ABS_E_ARG, "linear: a device pointer is NULL");
  const LinearPlan q = linear_plan(*p, true, op_aligned(x, 16), op_aligned(w, 16), op_aligned(dy, 16), keep != nullptr);
  if (q.bytes && (!ws || (uintptr_t)ws & 255)) return op_fail(ABS_E_ARG, "linear: d_workspace must be 256-byte aligned");
  if (bytes < q.bytes) return op_fail(ABS_E_WORKSPACE, "linear: workspace too small");
  const hipError_t e = p->dtype == ABS_X_BF16 ? backward_run<uint16_t>(*p, q, x, w, z, dy, dx, dw, keep, db, (char*)ws, s)
                                              : backward_run<float>(*p, q, x, w, z, dy, dx, dw, keep, db, (char*)ws, s);
  return op_hip("abs_linear_backward", e);
}

}  // namespace

// (the library's own calls: operands aligned, pitches checked where the arrays are laid out)
size_t op_linear_shares_size(const abs_linear* p, int32_t backward) noexcept { return linear_plan(*p, backward != 0, false, false, false, true).bytes; }
int op_linear_forward_shares(const abs_linear* p, const void* d_x, const void* d_w, void* d_workspace, size_t workspace_bytes, void* hip_stream,
                             OpShares* product) noexcept {
  if (const char* why = linear_problem(p, false)) return op_fail(ABS_E_ARG, why);
  return forward_call(p, d_x, d_w, nullptr, nullptr, nullptr, nullptr, product, d_workspace, workspace_bytes, (hipStream_t)hip_stream);
}
int op_linear_backward_shares(const abs_linear* p, const void* d_x, const void* d_w, const void* d_z, const void* d_dy, void* d_dx, float* d_db,
                              void* d_workspace, size_t workspace_bytes, void* hip_stream, OpShares* dw) noexcept {
  if (const char* why = linear_problem(p, true)) return op_fail(ABS_E_ARG, why);
  return backward_call(p, d_x, d_w, d_z, d_dy, d_dx, nullptr, dw, d_db, d_workspace, workspace_bytes, (hipStream_t)hip_stream);
}

}  // namespace abs_impl

using namespace abs_impl;

extern "C" {

size_t abs_linear_workspace_size(const abs_linear* p, int32_t backward, int32_t aligned) {
  if (const char* why = linear_problem(p, backward != 0)) { op_fail(ABS_E_ARG, why); return 0; }
  return p->rows ? linear_plan(*p, backward != 0, aligned != 0, aligned != 0, aligned != 0).bytes : 0;
}

int abs_linear_forward(const abs_linear* p, const void* d_x, const void* d_w, const float* d_b, const void* d_r,
                       void* d_y, void* d_z, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (const char* why = linear_problem(p, false)) return op_fail(ABS_E_ARG, why);
  if (bad_pitch(p->ldy, p->d_out) || (d_z && bad_pitch(p->ldz, p->d_out)) || (d_r && bad_pitch(p->ldr, p->d_out)))
    return op_fail(ABS_E_ARG, "linear: a pitch is below the row's length, or 2^32 or more");
  if (p->rows == 0) return ABS_OK;
  return forward_call(p, d_x, d_w, d_b, d_r, d_y, d_z, nullptr, d_workspace, workspace_bytes, (hipStream_t)hip_stream);
}

int abs_linear_backward(const abs_linear* p, const void* d_x, const void* d_w, const void* d_z, const void* d_dy,
                        void* d_dx, void* d_dw, float* d_db, void* d_workspace, size_t workspace_bytes,
                        void* hip_stream) {
  if (const char* why = linear_problem(p, true)) return op_fail(ABS_E_ARG, why);
  if (bad_pitch(p->lddy, p->d_out) || (d_dx && bad_pitch(p->lddx, p->d_in)) || (d_dw && bad_pitch(p->lddw, p->d_out)) ||
      (p->act != ABS_ACT_NONE && bad_pitch(p->ldz, p->d_out)))
    return op_fail(ABS_E_ARG, "linear: a pitch is below the row's length, or 2^32 or more");
  const uintptr_t all = (uintptr_t)d_x | (uintptr_t)d_w | (uintptr_t)d_z | (uintptr_t)d_dy | (uintptr_t)d_dx | (uintptr_t)d_dw;
  if (all & (uintptr_t)(op_size(p->dtype) - 1) || (uintptr_t)d_db & 3) return op_fail(ABS_E_ARG, "linear: a pointer is not aligned to its elements");
  const hipStream_t s = (hipStream_t)hip_stream;
  if (p->rows == 0) {                       // sums over nothing
    hipError_t e = hipSuccess;
    if (d_dw) {
      const unsigned blocks = few_blocks((int64_t)p->d_in * p->d_out);
      if (p->dtype == ABS_X_BF16) linear_zero_kernel<uint16_t><<<blocks, 256, 0, s>>>((uint16_t*)d_dw, p->lddw, p->d_in, p->d_out);
      else                        linear_zero_kernel<float><<<blocks, 256, 0, s>>>((float*)d_dw, p->lddw, p->d_in, p->d_out);
      e = hipGetLastError();
    }
    if (e == hipSuccess && d_db) { linear_zero_kernel<float><<<few_blocks(p->d_out), 256, 0, s>>>(d_db, p->d_out, 1, p->d_out); e = hipGetLastError(); }
    return op_hip("abs_linear_backward", e);
  }
  return backward_call(p, d_x, d_w, d_z, d_dy, d_dx, d_dw, nullptr, d_db, d_workspace, workspace_bytes, s);
}

}  // extern "C"
